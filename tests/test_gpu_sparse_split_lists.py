"""A few queries with long lists: the lists are cut into ranges whose parts a second kernel joins, launched while the first still
runs.  Calls one behind the other in one workspace must each join their own parts."""
import pytest

from helpers import dev_bf16
from paper_2603_17051_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n_q", [(1, 5), (2, 40), (12, 128)])
def test_calls_in_one_workspace_join_their_own_parts(D, H, n_q):
    import torch
    from paper_2603_17051_b200 import binding as A
    n_kc, block, n = 4096, 64, 60
    k, v = (dev_bf16(synth.normal_bf16(700 + i, (1, n_kc, H, D))) for i in range(2))
    g = torch.Generator().manual_seed(H)
    qs = [dev_bf16(synth.normal_bf16(710 + i, (1, n_q, H, D))) for i in range(6)]
    lists = [torch.stack([torch.randperm(64, generator=g)[:n] for _ in range(H)]).int().view(1, H, 1, n).cuda() for _ in qs]
    need = A.astro_sparse_attn_fwd_workspace_bytes(1, H, D, n_q, n, block)
    assert need > 0
    alone = []
    for q, b in zip(qs, lists):
        alone.append(A.astro_sparse_attn_fwd(None, q, k, v, b, block, D ** -0.5))
        torch.cuda.synchronize()
    shared = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(20):
        got = [A.astro_sparse_attn_fwd(None, q, k, v, b, block, D ** -0.5, workspace=shared) for q, b in zip(qs, lists)]
        torch.cuda.synchronize()
        for (o, lse), (po, plse) in zip(got, alone):
            assert torch.equal(o, po) and torch.equal(lse, plse)
