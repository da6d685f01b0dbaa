"""Places that only large or unusual inputs reach: offsets beyond 32 bits, long lists, a first call inside a captured graph."""
import subprocess
import sys

import numpy as np
import pytest

from helpers import f64
from oracle import rope as rope_orc
from oracle import sparse_attn as orc

pytestmark = pytest.mark.gpu


def test_caches_and_strides_beyond_32_bits():
    import torch
    from paper_2603_17051_b200 import binding as A
    H, D, T, S, L, block = 1, 64, 4096, 1, 15, 128
    B = 600                                              # 600 * 16 * 4096 * 64 elements: 5.0 GB of keys
    nbytes = A.astro_kvcache_storage_bytes(B, H, D, T, S, L)
    assert nbytes > 2 ** 32
    k, v = (torch.zeros(nbytes, dtype=torch.uint8, device="cuda") for _ in range(2))
    big = A.astro_kvcache_create(B, H, D, T, S, L, k_storage=k, v_storage=v)
    A.astro_kvcache_set_state(big, A.KVCacheState(1, 13, 3, 99))   # frames in slots 0, 14, 15, 1
    last = torch.randn(2, H, S + L, T, D, device="cuda").bfloat16()
    k.view(torch.bfloat16)[-last[0].numel():] = last[0].flatten()
    v.view(torch.bfloat16)[-last[1].numel():] = last[1].flatten()
    one = A.astro_kvcache_create(1, H, D, T, S, L, k_storage=last[0].clone(), v_storage=last[1].clone())
    A.astro_kvcache_set_state(one, A.KVCacheState(1, 13, 3, 99))
    q = torch.zeros(B, 3, H, D, device="cuda").bfloat16()
    q[-1] = torch.randn(3, H, D, device="cuda").bfloat16()
    pb, po = A.astro_block_pool(big, block), A.astro_block_pool(one, block)
    assert torch.equal(pb[-1], po[0])
    sb = A.astro_block_select(big, pb, q, None, block, 9)
    so = A.astro_block_select(one, po, q[-1:].contiguous(), None, block, 9)
    assert torch.equal(sb[-1], so[0])
    for n_q in (3, 1):                                   # the MMA kernel and the one for single queries
        x, y = (A.astro_sparse_attn_fwd(c, z[:, :n_q].contiguous(), None, None, s, block, 0.125)
                for c, z, s in ((big, q, sb), (one, q[-1:], so)))
        assert (x[0][-1].float() - y[0][0].float()).abs().max() <= 2 ** -6 and (x[1][-1] - y[1][0]).abs().max() <= 1e-5
        d_o = torch.ones_like(x[0])
        g = A.astro_sparse_attn_bwd(big, q[:, :n_q].contiguous(), None, None, sb, block, *x, d_o, 0.125)[0][-1]
        w = A.astro_sparse_attn_bwd(one, q[-1:, :n_q].contiguous(), None, None, so, block, *y, d_o[-1:].contiguous(), 0.125)[0][0]
        assert (g.float() - w.float()).abs().max() <= 2 ** -6
    small = A.astro_kvcache_create(2, H, D, T, 0, 2)
    A.astro_kvcache_fork(small, big, parents=torch.tensor([B - 1, 0], dtype=torch.int32, device="cuda"), frames=[3, 0])
    fk, _ = A.astro_kvcache_export(small)
    assert torch.equal(fk[0, :T, 0], last[0, 0, 1]) and torch.equal(fk[0, T:, 0], last[0, 0, 0]) and not fk[1].any()
    A.astro_last_device_status()
    # a rotary input whose second sample starts 2^31 elements on
    rope = A.astro_rope_create(D, D, "halves", (32,))
    room = k.view(torch.bfloat16)
    x = room.as_strided((2, 5, 1, D), (2 ** 31 - 2 ** 31 % 64, D, D, 1))
    pos = torch.arange(5, dtype=torch.int32, device="cuda").view(1, 5, 1)
    x[1] = torch.randn(5, 1, D, device="cuda").bfloat16()
    far, _ = A.astro_rope_apply(rope, x, None, pos)
    near, _ = A.astro_rope_apply(rope, x[1:].contiguous(), None, pos)
    assert torch.equal(far[1:], near)
    A.astro_rope_apply(rope, x, None, pos, q_out=x)      # in place, so far offsets on the way out too
    assert torch.equal(x[1:], near)


@pytest.mark.parametrize("n_q", [1, 2, 40, 300])
def test_lists_longer_than_the_keys(n_q):
    """Thousands of entries, most of them naming nothing: repeats count as often as they stand."""
    import torch
    from paper_2603_17051_b200 import binding as A
    H, D, n_kc, block, n = 1, 64, 150, 32, 5000
    g = torch.Generator().manual_seed(n_q)
    q, k, v, d_o = (torch.randn((1, m, H, D), generator=g).bfloat16() for m in (n_q, n_kc, n_kc, n_q))
    blocks = torch.full((1, H, -(-n_q // 128), n), -1, dtype=torch.int32)
    for i in range(blocks.shape[2]):
        at = torch.randperm(n, generator=g)[:37]
        blocks[0, 0, i, at] = torch.randint(0, 5, (37,), generator=g).int()
    ranges = orc.key_blocks(0, 1, n_kc, block)
    f = [x.double().numpy()[0, :, 0] for x in (q, k, v, d_o)]
    ref = orc.attend(f[0], f[1], f[2], blocks[0, 0].numpy(), ranges, 0.125, f[3], 0)
    dev = [x.cuda() for x in (q, k, v, d_o)]
    o, lse = A.astro_sparse_attn_fwd(None, *dev[:3], blocks.cuda(), block, 0.125)
    grads = A.astro_sparse_attn_bwd(None, *dev[:3], blocks.cuda(), block, o, lse, dev[3], 0.125)
    A.astro_last_device_status()
    assert np.abs(f64(o)[0, :, 0] - ref[0]).max() <= 2e-2 and np.abs(f64(lse)[0, 0] - ref[1]).max() <= 1e-4
    for got, want in zip(grads, ref[2:]):
        assert np.linalg.norm(f64(got)[0, :, 0] - want) <= 1e-2 * np.linalg.norm(want)


FIRST = """
import torch
from paper_2603_17051_b200 import binding as A
q, k, v = (torch.randn(2, n, 2, 64, device="cuda").bfloat16() for n in (%d, 90, 90))
pos = torch.arange(90, dtype=torch.int32, device="cuda").view(1, 90, 1)
rope = A.astro_rope_create(64, 64, "halves", (32,))
sel = torch.tensor([0, 2], dtype=torch.int32, device="cuda").expand(2, 2, 1, 2).contiguous()
d_o = torch.ones_like(q)

def whole():
    kr, _ = A.astro_rope_apply(rope, k, None, pos)
    picked = A.astro_block_select(None, None, q, kr, 32, 2)
    o, lse = A.astro_sparse_attn_fwd(None, q, kr, v, sel, 32, 0.125)
    return (kr, picked, o, lse) + A.astro_sparse_attn_bwd(None, q, kr, v, sel, 32, o, lse, d_o, 0.125)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = whole()
graph.replay()
torch.cuda.synchronize()
want = whole()
A.astro_last_device_status()
assert all(torch.equal(a, b) for a, b in zip(out, want))
print("same")
"""


@pytest.mark.parametrize("n_q", [1, 70])
def test_first_calls_of_a_process_inside_a_captured_graph(n_q):
    run = subprocess.run([sys.executable, "-c", FIRST % n_q], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "same" in run.stdout, run.stderr[-2000:]


def test_far_positions_of_every_type_stay_exact():
    import torch
    from paper_2603_17051_b200 import binding as A
    f, axis = rope_orc.frequencies((48,), 10000.0)
    rope = A.astro_rope_create(96, 96, "interleaved", (48,))
    pos = torch.tensor([0, 1, -1, 10 ** 6, 2 ** 30 + 1, -(2 ** 31)], dtype=torch.int32, device="cuda").view(1, 6, 1)
    x = torch.ones(1, 6, 1, 96, device="cuda")
    y, _ = A.astro_rope_apply(rope, x, None, pos)
    # the table's frequencies differ from the oracle's in their last bit: use the library's
    freq = np.array(A.astro_rope_frequencies(rope)[0])
    want = rope_orc.rotate(f64(x), pos.cpu().numpy(), freq, axis, "interleaved")
    assert np.abs(f64(y) - want).max() <= 1e-6 and np.allclose(freq, f, rtol=1e-13)
