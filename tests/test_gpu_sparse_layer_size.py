"""The operators over chosen blocks at the size of a video transformer's layer: 4680 queries, 18 frames of 1560 tokens, 12 heads,
blocks of 120 tokens, 64 of 273 per query block.  Two heads are compared with fp64 torch, every other with the call repeated."""
import pytest

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8     # half a bf16 step, relative


def attention_fp64(q, k, v, d_o, blocks, block, scale):
    """O, LSE, dQ, dK, dV of one head over the keys of the listed blocks (full blocks, no repeats), and sum_j p_j |v_j|."""
    import torch
    n_q = q.shape[0]
    o, lse, dq, o_abs = torch.zeros_like(q), torch.zeros_like(q[:, 0]), torch.zeros_like(q), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    at0 = torch.arange(block, device=q.device)
    for i in range(blocks.shape[0]):
        at = (blocks[i].long()[:, None] * block + at0).flatten()
        r = slice(i * 128, min(n_q, i * 128 + 128))
        s = q[r] @ k[at].T * scale
        lse[r] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[r][:, None])
        o[r], o_abs[r] = p @ v[at], p @ v[at].abs()
        ds = p * (d_o[r] @ v[at].T - (d_o[r] * o[r]).sum(1, keepdim=True)) * scale
        dq[r] = ds @ k[at]
        dk.index_add_(0, at, ds.T @ q[r])
        dv.index_add_(0, at, p.T @ d_o[r])
    return o, lse, dq, dk, dv, o_abs


def test_choice_attention_and_gradients_at_the_size_of_a_layer():
    import torch
    from paper_2603_17051_b200 import binding as A
    H, D, T, S, L, n, block, n_select, scale = 12, 128, 1560, 3, 18, 4680, 120, 64, 128 ** -0.5
    g = torch.Generator(device="cuda").manual_seed(2)
    normal = lambda m: torch.randn((1, m, H, D), generator=g, device="cuda").bfloat16()  # noqa: E731
    cache = A.astro_kvcache_create(1, H, D, T, S, L)
    kx, vx = normal(20 * T), normal(20 * T)
    for first, count in ((0, 18), (18, 2)):                  # two frames leave the window, two more wrap around
        if first:
            A.astro_kvcache_evict(cache, 2)
        cut = slice(first * T, (first + count) * T)
        A.astro_kvcache_append(cache, kx[:, cut].contiguous(), vx[:, cut].contiguous(), count)
    held = [0, 1, 2] + list(range(5, 20))
    rows = (torch.tensor(held, device="cuda")[:, None] * T + torch.arange(T, device="cuda")).flatten()
    q, k, v, d_o = (normal(n) for _ in range(4))
    pooled = A.astro_block_pool(cache, block)
    sel = A.astro_block_select(cache, pooled, q, k, block, n_select, keep=A.KEEP_SINK | A.KEEP_CHUNK)
    o, lse = A.astro_sparse_attn_fwd(cache, q, k, v, sel, block, scale)
    grads = A.astro_sparse_attn_bwd(cache, q, k, v, sel, block, o, lse, d_o, scale)
    A.astro_last_device_status()
    assert sel.shape == (1, H, 37, n_select)
    score = (D + 8) * 2.0 ** -24 * 40.0                      # fp32 sums of D products below scale * sum |q_d k_d| < 40, the exponent's rounding
    for h in (0, H - 1):
        K, V = (torch.cat([c[0, rows, h], x[0, :, h]]).double() for c, x in ((kx, k), (vx, v)))
        mean = K.view(273, block, D).mean(1).float().double()
        qm = torch.stack([x.double().mean(0) for x in q[0, :, h].split(128)]).float().double()
        s = qm @ mean.T
        s[:, :39] = float("inf")                             # sink and chunk blocks come first
        s[:, 234:] = float("inf")
        want = s.sort(dim=1, descending=True, stable=True).indices[:, :n_select].sort(1).values
        assert torch.equal(sel[0, h].long(), want)
        r_o, r_lse, r_dq, r_dk, r_dv, o_abs = attention_fp64(q[0, :, h].double(), K, V, d_o[0, :, h].double(), sel[0, h], block, scale)
        err = (o[0, :, h].double() - r_o).abs()
        assert (err <= HALF * r_o.abs() + (HALF + 2 * score) * o_abs * (1 + HALF)).all()
        assert (lse[0, h].double() - r_lse).abs().max() <= score + 2.0 ** -22 * r_lse.abs().max()
        for got, ref in zip(grads, (r_dq, r_dk[18 * T:], r_dv[18 * T:])):
            assert (got[0, :, h].double() - ref).norm() <= 1e-2 * ref.norm()
    again = A.astro_sparse_attn_fwd(cache, q, k, v, sel, block, scale)
    twice = A.astro_sparse_attn_bwd(cache, q, k, v, sel, block, o, lse, d_o, scale)
    assert all(torch.equal(a, b) for a, b in zip((o, lse) + grads, again + twice))
