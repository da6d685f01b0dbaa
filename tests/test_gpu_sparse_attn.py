"""GPU parity of attention over lists of key blocks against the fp64 oracle: forward, backward, and a run of the operators
together."""
import numpy as np
import pytest

from helpers import check_grads, dev_bf16, f64
from oracle import sparse_attn as orc
from oracle.rolling_attn import bf16_bits_to_f64
from paper_2603_17051_b200 import synth
from test_gpu_block_select import ring

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8     # half a bf16 step, relative


def lists(rng, B, H, nqb, n_blocks, n_select, kind):
    """int32 lists: random without repeats; `odd` adds entries out of range, repeats, empty and one-entry lists."""
    out = np.full((B, H, nqb, n_select), -1, np.int32)
    for idx in np.ndindex(B, H, nqb):
        pick = rng.permutation(n_blocks)[:n_select]
        out[idx][:len(pick)] = pick
        if kind == "odd":
            how = rng.integers(0, 6)
            if how == 0:
                out[idx] = -1
            elif how == 1:
                out[idx] = [n_blocks, -7, 2 ** 31 - 1, -2 ** 31][:n_select] + [-1] * max(0, n_select - 4)
            elif how == 2:
                out[idx][1:] = -1
            elif how == 3 and n_select > 1:
                out[idx][-1] = out[idx][0]
            elif how == 4:
                out[idx][:n_select // 2] = -1
        elif kind == "ascending":
            out[idx][:len(pick)] = np.sort(pick)
    return out


def reference(q, k, v, kx, vx, blocks, ranges, scale, n_ctx, d_o=None):
    """Oracle over all heads, plus sum_j p_j |v_j| and the largest scale * sum |q_d k_d| for the bounds."""
    B, n_q, H, D = q.shape
    outs = None
    o_abs = np.zeros_like(q)
    for b in range(B):
        for h in range(H):
            bc = min(b, kx.shape[0] - 1)
            kk, vv = (np.concatenate([x[bc, :, h], y[b, :, h]]) for x, y in ((kx, k), (vx, v)))
            r = orc.attend(q[b, :, h], kk, vv, blocks[b, h], ranges, scale, None if d_o is None else d_o[b, :, h], n_ctx)
            o_abs[b, :, h] = orc.attend(q[b, :, h], kk, np.abs(vv), blocks[b, h], ranges, scale)[0]
            if outs is None:
                outs = [np.zeros((B, n_q, H, D)), np.zeros((B, H, n_q))] + [np.zeros((B,) + x.shape[:1] + (H, D)) for x in r[2:]]
            outs[0][b, :, h], outs[1][b, h] = r[0], r[1]
            for i in range(2, len(r)):
                outs[i][b, :, h] = r[i]
    return outs, o_abs


def check_forward(o, lse, ref, o_abs, q, scale, D, tag):
    """O: its own rounding and that of every weight to bf16 (half a step each); scores: fp32 sums of D products, each
    partial sum of at most scale * sum |q_d k_d| <= about 40 here, and the exponent's own rounding."""
    score = (D + 8) * 2.0 ** -24 * 40.0 * max(1.0, scale * np.sqrt(D))
    want_o, want_lse = ref[0], ref[1]
    err = np.abs(f64(o) - want_o)
    bound = HALF * np.abs(want_o) + (HALF + 2 * score) * o_abs * (1 + HALF) + 1e-30
    assert (err <= bound).all(), "%s O %.3e over its bound" % (tag, (err - bound).max())
    got = f64(lse)
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got), empty), tag
    assert (np.abs(got[~empty] - want_lse[~empty]) <= score + 2.0 ** -22 * np.abs(want_lse[~empty]) + 1e-6).all(), tag
    e = np.moveaxis(empty, 1, 2)
    assert not f64(o)[e].any(), tag + ": queries without a key"


SHAPES = [  # Bc, B, H, D, T, S, L, evicted, held, n_q, n_kc, block, n_select
    (1, 1, 2, 64, 16, 0, 6, 0, 3, 48, 48, 16, 5),
    (1, 3, 2, 128, 100, 1, 6, 3, 5, 300, 130, 64, 7),
    (2, 2, 2, 128, 121, 2, 3, 2, 4, 1, 1, 120, 4),
    (1, 1, 1, 64, 7, 0, 9, 4, 6, 700, 0, 8, 3),
    (1, 2, 2, 64, 40, 3, 2, 0, 2, 5, 1000, 24, 40),
    (1, 1, 1, 128, 33, 0, 3, 0, 0, 129, 500, 128, 2),
    (1, 1, 1, 128, 260, 1, 3, 2, 3, 257, 90, 104, 9),
    (2, 2, 1, 128, 96, 0, 4, 1, 4, 128, 128, 96, 5),
    (1, 1, 3, 64, 130, 0, 4, 1, 3, 200, 77, 40, 14),
    (1, 4, 12, 128, 61, 0, 30, 5, 28, 3, 2, 32, 57),
    (1, 1, 1, 64, 1, 0, 40, 7, 33, 1, 0, 128, 33),
    (1, 3, 2, 128, 70, 1, 5, 2, 6, 2, 1, 64, 13),
    (2, 2, 5, 64, 97, 0, 12, 4, 12, 1, 1, 96, 20),
    (1, 1, 1, 128, 50, 0, 30, 3, 30, 2, 0, 8, 200),
    (1, 5, 33, 64, 31, 0, 4, 1, 4, 1, 3, 32, 5),
    (1, 1, 2, 128, 80, 2, 9, 3, 11, 5, 4, 40, 22),
]


@pytest.mark.parametrize("kind", ["ascending", "plain", "odd"])
@pytest.mark.parametrize("Bc,B,H,D,T,S,L,evicted,held,n_q,n_kc,block,n_select", SHAPES)
def test_forward_matches_the_oracle(Bc, B, H, D, T, S, L, evicted, held, n_q, n_kc, block, n_select, kind):
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, kx, vx, frames = ring(A, Bc, H, D, T, S, L, evicted, held, 1500, poison=True)
    bits = [synth.normal_bf16(1900 + i, (B, n, H, D)) for i, n in enumerate((n_q, max(1, n_kc), max(1, n_kc)))]
    q, k, v = (dev_bf16(x) for x in bits)
    qf, kf, vf = (bf16_bits_to_f64(x) for x in bits)
    ranges = orc.key_blocks(frames, T, n_kc, block)
    blocks = lists(np.random.default_rng(n_q + block), B, H, -(-n_q // 128), len(ranges), n_select, kind)
    scale = D ** -0.5
    ref, o_abs = reference(qf, kf[:, :n_kc], vf[:, :n_kc], kx, vx, blocks, ranges, scale, frames * T)
    tb = torch.from_numpy(blocks).cuda()
    for mode in (0, 1):
        A.astro_debug_forward_mode(mode)
        try:
            o, lse = A.astro_sparse_attn_fwd(cache, q, k if n_kc else None, v if n_kc else None, tb, block, scale)
        finally:
            A.astro_debug_forward_mode(0)
        A.astro_last_device_status()
        check_forward(o, lse, ref, o_abs, qf, scale, D, "%s mode %d" % (kind, mode))


@pytest.mark.parametrize("D", [64, 128])
def test_units_that_need_the_careful_pass_between_units_that_do_not(D):
    """More units than SMs; in some of them a later block's scores exceed those of the first by far more than 2^100."""
    import torch
    from paper_2603_17051_b200 import binding as A
    B, H, n_q, n_kc, block = 2, 4, 128 * 21 + 5, 640, 64
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((B, n, H, D), generator=g).bfloat16() for n in (n_q, n_kc, n_kc))
    k[:, 320:384] *= 30.0                                 # block 5: scores up to hundreds (scale 1)
    k[:, 0:64] *= 0.01
    rng = np.random.default_rng(1)
    ranges = orc.key_blocks(0, 1, n_kc, block)
    blocks = lists(rng, B, H, 22, len(ranges), 4, "plain")
    blocks[:, :, ::3] = [0, 1, 5, 2]                      # reference from block 0, then block 5
    qf, kf, vf = (x.double().numpy() for x in (q, k, v))
    none = np.zeros((1, 0, H, D))
    ref, o_abs = reference(qf, kf, vf, none, none, blocks, ranges, 1.0, 0)
    o, lse = A.astro_sparse_attn_fwd(None, q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(blocks).cuda(), block, 1.0)
    A.astro_last_device_status()
    # scores here reach 30 * 40: the fp32 score error grows with them
    err = np.abs(f64(o) - ref[0])
    score = (D + 8) * 2.0 ** -24 * np.abs(ref[1]).max() * 4
    assert (err <= HALF * np.abs(ref[0]) + (HALF + 2 * score) * o_abs * 1.01).all()
    assert np.abs(f64(lse) - ref[1]).max() <= score


def test_many_short_lists_per_cta_and_single_tile_units():
    import torch
    from paper_2603_17051_b200 import binding as A
    B, H, D, n_q, n_kc, block = 3, 5, 64, 128 * 40, 256, 32
    bits = [synth.normal_bf16(40 + i, (B, n, H, D)) for i, n in enumerate((n_q, n_kc, n_kc))]
    qf, kf, vf = (bf16_bits_to_f64(x) for x in bits)
    ranges = orc.key_blocks(0, 1, n_kc, block)
    blocks = lists(np.random.default_rng(3), B, H, 40, len(ranges), 3, "odd")
    none = np.zeros((1, 0, H, D))
    ref, o_abs = reference(qf, kf, vf, none, none, blocks, ranges, 0.125, 0)
    o, lse = A.astro_sparse_attn_fwd(None, *(dev_bf16(x) for x in bits), torch.from_numpy(blocks).cuda(), block, 0.125)
    A.astro_last_device_status()
    check_forward(o, lse, ref, o_abs, qf, 0.125, D, "short lists")


@pytest.mark.parametrize("D", [64, 128])
def test_single_tile_units_with_and_without_queries_in_every_quarter(D):
    """A CTA meets full and nearly empty query blocks in turn, one key tile each: what one unit leaves for the epilogue must
    not be overwritten by the unit after the next."""
    import torch
    from paper_2603_17051_b200 import binding as A
    B, H, n_q, n_kc, block = 8, 40, 128 * 2 + 5, 96, 32
    bits = [synth.normal_bf16(60 + i, (B, n, H, D)) for i, n in enumerate((n_q, n_kc, n_kc))]
    qf, kf, vf = (bf16_bits_to_f64(x) for x in bits)
    ranges = orc.key_blocks(0, 1, n_kc, block)
    blocks = lists(np.random.default_rng(8), B, H, 3, len(ranges), 3, "odd")
    none = np.zeros((1, 0, H, D))
    scale = D ** -0.5
    ref, o_abs = reference(qf, kf, vf, none, none, blocks, ranges, scale, 0)
    q, k, v = (dev_bf16(x) for x in bits)
    tb = torch.from_numpy(blocks).cuda()
    first = None
    for _ in range(5):
        o, lse = A.astro_sparse_attn_fwd(None, q, k, v, tb, block, scale)
        A.astro_last_device_status()
        if first is None:
            first = o.clone()
            check_forward(o, lse, ref, o_abs, qf, scale, D, "single tiles")
        assert torch.equal(o, first)


def test_every_block_chosen_is_dense_attention():
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, _, _, frames = ring(A, 1, 2, 128, 130, 1, 5, 2, 5, 77)
    q, k, v = (dev_bf16(synth.normal_bf16(80 + i, (2, 390, 2, 128))) for i in range(3))
    n = sum(A.astro_block_count(cache, 390, 64))
    every = torch.arange(n, dtype=torch.int32, device="cuda").expand(2, 2, 4, n).contiguous()
    o, lse = A.astro_sparse_attn_fwd(cache, q, k, v, every, 64, 0.09)
    od, ld = A.astro_chunk_attn_fwd(cache, q, k, v, 0.09)
    assert (o.float() - od.float()).abs().max() <= 1e-2 and (lse - ld).abs().max() <= 1e-4


def test_refusals_of_the_forward():
    import torch
    from paper_2603_17051_b200 import binding as A
    q = torch.zeros(1, 200, 2, 64, device="cuda").bfloat16()
    blocks = torch.zeros(1, 2, 2, 3, dtype=torch.int32, device="cuda")
    run = lambda **kw: A.astro_sparse_attn_fwd(**{**dict(cache=None, q=q, k_chunk=q, v_chunk=q, blocks=blocks, block_tokens=64, scale=0.1), **kw})  # noqa: E731
    run()
    for bad in (dict(blocks=blocks.long()), dict(blocks=blocks[:, :, :1].contiguous()), dict(blocks=blocks.cpu()), dict(q=q.half()),
                dict(k_chunk=q[:, :100].contiguous()), dict(o=q[:, :100].contiguous()), dict(v_chunk=q.transpose(0, 1))):
        with pytest.raises(ValueError):
            run(**bad)
    for bad, status in ((dict(block_tokens=20), 2), (dict(block_tokens=256), 2), (dict(scale=-1.0), 2), (dict(k_chunk=None, v_chunk=None), 2),
                        (dict(v_chunk=None), 1)):
        with pytest.raises(A.AstroError) as e:
            run(**bad)
        assert e.value.status == status
    few = torch.zeros(1, 2, 1, 40, dtype=torch.int32, device="cuda")
    need = A.astro_sparse_attn_fwd_workspace_bytes(1, 2, 64, 5, 40, 64)
    assert need > 0 and A.astro_sparse_attn_fwd_workspace_bytes(1, 2, 64, 1, 40, 64) == 0
    with pytest.raises(A.AstroError) as e:
        run(q=q[:, :5].contiguous(), blocks=few, workspace=torch.empty(need - 4, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 4


@pytest.mark.parametrize("kind", ["ascending", "plain", "odd"])
@pytest.mark.parametrize("Bc,B,H,D,T,S,L,evicted,held,n_q,n_kc,block,n_select", SHAPES)
def test_backward_matches_the_oracle_and_repeats_itself(Bc, B, H, D, T, S, L, evicted, held, n_q, n_kc, block, n_select, kind):
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, kx, vx, frames = ring(A, Bc, H, D, T, S, L, evicted, held, 2500, poison=True)
    bits = [synth.normal_bf16(2900 + i, (B, n, H, D)) for i, n in enumerate((n_q, max(1, n_kc), max(1, n_kc), n_q))]
    q, k, v, d_o = (dev_bf16(x) for x in bits)
    qf, kf, vf, gf = (bf16_bits_to_f64(x) for x in bits)
    k, v = (k, v) if n_kc else (None, None)
    ranges = orc.key_blocks(frames, T, n_kc, block)
    blocks = lists(np.random.default_rng(n_q + block), B, H, -(-n_q // 128), len(ranges), n_select, kind)
    scale = D ** -0.5
    ref, _ = reference(qf, kf[:, :n_kc], vf[:, :n_kc], kx, vx, blocks, ranges, scale, frames * T, gf)
    tb = torch.from_numpy(blocks).cuda()
    o, lse = A.astro_sparse_attn_fwd(cache, q, k, v, tb, block, scale)
    got = A.astro_sparse_attn_bwd(cache, q, k, v, tb, block, o, lse, d_o, scale)
    A.astro_last_device_status()
    check_grads(got, ref[2:] if n_kc else (ref[2],), tag=kind)
    empty = np.moveaxis(np.isneginf(ref[1]), 1, 2)
    assert not f64(got[0])[empty].any()
    if n_kc:                                              # a chunk block that no list names
        for b in range(B):
            for h in range(H):
                for j, (first, end) in enumerate(ranges):
                    if first >= frames * T and not (blocks[b, h] == j).any():
                        rows = slice(first - frames * T, end - frames * T)
                        assert not f64(got[1])[b, rows, h].any() and not f64(got[2])[b, rows, h].any()
    again = A.astro_sparse_attn_bwd(cache, q, k, v, tb, block, o, lse, d_o, scale)
    assert all(x is None or torch.equal(x, y) for x, y in zip(got, again))


def test_gradients_agree_with_differences_of_the_forward():
    """Directional derivatives of sum(dO * O) from the kernel's forward itself."""
    import torch
    from paper_2603_17051_b200 import binding as A
    g = torch.Generator().manual_seed(31)
    B, H, D, n_q, n_kc, block = 1, 2, 64, 200, 192, 64
    q, k, v, d_o = ((torch.randn((B, n, H, D), generator=g) * 0.5).bfloat16().cuda() for n in (n_q, n_kc, n_kc, n_q))
    tb = torch.tensor([[0, 2], [1, 2]], dtype=torch.int32, device="cuda").expand(B, H, 2, 2).contiguous()
    run = lambda q, k, v: A.astro_sparse_attn_fwd(None, q, k, v, tb, block, 0.125)  # noqa: E731
    o, lse = run(q, k, v)
    grads = A.astro_sparse_attn_bwd(None, q, k, v, tb, block, o, lse, d_o, 0.125)
    step = 0.25
    for i, x in enumerate((q, k, v)):
        # along the gradient itself, so that the slope is far above what bf16 outputs round away
        d = (grads[i].float() / grads[i].float().norm() * x.float().norm()).bfloat16()
        ins = [q, k, v]
        sides = []
        for sign in (1, -1):
            moved = list(ins)
            moved[i] = (x.float() + sign * step * d.float()).bfloat16()
            sides.append((run(*moved)[0].double() * d_o.double()).sum().item())
        true_step = ((x.float() + step * d.float()).bfloat16().double() - (x.float() - step * d.float()).bfloat16().double())
        slope, want = sides[0] - sides[1], (true_step * grads[i].double()).sum().item()
        assert abs(slope - want) <= 0.05 * abs(want), (i, slope, want)


def test_a_stream_a_captured_graph_and_two_calls_at_once():
    import torch
    from paper_2603_17051_b200 import binding as A
    cache, _, _, _ = ring(A, 1, 2, 64, 50, 0, 5, 2, 4, 301)
    q, k, v, d_o = (dev_bf16(synth.normal_bf16(310 + i, (2, 150, 2, 64))) for i in range(4))
    n = sum(A.astro_block_count(cache, 150, 32))
    sel = A.astro_block_select(cache, A.astro_block_pool(cache, 32), q, k, 32, 6)

    def whole(stream=None):
        o, lse = A.astro_sparse_attn_fwd(cache, q, k, v, sel, 32, 0.125, stream=stream)
        return (o, lse) + A.astro_sparse_attn_bwd(cache, q, k, v, sel, 32, o, lse, d_o, 0.125, stream=stream)

    want = whole()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got_a, got_b = whole(a), whole(b)                     # two at once, each with scratch of its own
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(want, got_a, got_b))
    graph = torch.cuda.CUDAGraph()
    a.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=a):
        out = whole()
    for x in (q, k, v, d_o):
        x.copy_(x.flip(1))
    sel.copy_((sel + 1) % n)
    want = whole()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, out))


def test_the_operators_together_in_a_streaming_rollout():
    """Positions, append, pooled means, choice, attention and update over several chunks, then a fork of the cache: every
    chunk's results against the oracle fed with the same (rotated) keys."""
    import torch
    from oracle import rope as rope_orc
    from paper_2603_17051_b200 import binding as A
    B, H, D, T, S, L, c, block, n_select = 2, 2, 64, 24, 1, 5, 2, 24, 4
    rope = A.astro_rope_create(D, D, "interleaved", (12, 10, 10))
    f, axis = rope_orc.frequencies((12, 10, 10), 10000.0)
    cache = A.astro_kvcache_create(B, H, D, T, S, L)
    pooled = torch.zeros((B, H, S + L, 1, D), device="cuda")
    held_k, held_v = [], []
    for chunk in range(5):
        M = c * T
        q, k, v, d_o = (dev_bf16(synth.normal_bf16(4000 + 10 * chunk + i, (B, M, H, D))) for i in range(4))
        t = torch.arange(M)
        pos = torch.stack([chunk * c + t // T, t % T // 6, t % 6], -1).int()[None].contiguous().cuda()
        qr, kr = A.astro_rope_apply(rope, q, k, pos)
        want = rope_orc.rotate(f64(q), pos.cpu().numpy(), f, axis, "interleaved")
        assert np.abs(f64(qr) - want).max() <= HALF * np.abs(want).max() * 1.01
        sink, win, _ = A.astro_kvcache_query(cache)
        if sink + win > S + L - c:
            over = sink + win - (S + L - c)
            A.astro_kvcache_evict(cache, over)
            del held_k[S:S + over], held_v[S:S + over]
        sel = A.astro_block_select(cache, pooled, qr, kr, block, n_select, keep=A.KEEP_CHUNK)
        o, lse = A.astro_sparse_attn_fwd(cache, qr, kr, v, sel, block, D ** -0.5)
        grads = A.astro_sparse_attn_bwd(cache, qr, kr, v, sel, block, o, lse, d_o, D ** -0.5)
        dq, dk = A.astro_rope_apply(rope, grads[0], grads[1], pos, inverse=True)
        A.astro_last_device_status()
        frames = len(held_k)
        kx, vx = (np.concatenate(x, 1) if x else np.zeros((B, 0, H, D)) for x in (held_k, held_v))
        ranges = orc.key_blocks(frames, T, M, block)
        kept = set(range(frames, len(ranges)))
        lists_ = np.zeros(tuple(sel.shape), np.int64)
        for b in range(B):
            for h in range(H):
                lists_[b, h] = orc.select(f64(qr)[b, :, h], np.concatenate([kx[b, :, h], f64(kr)[b, :, h]]), ranges, n_select, kept)
        assert np.array_equal(sel.cpu().numpy(), lists_)
        ref, o_abs = reference(f64(qr), f64(kr), f64(v), kx, vx, lists_, ranges, D ** -0.5, frames * T, f64(d_o))
        check_forward(o, lse, ref, o_abs, f64(qr), D ** -0.5, D, "chunk %d" % chunk)
        check_grads(grads, ref[2:], tag="chunk %d" % chunk)
        back = rope_orc.rotate(ref[2], pos.cpu().numpy(), f, axis, "interleaved", inverse=True)
        assert np.linalg.norm(f64(dq) - back) <= 2e-2 * np.linalg.norm(back) and dk.shape == k.shape
        A.astro_kvcache_append(cache, kr, v, c)
        sink, win, _ = A.astro_kvcache_query(cache)
        A.astro_block_pool(cache, block, first_frame=sink + win - c, n_frames=c, pooled=pooled)
        for i in range(c):
            held_k.append(f64(kr)[:, i * T:(i + 1) * T]); held_v.append(f64(v)[:, i * T:(i + 1) * T])
    # sample 1 goes on twice
    twin = A.astro_kvcache_create(B, H, D, T, S, L)
    A.astro_kvcache_fork(twin, cache, parents=torch.tensor([1, 1], dtype=torch.int32, device="cuda"))
    q2 = qr[1:].expand(2, -1, -1, -1).contiguous()
    p2 = A.astro_block_pool(twin, block)
    s2 = A.astro_block_select(twin, p2, q2, None, block, n_select)
    o2, _ = A.astro_sparse_attn_fwd(twin, q2, None, None, s2, block, D ** -0.5)
    assert torch.equal(s2[0], s2[1]) and torch.equal(o2[0], o2[1])


def test_refusals_of_the_backward():
    import torch
    from paper_2603_17051_b200 import binding as A
    q = torch.zeros(1, 200, 2, 64, device="cuda").bfloat16()
    blocks = torch.zeros(1, 2, 2, 3, dtype=torch.int32, device="cuda")
    o, lse = A.astro_sparse_attn_fwd(None, q, q, q, blocks, 64, 0.1)
    run = lambda **kw: A.astro_sparse_attn_bwd(**{**dict(cache=None, q=q, k_chunk=q, v_chunk=q, blocks=blocks, block_tokens=64, o=o, lse=lse, d_o=q, scale=0.1), **kw})  # noqa: E731
    run()
    for bad in (dict(lse=lse.double()), dict(lse=lse[:, :, :100].contiguous()), dict(d_o=q[:, :100].contiguous()), dict(o=o.float()),
                dict(dk_chunk=q[:, :100].contiguous()), dict(d_o=q.cpu())):
        with pytest.raises(ValueError):
            run(**bad)
    for bad, status in ((dict(block_tokens=4), 2), (dict(scale=float("nan")), 2), (dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")), 4)):
        with pytest.raises(A.AstroError) as e:
            run(**bad)
        assert e.value.status == status
