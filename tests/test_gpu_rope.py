"""GPU parity of rotary positions against the fp64 oracle, forward and transposed."""
import numpy as np
import pytest

from oracle import rope as orc

pytestmark = pytest.mark.gpu

# half a step of the type (the one rounding of a result), relative to the rotated pair's length
HALF_STEP = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}
# fp32 arithmetic before that: the fraction of a turn is rounded to fp32 (2^-25 of a turn = 1.9e-7 rad), sine and cosine
# are within 2 steps, and two products and a sum add 2 more half steps each: below 1e-6 of the pair's length
ARITHMETIC = 1e-6


def make(B, n, H, D, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, n, H, D), generator=g).to(getattr(torch, dtype)).cuda()


def positions_for(B, n, axes, far, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-far, far, (B, n, axes), generator=g, dtype=torch.int32).cuda()


def check(got, x, pos, f, axis, layout, size, inverse, tag):
    ref = orc.rotate(x.double().cpu().numpy(), pos.cpu().numpy(), f, axis, layout, size, inverse)
    y = got.double().cpu().numpy()
    pairs = len(f)
    rot, rest = 2 * pairs, slice(2 * pairs, None)
    assert np.array_equal(y[..., rest], ref[..., rest]), tag + ": copied part"
    xs = x.double().cpu().numpy()[..., :rot]
    a, b = (xs[..., 0::2], xs[..., 1::2]) if layout == "interleaved" else (xs[..., :pairs], xs[..., pairs:])
    length = size * np.sqrt(a * a + b * b)
    length = np.stack([length, length], -1).reshape(xs.shape) if layout == "interleaved" else np.concatenate([length, length], -1)
    kind = str(got.dtype).replace("torch.", "")
    tiny = 2.0 ** -24 if kind == "float16" else 1e-37          # fp16 results below its normal range
    bound = HALF_STEP[kind] * np.abs(ref[..., :rot]) + (ARITHMETIC * (1 + HALF_STEP[kind])) * length + tiny
    err = np.abs(y[..., :rot] - ref[..., :rot])
    assert (err <= bound).all(), "%s: %.3e over its bound" % (tag, (err - bound).max())


@pytest.mark.parametrize("layout", ["interleaved", "halves"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("B,n,H,D,cut", [(1, 1, 1, 8, (4,)), (4, 1, 12, 128, (64,)), (2, 37, 3, 64, (16,)), (1, 130, 12, 128, (22, 21, 21)),
                                         (3, 5, 2, 96, (46,)), (2, 19, 5, 72, (3, 2)), (1, 9, 1, 256, (60, 68)), (2, 11, 40, 128, (1,)),
                                         (1, 700, 2, 128, (32, 16, 8, 4))])
def test_rotation_matches_the_oracle(B, n, H, D, cut, dtype, layout):
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(D, 2 * sum(cut), layout, cut)
    f, axis = orc.frequencies(cut, 10000.0)
    q, k = make(B, n, H, D, dtype, 1), make(B, n, H, D, dtype, 2)
    for pos_batch in {1, B}:
        pos = positions_for(pos_batch, n, len(cut), 2000, 3)
        for inverse in (False, True):
            qo, ko = A.astro_rope_apply(rope, q, k, pos, inverse=inverse)
            check(qo, q, pos, f, axis, layout, 1.0, inverse, "q")
            check(ko, k, pos, f, axis, layout, 1.0, inverse, "k")


@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("base", 8.0), ("ramp", 16.0)])
@pytest.mark.parametrize("scaled_axes", [None, (0,)])
def test_stretched_contexts_and_far_positions(scaling, factor, scaled_axes):
    from paper_2603_17051_b200 import binding as A
    cut = (22, 21, 21)
    rope = A.astro_rope_create(128, 128, "interleaved", cut, base=500000.0, scaling=scaling, factor=factor,
                               scaled_axes=scaled_axes, original_length=1000, ramp_low=2, ramp_high=20)
    f, axis = orc.frequencies(cut, 500000.0, scaling, factor, scaled_axes, 1000, 2, 20)
    got_f, size = A.astro_rope_frequencies(rope)
    assert np.allclose(got_f, f, rtol=1e-13) and abs(size - orc.magnitude(scaling, factor)) < 1e-14
    q = make(2, 33, 4, 128, "float32", 4)
    pos = positions_for(1, 33, 3, 2 ** 31 - 1, 5)
    pos[0, 0] = -2 ** 31
    pos[0, 1] = 2 ** 31 - 1
    # the angle's own error: the oracle's fp64 angle of up to 2^31 rad is 2^-22 rad off (half a step), the table's
    # frequency differs from the oracle's in its last bits (1e-13 relative at most, 2e-4 rad at 2^31): compare with the
    # library's frequencies
    qo, none = A.astro_rope_apply(rope, q, None, pos)
    assert none is None
    check(qo, q, pos, np.array(got_f), axis, "interleaved", size, False, scaling)


def test_gradient_is_the_transpose_and_agrees_with_differences():
    """<R x, g> = <x, R^T g> for the computed R and R^T, and the derivative of sum(g * R x) along a direction."""
    import torch
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(64, 48, "halves", (24,), scaling="ramp", factor=4.0, original_length=64)
    x, g, d = (make(2, 21, 3, 64, "float32", s) for s in (6, 7, 8))
    pos = positions_for(2, 21, 1, 500, 9)
    y, _ = A.astro_rope_apply(rope, x, None, pos)
    gx, _ = A.astro_rope_apply(rope, g, None, pos, inverse=True)
    left, right = (y.double() * g.double()).sum().item(), (x.double() * gx.double()).sum().item()
    scale = (y.double().norm() * g.double().norm()).item()
    assert abs(left - right) <= 2e-6 * scale          # two roundings of 2^-24 and ARITHMETIC, summed against the norms
    eps = 2.0 ** -4                                    # the map is linear: a wide step has no truncation error
    up, _ = A.astro_rope_apply(rope, x + eps * d, None, pos)
    down, _ = A.astro_rope_apply(rope, x - eps * d, None, pos)
    slope = ((up.double() - down.double()) / (2 * eps) * g.double()).sum().item()
    want = (gx.double() * d.double()).sum().item()
    assert abs(slope - want) <= 4e-6 / eps * scale


def test_strided_views_in_place_and_different_head_counts():
    import torch
    from paper_2603_17051_b200 import binding as A
    cut = (32, 32)
    f, axis = orc.frequencies(cut, 10000.0)
    rope = A.astro_rope_create(128, 128, "interleaved", cut)
    B, n = 2, 29
    qkv = torch.randn(B, n, 3, 6, 128, device="cuda").bfloat16()       # a fused projection's output
    before = qkv.clone()
    q, k = qkv[:, :, 0], qkv[:, :, 1]
    pos = positions_for(B, n, 2, 300, 11)
    qo, ko = A.astro_rope_apply(rope, q, k, pos)
    assert qo.is_contiguous() and torch.equal(qkv, before)
    check(qo, q, pos, f, axis, "interleaved", 1.0, False, "strided q")
    check(ko, k, pos, f, axis, "interleaved", 1.0, False, "strided k")
    A.astro_rope_apply(rope, q, k, pos, q_out=q, k_out=k)               # in place, inside the fused tensor
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, :, 2], before[:, :, 2])
    # heads first in memory, and fewer key heads
    qh = torch.randn(B, 6, n, 128, device="cuda").half().transpose(1, 2)
    kh = torch.randn(B, n, 2, 128, device="cuda").half()
    qo, ko = A.astro_rope_apply(rope, qh, kh, pos)
    check(qo, qh, pos, f, axis, "interleaved", 1.0, False, "head-major q")
    check(ko, kh, pos, f, axis, "interleaved", 1.0, False, "two key heads")
    # one row broadcast over the heads: stride 0 is fine for reading, not for writing
    row = torch.randn(B, n, 1, 128, device="cuda").expand(B, n, 4, 128)
    ro, _ = A.astro_rope_apply(rope, row, None, pos)
    check(ro, row, pos, f, axis, "interleaved", 1.0, False, "broadcast")
    with pytest.raises(A.AstroError) as e:
        A.astro_rope_apply(rope, ro, None, pos, q_out=torch.empty_like(ro[:, :, :1]).expand(B, n, 4, 128))
    assert e.value.status == 2


def test_stream_graph_and_empty_call():
    import torch
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(64, 64, "halves", (32,))
    f, axis = orc.frequencies((32,), 10000.0)
    q, k = make(1, 50, 2, 64, "bfloat16", 12), make(1, 50, 2, 64, "bfloat16", 13)
    pos = positions_for(1, 50, 1, 100, 14)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        A.astro_rope_apply(rope, q, k, pos, q_out=qo, k_out=ko)
    q.copy_(make(1, 50, 2, 64, "bfloat16", 15))
    pos += 7
    graph.replay()
    torch.cuda.synchronize()
    check(qo, q, pos, f, axis, "halves", 1.0, False, "replayed")
    e, _ = A.astro_rope_apply(rope, q[:, :0], None, pos[:, :0])
    assert e.shape == (1, 0, 2, 64)


def test_refusals_of_the_binding():
    import torch
    from paper_2603_17051_b200 import binding as A
    rope = A.astro_rope_create(64, 64, "halves", (32,))
    q = make(1, 4, 2, 64, "bfloat16", 1)
    pos = positions_for(1, 4, 1, 9, 2)
    for bad in (dict(positions=pos.long()), dict(positions=pos[:, :3].contiguous()), dict(positions=pos.cpu()),
                dict(q=q[..., :32]), dict(q=q.double()), dict(q=q.cpu()), dict(k=q.float()), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        args = dict(q=q, k=None, positions=pos)
        args.update(bad)
        with pytest.raises(ValueError):
            A.astro_rope_apply(rope, args["q"], args["k"], args["positions"])
