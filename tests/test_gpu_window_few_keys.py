"""Window attention's gradients of rows that see few keys, of which one has nearly all the weight: in short sequences, in short ones of
a padded batch, and everywhere where the window is narrow.  delta comes from the weights there, not from the rounded O."""
import pytest

from attn_bounds import check

pytestmark = pytest.mark.gpu


def modules():
    import torch
    from paper_2603_17051_b200 import binding as A
    return torch, A


def gradients(torch, q, k, v, d_o, scale, see):
    """dQ, dK and dV's parts of one head in 64 bits, each with a bound of which the part that comes from dS is relative to dS itself: its
    rounding and the output's, 2^-8 of each term, the polynomial exp2 of dK's weights (7.6e-5) beside fp32's products of D terms and
    exp2 of arguments up to |x| (2^-18 of the sizes that go into them)."""
    h8 = 2.0 ** -8
    x = torch.where(see, scale * (q @ k.T), -torch.inf)
    p = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)
    dp = d_o @ v.T
    ds = p * (dp - (p * dp).sum(1, keepdim=True))
    size = scale * (q.abs() @ k.abs().T) * see
    fp32 = 2.0 ** -18 * (1 + size.amax(1, keepdim=True)) * p * ((d_o.abs() @ v.abs().T) * see).amax(1, keepdim=True)
    err = h8 * ds.abs() + fp32
    dq = scale * (ds @ k)
    err_k = err + 2.0 ** -13 * ds.abs()
    return (dq, 1.1 * (scale * (err @ k.abs()) + h8 * dq.abs()) + 1e-7), (scale * (ds.T @ q), scale * (err_k.T @ q.abs()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,block,window,sink,lengths", [
    (500, 1, 2, 0, None), (500, 1, 3, 0, None), (500, 1, 2, 1, None), (1030, 1, 17, 5, None), (300, 1, 60, 4, None), (300, 1, 20, 44, (300, 129)),
    (700, 10, 30, 0, None), (257, 64, 64, 0, None), (640, 20, 40, 24, (640, 333)),
    (65, 1, None, 0, (64, 3)), (65, 1, None, 0, (2, 64)), (100, 1, None, 0, (3, 64)), (2000, 1, None, 0, (5, 33)), (400, 50, 100, 200, (64, 1)),
    (400, 1, 300, 100, (63, 64)), (400, 500, 600, 0, (17, 2)),
])
def test_few_keys_of_which_one_has_nearly_all_the_weight(D, n, block, window, sink, lengths):
    torch, A = modules()
    B, H, G, scale = 2, 4, 2, 4.0 / D ** 0.5
    g = torch.Generator(device="cuda").manual_seed(n + D)
    q, k, v, d_o = (torch.randn(B, n, h, D, generator=g, device="cuda").bfloat16() for h in (H, G, G, H))
    form = dict(block_tokens=block, window_tokens=window, sink_tokens=sink,
                lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    o, lse = A.astro_window_attn_fwd(q, k, v, scale, **form)
    grads = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, scale, **form)
    A.astro_last_device_status()
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    end = (i // block + 1) * block
    for b in range(B):
        length = n if lengths is None else lengths[b]
        see = (j < end) & ((j < sink) | (j >= end - (10 ** 9 if window is None else window))) & (j < length) & (i < length)
        assert see.sum(1).max() <= 64
        for kv in range(G):
            dk, dk_err = 0, 0
            for h in range(kv * (H // G), (kv + 1) * (H // G)):
                dq, part = gradients(torch, *(t[b, :, x].double() for t, x in ((q, h), (k, kv), (v, kv), (d_o, h))), scale, see)
                check(grads[0][b, :, h], dq, "dQ sample %d head %d" % (b, h))
                dk, dk_err = dk + part[0], dk_err + part[1]
            check(grads[1][b, :, kv], (dk, 1.1 * (dk_err + 2.0 ** -8 * dk.abs()) + 1e-7), "dK sample %d head %d" % (b, kv))


@pytest.mark.parametrize("n", [64, 65, 300])
def test_padding_does_not_change_a_samples_gradients(n):
    """A sample of 40 tokens alone and in padded batches: the same bits."""
    torch, A = modules()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, d_o = (torch.randn(1, 40, h, 64, generator=g, device="cuda").bfloat16() for h in (4, 2, 2, 4))
    scale = 0.5
    o, lse = A.astro_window_attn_fwd(q, k, v, scale)
    want = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, scale)
    wide = [torch.full((2, n, t.shape[2], 64), float("nan"), dtype=t.dtype, device="cuda") for t in (q, k, v, d_o)]
    for t, x in zip(wide, (q, k, v, d_o)):
        t[0] = 1.0
        t[1, :40] = x[0]
    lengths = torch.tensor([n, 40], dtype=torch.int32, device="cuda")
    o, lse = A.astro_window_attn_fwd(*wide[:3], scale, lengths=lengths)
    got = A.astro_window_attn_bwd(*wide[:3], o, lse, wide[3], scale, lengths=lengths)
    assert all(torch.equal(a[1, :40], b[0]) for a, b in zip(got, want))


def test_strided_rows_and_a_captured_call():
    """Narrow windows over strided inputs; lengths that change between replays decide anew what a sample is."""
    torch, A = modules()
    B, n, H, D = 2, 300, 3, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    packed = torch.randn(B, n, 3, H, D, generator=g, device="cuda").bfloat16()
    q, k, v = (packed[:, :, i] for i in range(3))
    d_o = torch.randn(B, n, H, D, generator=g, device="cuda").bfloat16()
    lengths = torch.tensor([300, 20], dtype=torch.int32, device="cuda")
    for form in (dict(window_tokens=5, sink_tokens=2), dict(lengths=lengths)):
        run = lambda *x: [*(f := A.astro_window_attn_fwd(*x, 0.3, **form)), *A.astro_window_attn_bwd(*x, *f, d_o, 0.3, **form)]  # noqa: E731, B023
        want = run(q.contiguous(), k.contiguous(), v.contiguous())
        assert all(torch.equal(a, b) for a, b in zip(run(q, k, v), want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            inside = run(q, k, v)
        for x in (64, 65, 0, 300, 7):
            lengths[0] = x
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(inside, run(q, k, v)))
        del graph
