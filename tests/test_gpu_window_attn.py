"""Attention of whole sequences with a sliding window and sinks on the GPU, against attention in 64 bits with the mask written
out (attn_bounds.py)."""
import pytest

from attn_bounds import check, head

pytestmark = pytest.mark.gpu


def modules():
    import torch
    from paper_2603_17051_b200 import binding as A
    return torch, A


def mask(torch, n, length, block, window, sink):
    i = torch.arange(n, device="cuda")[:, None]
    j = torch.arange(n, device="cuda")[None]
    end = (i // block + 1) * block
    return (j < end) & ((j < sink) | (j >= end - window)) & (j < length) & (i < length)


def tensors(torch, B, n, H, G, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(B, n, h, D, generator=g, device="cuda").bfloat16() for h in (H, G, G, H)]


def compare(torch, A, q, k, v, d_o, block, window, sink, lengths=None, scale=None, tag="", at=None):
    """Every head of every sample (or those in `at`) against the oracle; returns what the calls returned."""
    B, n, H, D = q.shape
    G = k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    form = dict(block_tokens=block, window_tokens=window, sink_tokens=sink,
                lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    o, lse = A.astro_window_attn_fwd(q, k, v, scale, **form)
    grads = None if d_o is None else A.astro_window_attn_bwd(q, k, v, o, lse, d_o, scale, **form)
    A.astro_last_device_status()
    reach = 10 ** 9 if window is None else window
    for b in range(B):
        length = n if lengths is None else min(max(lengths[b], 0), n)
        see = mask(torch, n, length, block, reach, sink)
        for kv in range(G):
            dk, dv = [], []
            for h in range(kv * (H // G), (kv + 1) * (H // G)):
                if at is not None and (b, h) not in at:
                    continue
                x = [t[b, :, i].double() for t, i in ((q, h), (k, kv), (v, kv))]
                for t in x:
                    t[length:] = 0.0                         # whatever the padding holds
                g = None
                if d_o is not None:
                    g = d_o[b, :, h].double()
                    g[length:] = 0.0
                want = head(*x, scale, see, g)
                name = "%s sample %d head %d " % (tag, b, h)
                check(o[b, :, h], want["o"], name + "O")
                check(lse[b, h], want["lse"], name + "LSE")
                if g is not None:
                    check(grads[0][b, :, h], want["dq"], name + "dQ")
                    dk.append(want["dk"])
                    dv.append(want["dv"])
            if dk and len(dk) == H // G:
                for got, parts, which in ((grads[1], dk, "dK"), (grads[2], dv, "dV")):
                    check(got[b, :, kv], tuple(sum(p[i] for p in parts) for i in range(2)), "%s sample %d shared head %d %s" % (tag, b, kv, which))
            if d_o is not None:
                assert not grads[0][b, length:].any() and not grads[1][b, length:].any() and not grads[2][b, length:].any()
        assert not o[b, length:].any() and (lse[b, :, length:] == -torch.inf).all()
    return o, lse, grads


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,block,window,sink", [(1, 1, None, 0), (2, 1, 1, 1), (127, 1, None, 0), (128, 1, 7, 3), (129, 3, 5, 0), (257, 100, 200, 100),
                                                 (300, 100, 100, 0), (640, 128, 256, 128), (385, 1, 128, 4), (500, 37, 150, 130), (700, 1, 300, 200),
                                                 (900, 450, 500, 20), (1000, 2000, 3000, 5), (777, 1, 40, 777)])
def test_masks(D, n, block, window, sink):
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 1, n, 2, 2, D, n)
    compare(torch, A, q, k, v, d_o, block, window, sink)


@pytest.mark.parametrize("H,G", [(1, 1), (4, 2), (6, 2), (12, 1)])
@pytest.mark.parametrize("lengths", [None, (300, 0, 129), (-5, 1000, 255), (1, 256, 384)])
def test_shared_heads_and_lengths(H, G, lengths):
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 3, 384, H, G, 64, H)
    compare(torch, A, q, k, v, d_o, 1, 200, 3, lengths)
    compare(torch, A, q, k, v, d_o, 150, 200, 10, lengths)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block,window,sink", [(1, 90, 5), (70, 140, 30), (400, 400, 0)])
def test_what_the_padding_holds_does_not_matter(D, block, window, sink):
    torch, A = modules()
    lengths = (200, 333)
    clean = tensors(torch, 2, 400, 4, 2, D, 1)
    for fill in (float("nan"), float("inf"), 3e38):
        dirty = [t.clone() for t in clean]
        for t in dirty:
            for b, length in enumerate(lengths):
                t[b, length:] = fill
        got = compare(torch, A, *dirty, block, window, sink, lengths)
        want = compare(torch, A, *clean, block, window, sink, lengths)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert all(torch.equal(x, y) for x, y in zip(got[2], want[2]))


def test_strided_inputs():
    torch, A = modules()
    B, n, H, D = 2, 300, 3, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    packed = torch.randn(B, n, 3, H, D, generator=g, device="cuda").bfloat16()
    q, k, v = (packed[:, :, i] for i in range(3))
    d_o = torch.randn(B, n, H, D, generator=g, device="cuda").bfloat16()
    got = compare(torch, A, q, k, v, d_o, 50, 100, 20)
    want = compare(torch, A, q.contiguous(), k.contiguous(), v.contiguous(), d_o, 50, 100, 20)
    assert all(torch.equal(x, y) for x, y in zip((*got[:2], *got[2]), (*want[:2], *want[2])))
    by_head = packed.permute(0, 3, 2, 1, 4).contiguous()     # [B, H, 3, n, D]
    q, k, v = (by_head[:, :, i].transpose(1, 2) for i in range(3))
    got = compare(torch, A, q, k, v, d_o, 50, 100, 20)
    assert all(torch.equal(x, y) for x, y in zip((*got[:2], *got[2]), (*want[:2], *want[2])))


@pytest.mark.parametrize("what", ["k", "v", "q", "d_o"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("block,window,sink", [(1, 100, 2), (100, 200, 50)])
def test_nan_and_infinity_reach_those_who_see_them_alone(what, value, block, window, sink):
    """One element of one token: results in which the token has no part are those of clean inputs, to their bounds."""
    torch, A = modules()
    n, D, at = 400, 64, 210
    q, k, v, d_o = tensors(torch, 1, n, 2, 2, D, 5)
    form = dict(block_tokens=block, window_tokens=window, sink_tokens=sink)
    clean_o, clean_lse = A.astro_window_attn_fwd(q, k, v, 0.125, **form)
    clean = A.astro_window_attn_bwd(q, k, v, clean_o, clean_lse, d_o, 0.125, **form)
    bad = {"q": q, "k": k, "v": v, "d_o": d_o}
    bad[what] = bad[what].clone()
    bad[what][0, at, 0, 9] = value
    o, lse = A.astro_window_attn_fwd(bad["q"], bad["k"], bad["v"], 0.125, **form)
    grads = A.astro_window_attn_bwd(bad["q"], bad["k"], bad["v"], o, lse, bad["d_o"], 0.125, **form)
    A.astro_last_device_status()
    see = mask(torch, n, n, block, window, sink)
    touched = see[:, at] if what in "kv" else torch.arange(n, device="cuda") == at        # queries whose row it is in
    if what == "d_o":
        assert torch.equal(o, clean_o) and torch.equal(lse, clean_lse)
    else:
        assert (o[0, ~touched, 0].float() - clean_o[0, ~touched, 0].float()).abs().max() <= 2.0 ** -6
        assert not o[0, touched, 0].isfinite().all() and torch.equal(o[:, :, 1], clean_o[:, :, 1])
        rows = o[0, touched, 0].isfinite()
        assert not (rows.all(-1) if what == "v" else rows.any(-1)).any() or value == float("inf") and what != "v"
    keys = see[touched].any(0)                               # tokens whose dK and dV such a query has a part in
    for got, want, free in ((grads[0], clean[0], ~touched), (grads[1], clean[1], ~keys), (grads[2], clean[2], ~keys)):
        assert got[0, free, 0].isfinite().all()
        assert (got[0, free, 0].float() - want[0, free, 0].float()).abs().max() <= 2.0 ** -5 * (1 + want[0, free, 0].float().abs().max())
        assert torch.equal(got[:, :, 1], want[:, :, 1])


@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_leave_the_range_of_one_reference(D):
    """Later and earlier keys far above the diagonal tile's: the row sums overflow any reference taken there."""
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 1, 700, 2, 1, D, 6)
    k[:, 20] *= 60
    k[:, 333] *= 40
    q = q * 4
    compare(torch, A, q, k, v, d_o, 300, 600, 30, scale=0.25)


def test_the_second_pass_alone():
    torch, A = modules()
    try:
        A.astro_debug_forward_mode(A.FWD_MODE_SAFE_ONLY)
        for D in (64, 128):
            q, k, v, _ = tensors(torch, 2, 300, 4, 2, D, 7)
            compare(torch, A, q, k, v, None, 70, 100, 20, (300, 131))
            compare(torch, A, q, k, v, None, 1, 60, 0)
    finally:
        A.astro_debug_forward_mode(A.FWD_MODE_NORMAL)


def test_more_units_than_multiprocessors_and_repeated_calls():
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 3, 1100, 40, 20, 64, 8)    # 1080 units of 1 to 9 tiles
    first = compare(torch, A, q, k, v, d_o, 1, None, 0, at={(0, 0), (0, 1), (2, 38), (2, 39)})
    for _ in range(3):
        o, lse = A.astro_window_attn_fwd(q, k, v, 0.125)
        grads = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, 0.125)
        assert all(torch.equal(x, y) for x, y in zip((*first[:2], *first[2]), (o, lse, *grads)))


def test_the_same_as_a_stream_through_a_cache():
    """Blocks of a sequence at once, and one after the other through a rolling cache with sinks, in 16 and in 8 bits."""
    torch, A = modules()
    B, H, D, T, c, S, L, chunks = 2, 2, 128, 50, 2, 1, 5, 6
    n = chunks * c * T
    q, k, v, _ = tensors(torch, B, n, H, H, D, 9)
    for create, attend in ((A.astro_kvcache_create, A.astro_chunk_attn_fwd), (A.astro_kvcache8_create, A.astro_chunk_attn8_fwd)):
        cache = create(B, H, D, T, S, L)
        if cache.bits == 8:                                  # its rows are what 8 bits hold of them, a chunk's own included
            whole = A.astro_kvcache8_create(B, H, D, T, 0, chunks * c)
            A.astro_kvcache8_append(whole, k, v, chunks * c)
            kk, vv = A.astro_kvcache8_read(whole)
        else:
            kk, vv = k, v
        o, lse = A.astro_window_attn_fwd(q, kk, vv, 0.1, block_tokens=c * T, window_tokens=L * T, sink_tokens=S * T)
        for x in range(chunks):
            sink, win, _ = A.astro_kvcache_query(cache)
            if sink + win > S + L - c:
                A.astro_kvcache_evict(cache, sink + win - (S + L - c))
            part = slice(x * c * T, (x + 1) * c * T)
            cut = lambda t: t[:, part].contiguous()  # noqa: E731
            got, got_lse = attend(cache, cut(q), cut(kk), cut(vv), 0.1)
            assert (got.float() - o[:, part].float()).abs().max() <= 2.0 ** -7 * 2
            assert (got_lse - lse[:, :, part]).abs().max() <= 1e-5
            A.astro_kvcache_append(cache, cut(kk), cut(vv), c)


def test_layer_size():
    torch, A = modules()
    n, block, window, sink = 32760, 4680, 18720, 4680
    q, k, v, d_o = tensors(torch, 1, n, 12, 12, 128, 10)
    form = dict(block_tokens=block, window_tokens=window, sink_tokens=sink)
    o, lse = A.astro_window_attn_fwd(q, k, v, 128 ** -0.5, **form)
    grads = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, 128 ** -0.5, **form)
    A.astro_last_device_status()
    h = 7
    rows = torch.cat([torch.arange(0, 40), torch.arange(4600, 4760), torch.arange(23390, 23410), torch.arange(32700, 32760)]).cuda()
    x = [t[0, :, h].double() for t in (q, k, v)]
    end = (rows[:, None] // block + 1) * block
    j = torch.arange(n, device="cuda")[None]
    see = (j < end) & ((j < sink) | (j >= end - window))
    want = head(x[0][rows], x[1], x[2], 128 ** -0.5, see, d_o[0, rows, h].double())
    check(o[0, rows, h], want["o"], "O")
    check(lse[0, h, rows], want["lse"], "LSE")
    check(grads[0][0, rows, h], want["dq"], "dQ")
    total = [torch.zeros(n, 128, dtype=torch.float64, device="cuda") for _ in range(4)]
    for i in range(0, n, 2340):
        see = mask(torch, n, n, block, window, sink)[i:i + 2340] if i == 0 else None
        r = torch.arange(i, i + 2340, device="cuda")[:, None]
        end = (r // block + 1) * block
        see = (j < end) & ((j < sink) | (j >= end - window))
        part = head(x[0][i:i + 2340], x[1], x[2], 128 ** -0.5, see, d_o[0, i:i + 2340, h].double())
        for t, p in zip(total, (*part["dk"], *part["dv"])):
            t += p
    check(grads[1][0, :, h], (total[0], total[1]), "dK")
    check(grads[2][0, :, h], (total[2], total[3]), "dV")


def test_a_captured_call_one_on_another_stream_and_an_empty_one():
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 2, 333, 4, 2, 128, 11)
    lengths = torch.tensor([333, 100], dtype=torch.int32, device="cuda")
    form = dict(block_tokens=1, window_tokens=90, sink_tokens=4, lengths=lengths)
    want = A.astro_window_attn_fwd(q, k, v, 0.1, **form)
    grads = A.astro_window_attn_bwd(q, k, v, *want, d_o, 0.1, **form)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = A.astro_window_attn_fwd(q, k, v, 0.1, stream=side, **form)
    got_grads = A.astro_window_attn_bwd(q, k, v, *got, d_o, 0.1, stream=side, **form)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*want, *grads), (*got, *got_grads)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = A.astro_window_attn_fwd(q, k, v, 0.1, **form)
        inside_grads = A.astro_window_attn_bwd(q, k, v, *inside, d_o, 0.1, **form)
    for shift in (100, 57):                                  # lengths are read when the graph runs
        lengths[1] = shift
        want = A.astro_window_attn_fwd(q, k, v, 0.1, **form)
        grads = A.astro_window_attn_bwd(q, k, v, *want, d_o, 0.1, **form)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*want, *grads), (*inside, *inside_grads)))
    del graph
    none = q[:, :0].contiguous()
    o, lse = A.astro_window_attn_fwd(none, k[:, :0].contiguous(), v[:, :0].contiguous(), 0.1)
    assert o.shape == (2, 0, 4, 128) and lse.shape == (2, 4, 0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths", [None, (4200,), (900,), (0,), (4195,)])
def test_sinks_that_many_queries_of_many_heads_see(D, lengths):
    """The sinks' key tiles are divided among CTAs and joined."""
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 1, 4200, 12, 1, D, 15)
    compare(torch, A, q, k, v, d_o, 1, 256, 100, lengths)


def test_nan_in_a_divided_key_tile():
    """In a query that the sinks' keys see, and in one that a key of the same tile does not see."""
    torch, A = modules()
    n, D = 4200, 64
    q, k, v, d_o = tensors(torch, 1, n, 8, 1, D, 16)
    form = dict(block_tokens=1, window_tokens=256, sink_tokens=40)
    o, lse = A.astro_window_attn_fwd(q, k, v, 0.125, **form)
    d_o[0, 3000, 2, 5] = float("nan")
    _, dk, dv = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, 0.125, **form)
    A.astro_last_device_status()
    i = torch.arange(n, device="cuda")
    seen = (i < 40) | ((i > 3000 - 256) & (i <= 3000))
    assert dk[0, seen].isnan().any(-1).all() and dk[0, ~seen].isfinite().all()
    assert dv[0, seen][..., 5].isnan().all() and dv[0, ~seen].isfinite().all()


def test_units_of_one_tile():
    """A CTA's look-ahead spans several units: short sequences, many of them, dead ones among them."""
    torch, A = modules()
    B, n, H = 500, 100, 3
    g = torch.Generator(device="cuda").manual_seed(17)
    q, k, v, d_o = tensors(torch, B, n, H, 1, 64, 17)
    lengths = torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lengths[::7] = 0
    at = {(b, h) for b in range(0, B, 17) for h in range(H)} | {(b, h) for b in (7, 499) for h in range(H)}
    compare(torch, A, q, k, v, d_o, 10, 30, 5, lengths.tolist(), at=at)


def test_everything_nan():
    """Sequences of which every result is NaN: every tile is done again, which ends as soon as a row is NaN throughout."""
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 1, 8192, 12, 4, 128, 18)
    form = dict(block_tokens=1, window_tokens=5000, sink_tokens=100)
    o, lse = A.astro_window_attn_fwd(q, k, v, 0.1, **form)
    nan = torch.full_like(q, float("nan"))
    bad, bad_lse = A.astro_window_attn_fwd(nan, k, v, 0.1, **form)
    grads = A.astro_window_attn_bwd(q, k, v, o, lse, nan, 0.1, **form)
    A.astro_last_device_status()
    assert bad.isnan().all() and bad_lse.isnan().all() and all(g.isnan().all() for g in grads)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2, 3, 5, 64])
def test_rows_of_which_one_key_has_nearly_all_the_weight(D, n):
    """dS is far smaller than delta there: in short sequences delta comes from the weights, not from the rounded O.  Then every
    error of dQ and dK is relative to dS itself: its rounding and the output's, 2^-8 of each term, beside fp32's."""
    torch, A = modules()
    q, k, v, d_o = tensors(torch, 3, n, 4, 2, D, 19)
    k[:, 0] = (k[:, 0].float() + 5 * q[:, :, :1].float().mean(1) / D ** 0.5).bfloat16()
    scale = 4.0 / D ** 0.5
    o, lse = A.astro_window_attn_fwd(q, k, v, scale)
    grads = A.astro_window_attn_bwd(q, k, v, o, lse, d_o, scale)
    see = mask(torch, n, n, 1, 10 ** 9, 0)
    h8 = 2.0 ** -8
    for b in range(3):
        for kv in range(2):
            dk, dk_err = 0, 0
            for h in (2 * kv, 2 * kv + 1):
                qq, kk, vv, gg = (t[b, :, i].double() for t, i in ((q, h), (k, kv), (v, kv), (d_o, h)))
                x = torch.where(see, scale * (qq @ kk.T), -torch.inf)
                p = torch.softmax(x, 1)
                dp = gg @ vv.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                # fp32: products of D terms and exp2 of arguments up to |x|, relative to the sizes that go into them
                size = scale * (qq.abs() @ kk.abs().T) * see
                fp32 = 2.0 ** -18 * (1 + size.amax(1, keepdim=True)) * p * (gg.abs() @ vv.abs().T).amax(1, keepdim=True)
                err = h8 * ds.abs() + fp32
                dq = scale * (ds @ kk)
                check(grads[0][b, :, h], (dq, 1.1 * (scale * (err @ kk.abs()) + h8 * dq.abs()) + 1e-7), "dQ")
                dk = dk + scale * (ds.T @ qq)
                dk_err = dk_err + scale * (err.T @ qq.abs())
            check(grads[1][b, :, kv], (dk, 1.1 * (dk_err + h8 * dk.abs()) + 1e-7), "dK")


def test_rows_of_one_key_have_no_gradient():
    torch, A = modules()
    for block, window, sink, lengths in ((1, 1, 0, None), (1, 50, 0, None), (1, 1, 1, (300, 1)), (10, 20, 3, (1, 1)), (1, None, 4, (1, 300))):
        q, k, v, d_o = tensors(torch, 2, 300, 4, 2, 64, 20)
        _, _, (dq, dk, dv) = compare(torch, A, q, k, v, d_o, block, window, sink, lengths)
        one = torch.stack([mask(torch, 300, 300 if lengths is None else n, block, 10 ** 9 if window is None else window, sink).sum(1) == 1
                           for n in (lengths or (300, 300))])
        assert not dq[one].any()
        if block == 1 and window == 1 and sink == 0:
            assert not dk.any() and torch.equal(dv, d_o.unflatten(2, (2, 2)).float().sum(3).bfloat16())
