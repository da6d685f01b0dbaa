"""Attention over a cache in 8 bits on the GPU, against attention in 64 bits over what the cache holds (attn_bounds.py)."""
import pytest

from attn_bounds import check, head

pytestmark = pytest.mark.gpu


def modules():
    import torch
    from paper_2603_17051_b200 import binding as A
    return torch, A


def filled(torch, A, Bc, H, D, T, S, L, held, head_at, seed, spread=0.5):
    """A cache of `held` frames whose window starts at ring slot head_at."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = A.astro_kvcache8_create(Bc, H, D, T, S, L)
    for s in (cache.k_storage, cache.v_storage):
        s.fill_(0x7f)                                        # NaN in every row that is not written
    sink = min(S, held)
    size = torch.exp(spread * torch.randn(2, H, D, generator=g, device="cuda"))
    k, v = ((torch.randn(Bc, held * T, H, D, generator=g, device="cuda") * size[i]).bfloat16() for i in range(2))
    cut = lambda x, a, b: x[:, a * T:b * T].contiguous()  # noqa: E731
    if sink:
        A.astro_kvcache8_append(cache, cut(k, 0, sink), cut(v, 0, sink), sink)
    if held > sink:
        A.astro_kvcache_set_state(cache, A.KVCacheState(sink, head_at, 1, sink + 1))    # an empty window starts at 0: hold one,
        A.astro_kvcache_evict(cache, 0)
        if held - sink > 1:
            A.astro_kvcache8_append(cache, cut(k, sink + 1, held), cut(v, sink + 1, held), held - sink - 1)
        A.astro_kvcache_set_state(cache, A.KVCacheState(sink, (head_at - 1) % L, 1, sink + 1))  # and write it last
        if L > 1:
            A.astro_kvcache8_append(cache, cut(k, sink, sink + 1), cut(v, sink, sink + 1), 1)
        else:
            A.astro_kvcache_set_state(cache, A.KVCacheState(sink, 0, 0, sink))
            A.astro_kvcache8_append(cache, cut(k, sink, sink + 1), cut(v, sink, sink + 1), 1)
        A.astro_kvcache_set_state(cache, A.KVCacheState(sink, head_at, held - sink, held))
    return cache


def compare(torch, A, cache, q, kc, vc, scale, d_o=None, tag="", rows=None, heads=None):
    B, n_q, H, D = q.shape
    o, lse = A.astro_chunk_attn8_fwd(cache, q, kc, vc, scale)
    grads = None if d_o is None else A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, scale)
    A.astro_last_device_status()
    if cache is not None:
        k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
        n_ctx = k8.shape[1]
    else:
        n_ctx = 0
    for b in range(B):
        for h in range(H) if heads is None else heads:
            parts = []
            for x, y in ((k8 if n_ctx else None, kc), (v8 if n_ctx else None, vc)):
                got = ([x[b if x.shape[0] > 1 else 0, :, h]] if n_ctx else []) + ([] if y is None else [y[b, :, h].double()])
                parts.append(torch.cat(got))
            want = head(q[b, :, h].double(), *parts, scale, d_o=None if d_o is None else d_o[b, :, h].double())
            name = "%s sample %d head %d " % (tag, b, h)
            check(o[b, :, h], want["o"], name + "O")
            check(lse[b, h], want["lse"], name + "LSE")
            if d_o is not None:
                check(grads[0][b, :, h], want["dq"], name + "dQ")
                if kc is not None:
                    check(grads[1][b, :, h], tuple(x[n_ctx:] for x in want["dk"]), name + "dK")
                    check(grads[2][b, :, h], tuple(x[n_ctx:] for x in want["dv"]), name + "dV")
    return o, lse


def tensors(torch, B, n_q, n_kc, H, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda n: torch.randn(B, n, H, D, generator=g, device="cuda").bfloat16() if n else None  # noqa: E731
    return make(n_q), make(n_kc), make(n_kc), make(n_q)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [1, 2, 7, 8, 9, 16, 17, 63, 64, 65, 130, 1000])
def test_numbers_of_queries(D, n_q):
    torch, A = modules()
    cache = filled(torch, A, 2, 3, D, 37, 1, 6, 6, 4, n_q)
    q, kc, vc, d_o = tensors(torch, 2, n_q, 11, 3, D, n_q + 100)
    compare(torch, A, cache, q, kc, vc, D ** -0.5, d_o)


@pytest.mark.parametrize("D,H,n_q", [(64, 40, 100), (64, 40, 300), (128, 40, 300), (128, 20, 1500)])
def test_queries_on_both_sides_of_the_choice_between_the_kernels(D, H, n_q):
    torch, A = modules()
    cache = filled(torch, A, 1, H, D, 100, 1, 6, 7, 4, n_q)
    q, kc, vc, d_o = tensors(torch, 1, n_q, 50, H, D, n_q)
    compare(torch, A, cache, q, kc, vc, D ** -0.5, d_o, heads=(0, H - 1))


@pytest.mark.parametrize("n_q", [1, 12, 100])
@pytest.mark.parametrize("T,S,L,held,at", [(1, 0, 1, 1, 0), (1, 4, 600, 530, 590), (1, 4, 20, 3, 0), (15, 0, 1, 1, 0), (16, 1, 3, 4, 2), (17, 2, 5, 6, 3),
                                           (129, 0, 4, 3, 3), (500, 3, 3, 5, 1)])
@pytest.mark.parametrize("n_kc", [0, 1, 16, 45])
def test_lengths_and_places_of_the_context(n_q, T, S, L, held, at, n_kc):
    torch, A = modules()
    for Bc in (1, 2):
        cache = filled(torch, A, Bc, 2, 64, T, S, L, held, at, T + n_kc)
        q, kc, vc, d_o = tensors(torch, 2, n_q, n_kc, 2, 64, held)
        compare(torch, A, cache, q, kc, vc, 0.125, d_o if n_q > 1 else None, "cache batch %d" % Bc)


def test_without_a_context():
    torch, A = modules()
    empty = A.astro_kvcache8_create(1, 2, 128, 4, 1, 2)
    for n_q in (1, 20, 70):
        q, kc, vc, d_o = tensors(torch, 2, n_q, 33, 2, 128, n_q)
        o, lse = compare(torch, A, empty, q, kc, vc, 0.1, d_o)
        again = A.astro_chunk_attn8_fwd(None, q, kc, vc, 0.1)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
        compare(torch, A, None, q, kc, vc, 0.1, d_o)


@pytest.mark.parametrize("n_q", [1, 3, 40, 300])
def test_large_scores_and_large_values(n_q):
    """Scores of several hundred, rising along the keys; values and keys of very different sizes from row to row."""
    torch, A = modules()
    B, H, D, T, L = 1, 2, 128, 64, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = A.astro_kvcache8_create(B, H, D, T, 0, L)
    n = T * L
    ramp = torch.linspace(0.1, 4.0, n, device="cuda").view(1, n, 1, 1)
    size = torch.exp2(torch.randint(-40, 40, (B, n, H, 1), generator=g, device="cuda").float())
    k = (torch.randn(B, n, H, D, generator=g, device="cuda") * ramp).bfloat16()
    v = (torch.randn(B, n, H, D, generator=g, device="cuda") * size).bfloat16()
    A.astro_kvcache8_append(cache, k, v, L)
    q, kc, vc, _ = tensors(torch, B, n_q, 5, H, D, 4)
    compare(torch, A, cache, q * 3, kc, vc, 1.0)


@pytest.mark.parametrize("n_q", [1, 20, 100])
def test_nan_in_one_element_of_a_value_reaches_that_element_alone(n_q):
    torch, A = modules()
    cache = A.astro_kvcache8_create(1, 1, 64, 40, 0, 2)
    q, k, v, _ = tensors(torch, 1, max(n_q, 80), 80, 1, 64, 5)
    q = q[:, :n_q].contiguous()
    v[0, 41, 0, 7] = float("inf")
    A.astro_kvcache8_append(cache, k, v, 2)
    o, lse = A.astro_chunk_attn8_fwd(cache, q, None, None, 0.125)
    bad = o.isnan()
    assert bad[..., 7].all() and bad.sum() == n_q and lse.isfinite().all()


@pytest.mark.parametrize("shape", ["rollout", "update"])
def test_layer_size(shape):
    torch, A = modules()
    B, n_q, S, L, held = (4, 1, 3, 12, 12) if shape == "rollout" else (1, 4680, 3, 18, 18)
    cache = filled(torch, A, B, 12, 128, 1560, S, L, held, 1, 6)
    q, kc, vc, d_o = tensors(torch, B, n_q, n_q, 12, 128, 7)
    heads = range(12) if n_q == 1 else (0, 11)
    if n_q == 1:
        compare(torch, A, cache, q, kc, vc, 128 ** -0.5, heads=heads)
        return
    o, lse = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 128 ** -0.5)
    dense = A.astro_kvcache_create(1, 12, 128, 1560, S, L)
    A.astro_kvcache_append(dense, *A.astro_kvcache8_read(cache), held)
    want, want_lse = A.astro_chunk_attn_fwd(dense, q, kc, vc, 128 ** -0.5)     # the same rows in 16 bits, tiles cut elsewhere
    assert (o.float() - want.float()).abs().max() <= 2.0 ** -8 * 2 and (lse - want_lse).abs().max() <= 1e-5
    got, ref = (f(c, q, kc, vc, o, lse, d_o, 128 ** -0.5) for f, c in ((A.astro_chunk_attn8_bwd, cache), (A.astro_chunk_attn_bwd, dense)))
    for a, r in zip(got, ref):
        assert (a.float() - r.float()).norm() <= 2.0 ** -8 * r.float().norm()
    # dV is the same sum; in dK the fp32 sum delta runs in another order (2^-20 of its terms), which may turn single roundings of dS by a step
    assert torch.equal(got[2], ref[2])


def test_a_captured_call_and_one_on_another_stream():
    torch, A = modules()
    cache = filled(torch, A, 2, 2, 128, 50, 1, 4, 5, 2, 8)
    for n_q in (1, 9, 100):
        q, kc, vc, d_o = tensors(torch, 2, n_q, 7, 2, 128, 9)
        want = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.1)
        grads = A.astro_chunk_attn8_bwd(cache, q, kc, vc, *want, d_o, 0.1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.1, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            inside = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.1)
            inside_grads = A.astro_chunk_attn8_bwd(cache, q, kc, vc, *inside, d_o, 0.1)
        for x in (*inside, *inside_grads):
            x.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*want, *grads), (*inside, *inside_grads)))
        del graph


@pytest.mark.parametrize("n_q,n_kc", [(1, 1), (3, 0), (5, 5), (17, 20), (64, 64)])
@pytest.mark.parametrize("B", [2, 7, 33])
def test_queries_of_many_samples_over_one_prefix(n_q, n_kc, B):
    """They are rows of one list; a sample's chunk is its own, whatever the others' hold."""
    torch, A = modules()
    cache = filled(torch, A, 1, 2, 64, 1, 3, 400, 350, 100, B)
    q, kc, vc, _ = tensors(torch, B, n_q, n_kc, 2, 64, n_q + B)
    o, lse = compare(torch, A, cache, q, kc, vc, 0.125)
    if n_kc:
        kc, vc = kc.clone(), vc.clone()
        kc[0] = float("nan")
        vc[0] = float("inf")
        bad, bad_lse = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.125)
        assert bad[0].isnan().any() and torch.equal(bad[1:], o[1:]) and torch.equal(bad_lse[1:], lse[1:])


def test_sizes_of_queries_keys_and_weights_that_fp16_does_not_hold():
    """Queries of 2^-60 and 2^60, keys the other way round, one sample's scores far from another's."""
    torch, A = modules()
    g = torch.Generator(device="cuda").manual_seed(12)
    cache = A.astro_kvcache8_create(1, 2, 128, 100, 0, 2)
    up = torch.tensor([2.0 ** 60, 2.0 ** -60], device="cuda").view(1, 1, 2, 1)
    k = (torch.randn(1, 200, 2, 128, generator=g, device="cuda") * up).bfloat16()
    v = torch.randn(1, 200, 2, 128, generator=g, device="cuda").bfloat16()
    A.astro_kvcache8_append(cache, k, v, 2)
    for n_q in (1, 4, 9):
        q = (torch.randn(2, n_q, 2, 128, generator=g, device="cuda") / up).bfloat16()
        q[0, 0, 0, 5] = 0.0
        compare(torch, A, cache, q, None, None, 0.09)


def test_offsets_beyond_32_bits():
    """A cache of 2.4 million tokens of 2048 bytes."""
    torch, A = modules()
    H, D, L = 16, 128, 2400000
    cache = A.astro_kvcache8_create(1, H, D, 1, 0, L)
    n = 4000
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - n, 0, 0))
    A.astro_kvcache_set_state(cache, A.KVCacheState(0, L - n, 1, 1))
    g = torch.Generator(device="cuda").manual_seed(13)
    k, v = (torch.randn(1, 2 * n, H, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    A.astro_kvcache8_append(cache, k[:, 1:].contiguous(), v[:, 1:].contiguous(), 2 * n - 1)
    A.astro_kvcache_evict(cache, 1)                              # the slot that was never written
    for n_q in (2, 70):
        q, kc, vc, _ = tensors(torch, 1, n_q, 3, H, D, 14)
        compare(torch, A, cache, q, kc, vc, D ** -0.5, heads=(0, 15))


@pytest.mark.parametrize("n_ctx,n_kc", [(1, 0), (0, 1), (1, 1), (3, 0), (40, 24)])
def test_few_keys(n_ctx, n_kc):
    """One key alone has no gradient; over a few, dS can be far smaller than delta, which then comes from the weights."""
    torch, A = modules()
    for Bc in (1, 2):
        cache = A.astro_kvcache8_create(Bc, 4, 64, 1, 0, 64)
        g = torch.Generator(device="cuda").manual_seed(n_ctx)
        if n_ctx:
            A.astro_kvcache8_append(cache, *(torch.randn(Bc, n_ctx, 4, 64, generator=g, device="cuda").bfloat16() for _ in range(2)), n_ctx)
        q, kc, vc, d_o = tensors(torch, 2, 9, n_kc, 4, 64, n_kc)
        o, lse = compare(torch, A, cache, q, kc, vc, 0.5, d_o)
        dq, dk, dv = A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, 0.5)
        if n_ctx + n_kc == 1:
            assert not dq.any() and (not n_kc or not dk.any())
            continue
        k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
        for b in range(2):
            for h in range(4):
                kk, vv = (torch.cat([x[b if Bc > 1 else 0, :, h]] + ([y[b, :, h].double()] if n_kc else [])) for x, y in ((k8, kc), (v8, vc)))
                qq, gg = q[b, :, h].double(), d_o[b, :, h].double()
                p = torch.softmax(0.5 * qq @ kk.T, 1)
                dp = gg @ vv.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                size = 0.5 * (qq.abs() @ kk.abs().T).amax(1, keepdim=True)
                err = 2.0 ** -8 * ds.abs() + 2.0 ** -18 * (1 + size) * p * (gg.abs() @ vv.abs().T).amax(1, keepdim=True)
                want = 0.5 * ds @ kk
                check(dq[b, :, h], (want, 1.1 * (0.5 * err @ kk.abs() + 2.0 ** -8 * want.abs()) + 1e-7), "dQ")


def test_one_key_of_nan():
    torch, A = modules()
    q, kc, vc, d_o = tensors(torch, 1, 9, 1, 4, 64, 3)
    q[0, 4, 1] = float("nan")
    o, lse = A.astro_chunk_attn8_fwd(None, q, kc, vc, 0.5)
    dq, dk, dv = A.astro_chunk_attn8_bwd(None, q, kc, vc, o, lse, d_o, 0.5)
    bad = torch.zeros(9, 4, dtype=torch.bool, device="cuda")
    bad[4, 1] = True
    assert dq[0, bad].isnan().all() and not dq[0, ~bad].any()
    assert dk[0, 0, 1].isnan().all() and not dk[0, 0, [0, 2, 3]].any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Bc,B,n_q,held,n_kc", [(2, 2, 5, 3000, 5), (1, 3, 130, 2100, 200), (1, 1, 1, 8001, 0), (1, 1, 129, 0, 2500), (1, 2, 7, 1000, 1200)])
def test_backward_of_few_queries_over_many_keys(D, Bc, B, n_q, held, n_kc):
    """Here the keys of a query tile are divided among CTAs, in the middle of the context, at its ragged end, in the chunk."""
    torch, A = modules()
    cache = A.astro_kvcache8_create(Bc, 2, D, 1, 100, 9000)
    g = torch.Generator(device="cuda").manual_seed(held + D)
    if held:
        A.astro_kvcache8_append(cache, *(torch.randn(Bc, held, 2, D, generator=g, device="cuda").bfloat16() for _ in range(2)), held)
    q, kc, vc, d_o = tensors(torch, B, n_q, n_kc, 2, D, n_q + D)
    o, lse = compare(torch, A, cache, q, kc, vc, D ** -0.5, d_o)
    first = A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, D ** -0.5)
    again = A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, D ** -0.5)
    assert all(x is y or torch.equal(x, y) for x, y in zip(first, again))
    need = A.astro_chunk_attn8_bwd_workspace_bytes(cache, B, n_q, n_kc)
    with pytest.raises(A.AstroError):
        A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, D ** -0.5, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Bc,n_q,held,n_kc", [(1, 3, 324, 1), (2, 8, 3000, 70), (1, 1, 65, 0), (2, 5, 0, 600), (1, 7, 129, 130)])
def test_few_queries_of_which_one_key_has_nearly_all_the_weight(D, Bc, n_q, held, n_kc):
    """delta of few queries comes from the weights: the errors of dQ and dK are relative to dS (its rounding, the output's: 2^-8 of
    each term) beside fp32's, 2^-18 of a weight and its products, which counts the score's own size."""
    torch, A = modules()
    B, Hh, scale = 2, 3, 4.0 / D ** 0.5
    q, kc, vc, d_o = tensors(torch, B, n_q, n_kc, Hh, D, 3 * D + n_q)
    cache = A.astro_kvcache8_create(Bc, Hh, D, 1, 10, 4000)
    g = torch.Generator(device="cuda").manual_seed(held + D)
    if held:
        ck, cv = (torch.randn(Bc, held, Hh, D, generator=g, device="cuda").bfloat16() for _ in range(2))
        ck[:, held // 2] = (ck[:, held // 2].float() + 4 * q[:Bc, 0].float() / D ** 0.5 * 2).bfloat16()
        A.astro_kvcache8_append(cache, ck, cv, held)
        k8, v8 = (x.double() for x in A.astro_kvcache8_read(cache, dtype=torch.float32))
    else:
        kc[:, 7] = (kc[:, 7].float() + 8 * q[:, 0].float() / D ** 0.5).bfloat16()
        k8 = v8 = torch.zeros(Bc, 0, Hh, D, dtype=torch.float64, device="cuda")
    o, lse = A.astro_chunk_attn8_fwd(cache, q, kc, vc, scale)
    dq, dk, dv = A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, scale)
    A.astro_last_device_status()
    for b in range(B):
        for h in range(Hh):
            kk, vv = (torch.cat([x[b if Bc > 1 else 0, :, h]] + ([y[b, :, h].double()] if n_kc else [])) for x, y in ((k8, kc), (v8, vc)))
            qq, gg = q[b, :, h].double(), d_o[b, :, h].double()
            p = torch.softmax(scale * qq @ kk.T, 1)
            dp = gg @ vv.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            size = scale * (qq.abs() @ kk.abs().T).amax(1, keepdim=True)
            err = 2.0 ** -8 * ds.abs() + 2.0 ** -18 * (1 + size) * p * (gg.abs() @ vv.abs().T).amax(1, keepdim=True)
            want = scale * ds @ kk
            check(dq[b, :, h], (want, 1.1 * (scale * err @ kk.abs() + 2.0 ** -8 * want.abs()) + 1e-7), "dQ")
            if n_kc:
                err = err + 2.0 ** -13 * p * (dp - (p * dp).sum(1, keepdim=True)).abs()     # the polynomial exp2 of dK/dV: 7.6e-5
                want, err = (scale * (ds.T @ qq))[held:], (scale * (err.T @ qq.abs()))[held:]
                check(dk[b, :, h], (want, 1.1 * (err + 2.0 ** -8 * want.abs()) + 1e-7), "dK")


@pytest.mark.parametrize("n_q", [3, 100])
def test_a_captured_backward_of_few_queries(n_q):
    """Captured, replayed twice on new inputs, beside eager calls with a workspace of their own."""
    torch, A = modules()
    B, H, D, held, n_kc = 2, 3, 64, 1900, 40
    cache = A.astro_kvcache8_create(B, H, D, 1, 0, held)
    g = torch.Generator(device="cuda").manual_seed(n_q)
    A.astro_kvcache8_append(cache, *(torch.randn(B, held, H, D, generator=g, device="cuda").bfloat16() for _ in range(2)), held)
    q, kc, vc, d_o = tensors(torch, B, n_q, n_kc, H, D, n_q)
    o, lse = A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.2)
    need = A.astro_chunk_attn8_bwd_workspace_bytes(cache, B, n_q, n_kc)
    out = [torch.empty_like(q), torch.empty_like(kc), torch.empty_like(vc)]
    given = dict(zip(("dq", "dk_chunk", "dv_chunk"), out), workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, 0.2, **given)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, 0.2, **given)
    for seed in (5, 6):
        for x, new in zip((q, kc, vc, d_o), tensors(torch, B, n_q, n_kc, H, D, seed)):
            x.copy_(new)
        A.astro_chunk_attn8_fwd(cache, q, kc, vc, 0.2, o=o, lse=lse)
        graph.replay()
        eager = A.astro_chunk_attn8_bwd(cache, q, kc, vc, o, lse, d_o, 0.2)
        assert all(torch.equal(x, y) for x, y in zip(out, eager))
