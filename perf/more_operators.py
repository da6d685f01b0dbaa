"""More operators around the rolling cache that are measured: the cache held in 8 bits (writing, reading back, attention
over it, forward and backward) and attention of whole sequences with a sliding window and sinks (forward and backward).

`run` computes an operator in elementary torch operations, or, where `own` is true, through the package's binding.
`exact` computes the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LARGEST, LOWEST_EXP = 448.0, -124      # e4m3's largest number; the smallest exponent of a row's factor


# ------------------------------------------------------------------------------------------------ cases

def listed():
    dit = dict(heads=12, head_dim=128, tokens_per_frame=1560)
    return [
        # one new token for each of 4 samples into a cache of single tokens, and what it now stands for: latency
        dict(name="store_one_token", op="store", batch=4, heads=12, head_dim=128, tokens_per_frame=1, sink=4, window=4096, frames=1,
             dtype="bf16", out="bf16"),
        # the clean keys and values of a 3-frame chunk for 4 samples, written and read back for the next step
        dict(name="store_chunk", op="store", batch=4, sink=3, window=12, frames=3, dtype="bf16", out="bf16", **dit),
        # the whole full-length context read back
        dict(name="read_context", op="read", batch=1, sink=3, window=18, held=18, out="bf16", **dit),
        # its last frames in fp32, odd frame length
        dict(name="read_frames", op="read", batch=2, heads=2, head_dim=64, tokens_per_frame=99, sink=1, window=6, held=6, out="fp32"),
        # one query per sample over 12 frames of its own
        dict(name="attend8_one_query", op="attend", batch=4, shared=False, sink=3, window=12, held=12, n_q=1, n_kc=1, grad=False, **dit),
        # a few queries of every candidate of a group over one shared prefix of single tokens
        dict(name="attend8_few_queries", op="attend", batch=8, shared=True, heads=12, head_dim=64, tokens_per_frame=1, sink=4,
             window=8192, held=8001, n_q=5, n_kc=5, grad=False),
        # one denoising step of a chunk over the full context
        dict(name="attend8_chunk", op="attend", batch=1, shared=False, sink=3, window=18, held=18, n_q=4680, n_kc=4680, grad=False, **dit),
        # the clip-window update of a 2-sample batch
        dict(name="attend8_train", op="attend", batch=2, shared=False, sink=3, window=18, held=18, n_q=4680, n_kc=4680, grad=True, **dit),
        # short sequences of two lengths, forward
        dict(name="window_small", op="window", batch=2, n=300, heads=2, kv_heads=2, head_dim=64, block=100, window=200, sink=100,
             ragged=True, grad=False),
        # a prompt of a whole video, seven chunks of 3 frames, 3 sink frames, a window of 12
        dict(name="window_video", op="window", batch=1, n=32760, heads=12, kv_heads=12, head_dim=128, block=4680, window=18720, sink=4680,
             ragged=False, grad=False),
        # single tokens, keys and values shared by three heads each, sequences of different lengths: a training step
        dict(name="window_tokens", op="window", batch=2, n=4097, heads=12, kv_heads=4, head_dim=64, block=1, window=1024, sink=4,
             ragged=True, grad=True),
        # the video's training step
        dict(name="window_train", op="window", batch=1, n=32760, heads=12, kv_heads=12, head_dim=128, block=4680, window=18720, sink=4680,
             ragged=False, grad=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["store", "read", "attend", "attend", "attend", "window", "window", "window"])
    head_dim, heads = rng.choice([64, 128, 128]), rng.choice([1, 2, 12])
    if op == "window":
        n = _spread(rng, 1, 16384)
        block = rng.choice([1, 1, _spread(rng, 2, 256), 1560, _spread(rng, 100, 4680)])
        kv_heads = rng.choice([h for h in (1, 2, 4, 12) if heads % h == 0])
        return dict(op=op, batch=rng.randint(1, 2), n=n, heads=heads, kv_heads=kv_heads, head_dim=head_dim, block=block,
                    window=block + _spread(rng, 1, 16384), sink=rng.choice([0, 4, _spread(rng, 1, 4680)]), ragged=rng.random() < 0.5,
                    grad=rng.random() < 0.5)
    tokens = rng.choice([1, _spread(rng, 2, 1560), 1560])
    sink, window = (rng.randint(0, 3), rng.randint(4, 18)) if tokens > 1 else (rng.randint(0, 8), _spread(rng, 64, 16384))
    held = sink + rng.randint(1, window)
    size = dict(heads=heads, head_dim=head_dim, tokens_per_frame=tokens, sink=sink, window=window)
    if op == "store":
        return dict(op=op, batch=rng.randint(1, 4), frames=rng.randint(1, min(window, 3 if tokens > 1 else 4096)),
                    dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), out=rng.choice(["bf16", "fp32"]), **size)
    if op == "read":
        return dict(op=op, batch=rng.randint(1, 2), held=held, out=rng.choice(["bf16", "bf16", "fp16", "fp32"]), **size)
    n_kc = rng.choice([0, 1, _spread(rng, 2, 64), _spread(rng, 8, 4680)])
    n_q = rng.choice([1, max(1, n_kc), _spread(rng, 1, 64), _spread(rng, 1, 4680)])
    return dict(op=op, batch=rng.randint(1, 2), shared=rng.random() < 0.3, held=held, n_q=n_q, n_kc=n_kc, grad=rng.random() < 0.5, **size)


def _pairs(c):
    """Pairs of a query and a key that it sees, of full sequences."""
    block, reach, sink, n = c["block"], c["window"], c["sink"], c["n"]
    pairs = 0
    for b in range(-(-n // block)):
        hi, low = min(n, (b + 1) * block), max(0, (b + 1) * block - reach)
        pairs += (hi - b * block) * (hi - max(low, min(sink, hi)) + min(sink, hi))
    return pairs


def work(case):
    c = case
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    if c["op"] in ("store", "read"):
        rows = 2 * c["batch"] * c["heads"] * c["tokens_per_frame"] * (c["frames"] if c["op"] == "store" else c["held"])
        held = rows * (c["head_dim"] + 1)
        out = rows * c["head_dim"] * size[c["out"]]
        if c["op"] == "read":
            return {"bytes": held + out, "flops": 0}
        return {"bytes": rows * c["head_dim"] * size[c["dtype"]] + held + out, "flops": 0}
    B, H, D = c["batch"], c["heads"], c["head_dim"]
    if c["op"] == "window":
        pairs = (0.75 if c["ragged"] else 1.0) * B * H * _pairs(c)
        moved = 2 * B * c["n"] * D * (2 * H + 2 * c["kv_heads"]) + 4 * B * H * c["n"]
        if c["grad"]:
            moved += 2 * B * c["n"] * D * (2 * H + 2 * c["kv_heads"])
        return {"bytes": moved, "flops": (14.0 if c["grad"] else 4.0) * pairs * D}
    ctx, n_q, n_kc = c["held"] * c["tokens_per_frame"], c["n_q"], c["n_kc"]
    moved = 2 * (1 if c["shared"] else B) * ctx * H * (D + 1) + 4 * B * (n_q + n_kc) * H * D + 4 * B * H * n_q
    flops = 4.0 * B * H * n_q * (ctx + n_kc) * D
    if c["grad"]:
        moved += 4 * B * (n_q + n_kc) * H * D
        flops += 6.0 * B * H * n_q * (ctx + n_kc) * D + 4.0 * B * H * n_q * n_kc * D
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------------------------------------------------ inputs

def _row_factors(x):
    """e of every row [..., D] in 32 bits: the smallest whole number with max |x| <= 448 * 2^e over the row's finite values."""
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    part, whole = torch.frexp(top)                               # top = part * 2^whole, 448 = 0.875 * 2^9
    e = whole - 9 + (part > 0.875).int()
    return torch.where(top > 0, e, LOWEST_EXP).clamp(min=LOWEST_EXP)


def _power(e):
    """2^e in 32 bits, exactly."""
    return ((e + 127) << 23).view(torch.float32).unsqueeze(-1)


def _held_in_8(x):
    """(values in e4m3, e) of rows in any type: a row is held as its e and e4m3(x / 2^e), what is not finite as NaN."""
    x = x.float()
    e = _row_factors(x)
    return (x * _power(-e)).to(torch.float8_e4m3fn), e


def _stands_for(codes, e):
    return codes.float() * _power(e)


def _contents(case, normal, g, batch, frames):
    """Keys and values of `frames` frames [batch, tokens, H, D]: elements of a head differ in size, a few by much."""
    H, D, T = case["heads"], case["head_dim"], case["tokens_per_frame"]
    out = []
    for _ in range(2):
        size = torch.exp(0.5 * torch.randn(H, D, generator=g, device="cuda"))
        out.append((normal(batch, frames * T, H, D, dtype=torch.float32) * size).to(TYPES[case.get("dtype", "bf16")]))
    return out


def _frames_of(x, case, first, count):
    T = case["tokens_per_frame"]
    return x[:, first * T:(first + count) * T].contiguous()


def _filled(case, batch, k, v):
    """A cache that holds the frames of k and v; its window starts at the second slot of its ring where it has one, so a full
    ring wraps.  (A window that becomes empty starts at the first slot again.)"""
    from paper_2603_17051_b200 import binding as A
    sink, held = min(case["sink"], case["held"]), case["held"]
    cache = A.astro_kvcache8_create(batch, case["heads"], case["head_dim"], case["tokens_per_frame"], case["sink"], case["window"])

    def put(first, count):
        if count:
            A.astro_kvcache8_append(cache, _frames_of(k, case, first, count), _frames_of(v, case, first, count), count)

    put(0, sink)
    if held > sink and case["window"] > 1:
        beside = min(held - sink, case["window"] - 1)
        put(sink, 1)                                             # into the ring's first slot, and out again behind the next ones
        put(sink, beside)
        A.astro_kvcache_evict(cache, 1)
        put(sink + beside, held - sink - beside)
        state = A.astro_kvcache_get_state(cache)
        assert (state.sink_held, state.window_head, state.window_held) == (sink, 1, held - sink)
    else:
        put(sink, held - sink)
    return cache


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape, dtype=torch.bfloat16: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    s = dict(case)
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    if case["op"] == "window":
        s["q"] = normal(B, case["n"], H, D)
        s["k"], s["v"] = (normal(B, case["n"], case["kv_heads"], D) for _ in range(2))
        s["scale"] = D ** -0.5
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(case["n"] // 2, case["n"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        if case["grad"]:
            s["d_o"] = normal(B, case["n"], H, D)
        if own:
            from paper_2603_17051_b200 import binding as A
            if case["grad"]:
                need = A.astro_window_attn_bwd_workspace_bytes(B, H, case["n"], D)
                s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] == "store":
        s["k"], s["v"] = _contents(case, normal, g, B, case["frames"])
        if own:
            from paper_2603_17051_b200 import binding as A
            s["cache"] = A.astro_kvcache8_create(B, H, D, case["tokens_per_frame"], case["sink"], case["window"])
            # a frame in the middle of the ring is held already, where the new ones leave room for it; they go behind it
            s["beside"] = 1 if case["frames"] < case["window"] else 0
            A.astro_kvcache_set_state(s["cache"], A.KVCacheState(case["sink"], case["window"] // 2, s["beside"], case["sink"] + s["beside"]))
            s["before"] = A.astro_kvcache_get_state(s["cache"])
            assert s["before"].window_head == case["window"] // 2 * s["beside"]
        return s
    of = 1 if case.get("shared") else B
    k, v = _contents(case, normal, g, of, case["held"])
    if own:
        s["cache"] = _filled(case, of, k, v)
    else:
        s["k8"], s["v8"] = _held_in_8(k), _held_in_8(v)
    if case["op"] == "read":
        return s
    n_q, n_kc = case["n_q"], case["n_kc"]
    s["q"] = normal(B, n_q, H, D)
    s["k"], s["v"] = (normal(B, n_kc, H, D) if n_kc else None for _ in range(2))
    s["scale"] = D ** -0.5
    if case["grad"]:
        s["d_o"] = normal(B, n_q, H, D)
    if own:
        from paper_2603_17051_b200 import binding as A
        need = A.astro_chunk_attn8_fwd_workspace_bytes(s["cache"], B, n_q, n_kc)
        if case["grad"]:
            need = max(need, A.astro_chunk_attn8_bwd_workspace_bytes(s["cache"], B, n_q, n_kc))
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _softmax_rows(score):
    """(weights, LSE) of rows of scores, in place; a row without a key has weights of 0 and an LSE of -infinity."""
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    p /= torch.where(total > 0, total, 1.0)
    return p, lse


def _attended(s):
    B, H, D, n_q, n_kc = s["batch"], s["heads"], s["head_dim"], s["n_q"], s["n_kc"]
    k, v = (_stands_for(*s[x]).transpose(1, 2).expand(B, H, -1, D) for x in ("k8", "v8"))
    n_ctx = k.shape[2]
    if n_kc:
        k, v = (torch.cat([x, s[y].float().transpose(1, 2)], 2) for x, y in ((k, "k"), (v, "v")))
    back = lambda x: x.transpose(1, 2).to(torch.bfloat16)  # noqa: E731
    q, d_o = s["q"].float().transpose(1, 2), s["d_o"].float().transpose(1, 2) if s["grad"] else None
    outs, lses, dqs = [], [], []
    dk, dv = (torch.zeros(B, H, n_kc, D, device="cuda") for _ in range(2))
    for i in range(0, n_q, 1024):
        qi = q[:, :, i:i + 1024]
        p, lse = _softmax_rows((qi @ k.transpose(-1, -2)).mul_(s["scale"]))
        o = p @ v
        outs.append(o)
        lses.append(lse)
        if s["grad"]:
            gi = d_o[:, :, i:i + 1024]
            if n_kc:
                dv += p[..., n_ctx:].transpose(-1, -2) @ gi
            ds = (gi @ v.transpose(-1, -2)).sub_((gi * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
            dqs.append(ds @ k)
            if n_kc:
                dk += ds[..., n_ctx:].transpose(-1, -2) @ qi
    out = [back(torch.cat(outs, 2)).contiguous(), torch.cat(lses, 2).contiguous()]
    if s["grad"]:
        out.append(back(torch.cat(dqs, 2)).contiguous())
        if n_kc:
            out += [back(dk).contiguous(), back(dv).contiguous()]
    return out


def _windowed(s):
    """Row blocks of one choice of keys where a block of tokens is long, of 1024 rows with a mask where it is short."""
    B, n, H, G, D, block, sink = s["batch"], s["n"], s["heads"], s["kv_heads"], s["head_dim"], s["block"], s["sink"]
    k, v = (s[x].float().transpose(1, 2) for x in ("k", "v"))                   # [B, G, n, D]
    heads = lambda x: x.float().transpose(1, 2).unflatten(1, (G, H // G))  # noqa: E731
    q, d_o = heads(s["q"]), heads(s["d_o"]) if s["grad"] else None               # [B, G, heads of the group, n, D]
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), n, device="cuda")
    o, dq = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((B, G, H // G, n), -math.inf, device="cuda")
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    step = block if 512 <= block <= 8192 else 1024
    for i in range(0, n, step):
        rows = torch.arange(i, min(n, i + step), device="cuda")
        first, last = i // block, (min(n, i + step) - 1) // block
        low, high = max(0, (first + 1) * block - s["window"]), min(n, (last + 1) * block)
        front = min(sink, low)
        at = torch.cat([torch.arange(front, device="cuda"), torch.arange(low, high, device="cuda")])
        end = (rows // block + 1) * block
        see = (at < end[:, None]) & ((at < sink) | (at >= end[:, None] - s["window"]))
        see = see & (at < length[:, None, None]) & (rows[:, None] < length[:, None, None])
        see = see[:, None, None]
        pick = lambda x: (torch.cat([x[:, :, :front], x[:, :, low:high]], 2) if front else x[:, :, low:high]).unsqueeze(2)  # noqa: E731
        ki, vi, qi = pick(k), pick(v), q[..., i:i + step, :]
        p, lse[..., i:i + step] = _softmax_rows((qi @ ki.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~see, -math.inf))
        oi = p @ vi
        o[..., i:i + step, :] = oi
        if not s["grad"]:
            continue
        gi = d_o[..., i:i + step, :]
        pieces = ((dv, (p.transpose(-1, -2) @ gi).sum(2)),)
        ds = (gi @ vi.transpose(-1, -2)).sub_((gi * oi).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
        dq[..., i:i + step, :] = ds @ ki
        for whole, part in pieces + ((dk, (ds.transpose(-1, -2) @ qi).sum(2)),):
            whole[:, :, :front] += part[:, :, :front]
            whole[:, :, low:high] += part[:, :, front:]
    back = lambda x: x.transpose(1, 2).to(torch.bfloat16).contiguous()  # noqa: E731
    out = [back(o.flatten(1, 2)), lse.flatten(1, 2).contiguous()]
    return out + [back(dq.flatten(1, 2)), back(dk), back(dv)] if s["grad"] else out


def run(state):
    s = state
    if not own:
        if s["op"] == "store":
            return tuple(_stands_for(*_held_in_8(s[x])).to(TYPES[s["out"]]) for x in ("k", "v"))
        if s["op"] == "read":
            return tuple(_stands_for(*s[x]).to(TYPES[s["out"]]) for x in ("k8", "v8"))
        return _attended(s) if s["op"] == "attend" else _windowed(s)
    from paper_2603_17051_b200 import binding as A
    if s["op"] == "store":
        A.astro_kvcache_set_state(s["cache"], s["before"])
        A.astro_kvcache8_append(s["cache"], s["k"], s["v"], s["frames"])
        return A.astro_kvcache8_read(s["cache"], first_frame=s["sink"] + s["beside"], n_frames=s["frames"], dtype=TYPES[s["out"]])
    if s["op"] == "read":
        return A.astro_kvcache8_read(s["cache"], dtype=TYPES[s["out"]])
    if s["op"] == "attend":
        o, lse = A.astro_chunk_attn8_fwd(s["cache"], s["q"], s["k"], s["v"], s["scale"], workspace=s["workspace"])
        if not s["grad"]:
            return o, lse
        grads = A.astro_chunk_attn8_bwd(s["cache"], s["q"], s["k"], s["v"], o, lse, s["d_o"], s["scale"], workspace=s["workspace"])
        return [o, lse] + [x for x in grads if x is not None]
    mask = dict(block_tokens=s["block"], window_tokens=s["window"], sink_tokens=s["sink"], lengths=s["lengths"])
    o, lse = A.astro_window_attn_fwd(s["q"], s["k"], s["v"], s["scale"], **mask)
    if not s["grad"]:
        return o, lse
    return [o, lse, *A.astro_window_attn_bwd(s["q"], s["k"], s["v"], o, lse, s["d_o"], s["scale"], workspace=s["workspace"], **mask)]


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    def eight(x):
        """What a row held in 8 bits stands for: its values rounded, ties to even, to 3 bits behind the leading one, or
        to multiples of 2^(e-9) where they are small."""
        def two_to(e):
            return ((e.long() + 1023) << 52).view(torch.float64)

        x = x.double()
        top = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / LARGEST))
        e = e + (top > LARGEST * two_to(e)).double() - (top <= LARGEST * two_to(e - 1)).double()   # a logarithm next to a whole number
        e = torch.where(top > 0, e, float(LOWEST_EXP)).clamp(min=LOWEST_EXP)
        y = x * two_to(-e)
        step = two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(y / step) * step * two_to(e)

    def dense(q, k, v, see, scale, d_o):
        """One head: [O, LSE] or [O, LSE, dQ, dK, dV], rows a thousand at a time."""
        o, lse, dq, dk, dv = torch.zeros_like(q), q.new_zeros(len(q)), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for i in range(0, len(q), 1000):
            rows = slice(i, i + 1000)
            x = scale * (q[rows] @ k.T)
            if see is not None:
                x = torch.where(see(torch.arange(i, min(len(q), i + 1000), device="cuda")[:, None]), x, -math.inf)
            lse[rows] = torch.logsumexp(x, 1)
            p = torch.where(x == -math.inf, 0.0, torch.exp(x - lse[rows][:, None]))
            o[rows] = p @ v
            if d_o is not None:
                g = d_o[rows]
                ds = p * (g @ v.T - (g * o[rows]).sum(1, keepdim=True)) * scale
                dq[rows] = ds @ k
                dk += ds.T @ q[rows]
                dv += p.T @ g
        return [o, lse] if d_o is None else [o, lse, dq, dk, dv]

    s = prepare(case, seed)
    if case["op"] == "store":
        return tuple(eight(s[x]) for x in ("k", "v"))
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    if case["op"] == "window":
        n, group = case["n"], H // case["kv_heads"]
        outs = [s["q"].double() * 0, torch.zeros(B, H, n, dtype=torch.float64, device="cuda")]
        if case["grad"]:
            outs += [s["q"].double() * 0, s["k"].double() * 0, s["v"].double() * 0]
        j = torch.arange(n, device="cuda")[None]
        for b in range(B):
            length = n if s["lengths"] is None else int(s["lengths"][b])

            def see(i):
                before = torch.div(i, case["block"], rounding_mode="floor") * case["block"]     # tokens in front of i's block
                near = j >= before - (case["window"] - case["block"])
                return ((j < case["sink"]) | near) & (j < before + case["block"]) & (j < length) & (i < length)

            for h in range(H):
                d_o = s["d_o"][b, :, h].double() if case["grad"] else None
                got = dense(s["q"][b, :, h].double(), *(s[x][b, :, h // group].double() for x in "kv"), see, s["scale"], d_o)
                outs[0][b, :, h], outs[1][b, h] = got[:2]
                if case["grad"]:
                    outs[2][b, :, h] = got[2]
                    outs[3][b, :, h // group] += got[3]
                    outs[4][b, :, h // group] += got[4]
        return outs
    # the frames of a cache are inputs as they were before they were written: made again from the seed
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    frames = [eight(x) for x in _contents(case, lambda *shape, dtype: torch.randn(shape, generator=g, device="cuda").to(dtype), g,
                                          1 if case.get("shared") else B, case["held"])]
    if case["op"] == "read":
        return tuple(frames)
    n_q, n_kc, n_ctx = case["n_q"], case["n_kc"], case["held"] * case["tokens_per_frame"]
    outs = [s["q"].double() * 0, torch.zeros(B, H, n_q, dtype=torch.float64, device="cuda")]
    if case["grad"]:
        outs += [s["q"].double() * 0] + ([s["k"].double() * 0, s["v"].double() * 0] if n_kc else [])
    for b in range(B):
        for h in range(H):
            kv = [torch.cat([x[0 if case["shared"] else b, :, h]] + ([s[y][b, :, h].double()] if n_kc else [])) for x, y in zip(frames, "kv")]
            got = dense(s["q"][b, :, h].double(), *kv, None, s["scale"], s["d_o"][b, :, h].double() if case["grad"] else None)
            outs[0][b, :, h], outs[1][b, h] = got[:2]
            if case["grad"]:
                outs[2][b, :, h] = got[2]
                if n_kc:
                    outs[3][b, :, h], outs[4][b, :, h] = got[3][n_ctx:], got[4][n_ctx:]
    return outs
