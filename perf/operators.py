"""The operators around the rolling cache that are measured: rotary positions of queries and keys, the choice of key
blocks by a cheap score, attention over the chosen blocks (forward and backward), and forking a cache.

`run` computes an operator in elementary torch operations, or, where `own` is true, through the package's binding.
`exact` computes the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

QB = 128          # queries that share one choice of key blocks
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
KEEP_SINK, KEEP_CHUNK = 1, 2


# ------------------------------------------------------------------------------------------------ cases

def listed():
    dit = dict(heads=12, head_dim=128, tokens_per_frame=1560)
    video = dict(axis_pairs="22,21,21", layout="interleaved", rot_dim=128, base=10000.0, scaling="none", factor=1.0)
    return [
        # one new position for each of a group of 4: latency
        dict(name="rope_one_token", op="rope", batch=4, n=1, heads=12, head_dim=128, dtype="bf16", inverse=False,
             axis_pairs="64", layout="halves", rot_dim=128, base=10000.0, scaling="linear", factor=4.0, far=100000),
        # queries and keys of one 3-frame chunk of the video transformer: frame, row and column positions
        dict(name="rope_chunk", op="rope", batch=1, n=4680, heads=12, head_dim=128, dtype="bf16", inverse=False,
             far=21, **video),
        # their gradients for a group of 8 in fp32, half of each head rotated, stretched beyond the trained length
        dict(name="rope_gradient", op="rope", batch=8, n=4680, heads=12, head_dim=128, dtype="fp32", inverse=True,
             axis_pairs="32", layout="halves", rot_dim=64, base=10000.0, scaling="ramp", factor=8.0, far=1000000),
        # block means of the 3 frames that were just appended, for 4 samples
        dict(name="pool_appended", op="pool", batch=4, sink=3, window=12, held=12, frames=3, block=120, **dit),
        # the blocks for one query per sample
        dict(name="select_one_query", op="select", batch=4, shared=False, sink=3, window=12, held=12, n_q=1, n_kc=1, block=120, n_select=64,
             keep=KEEP_SINK | KEEP_CHUNK, **dit),
        # the blocks for every query block of a chunk against the full 18-frame context
        dict(name="select_chunk", op="select", batch=1, shared=False, sink=3, window=18, held=18, n_q=4680, n_kc=4680, block=120,
             n_select=96, keep=KEEP_SINK | KEEP_CHUNK, **dit),
        # one query per sample over its chosen blocks
        dict(name="attend_one_query", op="attend", batch=4, shared=False, sink=3, window=12, held=12, n_q=1, n_kc=1,
             block=120, n_select=32, empty=0, grad=False, **dit),
        # one denoising step of a chunk over a quarter of the full context
        dict(name="attend_chunk", op="attend", batch=1, shared=False, sink=3, window=18, held=18, n_q=4680, n_kc=4680,
             block=120, n_select=64, empty=0, grad=False, **dit),
        # a small training step: odd frame length, two blocks to a tile, some query blocks with nothing chosen
        dict(name="train_small", op="attend", batch=2, shared=True, heads=2, head_dim=64, tokens_per_frame=100, sink=1,
             window=6, held=5, n_q=300, n_kc=300, block=64, n_select=9, empty=3, grad=True),
        # the clip-window update: forward and backward of a 2-sample batch
        dict(name="train_clip", op="attend", batch=2, shared=False, sink=3, window=18, held=18, n_q=4680, n_kc=4680,
             block=120, n_select=64, empty=0, grad=True, **dit),
        # two samples continued twice each, few short frames
        dict(name="fork_small", op="fork", source=2, batch=4, heads=2, head_dim=64, tokens_per_frame=16, sink=0, window=6,
             held=6, frames=5),
        # the shared prefix copied out for a group of 8 that goes on separately
        dict(name="fork_group", op="fork", source=1, batch=8, sink=3, window=18, held=18, frames=18, **dit),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "pool", "select", "attend", "attend", "attend", "fork"])
    if op == "rope":
        heads, head_dim = rng.choice([1, 2, 12, 16]), rng.choice([64, 96, 128])
        n = _spread(rng, 1, 4680)
        batch = rng.randint(1, 8)
        axes = rng.choice([1, 3])
        rot = rng.choice([head_dim, head_dim // 2, head_dim - 4])
        half = rot // 2
        cut = [half] if axes == 1 else [half - 2 * (half // 3), half // 3, half // 3]
        return dict(op=op, batch=batch, n=n, heads=heads, head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    inverse=rng.random() < 0.5, axis_pairs=",".join(map(str, cut)), rot_dim=rot,
                    layout=rng.choice(["interleaved", "halves"]), base=rng.choice([10000.0, 500000.0]),
                    scaling=(s := rng.choice(["none", "linear", "base", "ramp"])), factor=1.0 if s == "none" else rng.choice([2.0, 8.0]),
                    far=_spread(rng, 16, 1000000))
    head_dim, heads = rng.choice([64, 128, 128]), rng.choice([1, 2, 12])
    tokens = rng.choice([_spread(rng, 5, 1560), 1560])
    sink, window = rng.randint(0, 3), rng.randint(4, 18)
    held = sink + rng.randint(1, window)
    size = dict(heads=heads, head_dim=head_dim, tokens_per_frame=tokens, sink=sink, window=window, held=held)
    if op == "fork":
        source = rng.choice([1, 2, 4])
        return dict(op=op, source=source, batch=rng.randint(1, 8), frames=rng.randint(1, min(held, 18)), **size)
    block = rng.choice([32, 40, 64, 96, 104, 120, 128])
    if op == "pool":
        return dict(op=op, batch=rng.randint(1, 4), frames=rng.randint(1, min(held, 3)), block=block, **size)
    n_kc = rng.choice([0, 1, _spread(rng, 8, 4680), _spread(rng, 8, 4680)])
    n_q = rng.choice([1, max(1, n_kc), _spread(rng, 1, 4680)])
    blocks = held * -(-tokens // block) + -(-n_kc // block)
    most = max(1, min(blocks, 7680 // block))
    if op == "select":
        return dict(op=op, batch=rng.randint(1, 2), shared=rng.random() < 0.3, n_q=n_q, n_kc=n_kc, block=block,
                    n_select=rng.randint(max(1, most // 4), most), keep=0, **size)
    return dict(op=op, batch=rng.randint(1, 2), shared=rng.random() < 0.3, n_q=n_q, n_kc=n_kc, block=block,
                n_select=rng.randint(max(1, most // 4), most), empty=rng.choice([0, 0, 4]), grad=rng.random() < 0.5, **size)


def work(case):
    c = case
    if c["op"] == "rope":
        rows = 2 * c["batch"] * c["n"] * c["heads"]
        size = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": 2 * rows * c["head_dim"] * size + 4 * c["n"] * len(_cut(c)), "flops": 3 * rows * c["rot_dim"]}
    row = c["heads"] * c["head_dim"] * 2                        # bytes of one token's keys
    if c["op"] == "fork":
        frame = c["tokens_per_frame"] * row * 2
        return {"bytes": frame * c["frames"] * (min(c["source"], c["batch"]) + c["batch"]), "flops": 0}
    if c["op"] == "pool":
        tokens = c["batch"] * c["frames"] * c["tokens_per_frame"]
        means = c["batch"] * c["frames"] * -(-c["tokens_per_frame"] // c["block"]) * c["heads"] * c["head_dim"]
        return {"bytes": tokens * row + 4 * means, "flops": tokens * row // 2}
    B, H, D = c["batch"], c["heads"], c["head_dim"]
    nqb, ctx, chunk = -(-c["n_q"] // QB), c["held"] * -(-c["tokens_per_frame"] // c["block"]), -(-c["n_kc"] // c["block"])
    if c["op"] == "select":
        return {"bytes": B * (c["n_q"] + c["n_kc"]) * row + 4 * (1 if c["shared"] else B) * ctx * H * D + 4 * B * H * nqb * c["n_select"],
                "flops": 2 * B * H * nqb * (ctx + chunk) * D}
    keys = min(c["n_select"] * c["block"], c["held"] * c["tokens_per_frame"] + c["n_kc"])   # seen by a query
    seen = min(nqb * keys, c["held"] * c["tokens_per_frame"] + c["n_kc"])                     # read at least once
    live = c["n_q"] if not c["empty"] else c["n_q"] * (c["empty"] - 1) / c["empty"]
    read = B * (2 * c["n_q"] + 2 * seen) * row + 4 * B * H * (c["n_q"] + nqb * c["n_select"])
    flops = 4.0 * B * H * live * keys * D
    if c["grad"]:
        share = c["n_kc"] / (c["held"] * c["tokens_per_frame"] + c["n_kc"])
        read += B * (2 * c["n_q"] + 2 * c["n_kc"]) * row
        flops += 6.0 * B * H * live * keys * D + 4.0 * B * H * live * keys * share * D
    return {"bytes": int(read), "flops": flops}


# ------------------------------------------------------------------------------------------------ inputs

def _cut(case):
    return [int(p) for p in case["axis_pairs"].split(",")]


def _slots(case):
    """Storage slots of the held frames, oldest first: the sink, then the window from a ring head of 1."""
    sink = min(case["sink"], case["held"])
    head = 1 % case["window"]
    return list(range(sink)) + [case["sink"] + (head + i) % case["window"] for i in range(case["held"] - sink)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape, dtype=torch.bfloat16: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    s = dict(case)
    if case["op"] == "rope":
        shape = (case["batch"], case["n"], case["heads"], case["head_dim"])
        s["q"], s["k"] = normal(*shape, dtype=TYPES[case["dtype"]]), normal(*shape, dtype=TYPES[case["dtype"]])
        s["positions"] = torch.randint(0, case["far"], (1, case["n"], len(_cut(case))), generator=g, device="cuda", dtype=torch.int32)
        if own:
            from paper_2603_17051_b200 import binding as A
            s["rope"] = A.astro_rope_create(case["head_dim"], case["rot_dim"], case["layout"], _cut(case), base=case["base"],
                                            scaling=case["scaling"], factor=case["factor"], original_length=4096)
        return s
    H, D, T = case["heads"], case["head_dim"], case["tokens_per_frame"]
    slots = _slots(case)
    of = case["source"] if case["op"] == "fork" else 1 if case.get("shared") else case["batch"]
    s["k_store"], s["v_store"] = (normal(of, H, case["sink"] + case["window"], T, D) for _ in range(2))
    s["slots"] = torch.tensor(slots, device="cuda")
    if case["op"] == "fork":
        s["parents"] = torch.randint(0, of, (case["batch"],), generator=g, device="cuda", dtype=torch.int32)
        s["kept"] = list(range(case["held"] - case["frames"], case["held"]))
    elif case["op"] == "pool":
        s["pooled"] = torch.zeros(of, H, case["sink"] + case["window"], -(-T // case["block"]), D, device="cuda")
    else:
        B, n_q, n_kc, block = case["batch"], case["n_q"], case["n_kc"], case["block"]
        s["q"] = normal(B, n_q, H, D)
        s["k"], s["v"] = (normal(B, n_kc, H, D) if n_kc else None for _ in range(2))
        if case["op"] == "select":
            s["pooled"] = _means(s["k_store"], block)
        else:
            ctx, chunk = case["held"] * -(-T // block), -(-n_kc // block)
            score = torch.rand(B, H, -(-n_q // QB), ctx + chunk, generator=g, device="cuda")
            picked = score.topk(min(case["n_select"], ctx + chunk)).indices.sort(-1).values.to(torch.int32)
            if case["empty"]:
                picked[:, :, case["empty"] - 1::case["empty"]] = -1
            s["blocks"] = picked.contiguous()
            s["scale"] = D ** -0.5
            if case["grad"]:
                s["d_o"] = normal(B, n_q, H, D)
    if own:
        from paper_2603_17051_b200 import binding as A
        sink = min(case["sink"], case["held"])

        def handle(batch, k, v):
            return A.astro_kvcache_create(batch, H, D, T, case["sink"], case["window"], k_storage=k, v_storage=v)

        s["cache"] = handle(of, s["k_store"], s["v_store"])
        ring = case["held"] - sink
        A.astro_kvcache_set_state(s["cache"], A.KVCacheState(sink, 1 % case["window"] if ring else 0, ring, case["held"]))
        if case["op"] == "fork":
            f = case["frames"]
            s["k_new"], s["v_new"] = (torch.empty(case["batch"], H, f, T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            s["fork"] = A.astro_kvcache_create(case["batch"], H, D, T, 0, f, k_storage=s["k_new"], v_storage=s["v_new"])
        elif case["op"] == "attend":
            need = A.astro_sparse_attn_fwd_workspace_bytes(case["batch"], H, D, case["n_q"], s["blocks"].shape[-1], case["block"])
            if case["grad"]:
                need = max(need, A.astro_sparse_attn_bwd_workspace_bytes(case["batch"], H, D, case["n_q"], case["n_kc"],
                                                                         s["blocks"].shape[-1], case["block"]))
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        elif case["op"] == "select":
            need = A.astro_block_select_workspace_bytes(case["batch"], H, D, case["n_q"], case["n_kc"], case["block"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _frequencies(c):
    """Radians per position of every pair, and the factor on cos and sin.  Stretched contexts: positions divided
    by the factor; or the base raised so that the slowest pair is divided by it; or a ramp that divides the pairs
    that turn at most once over the trained length, leaves those that turn 32 times or more, and blends between."""
    amount, size = c["factor"], 1.0

    def axis(pairs):
        base = c["base"]
        if c["scaling"] == "base" and pairs > 1:
            base *= amount ** (pairs / (pairs - 1))
        f = base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
        if c["scaling"] == "linear":
            f = f / amount
        if c["scaling"] == "ramp":
            keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
            f = f * (keep + (1 - keep) / amount)
        return f

    if c["scaling"] == "ramp":
        size = 0.1 * math.log(amount) + 1
    cut = _cut(c)
    return torch.cat([axis(p) for p in cut]), torch.repeat_interleave(torch.arange(len(cut)), torch.tensor(cut)), size


def _rotated(s):
    freq, axis, size = _frequencies(s)
    angle = s["positions"].double()[..., axis.cuda()] * freq.cuda()           # far positions: the product needs 64 bits
    cos, sin = (angle.cos() * size).float().unsqueeze(2), (angle.sin() * size).float().unsqueeze(2)
    if s["inverse"]:
        sin = -sin
    rot, half = s["rot_dim"], s["rot_dim"] // 2

    def turn(x):
        y = x.float()
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if s["layout"] == "interleaved" else (y[..., :half], y[..., half:rot])
        u, v = a * cos - b * sin, a * sin + b * cos
        front = torch.stack([u, v], -1).flatten(-2) if s["layout"] == "interleaved" else torch.cat([u, v], -1)
        return torch.cat([front, y[..., rot:]], -1).to(x.dtype)

    return turn(s["q"]), turn(s["k"])


def _means(x, block):
    """Means over the blocks of `block` tokens (the last may be shorter) of x [..., tokens, D], summed in 64 bits."""
    T = x.shape[-2]
    nb = -(-T // block)
    padded = torch.nn.functional.pad(x.double(), (0, 0, 0, nb * block - T))
    count = (T - block * torch.arange(nb, device=x.device)).clamp(max=block).double()
    return (padded.unflatten(-2, (nb, block)).sum(-2) / count[:, None]).float()


def _selected(s):
    B, H, D = s["batch"], s["heads"], s["head_dim"]
    q = _means(s["q"].transpose(1, 2), QB)
    keys = s["pooled"][:, :, s["slots"]].flatten(2, 3).expand(B, H, -1, D)
    n_ctx = keys.shape[2]
    if s["n_kc"]:
        keys = torch.cat([keys, _means(s["k"].transpose(1, 2), s["block"])], 2)
    score = q.double() @ keys.double().transpose(-1, -2)
    if s["keep"] & KEEP_SINK:
        score[..., :min(s["sink"], s["held"]) * -(-s["tokens_per_frame"] // s["block"])] = math.inf
    if s["keep"] & KEEP_CHUNK:
        score[..., n_ctx:] = math.inf
    first = score.sort(dim=-1, descending=True, stable=True).indices[..., :s["n_select"]]
    return first.sort(-1).values.to(torch.int32)


def _gathered(s, store, chunk):
    """[B, H, block, token of the block, D] in 32 bits (zeros behind a block's end), and the tokens per block."""
    B, H, D, T, block = s["batch"], s["heads"], s["head_dim"], s["tokens_per_frame"], s["block"]
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, -x.shape[-2] % block)).unflatten(-2, (-1, block))  # noqa: E731
    count = lambda n: (n - block * torch.arange(-(-n // block), device=store.device)).clamp(max=block)  # noqa: E731
    all_, counts = cut(store[:, :, s["slots"]].float()).flatten(2, 3).expand(B, -1, -1, -1, -1), count(T).repeat(s["held"])
    if s["n_kc"]:
        all_, counts = torch.cat([all_, cut(chunk.float().transpose(1, 2))], 2), torch.cat([counts, count(s["n_kc"])])
    return all_, counts


def _attended(s):
    B, H, D, n_q = s["batch"], s["heads"], s["head_dim"], s["n_q"]
    nqb, block = -(-n_q // QB), s["block"]
    kb, counts = _gathered(s, s["k_store"], s["k"])
    vb, _ = _gathered(s, s["v_store"], s["v"])
    sel, there = s["blocks"].clamp(min=0).long(), s["blocks"] >= 0
    at = (torch.arange(B, device="cuda")[:, None, None, None], torch.arange(H, device="cuda")[:, None, None], sel)
    valid = ((torch.arange(block, device="cuda") < counts[sel][..., None]) & there[..., None]).flatten(-2).unsqueeze(-2)
    kg, vg = kb[at].flatten(3, 4), vb[at].flatten(3, 4)                       # [B, H, query block, keys, D]
    rows = lambda x: torch.nn.functional.pad(x.float().transpose(1, 2), (0, 0, 0, nqb * QB - n_q)).unflatten(2, (nqb, QB))  # noqa: E731
    back = lambda x: x.flatten(2, 3)[:, :, :n_q].transpose(1, 2).to(torch.bfloat16)  # noqa: E731
    q = rows(s["q"])
    score = (q @ kg.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~valid, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1).flatten(2)[:, :, :n_q]
    p /= torch.where(total > 0, total, 1.0)
    o = p @ vg
    if not s["grad"]:
        return back(o), lse.contiguous()
    d_o = rows(s["d_o"])
    ds = d_o @ vg.transpose(-1, -2)
    ds = ds.sub_((d_o * o).sum(-1, keepdim=True)).mul_(p)
    dq = (ds @ kg).mul_(s["scale"])
    out = [back(o), lse.contiguous(), back(dq)]
    if not s["n_kc"]:
        return out
    n_ctx, n_blocks = kb.shape[2] - -(-s["n_kc"] // block), kb.shape[2]
    flat = ((torch.arange(B * H, device="cuda").view(B, H, 1, 1)) * n_blocks + sel).flatten()

    def scattered(per_list):                                                 # sums over the lists, chunk blocks only
        whole = torch.zeros(B * H * n_blocks, block, D, device="cuda")
        whole.index_add_(0, flat, per_list.unflatten(3, (-1, block)).flatten(0, 3))
        own_blocks = whole.view(B, H, n_blocks, block, D)[:, :, n_ctx:].flatten(2, 3)
        return own_blocks[:, :, :s["n_kc"]].transpose(1, 2).to(torch.bfloat16)

    return out + [scattered((ds.transpose(-1, -2) @ q).mul_(s["scale"])), scattered(p.transpose(-1, -2) @ d_o)]


def run(state):
    s = state
    if not own:
        if s["op"] == "rope":
            return _rotated(s)
        if s["op"] == "pool":
            s["pooled"][:, :, s["slots"][-s["frames"]:]] = _means(s["k_store"][:, :, s["slots"][-s["frames"]:]], s["block"])
            return s["pooled"]
        if s["op"] == "select":
            return _selected(s)
        if s["op"] == "attend":
            return _attended(s)
        kept = s["slots"][s["kept"][0]:s["kept"][-1] + 1]
        return tuple(x[:, :, kept][s["parents"]] for x in (s["k_store"], s["v_store"]))
    from paper_2603_17051_b200 import binding as A
    if s["op"] == "rope":
        return A.astro_rope_apply(s["rope"], s["q"], s["k"], s["positions"], inverse=s["inverse"])
    if s["op"] == "pool":
        return A.astro_block_pool(s["cache"], s["block"], first_frame=s["held"] - s["frames"], n_frames=s["frames"], pooled=s["pooled"])
    if s["op"] == "select":
        return A.astro_block_select(s["cache"], s["pooled"], s["q"], s["k"], s["block"], s["n_select"], keep=s["keep"],
                                    workspace=s["workspace"])
    if s["op"] == "fork":
        A.astro_kvcache_fork(s["fork"], s["cache"], parents=s["parents"], frames=s["kept"])
        return s["k_new"], s["v_new"]
    o, lse = A.astro_sparse_attn_fwd(s["cache"], s["q"], s["k"], s["v"], s["blocks"], s["block"], s["scale"], workspace=s["workspace"])
    if not s["grad"]:
        return o, lse
    grads = A.astro_sparse_attn_bwd(s["cache"], s["q"], s["k"], s["v"], s["blocks"], s["block"], o, lse, s["d_o"], s["scale"],
                                    workspace=s["workspace"])
    return [o, lse] + [x for x in grads if x is not None]


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    def rotated(s):
        turns = []                                                               # one complex factor for each pair
        pair = 0
        for a, pairs in enumerate(_cut(s)):
            for i in range(pairs):
                base = s["base"]
                if s["scaling"] == "base" and pairs > 1:
                    base = base * s["factor"] ** (pairs / (pairs - 1))
                f = math.exp(-math.log(base) * i / pairs)
                if s["scaling"] == "linear":
                    f /= s["factor"]
                if s["scaling"] == "ramp":
                    share = min(1.0, max(0.0, (f * 4096 / math.tau - 1.0) / (32.0 - 1.0)))
                    f = f / s["factor"] * (1.0 - share) + f * share
                turns.append(s["positions"][..., a].double() * (-f if s["inverse"] else f))
                pair += 1
        size = 1 + 0.1 * math.log(s["factor"]) if s["scaling"] == "ramp" else 1.0
        angle = torch.stack(turns, -1).unsqueeze(2)
        z = torch.polar(torch.full_like(angle, size), angle)
        out = []
        for x in (s["q"], s["k"]):
            y = x.double().clone()
            if s["layout"] == "interleaved":
                first, second = slice(0, 2 * pair, 2), slice(1, 2 * pair, 2)
            else:
                first, second = slice(0, pair), slice(pair, 2 * pair)
            w = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
            y[..., first], y[..., second] = w.real, w.imag
            out.append(y)
        return tuple(out)

    def attended(s):
        """Every head apart, as attention over all keys with the keys of blocks that were not chosen masked out."""
        B, H, D, T, block, n_q, n_kc = (s[x] for x in ("batch", "heads", "head_dim", "tokens_per_frame", "block", "n_q", "n_kc"))
        frames = s["held"]
        per_frame = -(-T // block)
        key_block = [f * per_frame + t // block for f in range(frames) for t in range(T)]
        key_block = torch.tensor(key_block + [frames * per_frame + t // block for t in range(n_kc)], device="cuda")
        n_blocks = frames * per_frame + -(-n_kc // block)
        query_block = torch.arange(n_q, device="cuda") // QB
        o = torch.zeros(B, n_q, H, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(B, H, n_q, dtype=torch.float64, device="cuda")
        dq, dk, dv = torch.zeros_like(o), *(torch.zeros(B, n_kc, H, D, dtype=torch.float64, device="cuda") for _ in range(2))
        for b in range(B):
            bc = 0 if s["shared"] else b
            for h in range(H):
                k, v = (torch.cat([x[bc, h][s["slots"]].reshape(-1, D)] + ([y[b, :, h]] if n_kc else [])).double()
                        for x, y in ((s["k_store"], s["k"]), (s["v_store"], s["v"])))
                chosen = torch.zeros(-(-n_q // QB), n_blocks + 1, dtype=torch.bool, device="cuda")
                picked = s["blocks"][b, h].long()
                chosen.scatter_(1, torch.where(picked < 0, n_blocks, picked), True)
                see = chosen[:, key_block][query_block]
                q = s["q"][b, :, h].double()
                x = torch.where(see, s["scale"] * (q @ k.T), -math.inf)
                lse[b, h] = torch.logsumexp(x, 1)
                p = torch.where(see, torch.exp(x - lse[b, h][:, None]), 0.0)
                o[b, :, h] = p @ v
                if s["grad"]:
                    g = s["d_o"][b, :, h].double()
                    ds = p * (g @ v.T - (g * o[b, :, h]).sum(1, keepdim=True)) * s["scale"]
                    dq[b, :, h] = ds @ k
                    dk[b, :, h] = (ds.T @ q)[frames * T:]
                    dv[b, :, h] = (p.T @ g)[frames * T:]
        return [o, lse] if not s["grad"] else [o, lse, dq] + ([dk, dv] if n_kc else [])

    s = prepare(case, seed)
    if case["op"] == "select":
        return None                                                          # whole numbers
    if case["op"] == "fork":
        kept = [_slots(case)[f] for f in s["kept"]]
        return tuple(torch.stack([torch.stack([x[int(p), :, f] for f in kept], 1) for p in s["parents"].tolist()]).double()
                     for x in (s["k_store"], s["v_store"]))
    if case["op"] == "rope":
        return rotated(s)
    if case["op"] == "pool":
        out = s["pooled"].double()
        for f in range(case["held"] - case["frames"], case["held"]):
            frame = s["k_store"][:, :, _slots(case)[f]].double()
            for j in range(out.shape[3]):
                out[:, :, _slots(case)[f], j] = frame[:, :, j * case["block"]:(j + 1) * case["block"]].mean(2)
        return out
    return attended(s)
