"""Performance cases of the decode-instance operators: the calls that one decode step of a served model makes.

Three kinds, one for each operator, all through the package's public calls:

* ``append``    -- ``ctr.ctr_kv_append``: queries and keys rotated at their positions, keys and values put into the paged cache.
* ``attention`` -- ``ctr.ctr_tree_attention``: each sequence's new tokens (one, a chain, or a tree of drafted ones) over the cache.
* ``sample``    -- ``ctr.ctr_sample``: a token per row from its logits and a given uniform.

``own = False`` computes the same outputs with elementary torch operations in fp32.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# the sampler's 2^f on [-1/2, 1/2]: its definition's coefficients, highest power first
EXP2 = tuple(float.fromhex(h) for h in ("0x1.5bba14p-10", "0x1.3cea88p-7", "0x1.c6b752p-5", "0x1.ebf9bcp-3", "0x1.62e42ap-1", "0x1p+0"))


def listed():
    return [
        # one decode step of a small pool instance: a handful of active sequences, a model with two KV heads
        {"name": "append_tick", "kind": "append", "n": 7, "heads": 16, "kv": 2, "d": 128, "rot": 128, "inter": False,
         "dtype": "bf16", "page": 16, "scaled": False, "first": 838, "pad": False},
        # a full decode batch in a captured graph: padded rows, half of each head rotated in neighbouring pairs
        {"name": "append_decode", "kind": "append", "n": 512, "heads": 32, "kv": 8, "d": 128, "rot": 64, "inter": True,
         "dtype": "fp16", "page": 32, "scaled": False, "first": 1000, "pad": True},
        # two dozen sequences' trees of 64 drafted tokens
        {"name": "append_tree", "kind": "append", "n": 1536, "heads": 64, "kv": 8, "d": 64, "rot": 64, "inter": False,
         "dtype": "bf16", "page": 64, "scaled": False, "first": 2048, "pad": False},
        # two batches of prompts (8,192 tokens each) deep in a context scaled beyond its trained length
        {"name": "append_prompt", "kind": "append", "n": 16384, "heads": 32, "kv": 8, "d": 128, "rot": 128, "inter": False,
         "dtype": "bf16", "page": 64, "scaled": True, "first": 100_003, "pad": False},
        # a lone interactive request at the mean prompt length
        {"name": "attn_one", "kind": "attention", "b": 1, "heads": 16, "kv": 2, "d": 128, "dtype": "bf16", "page": 16,
         "nodes": 1, "tree": False, "ctx": 838, "spread": 0.0},
        # a decode instance's batch: one token each, lognormal contexts, about 100,000 resident tokens
        {"name": "attn_decode", "kind": "attention", "b": 96, "heads": 32, "kv": 8, "d": 128, "dtype": "bf16", "page": 16,
         "nodes": 1, "tree": False, "ctx": 640, "spread": 1.0},
        # verification of ragged trees of up to 16 drafted tokens
        {"name": "attn_verify", "kind": "attention", "b": 32, "heads": 32, "kv": 8, "d": 128, "dtype": "fp16", "page": 64,
         "nodes": 16, "tree": True, "ctx": 1024, "spread": 0.6},
        # wide trees over long prompts: 64 drafted tokens, eight query heads to a KV head
        {"name": "attn_fan", "kind": "attention", "b": 16, "heads": 64, "kv": 8, "d": 128, "dtype": "bf16", "page": 64,
         "nodes": 64, "tree": True, "ctx": 8192, "spread": 0.0},
        # an instance's whole capacity (200,000 tokens) in two sequences: few rows over a long axis, a short chain
        {"name": "attn_long", "kind": "attention", "b": 2, "heads": 32, "kv": 8, "d": 64, "dtype": "fp16", "page": 32,
         "nodes": 5, "tree": False, "ctx": 99_989, "spread": 0.0},
        # a few interactive requests: top-k and top-p together
        {"name": "sample_tick", "kind": "sample", "n": 3, "vocab": 32_000, "dtype": "fp32", "mode": "both"},
        # a full batch over a large vocabulary, every request with settings of its own
        {"name": "sample_batch", "kind": "sample", "n": 256, "vocab": 131_072, "dtype": "bf16", "mode": "mixed"},
        # nucleus and min-p without top-k, odd vocabulary: the whole row's mass counts
        {"name": "sample_nucleus", "kind": "sample", "n": 96, "vocab": 100_003, "dtype": "fp32", "mode": "mass"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attention", "attention", "sample"))
    if kind == "append":
        kv = rng.choice((1, 2, 4, 8))
        d = rng.choice((64, 80, 128, 128, 256))
        heads = kv * rng.choice((1, 2, 4, 5, 8))
        return {"kind": kind, "n": _log(rng, 1, min(16_384, 100_000_000 // ((heads + 2 * kv) * d))), "heads": heads, "kv": kv,
                "d": d, "rot": rng.choice((d, d, d // 2)), "inter": rng.random() < 0.4, "dtype": rng.choice(("bf16", "fp16")),
                "page": rng.choice((16, 32, 64, 128)), "scaled": rng.random() < 0.3, "first": _log(rng, 1, 500_000),
                "pad": rng.random() < 0.3}
    if kind == "attention":
        kv, d = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128))
        nodes = rng.choice((1, 1, 1, _log(rng, 2, 64), _log(rng, 2, 64)))
        ctx = _log(rng, 1, 100_000)
        # resident tokens: at most the capacity of an instance, and what the largest listed case computes
        return {"kind": kind, "b": _log(rng, 1, max(1, min(256, 100_000 // (ctx + nodes)))), "heads": kv * rng.choice((1, 2, 4, 7, 8)),
                "kv": kv, "d": d, "dtype": rng.choice(("bf16", "fp16")), "page": rng.choice((16, 32, 64, 128)), "nodes": nodes,
                "tree": rng.random() < 0.6, "ctx": ctx, "spread": 0.0 if ctx > 5000 else rng.choice((0.0, 0.6))}
    vocab = _log(rng, 1000, 160_000)
    return {"kind": kind, "n": _log(rng, 1, min(512, 33_000_000 // vocab)), "vocab": vocab, "dtype": rng.choice(("bf16", "fp16", "fp32")),
            "mode": rng.choice(("both", "mixed", "mass", "plain"))}


# ---------------------------------------------------------------- inputs
def _lengths(case, seed):
    """Each sequence's (context, new tokens), host integers: the case's own set of both, the contexts in the seed's order."""
    b, nodes = case["b"], case["nodes"]
    g = torch.Generator().manual_seed(b)
    z = torch.randn(b, generator=g, dtype=torch.float64)
    # about half of the trees are full
    new = torch.full((b,), nodes) if nodes == 1 else torch.randint(1, 2 * nodes + 1, (b,), generator=g).clamp(max=nodes)
    new[0] = nodes
    ctx = (case["ctx"] * torch.exp(case["spread"] * z)).round().clamp(1, 12 * case["ctx"]).long()
    return ctx[torch.randperm(b, generator=torch.Generator().manual_seed(seed))], new


def _turns(half, base, factor):
    """Frequency of each pair in turns per position, as a 64-bit fraction; `factor` stretches the slow pairs."""
    freq = [base ** (-i / half) / (2 * math.pi) for i in range(half)]
    if factor > 1:  # a pair that turns less than once in 8,192 positions is slowed by the factor, a fast one (32 times) is kept
        keep = [min(1.0, max(0.0, (f * 8192 - 1) / 31)) for f in freq]
        freq = [f * (k + (1 - k) / factor) for f, k in zip(freq, keep)]
    words = [int(f * 2.0 ** 64) for f in freq]
    return torch.tensor([w - (1 << 64) if w >= 1 << 63 else w for w in words], dtype=torch.int64, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "append":
        n, heads, kv, d, page = case["n"], case["heads"], case["kv"], case["d"], case["page"]
        # q, k and v are views of one fused projection's output
        qkv = torch.randn(n, heads + 2 * kv, d, device=DEV, generator=g, dtype=torch.float32).to(dt)
        pages = -(-n // page) + 3  # the first page takes no token
        slots = page + torch.randperm((pages - 1) * page // 8, device=DEV, generator=g)[:, None] * 8 + torch.arange(8, device=DEV)
        slots = slots.reshape(-1)[:n].contiguous()  # runs of eight: a page's tokens lie together, in any order of pages
        if case["pad"]:
            slots = torch.where(torch.rand(n, device=DEV, generator=g) < 0.06, -1, slots)
        positions = case["first"] + torch.arange(n, device=DEV) if n > 1000 else torch.randint(
            0, 2 * case["first"] + 1, (n,), device=DEV, generator=g)
        return {"case": case, "q": qkv[:, :heads], "k": qkv[:, heads:heads + kv], "v": qkv[:, heads + kv:], "slots": slots,
                "positions": positions, "turns": _turns(case["rot"] // 2, 500_000.0, 8.0 if case["scaled"] else 1.0),
                "scale": 0.1 * math.log(8.0) + 1 if case["scaled"] else 1.0, "q_out": torch.empty(n, heads, d, device=DEV, dtype=dt),
                "k_cache": torch.zeros(pages, kv, page, d, device=DEV, dtype=dt), "v_cache": torch.zeros(pages, kv, page, d, device=DEV, dtype=dt)}
    if case["kind"] == "attention":
        heads, kv, d, page = case["heads"], case["kv"], case["d"], case["page"]
        ctx, new = _lengths(case, seed)
        total = int(new.sum())
        lens = ctx + new
        need = (lens + page - 1) // page
        width = int(need.max())
        gc = torch.Generator().manual_seed(seed + 1)
        perm = torch.randperm(int(need.sum()), generator=gc).int()
        table = torch.zeros(case["b"], width, dtype=torch.int32)
        cols = torch.arange(width)[None, :] < need[:, None]
        table[cols] = perm
        start = torch.zeros(case["b"] + 1, dtype=torch.int64)
        start[1:] = new.cumsum(0)
        # node i of a sequence hangs from one of the last few nodes before it (a tree) or from the one before it (a chain)
        node = torch.arange(total) - start[:-1].repeat_interleave(new)
        back = torch.randint(1, 7, (total,), generator=gc) if case["tree"] else torch.ones(total, dtype=torch.int64)
        mask = torch.zeros(total, dtype=torch.int64)
        for t, (i, s) in enumerate(zip(node.tolist(), back.tolist())):
            mask[t] = (int(mask[t - s]) if i - s >= 0 else 0) | ((1 << i) if i < 63 else -(1 << 63))
        pages = int(need.sum())
        cache = [torch.randn(pages, kv, page, d, device=DEV, generator=g, dtype=torch.float32).to(dt) for _ in range(2)]
        q = (1.5 * torch.randn(total, heads, d, device=DEV, generator=g, dtype=torch.float32)).to(dt)
        return {"case": case, "q": q, "k_cache": cache[0], "v_cache": cache[1], "q_start": start.int().to(DEV), "kv_len": lens.int().to(DEV),
                "table": table.to(DEV), "mask": mask.to(DEV), "scale": d ** -0.5, "out": torch.empty_like(q),
                "lse": torch.empty(total, heads, device=DEV), "longest": width * page}
    n, vocab, mode = case["n"], case["vocab"], case["mode"]
    # a broad bulk and a few dozen peaks of decreasing height, their count and height of each row's own
    x = 1.5 * torch.randn(n, vocab, device=DEV, generator=g)
    at = torch.randint(0, vocab, (n, 48), device=DEV, generator=g)
    top = 8 + 6 * torch.rand(n, 1, device=DEV, generator=g)
    fall = 0.1 + 0.9 * torch.rand(n, 1, device=DEV, generator=g)
    x.scatter_(1, at, top - fall * torch.arange(48, device=DEV) + 0.5 * torch.randn(n, 48, device=DEV, generator=g))
    rand = torch.rand(4, n, device=DEV, generator=g)
    temperature = 0.5 + 0.7 * rand[0]
    top_k = torch.randint(1, 101, (n,), device=DEV, generator=g, dtype=torch.int32)
    top_p, min_p = 0.8 + 0.19 * rand[1], 0.1 * rand[2]
    row = torch.arange(n, device=DEV)
    if mode == "both":
        top_k.fill_(50)
        min_p.zero_()
    elif mode == "mass":
        top_k.zero_()
    elif mode == "plain":
        top_k.zero_()
        top_p.fill_(1.0)
        min_p.zero_()
    else:  # a few greedy rows, a few with every token kept, a third without top-k
        temperature = torch.where(row % 16 == 5, 0.0, temperature)
        top_k = torch.where(row % 3 == 1, 0, top_k)
        top_p = torch.where(row % 8 == 4, 1.0, top_p)
        min_p = torch.where(row % 2 == 0, 0.0, min_p)
    return {"case": case, "logits": x.to(dt), "temperature": temperature, "top_k": top_k.int(), "top_p": top_p, "min_p": min_p,
            "u": rand[3].contiguous(), "token": torch.empty(n, dtype=torch.int32, device=DEV),
            "logprob": torch.empty(n, device=DEV), "n_kept": torch.empty(n, dtype=torch.int32, device=DEV)}


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return {"append": _append, "attention": _attention, "sample": _sample}[kind](state)


def _own_append(s):
    from paper_2609_16206_gb300 import ctr
    if "cache" not in s:  # the handles that a program keeps beside its cache
        s["cache"] = ctr.KvCache(s["k_cache"], s["v_cache"])
        s["rope"] = ctr.Rope(s["turns"], interleaved=s["case"]["inter"], scale=s["scale"])
    ctr.ctr_kv_append(s["cache"], s["rope"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"])
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attention(s):
    from paper_2609_16206_gb300 import ctr
    c = s["case"]
    if "cache" not in s:
        s["cache"] = ctr.KvCache(s["k_cache"], s["v_cache"])
        s["workspace"] = ctr.attention_workspace(s["cache"], c["heads"], c["b"], c["nodes"])
    ctr.ctr_tree_attention(s["cache"], s["q"], s["q_start"], s["kv_len"], s["table"], s["out"], s["workspace"], max_nodes=c["nodes"],
                           tree_mask=s["mask"], lse=s["lse"], scale=s["scale"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_sample(s):
    from paper_2609_16206_gb300 import ctr
    ctr.ctr_sample(s["logits"], s["temperature"], s["u"], s["token"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                   logprob=s["logprob"], n_kept=s["n_kept"])
    return {"token": s["token"], "logprob": s["logprob"], "n_kept": s["n_kept"]}


_OWN = {"append": _own_append, "attention": _own_attention, "sample": _own_sample}


# ---------------------------------------------------------------- plain forms, fp32
def _append(s):
    c = s["case"]
    half, page = c["rot"] // 2, c["page"]
    turn = ((s["positions"][:, None] * s["turns"][None, :]) >> 32).float() * 2.0 ** -31  # signed half-turns: the product wraps
    cos = (torch.cos(turn * math.pi) * s["scale"])[:, None, :]
    sin = (torch.sin(turn * math.pi) * s["scale"])[:, None, :]

    def rotate(x):
        f = x.float()
        out = f.clone()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["inter"] else (slice(0, half), slice(half, 2 * half))
        out[..., a] = f[..., a] * cos - f[..., b] * sin
        out[..., b] = f[..., a] * sin + f[..., b] * cos
        return out.to(x.dtype)

    put = s["slots"] >= 0
    slot = torch.where(put, s["slots"], 0)  # padding rows write the first page's first token back as it is
    at, off = slot // page, slot % page
    for cache, new in ((s["k_cache"], rotate(s["k"])), (s["v_cache"], s["v"])):
        cache[at, :, off] = torch.where(put[:, None, None], new, cache[at, :, off])
    return {"q": rotate(s["q"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attention(s):
    c = s["case"]
    b, kv, d, t, longest = c["b"], c["kv"], c["d"], c["nodes"], s["longest"]
    group = c["heads"] // kv
    table = s["table"].long()
    k, v = (x[table].float().permute(0, 2, 1, 3, 4).reshape(b, kv, longest, d) for x in (s["k_cache"], s["v_cache"]))
    start, lens = s["q_start"].long(), s["kv_len"].long()
    new = start[1:] - start[:-1]
    node = torch.arange(t, device=DEV)[None, :]
    row = (start[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().reshape(b, t, kv, group, d).permute(0, 2, 3, 1, 4).reshape(b, kv, group * t, d)
    score = torch.matmul(q, k.transpose(2, 3)).reshape(b, kv, group, t, longest) * s["scale"]
    at = torch.arange(longest, device=DEV) - (lens - new)[:, None]  # below 0: context, then the node's number
    bit = (s["mask"][row][:, :, None] >> at.clamp(0, 63)[:, None, :]) & 1
    seen = (at < 0)[:, None, :] | ((at < new[:, None])[:, None, :] & (bit == 1))
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - base)
    total = p.sum(-1, keepdim=True)
    v = torch.where((at < new[:, None])[:, None, :, None], v, 0.0)
    out = torch.matmul((p / torch.where(total > 0, total, 1.0)).reshape(b, kv, group * t, longest), v)
    lse = (base + torch.log(total)).reshape(b, kv * group, t)
    out = out.reshape(b, kv * group, t, d).permute(0, 2, 1, 3)
    live = (node < new[:, None]).reshape(-1).nonzero()[:, 0]
    return {"out": out.reshape(b * t, kv * group, d)[live].to(s["q"].dtype), "lse": lse.permute(0, 2, 1).reshape(b * t, -1)[live]}


def _weights(x, rate):
    """round(2^31 2^(x rate)) for x <= 0, in fp32 with every step rounded."""
    y = (x * rate).clamp(min=-64.0)
    k = torch.round(y)
    f = y - k
    p = torch.full_like(f, EXP2[0])
    for coef in EXP2[1:]:
        p = p * f
        p = p + coef
    return torch.round(p * ((k.int() + (31 + 127)) << 23).view(torch.float32)).long()


def _share(total, part):
    """floor(total part / 2^31) for part <= 2^31 without the 64-bit overflow of the product."""
    return (total >> 31) * part + (((total & 0x7FFFFFFF) * part) >> 31)


def _sample(s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    n, vocab = x.shape
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    top = value[:, :1]
    some = top > -math.inf
    greedy = ~(s["temperature"] > 0)[:, None]
    rate = torch.div(torch.full_like(s["temperature"], 1.4426950408889634), s["temperature"]).clamp(max=3e38)[:, None]
    w = _weights(torch.where(value == top, 0.0, value - top), torch.where(greedy, 1.0, rate))
    w = torch.where(value > -math.inf, w, 0)
    rank = torch.arange(vocab, device=DEV)[None, :]
    k = torch.where(s["top_k"] > 0, s["top_k"].long(), vocab)[:, None]
    w = torch.where(rank < torch.where(greedy, 1, k), w, 0)
    before = w.cumsum(1) - w
    goal = _share(before[:, -1:] + w[:, -1:], (s["top_p"].clamp(0, 1) * 2.0 ** 31).long()[:, None])
    w = torch.where((before < goal) | (rank == 0) | (s["top_p"] >= 1)[:, None], w, 0)
    least = (s["min_p"].clamp(0, 1) * 2.0 ** 31).long()[:, None]
    w = torch.where(w >= least, w, 0)
    kept = (w > 0).sum(1)
    mass = w.sum(1, keepdim=True)
    placed = torch.zeros_like(w).scatter_(1, index, w)
    goal = _share(mass, (s["u"] * 2.0 ** 31).long().clamp(0, (1 << 31) - 1)[:, None])
    token = (placed.cumsum(1) <= goal).sum(1).clamp(max=vocab - 1)
    share = placed.gather(1, token[:, None]).float() / mass.float()
    some = some[:, 0]
    return {"token": torch.where(some, token, -1).int(), "logprob": torch.where(some, torch.log(share[:, 0]), -math.inf),
            "n_kept": torch.where(some, kept, 0).int()}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["kind"] == "append":
        values = case["n"] * (case["heads"] + 2 * case["kv"]) * case["d"]
        return {"bytes": 2 * values * size + 16 * case["n"] + 4 * case["rot"],
                "flops": 3 * case["n"] * (case["heads"] + case["kv"]) * case["rot"]}
    if case["kind"] == "attention":
        ctx, new = _lengths(case, 0)
        lens = ctx + new
        cache = 2 * int(lens.sum()) * case["kv"] * case["d"] * size
        rows = int(new.sum()) * case["heads"]
        return {"bytes": cache + rows * (2 * case["d"] * size + 4) + 8 * int(new.sum()) + 4 * int((lens // case["page"] + 1).sum()),
                "flops": 4 * case["d"] * case["heads"] * int((lens * new).sum())}
    return {"bytes": case["n"] * (case["vocab"] * size + 32), "flops": 15 * case["n"] * case["vocab"]}


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, s)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    return _exact_sample(s)


def _exact_append(case, s):
    n, page, rot = case["n"], case["page"], case["rot"]
    pos, turns = s["positions"].tolist(), [t % (1 << 64) for t in s["turns"].tolist()]
    phase = torch.tensor([[((p * t) % (1 << 64)) / 2.0 ** 64 for t in turns] for p in pos], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(phase, s["scale"]), 2 * math.pi * phase)[:, None, :]  # a rotation is a complex product

    def rotated(x):
        z = x.double()
        head, rest = z[..., :rot], z[..., rot:]
        pairs = head.unflatten(-1, (-1, 2)) if case["inter"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        head = pairs.flatten(-2) if case["inter"] else pairs.transpose(-1, -2).flatten(-2)
        return torch.cat((head, rest), -1)

    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    live = (s["slots"] >= 0).nonzero()[:, 0]
    at = s["slots"][live]
    kc.transpose(1, 2)[at // page, at % page] = rotated(s["k"])[live]
    vc.transpose(1, 2)[at // page, at % page] = s["v"].double()[live]
    return {"q": rotated(s["q"]), "k_cache": kc, "v_cache": vc}


def _exact_attention(case, s):
    kv, d, page = case["kv"], case["d"], case["page"]
    group = case["heads"] // kv
    outs, lses = [], []
    start = s["q_start"].tolist()
    for b, length in enumerate(s["kv_len"].tolist()):
        rows = slice(start[b], start[b + 1])
        t = start[b + 1] - start[b]
        pages = s["table"][b, : -(-length // page)].long()
        k, v = (x[pages].transpose(0, 1).reshape(kv, -1, d)[:, :length].double() for x in (s["k_cache"], s["v_cache"]))
        q = s["q"][rows].double().reshape(t, kv, group, d)
        a = torch.einsum("tkgd,kpd->ktgp", q, k) * s["scale"]
        words = [m % (1 << 64) for m in s["mask"][rows].tolist()]
        own_nodes = torch.tensor([[bool(w >> j & 1) for j in range(t)] for w in words], device=DEV)
        a[..., length - t:].masked_fill_(~own_nodes[None, :, None, :], -math.inf)
        lse = torch.logsumexp(a, -1)
        outs.append(torch.einsum("ktgp,kpd->tkgd", torch.exp(a - lse[..., None]), v).reshape(t, kv * group, d))
        lses.append(lse.permute(1, 0, 2).reshape(t, kv * group))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_sample(s):
    """The kept sets and tokens from the integer weights (fp64 arithmetic, rounded to fp32 where the definition rounds), row by
    row; the log-probability then from the true exponentials of the kept logits."""
    r32 = lambda v: v.float().double()  # noqa: E731
    result = []
    for i in range(s["logits"].shape[0]):
        x = s["logits"][i].double()
        temp, k = float(s["temperature"][i]), int(s["top_k"][i])
        order = torch.argsort(-x, stable=True)
        if not temp > 0:
            result.append(0.0)
            continue
        gap = r32(x - x[order[0]])
        y = r32(gap * float(torch.tensor(1.4426950408889634).div(s["temperature"][i].cpu()))).clamp(min=-64.0)
        whole = y.round()
        f = y - whole
        p = torch.full_like(f, EXP2[0])
        for coef in EXP2[1:]:
            p = r32(r32(p * f) + coef)
        w = torch.round(torch.ldexp(p, whole + 31)).long()
        if k > 0:
            w[order[k:]] = 0
        total = int(w.sum())
        p_part = int(float(s["top_p"][i]) * 2 ** 31)
        if p_part < 1 << 31:
            ranked = w[order]
            keep = int((ranked.cumsum(0) - ranked < (total * p_part >> 31)).sum())
            w[order[max(keep, 1):]] = 0
        w[w < int(float(s["min_p"][i]) * 2 ** 31)] = 0
        goal = int(w.sum()) * min(int(float(s["u"][i]) * 2 ** 31), (1 << 31) - 1) >> 31
        token = int(torch.searchsorted(w.cumsum(0), goal, right=True))
        kept = torch.where(w > 0, (x - x[order[0]]) / temp, -math.inf)
        result.append(float(kept[token] - torch.logsumexp(kept, 0)))
    return {"token": None, "logprob": torch.tensor(result, dtype=torch.float64), "n_kept": None}
