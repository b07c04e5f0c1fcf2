"""64-bit references of the decode-step operators, written from their definitions in include/ctr_decode.h (numpy, and
torch in fp64 for the long sums)."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # largest relative rounding error of a normal number
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half the smallest subnormal


def paged_cache(pages, kv, page, d, dtype, gen, order="phtd", device="cuda"):
    """k, v [pages, kv, page, d] of random values; `order`: how the dimensions lie in memory (d last)."""
    sizes = {"p": pages, "h": kv, "t": page}
    out = []
    for _ in range(2):
        x = torch.randn([sizes[c] for c in order[:3]] + [d], device=device, generator=gen).to(dtype)
        out.append(x.permute([order.index(c) for c in "pht"] + [3]))
    return out


# ---------------------------------------------------------------- append
def rotated(x, positions, turns, interleaved, scale):
    """fp64 rotation of [n, heads, d] (numpy), and per element |x| + |y| of its pair."""
    x = x.astype(np.float64)
    half = len(turns)
    words = [int(t) % (1 << 64) for t in turns]
    phi = np.array([[2 * math.pi * ((int(p) * w) % (1 << 64)) / 2.0 ** 64 for w in words] for p in positions]).reshape(len(positions), half)
    c, s = scale * np.cos(phi)[:, None, :], scale * np.sin(phi)[:, None, :]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out, size = x.copy(), np.zeros_like(x)
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out, size


# ---------------------------------------------------------------- attention
def attention(q, kc, vc, q_start, kv_len, table, mask, scale):
    """(out, lse, and the two tolerances) in fp64, row by row of each sequence.

    Tolerances: a score is a sum of d products in fp32, so off by at most (d + 4) 2^-24 sum |q k| scale =: e, which moves a
    probability by that relative amount; a probability is rounded to the dtype (unit u; in fp16 at least 2^-25 of the
    largest) and the sums run in fp32 with an exponential good to 2^-21: 2^-18 covers both.  So
    |out - exact| <= (u + 2 e + 2^-18) sum p |v| [+ floor] + u |out|,  |lse - exact| <= e + 2^-20 max(1, |lse|)."""
    kv, page, d = kc.shape[1], kc.shape[2], kc.shape[3]
    heads = q.shape[1]
    group = heads // kv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    ltol = torch.zeros_like(lse)
    u = UNIT[q.dtype]
    for b, length in enumerate(kv_len.tolist()):
        r0, r1 = int(q_start[b]), int(q_start[b + 1])
        t = r1 - r0
        if t == 0 or length == 0:
            continue
        pages = table[b, : -(-length // page)].long()
        k, v = (x[pages].transpose(0, 1).reshape(kv, -1, d)[:, :length].double() for x in (kc, vc))
        seen = torch.ones(t, length, dtype=torch.bool, device=q.device)
        for i in range(t):
            word = ((1 << (i + 1)) - 1) if mask is None else int(mask[r0 + i]) % (1 << 64)
            for j in range(t):
                if length - t + j >= 0:
                    seen[i, length - t + j] = bool(word >> j & 1)
        qq = q[r0:r1].double().reshape(t, kv, group, d)
        clean_k = torch.where(torch.isfinite(k), k, 0.0)
        a = torch.einsum("tkgd,kpd->tkgp", qq, k) * scale
        size = torch.einsum("tkgd,kpd->tkgp", qq.abs(), clean_k.abs()) * abs(scale)
        a = torch.where(seen[:, None, None, :], a, -math.inf)
        size = torch.where(seen[:, None, None, :], size, 0.0)
        live = seen.any(1)
        top = a.amax(-1)
        top = torch.where(torch.isfinite(top), top, 0.0)
        p = torch.exp(a - top[..., None])
        total = p.sum(-1)
        e = size.amax(-1) * (d + 4) * 2.0 ** -24
        # value rows that a query does not attend to have no part, whatever they hold
        vv = torch.where(torch.isfinite(v), v, 0.0)
        o = torch.einsum("tkgp,kpd->tkgd", p, vv) / torch.where(total > 0, total, 1.0)[..., None]
        if not torch.isfinite(v).all():
            for i in range(t):  # one that it does attend to makes that dimension NaN or infinite
                w = torch.where(seen[i][None, :, None], v, 0.0)
                bad = ~torch.isfinite(w).all(1)
                plain = torch.einsum("kgp,kpd->kgd", p[i], w) / total[i][..., None]
                o[i] = torch.where(bad[:, None, :].expand(-1, group, -1), plain, o[i])
        share = torch.einsum("tkgp,kpd->tkgd", p, vv.abs()) / torch.where(total > 0, total, 1.0)[..., None]
        floor = 0.0
        if q.dtype == torch.float16:
            floor = 2.0 ** -25 * torch.einsum("tp,kpd->tkd", seen.double(), vv.abs())[:, :, None, :] / total.clamp(min=1e-300)[..., None]
        out[r0:r1] = o.reshape(t, heads, d)
        tol[r0:r1] = ((u + 2 * e[..., None] + 2.0 ** -18) * share + floor + u * o.abs() + TINY[q.dtype]).reshape(t, heads, d)
        ll = torch.where(live[:, None, None], top + torch.log(total), -math.inf)
        lse[r0:r1] = ll.reshape(t, heads)
        ltol[r0:r1] = (e + 2.0 ** -20 * ll.abs().clamp(min=1.0)).reshape(t, heads)
    return out, lse, tol, ltol


# ---------------------------------------------------------------- sampling
def weights(x, temperature):
    """Integer weights (python ints in an object-free int64 array) of one row of fp32 logits; numpy rounds every fp32 step."""
    x = np.asarray(x, np.float32)
    x = np.where(np.isnan(x), np.float32(-np.inf), x)
    top = x.max()
    with np.errstate(all="ignore"):
        rate = np.minimum(np.float32(1.4426950408889634) / np.float32(temperature), np.float32(3e38)) if temperature > 0 else np.float32(1)
        y = np.where(x == top, np.float32(0), (x - top) * rate)
        y = np.fmax(y, np.float32(-64)).astype(np.float32)
    k = np.rint(y)
    f = (y - k).astype(np.float32)
    p = np.full_like(f, np.float32(float.fromhex("0x1.5bba14p-10")))
    for h in ("0x1.3cea88p-7", "0x1.c6b752p-5", "0x1.ebf9bcp-3", "0x1.62e42ap-1", "0x1p+0"):
        p = (p * f).astype(np.float32) + np.float32(float.fromhex(h))
    w = np.rint(np.ldexp(p.astype(np.float64), k.astype(np.int64) + 31)).astype(np.int64)
    return np.where(x > -np.inf, w, 0)


def sample_row(x, temperature, top_k, top_p, min_p, u):
    """(token, logprob, n_kept) of one row, in integers."""
    x = np.asarray(x, np.float32)
    x = np.where(np.isnan(x), np.float32(-np.inf), x)
    if not (x > -np.inf).any():
        return -1, -math.inf, 0
    greedy = not temperature > 0
    w = weights(x, temperature)
    order = np.argsort(-x.astype(np.float64), kind="stable")
    k = 1 if greedy else top_k if top_k > 0 else len(x)
    w[order[k:]] = 0
    if not greedy and top_p < 1:
        goal = int(w.sum()) * int(max(float(np.float32(top_p)), 0.0) * 2 ** 31) >> 31
        ranked = w[order]
        keep = max(1, int((np.cumsum(ranked) - ranked < goal).sum()))
        w[order[keep:]] = 0
    if min_p > 0:
        w[w < int(min(float(np.float32(min_p)), 1.0) * 2 ** 31)] = 0
    total = int(w.sum())
    goal = total * min(int(max(float(np.float32(u)), 0.0) * 2 ** 31), (1 << 31) - 1) >> 31
    token = int(np.searchsorted(np.cumsum(w), goal, side="right"))
    return token, math.log(int(w[token]) / total), int((w > 0).sum())
