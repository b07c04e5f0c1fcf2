"""ctr_kv_append against the rotation in 64 bits: a result may be off by the rounding to its type and by the fp32 steps
before it (angle within 2^-22, two products and a sum: 2^-20 of |x| + |y|)."""
import math

import numpy as np
import pytest
import torch

from decodeutil import TINY, UNIT, paged_cache, rotated
from gpuutil import need_gpu

pytestmark = pytest.mark.gpu


def _turns(half, base=10000.0):
    words = [int(base ** (-i / max(half, 1)) / (2 * math.pi) * 2.0 ** 64) for i in range(half)]
    return torch.tensor([w - (1 << 64) if w >= 1 << 63 else w for w in words], dtype=torch.int64, device="cuda")


def _check(ctr, n, heads, kv, d, rot, inter, dtype, page, order="phtd", scale=1.0, pad=0.0, offset=0, in_place=False,
           positions=None, seed=0, head_major=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = -(-max(n, 1) // page) + 2
    kc, vc = paged_cache(pages, kv, page, d, dtype, g, order)
    k0, v0 = kc.clone(), vc.clone()
    total = heads + 2 * kv
    buf = torch.randn(n * total * d + offset, device="cuda", generator=g).to(dtype)[offset:]
    qkv = buf.view(total, n, d).transpose(0, 1) if head_major else buf.view(n, total, d)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:n]
    if pad:
        slots = torch.where(torch.rand(n, device="cuda", generator=g) < pad, -1 - slots, slots)
    if positions is None:
        positions = torch.randint(0, 200_000, (n,), device="cuda", generator=g)
    turns = _turns(rot // 2)
    want_q, size_q = rotated(q.float().cpu().numpy(), positions.tolist(), turns.tolist(), inter, scale)
    want_k, size_k = rotated(k.float().cpu().numpy(), positions.tolist(), turns.tolist(), inter, scale)
    v_in = v.clone()
    q_out = q if in_place else torch.full((n, heads, d), 7.0, device="cuda").to(dtype)
    ctr.ctr_kv_append(ctr.KvCache(kc, vc), ctr.Rope(turns, inter, scale), q, k, v, positions, slots, q_out)
    torch.cuda.synchronize()

    def near(got, want, size):
        tol = UNIT[dtype] * np.abs(want) + 2.0 ** -20 * size + TINY[dtype]
        err = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
        assert (err <= tol).all(), float((err - tol).max())

    near(q_out, want_q, size_q)
    live = (slots >= 0).nonzero()[:, 0]
    at, off = slots[live] // page, slots[live] % page
    near(kc[at, :, off], want_k[live.cpu().numpy()], size_k[live.cpu().numpy()])
    assert torch.equal(vc[at, :, off], v_in[live])
    k0[at, :, off], v0[at, :, off] = kc[at, :, off], vc[at, :, off]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)  # nothing else was written


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (80, 80), (80, 40), (96, 96), (256, 256), (256, 64),
                                   (8, 8), (8, 2), (24, 6), (128, 0), (248, 246), (160, 16)])
def test_heads_and_rotated_parts(d, rot, inter, dtype):
    ctr = need_gpu()
    _check(ctr, 37, 6, 2, d, rot, inter, dtype, 16, seed=d + rot)


@pytest.mark.parametrize("n", [0, 1, 2, 3, 31, 257, 5003])
@pytest.mark.parametrize("heads,kv", [(1, 1), (16, 2), (7, 1), (40, 8), (0, 3)])
def test_token_counts_and_head_layouts(n, heads, kv):
    ctr = need_gpu()
    _check(ctr, n, heads, kv, 128, 128, False, torch.bfloat16, 32, seed=n + heads, pad=0.2)


@pytest.mark.parametrize("order", ["phtd", "pthd", "htpd", "thpd"])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_cache_layouts(order, page):
    ctr = need_gpu()
    _check(ctr, 130, 8, 4, 64, 64, True, torch.float16, page, order=order, seed=page)


@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("head_major", [False, True])
def test_views_and_alignment(offset, head_major):
    ctr = need_gpu()
    for inter in (False, True):
        _check(ctr, 65, 8, 2, 64, 64, inter, torch.bfloat16, 16, offset=offset, head_major=head_major, seed=5)


@pytest.mark.parametrize("inter", [False, True])
def test_in_place_and_scaled(inter):
    ctr = need_gpu()
    _check(ctr, 33, 8, 2, 128, 128, inter, torch.bfloat16, 16, in_place=True, scale=1.2079441541679836)


def test_far_positions():
    """The angle of a position past 2^32, and of a negative one, is as good as a near one's."""
    ctr = need_gpu()
    p = torch.tensor([0, 1, (1 << 24) + 1, (1 << 32) + 7, (1 << 40) + 3, (1 << 62) + 1, -1, -12345], device="cuda")
    _check(ctr, 8, 4, 2, 128, 128, False, torch.float16, 16, positions=p)


def test_slots_outside_the_cache_write_nothing():
    ctr = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    kc, vc = paged_cache(3, 2, 16, 64, torch.bfloat16, g)
    k0, v0 = kc.clone(), vc.clone()
    q = torch.randn(5, 4, 64, device="cuda", generator=g).bfloat16()
    k = torch.randn(5, 2, 64, device="cuda", generator=g).bfloat16()
    slots = torch.tensor([48, 1 << 40, -1, -(1 << 62), (1 << 63) - 1], device="cuda")
    out = torch.zeros_like(q)
    ctr.ctr_kv_append(ctr.KvCache(kc, vc), ctr.Rope(_turns(32)), q, k, k, torch.zeros(5, dtype=torch.int64, device="cuda"), slots, out)
    torch.cuda.synchronize()
    assert torch.equal(kc, k0) and torch.equal(vc, v0) and torch.equal(out, q)  # position 0 turns nothing


def test_a_cache_past_32_bit_offsets():
    """A token whose element offset in the cache is above 2^32."""
    ctr = need_gpu()
    pages = 2 * (1 << 32) // (1 * 1024 * 128) + 8
    kc = torch.zeros(pages, 1, 1024, 128, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    g = torch.Generator(device="cuda").manual_seed(2)
    k = torch.randn(2, 1, 128, device="cuda", generator=g).bfloat16()
    slots = torch.tensor([pages * 1024 - 1, (pages // 2) * 1024 + 3], device="cuda")
    q = torch.zeros(2, 0, 128, dtype=torch.bfloat16, device="cuda")
    ctr.ctr_kv_append(ctr.KvCache(kc, vc), ctr.Rope(_turns(64)), q, k, k, torch.zeros(2, dtype=torch.int64, device="cuda"), slots, q)
    torch.cuda.synchronize()
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(kc[s // 1024, 0, s % 1024], k[i, 0]) and torch.equal(vc[s // 1024, 0, s % 1024], k[i, 0])
    assert int((kc != 0).sum()) == int((k != 0).sum())


def test_non_finite_values_stay_in_their_pair():
    ctr = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(3)
    kc, vc = paged_cache(1, 1, 16, 64, torch.bfloat16, g)
    k = torch.randn(1, 1, 64, device="cuda", generator=g).bfloat16()
    k[0, 0, 3] = math.nan
    k[0, 0, 40] = math.inf
    pos = torch.tensor([11], device="cuda")
    ctr.ctr_kv_append(ctr.KvCache(kc, vc), ctr.Rope(_turns(32)), k, k, k, pos, torch.tensor([5], device="cuda"), torch.empty_like(k))
    got = kc[0, 0, 5].float()
    bad = ~torch.isfinite(got)
    assert bad.nonzero()[:, 0].tolist() == [3, 8, 35, 40]


def test_on_another_stream_and_in_a_graph():
    ctr = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(4)
    kc, vc = paged_cache(2, 2, 16, 64, torch.bfloat16, g)
    cache, rope = ctr.KvCache(kc, vc), ctr.Rope(_turns(32))
    q = torch.randn(3, 4, 64, device="cuda", generator=g).bfloat16()
    k = torch.randn(3, 2, 64, device="cuda", generator=g).bfloat16()
    pos, slots = torch.tensor([5, 6, 7], device="cuda"), torch.tensor([1, 20, 31], device="cuda")
    want = torch.empty_like(q)
    ctr.ctr_kv_append(cache, rope, q, k, k, pos, slots, want)
    torch.cuda.synchronize()
    kc_want = kc.clone()
    kc.zero_()
    side, out = torch.cuda.Stream(), torch.zeros_like(q)
    side.wait_stream(torch.cuda.current_stream())
    ctr.ctr_kv_append(cache, rope, q, k, k, pos, slots, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctr.ctr_kv_append(cache, rope, q, k, k, pos, slots, out)
    out.zero_()
    kc.copy_(kc_want * 0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(kc[0, :, 1], kc_want[0, :, 1])
