"""ctr_tree_attention against the softmax in 64 bits; the tolerances are derived in decodeutil.attention."""
import math

import numpy as np
import pytest
import torch

from decodeutil import attention, paged_cache
from gpuutil import need_gpu

pytestmark = pytest.mark.gpu


def _tree(new, rng, back=6):
    words = []
    for n in new:
        row = []
        for i in range(n):
            parent = i - int(rng.integers(1, back + 1))
            row.append((row[parent] if parent >= 0 else 0) | 1 << i)
        words += row
    return words


def _case(heads, kv, d, dtype, page, ctx, new, mask="tree", order="phtd", q_scale=1.5, seed=0, spare=0):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = [c + n for c, n in zip(ctx, new)]
    need = [-(-x // page) for x in lens]
    pages = sum(need) + 2
    kc, vc = paged_cache(pages, kv, page, d, dtype, g, order)
    perm = rng.permutation(pages)
    width = max(max(need), 1) + spare
    table = np.full((len(new), width), -7, np.int32)  # entries past a sequence are never read
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    rows = sum(new)
    q = (q_scale * torch.randn(rows, heads, d, device="cuda", generator=g)).to(dtype)
    words = None
    if mask == "tree":
        words = _tree(new, rng)
    elif mask == "random":
        words = [int(rng.integers(0, 1 << 63)) * 2 + int(rng.integers(0, 2)) for _ in range(rows)]
    elif mask == "none":
        words = [0] * rows
    tm = None if words is None else torch.tensor([w - (1 << 64) if w >= 1 << 63 else w for w in words], dtype=torch.int64, device="cuda")
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    return dict(q=q, kc=kc, vc=vc, start=start, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                table=torch.from_numpy(table).to("cuda"), mask=tm, max_nodes=max(max(new), 1), scale=d ** -0.5)


def _run(ctr, c, out=None, stream=None, lse=True):
    cache = ctr.KvCache(c["kc"], c["vc"])
    ws = ctr.attention_workspace(cache, c["q"].shape[1], c["lens"].numel(), c["max_nodes"])
    ws.fill_(0xA5)  # its contents need no initialisation
    out = torch.full_like(c["q"], 9.0) if out is None else out
    l = torch.full(c["q"].shape[:2], 9.0, device="cuda") if lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    ctr.ctr_tree_attention(cache, c["q"], c["start"], c["lens"], c["table"], out, ws, max_nodes=c["max_nodes"], tree_mask=c["mask"],
                           lse=l, scale=c["scale"], status=status, stream=stream)
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    return out, l


def _check(ctr, c, **kw):
    out, lse = _run(ctr, c, **kw)
    want, wl, tol, ltol = attention(c["q"], c["kc"], c["vc"], c["start"], c["lens"], c["table"], c["mask"], c["scale"])
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out), fin)
    over = ((out.double() - want).abs() - tol)[fin]
    assert over.numel() == 0 or float(over.max()) <= 0, float(over.max())
    if lse is not None:
        some = torch.isfinite(wl)
        assert torch.equal(lse == -math.inf, wl == -math.inf)
        over = ((lse.double() - wl).abs() - ltol)[some]
        assert over.numel() == 0 or float(over.max()) <= 0, float(over.max())
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(16, 2), (8, 8), (7, 1), (5, 5), (28, 4), (64, 1), (32, 8), (48, 2)])
def test_single_tokens(heads, kv, d, dtype):
    ctr = need_gpu()
    _check(ctr, _case(heads, kv, d, dtype, 16, [0, 1, 15, 16, 17, 63, 130, 700], [1] * 8, mask=None, seed=heads + d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_trees(group, page, d, dtype):
    ctr = need_gpu()
    _check(ctr, _case(2 * group, 2, d, dtype, page, [0, 1, 127, 128, 129, 500, 2000], [1, 2, 5, 16, 31, 33, 64], seed=page + group))


@pytest.mark.parametrize("nodes", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 32, 33, 63, 64])
@pytest.mark.parametrize("group", [1, 2, 4, 5, 8, 16])
def test_row_counts_of_a_kv_head(nodes, group):
    """group x nodes rows share a KV head: every tile height and its edges."""
    ctr = need_gpu()
    _check(ctr, _case(group, 1, 128, torch.bfloat16, 64, [300, 1], [nodes, nodes], mask="random", seed=nodes + group))


@pytest.mark.parametrize("mask", [None, "tree", "random", "none"])
@pytest.mark.parametrize("ctx", [0, 3, 200])
def test_masks(mask, ctx):
    """`none` with no context leaves every row empty; `random` leaves some."""
    ctr = need_gpu()
    for nodes in (1, 6, 40):
        _check(ctr, _case(8, 2, 64, torch.bfloat16, 16, [ctx, 0, ctx], [nodes, 1, nodes], mask=mask, seed=ctx))


@pytest.mark.parametrize("heads,kv,nodes", [(16, 2, 1), (16, 2, 8), (32, 2, 48)])
@pytest.mark.parametrize("ctx", [4096, 20_011, 100_003])
def test_long_axis_in_parts(ctx, heads, kv, nodes):
    ctr = need_gpu()
    _check(ctr, _case(heads, kv, 128, torch.bfloat16, 64, [ctx, 5, ctx // 3], [nodes, 1, nodes], seed=ctx))


@pytest.mark.parametrize("nodes", [1, 4, 24])
def test_many_ragged_sequences(nodes):
    ctr = need_gpu()
    rng = np.random.default_rng(7)
    b = 150
    ctx = [int(x) for x in np.exp(rng.uniform(0, 7.5, b))]
    new = [int(x) for x in rng.integers(0, nodes + 1, b)]  # some sequences bring nothing
    new[3] = nodes
    _check(ctr, _case(8, 4, 64, torch.float16, 32, ctx, new, seed=nodes, spare=3))


@pytest.mark.parametrize("order", ["phtd", "pthd", "htpd", "thpd"])
def test_cache_layouts(order):
    ctr = need_gpu()
    for nodes in (1, 48):
        _check(ctr, _case(8, 4, 128, torch.bfloat16, 32, [200, 77], [nodes, nodes], order=order))


def test_strided_rows_and_outputs():
    ctr = need_gpu()
    for nodes in (1, 40):
        c = _case(8, 2, 64, torch.bfloat16, 16, [100, 300], [nodes, nodes])
        want, _ = _run(ctr, c)
        wide = torch.randn(c["q"].shape[0], 14, 72, device="cuda").bfloat16()
        wide[:, 2:10, :64] = c["q"]
        out = torch.zeros(8, c["q"].shape[0], 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
        got, _ = _run(ctr, dict(c, q=wide[:, 2:10, :64]), out=out)
        assert torch.equal(got, want)


@pytest.mark.parametrize("heads,nodes", [(4, 1), (4, 3), (4, 30)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_attended_has_no_part(bad, heads, nodes):
    """Slots past a sequence's end, unused pages and new tokens outside a row's mask may hold anything."""
    ctr = need_gpu()
    c = _case(heads, 1, 128, torch.bfloat16, 64, [130, 61, 0], [nodes, nodes, nodes], seed=3)
    want, wl = _run(ctr, c)
    used = torch.zeros(c["kc"].shape[0], 64, dtype=torch.bool, device="cuda")
    for b, n in enumerate(c["lens"].tolist()):
        for p in range(n):
            used[int(c["table"][b, p // 64]), p % 64] = True
    for cache in (c["kc"], c["vc"]):
        cache.permute(0, 2, 1, 3)[~used] = bad
    got, gl = _run(ctr, c)
    assert torch.equal(got, want) and torch.equal(gl, wl)
    if nodes > 1:  # the last new token of sequence 0 is seen by itself only
        p = int(c["lens"][0]) - 1
        c["vc"][int(c["table"][0, p // 64]), 0, p % 64, 5] = bad
        c["mask"][:nodes - 1] &= ~(1 << (nodes - 1))
        c["mask"][nodes - 1] |= 1 << (nodes - 1)
        out, _ = _check(ctr, c)
        assert torch.isfinite(out[:nodes - 1]).all() and not torch.isfinite(out[nodes - 1, :, 5]).any()


@pytest.mark.parametrize("nodes", [1, 48])
def test_scores_of_any_size(nodes):
    """Scores in the thousands (one key takes all) and maxima that grow along the sequence."""
    ctr = need_gpu()
    _check(ctr, _case(8, 2, 64, torch.bfloat16, 16, [500, 40], [nodes, nodes], q_scale=300.0, seed=1))
    c = _case(8, 2, 64, torch.bfloat16, 16, [900, 300], [nodes, nodes], seed=2)
    for b, n in enumerate(c["lens"].tolist()):
        for p in range(n):
            c["kc"][int(c["table"][b, p // 16]), :, p % 16] *= 8.0 * p / n
    _check(ctr, c)


def test_zero_and_negative_scale():
    ctr = need_gpu()
    for nodes in (1, 40):
        for scale in (0.0, -0.125):
            c = _case(8, 2, 64, torch.float16, 16, [100, 17], [nodes, nodes])
            _check(ctr, dict(c, scale=scale))


def test_lengths_outside_the_table_are_held_to_it():
    ctr = need_gpu()
    c = _case(4, 2, 64, torch.bfloat16, 16, [30, 30], [1, 1], mask=None)
    c["lens"] = torch.tensor([48, -3], dtype=torch.int32, device="cuda")
    c["table"] = c["table"][:, :3].contiguous().clamp(min=0)
    out, lse = _run(ctr, dict(c, lens=torch.tensor([1 << 30, -3], dtype=torch.int32, device="cuda")))
    want, wl = _run(ctr, dict(c, lens=torch.tensor([c["table"].shape[1] * 16, 0], dtype=torch.int32, device="cuda")))
    assert torch.isfinite(out).all() and torch.equal(out[1], want[1]) and float(lse[1].max()) == -math.inf
    assert (out[1] == 0).all()


def test_pages_outside_the_cache_read_as_zeros():
    ctr = need_gpu()
    for nodes in (1, 40):
        c = _case(4, 2, 64, torch.bfloat16, 16, [100], [nodes], mask="tree")
        gone = int(c["table"][0, 2])
        for cache in (c["kc"], c["vc"]):
            cache[gone] = 0
        want, wl = _run(ctr, c)
        for bad in (c["kc"].shape[0], 1 << 30, -1):
            c["table"][0, 2] = bad
            got, gl = _run(ctr, c)
            assert torch.equal(got, want) and torch.equal(gl, wl)


def test_same_call_twice_gives_the_same_bits():
    ctr = need_gpu()
    for heads, kv, nodes in ((16, 2, 1), (32, 4, 64)):
        c = _case(heads, kv, 128, torch.bfloat16, 32, [30_000, 100, 9000], [nodes] * 3, seed=9)
        first = _run(ctr, c)
        for _ in range(5):
            again = _run(ctr, c)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_offsets_past_32_bits():
    ctr = need_gpu()
    for nodes in (1, 40):
        c = _case(4, 2, 128, torch.bfloat16, 1024, [1500], [nodes], seed=4)
        want, _ = _run(ctr, c)
        pages = (1 << 33) // (2 * 1024 * 128) // 2 + 4
        kc = torch.zeros(pages, 2, 1024, 128, dtype=torch.bfloat16, device="cuda")
        vc = torch.zeros_like(kc)
        table = torch.empty_like(c["table"])
        for i in range(c["table"].shape[1]):
            kc[pages - 1 - i], vc[pages - 1 - i] = c["kc"][int(c["table"][0, i])], c["vc"][int(c["table"][0, i])]
            table[0, i] = pages - 1 - i
        got, _ = _run(ctr, dict(c, kc=kc, vc=vc, table=table))
        assert torch.equal(got, want)
        del kc, vc


def test_without_lse_on_another_stream_and_in_a_graph():
    ctr = need_gpu()
    for nodes in (1, 40):
        c = _case(8, 2, 128, torch.bfloat16, 64, [5000, 30], [nodes, nodes])
        want, _ = _run(ctr, c)
        got, _ = _run(ctr, c, stream=torch.cuda.Stream(), lse=False)
        assert torch.equal(got, want)
        cache = ctr.KvCache(c["kc"], c["vc"])
        ws = ctr.attention_workspace(cache, 8, 2, nodes)
        out = torch.zeros_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctr.ctr_tree_attention(cache, c["q"], c["start"], c["lens"], c["table"], out, ws, max_nodes=nodes, tree_mask=c["mask"],
                                   scale=c["scale"])
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
