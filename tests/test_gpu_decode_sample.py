"""ctr_sample against the definition in integers: tokens and kept counts are equal, the log-probability is the fp32
rounding of one computed in 64 bits (2^-23 relative)."""
import math

import numpy as np
import pytest
import torch

from decodeutil import sample_row
from gpuutil import need_gpu

pytestmark = pytest.mark.gpu


def _run(ctr, logits, temperature, top_k=None, top_p=None, min_p=None, u=None, stream=None):
    n = logits.shape[0]

    def vec(x, dt):
        return None if x is None else torch.as_tensor(np.broadcast_to(np.asarray(x), (n,)).copy()).to(dt).to("cuda")
    t = dict(token=torch.full((n,), -9, dtype=torch.int32, device="cuda"), logprob=torch.full((n,), 9.0, device="cuda"),
             n_kept=torch.full((n,), -9, dtype=torch.int32, device="cuda"))
    args = dict(top_k=vec(top_k, torch.int32), top_p=vec(top_p, torch.float32), min_p=vec(min_p, torch.float32))
    tt, uu = vec(temperature, torch.float32), vec(u, torch.float32)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    ctr.ctr_sample(logits, tt, uu, t["token"], stream=stream, **args, **{k: t[k] for k in ("logprob", "n_kept")})
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in t.items()}


def _check(ctr, logits, temperature, top_k=0, top_p=1.0, min_p=0.0, u=0.5):
    n = logits.shape[0]
    got = _run(ctr, logits, temperature, top_k, top_p, min_p, u)
    x = logits.float().cpu().numpy()
    col = [np.broadcast_to(np.asarray(a), (n,)) for a in (temperature, top_k, top_p, min_p, u)]
    for r in range(n):
        token, lp, kept = sample_row(x[r], float(np.float32(col[0][r])), int(col[1][r]), *(float(np.float32(c[r])) for c in col[2:]))
        assert (int(got["token"][r]), int(got["n_kept"][r])) == (token, kept), (r, got["token"][r], token, got["n_kept"][r], kept)
        if math.isfinite(lp):
            assert abs(float(got["logprob"][r]) - lp) <= 2.0 ** -23 * abs(lp) + 1e-30, (r, got["logprob"][r], lp)
        else:
            assert float(got["logprob"][r]) == lp
    return got


def _logits(n, vocab, dtype, seed, bulk=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = bulk * torch.randn(n, vocab, device="cuda", generator=g)
    at = torch.randint(0, vocab, (n, 20), device="cuda", generator=g)
    x.scatter_(1, at, 10 - 0.4 * torch.arange(20, device="cuda").expand(n, 20) + torch.randn(n, 20, device="cuda", generator=g))
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [1, 2, 31, 1000, 4096, 32_000, 50_021, 131_072, 262_144])
def test_every_setting(vocab, dtype):
    ctr = need_gpu()
    n = 24
    rng = np.random.default_rng(vocab)
    x = _logits(n, vocab, dtype, vocab)
    k = rng.choice([0, 0, 1, 2, 5, 50, 100, 500, 1000, 5000], n)
    p = rng.choice([1.0, 1.0, 0.0, 0.05, 0.5, 0.9, 0.95, 0.999], n)
    m = rng.choice([0.0, 0.0, 0.01, 0.1, 1.0], n)
    t = rng.choice([0.0, 0.3, 0.7, 1.0, 1.5], n)
    _check(ctr, x, t, k, p, m, rng.random(n).astype(np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.9), (0, 0.3), (1, 1.0), (7, 1.0), (1024, 0.99), (3000, 1.0), (40_000, 0.97)])
def test_flat_rows(k, p, dtype):
    """Rows without peaks: the kept set is most of the vocabulary, with ties across it in bf16."""
    ctr = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(k)
    x = (0.1 * torch.randn(6, 32_003, device="cuda", generator=g)).to(dtype)
    _check(ctr, x, 1.0, k, p, 0.0, np.linspace(0, 0.999, 6))


@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.5), (1, 1.0), (100, 0.7), (2000, 1.0), (2999, 0.5)])
@pytest.mark.parametrize("level", [0.0, -0.0, -1e30, 65504.0])
def test_all_equal(level, k, p):
    """One tie over the whole row: the lowest indices are kept."""
    ctr = need_gpu()
    x = torch.full((4, 3000), level, device="cuda")
    if level == 0.0:
        x[:, ::3] = -0.0  # equal to 0
    _check(ctr, x, 0.8, k, p, 0.0, [0.0, 0.3, 0.7, 1 - 2.0 ** -24])


def test_ties_at_every_cut():
    ctr = need_gpu()
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.integers(0, 6, (40, 5000)).astype(np.float32)).to("cuda")
    _check(ctr, x, rng.uniform(0.2, 2, 40), rng.integers(0, 3000, 40), rng.uniform(0.1, 1.05, 40), 0.0, rng.random(40))


def test_masked_and_empty_rows():
    """-inf, the type's lowest value and NaN as masks; rows with nothing left, and with one token left."""
    ctr = need_gpu()
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for mask in (-math.inf, torch.finfo(dtype).min, math.nan):
            x = _logits(6, 20_000, dtype, 3)
            x[1] = mask
            x[2, :19_999] = mask
            x[3, 1:] = mask
            x[4, ::2] = mask
            x[5, 10_000:] = mask
            _check(ctr, x, 0.9, [0, 0, 0, 5, 50, 0], [0.9, 0.9, 0.9, 1.0, 0.8, 1.0], 0.0, [0.1, 0.5, 0.9, 0.2, 0.7, 0.99])


def test_infinite_logits():
    ctr = need_gpu()
    x = _logits(3, 5000, torch.float32, 8)
    x[0, 77] = math.inf
    x[1, [5, 900]] = math.inf
    _check(ctr, x, [0.7, 0.7, 0.0], [0, 0, 0], [0.9, 1.0, 1.0], 0.0, [0.4, 0.75, 0.2])


@pytest.mark.parametrize("temperature", [0.0, -1.0, math.nan, 1e-30, 1e-42, 0.01, 100.0, 1e30, math.inf])
def test_temperatures(temperature):
    ctr = need_gpu()
    x = _logits(5, 9001, torch.float32, 2)
    x[1, 44] = -math.inf
    _check(ctr, x, temperature, [0, 0, 40, 0, 0], [1.0, 0.9, 1.0, 0.5, 1.0], [0, 0, 0, 0, 0.2], [0.0, 0.3, 0.5, 0.7, 0.9999])


@pytest.mark.parametrize("u", [0.0, 2.0 ** -31, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, -1.0])
def test_uniforms_at_their_ends(u):
    ctr = need_gpu()
    _check(ctr, _logits(4, 3001, torch.bfloat16, 6), 1.0, [0, 10, 0, 0], [1.0, 1.0, 0.9, 0.1], 0.0, u)


def test_frequencies():
    """2^16 draws of one row: counts within 5 standard deviations of the softmax's probabilities."""
    ctr = need_gpu()
    n = 1 << 16
    row = _logits(1, 40, torch.float32, 1, bulk=1.0)
    u = (np.arange(n) + 0.5) / n
    got = _run(ctr, row.expand(n, 40).contiguous(), 1.3, None, None, None, np.random.default_rng(0).permutation(u))
    prob = torch.softmax(row[0].double() / 1.3, 0).cpu().numpy()
    counts = np.bincount(got["token"], minlength=40)
    assert np.all(np.abs(counts - n * prob) <= 5 * np.sqrt(n * prob * (1 - prob)) + 1)
    assert np.allclose(got["logprob"], np.log(prob)[got["token"]], atol=1e-6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,stride", [(0, 8192), (1, 8193), (3, 8200), (8, 8192)])
def test_strides_and_alignment(offset, stride, dtype):
    ctr = need_gpu()
    buf = _logits(1, 9 * stride + 16, dtype, 4)[0]
    x = buf[offset:offset + 9 * stride].view(9, stride)[:, :8191]
    _check(ctr, x, 0.8, [0, 3, 50, 0, 0, 200, 0, 0, 1500], [1, 1, .9, .9, .5, 1, .99, 1, 1], [0, 0, 0, 0, 0, 0, 0, .05, 0],
           np.linspace(0, .99, 9))


@pytest.mark.parametrize("n", [1, 2, 150, 700])
def test_row_counts(n):
    ctr = need_gpu()
    rng = np.random.default_rng(n)
    _check(ctr, _logits(n, 4001, torch.bfloat16, n), rng.uniform(0.3, 1.2, n), rng.integers(0, 60, n), rng.uniform(0.5, 1.1, n), 0.0,
           rng.random(n))


def test_no_rows_and_no_options():
    ctr = need_gpu()
    x = torch.empty(0, 100, device="cuda")
    empty = torch.empty(0, device="cuda")
    ctr.ctr_sample(x, empty, empty, torch.empty(0, dtype=torch.int32, device="cuda"))
    x = _logits(3, 2000, torch.float16, 5)
    want = _run(ctr, x, 0.9, 0, 1.0, 0.0, 0.6)
    got = _run(ctr, x, 0.9, u=0.6)
    assert np.array_equal(got["token"], want["token"])
    token = torch.empty(3, dtype=torch.int32, device="cuda")
    ctr.ctr_sample(x, torch.full((3,), 0.9, device="cuda"), torch.full((3,), 0.6, device="cuda"), token)
    assert np.array_equal(token.cpu().numpy(), want["token"])


def test_nan_settings_are_off():
    ctr = need_gpu()
    x = _logits(2, 2000, torch.float32, 5)
    want = _run(ctr, x, 0.9, 0, 1.0, 0.0, 0.6)
    got = _run(ctr, x, 0.9, 0, math.nan, math.nan, 0.6)
    assert all(np.array_equal(got[k], want[k]) for k in want)


def test_on_another_stream_and_in_a_graph():
    ctr = need_gpu()
    x = _logits(5, 33_000, torch.bfloat16, 12)
    want = _run(ctr, x, 0.9, 50, 0.9, 0.0, 0.3)
    got = _run(ctr, x, 0.9, 50, 0.9, 0.0, 0.3, stream=torch.cuda.Stream())
    assert all(np.array_equal(got[k], want[k]) for k in want)
    t, u = torch.full((5,), 0.9, device="cuda"), torch.full((5,), 0.3, device="cuda")
    k, p = torch.full((5,), 50, dtype=torch.int32, device="cuda"), torch.full((5,), 0.9, device="cuda")
    token = torch.zeros(5, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctr.ctr_sample(x, t, u, token, top_k=k, top_p=p)
    for _ in range(3):
        token.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(token.cpu().numpy(), want["token"])
