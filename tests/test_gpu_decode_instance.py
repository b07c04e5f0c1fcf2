"""The three operators together: a decode instance against the same transformer without a cache, draft trees against
their branches, and the simulated cluster that its calibration gives."""
import math

import numpy as np
import pytest
import torch

from gpuutil import gen, need_gpu, simulate
from paper_2609_16206_gb300 import workloads as W

pytestmark = pytest.mark.gpu


def _spec(decode, **kw):
    base = dict(layers=2, hidden=256, heads=8, kv_heads=2, head_dim=64, ffn=512, vocab=1000, dtype=torch.float16)
    base.update(kw)
    return decode.ModelSpec(**base)


def _plain_logits(inst, tokens):
    """The whole sequence at once in fp64, causal attention over the rotated keys."""
    s = inst.spec
    n = len(tokens)
    x = inst.embed[torch.tensor(tokens, device="cuda")].double()
    turns = [w % (1 << 64) for w in inst.rope.turns.tolist()]
    phi = torch.tensor([[2 * math.pi * ((p * w) % (1 << 64)) / 2.0 ** 64 for w in turns] for p in range(n)], dtype=torch.float64, device="cuda")
    c, sn, half = phi.cos()[:, None], phi.sin()[:, None], s.head_dim // 2

    def norm(v):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6)

    def rot(v):
        a, b = v[..., :half], v[..., half:]
        return torch.cat((a * c - b * sn, a * sn + b * c), -1)
    for layer in inst.layers:
        w = {k: v.double() for k, v in layer.items()}
        qkv = (norm(x) @ w["qkv"]).view(n, -1, s.head_dim)
        q, k, v = rot(qkv[:, :s.heads]), rot(qkv[:, s.heads:s.heads + s.kv_heads]), qkv[:, s.heads + s.kv_heads:]
        g = s.heads // s.kv_heads
        a = torch.einsum("thd,phd->htp", q, k.repeat_interleave(g, 1)) * s.head_dim ** -0.5
        a = a.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf).softmax(-1)
        x = x + torch.einsum("htp,phd->thd", a, v.repeat_interleave(g, 1)).reshape(n, -1) @ w["out"]
        up, gate = (norm(x) @ w["up"]).chunk(2, -1)
        x = x + (up * torch.nn.functional.silu(gate)) @ w["down"]
    return norm(x) @ inst.head.double()


def _near(got, want):
    """fp16 activations through two layers: about twenty roundings of 2^-11 on values whose sums have random signs, so a
    relative error of the whole vector below 20 2^-11 = 1 %."""
    err = (got.double() - want).norm() / want.norm()
    assert float(err) < 20 * 2.0 ** -11, float(err)


def test_decode_steps_equal_the_whole_sequence():
    need_gpu()
    from paper_2609_16206_gb300 import decode
    inst = decode.DecodeInstance(_spec(decode), max_seqs=3, kv_tokens=300, max_nodes=4)
    inst.reset([0, 0, 0])
    rng = np.random.default_rng(0)
    seqs = [rng.integers(0, 1000, 40).tolist() for _ in range(3)]
    last = None
    at = [0, 0, 0]
    for new in ([4, 1, 0], [3, 4, 4], [4, 4, 1], [1, 1, 1], [1, 1, 1], [4, 2, 3]):  # chains of tokens, one or none
        parents = [[i - 1 for i in range(n)] for n in new]
        tokens = [t for s, a, n in zip(seqs, at, new) for t in s[a:a + n]]
        last = inst.step(torch.tensor(tokens, device="cuda"), inst.plan(parents))
        inst.grow(new)
        at = [a + n for a, n in zip(at, new)]
    rows = np.cumsum([0] + new)
    for b in range(3):
        _near(last[rows[b]:rows[b + 1]], _plain_logits(inst, seqs[b][:at[b]])[at[b] - new[b]:])


def test_a_draft_tree_equals_its_branches():
    need_gpu()
    from paper_2609_16206_gb300 import decode
    inst = decode.DecodeInstance(_spec(decode), max_seqs=1, kv_tokens=300, max_nodes=64)
    rng = np.random.default_rng(1)
    prompt = rng.integers(0, 1000, 50).tolist()
    inst.reset([0])
    inst.step(torch.tensor(prompt, device="cuda"), inst.plan([[i - 1 for i in range(50)]]))
    inst.grow([50])
    parents = [-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, 40)]
    drafted = rng.integers(0, 1000, 40).tolist()
    logits = inst.step(torch.tensor(drafted, device="cuda"), inst.plan([parents]))
    for leaf in (39, 38, 17, 0):
        path, i = [], leaf
        while i >= 0:
            path.append(i)
            i = parents[i]
        path = path[::-1]
        want = _plain_logits(inst, prompt + [drafted[i] for i in path])[50:]
        _near(logits[path], want)


def test_sampling_ends_the_step():
    need_gpu()
    from paper_2609_16206_gb300 import decode
    inst = decode.DecodeInstance(_spec(decode), max_seqs=2, kv_tokens=100)
    inst.reset([0, 0])
    tokens = torch.tensor([1, 2], device="cuda")
    for _ in range(20):
        logits = inst.step(tokens, inst.plan())
        greedy = inst.sample(logits, torch.zeros(2, device="cuda"), temperature=0.0)
        assert torch.equal(greedy.long(), logits.float().argmax(-1))
        token = inst.sample(logits, torch.rand(2, device="cuda"), temperature=0.8, top_k=5)
        top = logits.float().topk(5).indices
        assert (top == token[:, None]).any(1).all()
        inst.grow([1, 1])
        tokens = token.long()
    with pytest.raises(ValueError):
        inst.reset([1000])


def test_calibration_gives_a_cluster_that_simulates(orc):
    ctr = need_gpu()
    from paper_2609_16206_gb300 import decode
    inst = decode.DecodeInstance(_spec(decode, head_dim=128, vocab=4000), max_seqs=32, kv_tokens=40_000)
    fit = decode.calibrate(inst, batches=(1, 8, 32), contexts=(64, 512, 1024), reps=3)
    assert len(fit.points) >= 6 and all(t > 0 for _, _, t in fit.points)
    assert fit.dec_base_us >= 0 and fit.dec_us_per_seq >= 0 and fit.dec_kv_tokens_per_us > 0
    cfg, cc = decode.calibrated_sim(fit, W.replica_sweep().sim)
    wl = W.replica_sweep(n_replicas=2, n_req=300)
    tr = gen(ctr, wl.trace, 2, 300)
    res = simulate(ctr, cfg, [cc], [W.POLICY_LEARNED], tr, 2, 300)
    assert (res["status"] == 0).all()
    for r in range(2):
        ref = orc.simulate(cfg, cc, W.POLICY_LEARNED, orc.gen_trace(wl.trace, 300, replica=r))
        assert int(res["hash"][r]) == ref["hash"]
