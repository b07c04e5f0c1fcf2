"""The decode instance's host-side helpers, without a GPU."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_16206_gb300 import decode  # noqa: E402
from paper_2609_16206_gb300 import workloads as W  # noqa: E402


def _turn(word):
    return (word % (1 << 64)) / 2.0 ** 64


def test_turns_are_the_frequencies():
    t = decode.rope_turns(128, 10000.0, device="cpu").tolist()
    for i, w in enumerate(t):
        assert abs(_turn(w) * 2 * math.pi - 10000.0 ** (-i / 64)) <= 1e-15
    lin = decode.rope_turns(128, 10000.0, factor=4.0, device="cpu").tolist()
    assert all(abs(_turn(a) - 4 * _turn(b)) <= 1e-15 for a, b in zip(t, lin))


def test_scaled_turns_keep_fast_pairs_and_divide_slow_ones():
    plain = decode.rope_turns(128, 10000.0, device="cpu").tolist()
    got = decode.rope_turns(128, 10000.0, factor=8.0, trained_len=4096, device="cpu").tolist()
    for a, b in zip(plain, got):
        turns = _turn(a) * 4096
        if turns >= 32:
            assert a == b
        elif turns <= 1:
            assert abs(_turn(a) - 8 * _turn(b)) <= 1e-15
        else:
            assert _turn(a) / 8 < _turn(b) < _turn(a)
    for bad in ((3, 1e4, 1.0), (-2, 1e4, 1.0), (4, 1.0, 1.0), (4, 1e4, 0.5)):
        with pytest.raises(ValueError):
            decode.rope_turns(*bad, device="cpu")


def test_tree_words_and_depths():
    parents = [-1, 0, 0, 1, -1, 4]
    assert decode.tree_words(parents) == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b110000]
    assert decode.tree_depths(parents) == [0, 1, 1, 2, 0, 1]
    chain = decode.tree_words([i - 1 for i in range(64)])
    assert chain[63] == -1 and chain[62] == (1 << 63) - 1
    for bad in ([0], [-2], [-1, 1], [-1] * 65):
        with pytest.raises(ValueError):
            decode.tree_words(bad)


def test_fit_finds_the_terms_and_holds_them_at_zero():
    pts = [(n, n * c, 150.0 + 1.5 * n + n * c / 400.0) for n in (1, 8, 32) for c in (64, 512, 2048)]
    f = decode.fit_steps(pts)
    assert abs(f.dec_base_us - 150) < 1e-6 and abs(f.dec_us_per_seq - 1.5) < 1e-6 and abs(f.dec_kv_tokens_per_us - 400) < 1e-4
    assert all(abs(f.step_us(n, kv) - t) < 1e-6 for n, kv, t in f.points)
    down = decode.fit_steps([(n, kv, 100.0 - 0.5 * n) for n in (1, 10, 20) for kv in (10, 1000)])
    assert down.dec_us_per_seq == 0.0 and down.dec_kv_tokens_per_us >= 1


def test_fitted_constants_are_the_simulators():
    f = decode.StepFit(150.4, 1.6, 399.7, ())
    cfg, cc = decode.calibrated_sim(f, W.replica_sweep().sim)
    assert (cfg.dec_base_us, cfg.dec_us_per_seq, cfg.dec_kv_tokens_per_us) == (150, 2, 400)
    assert cc.tau_dec_us == 152 and cfg.n_decode == W.replica_sweep().sim.n_decode
    cfg, _ = decode.calibrated_sim(decode.StepFit(0.0, 0.0, 2.0 ** 40, ()))
    assert cfg.dec_base_us == 1 and cfg.dec_kv_tokens_per_us == 1 << 31
