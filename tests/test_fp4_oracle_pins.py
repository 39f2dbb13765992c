"""The 4-bit oracle against its definition, value by value, and the rules' oracle against loops (no GPU)."""
import numpy as np

from oracle import fp4_oracle as fp4


def _nearest(v, e):
    """By brute force: the codes at the least distance, the even one of two."""
    best = sorted(range(8), key=lambda c: (abs(abs(v) - fp4.GRID[c] * 2.0 ** e), c % 2))[0]
    return float(np.copysign(fp4.GRID[best] * 2.0 ** e, v))


def test_round_is_the_nearest_of_the_grid():
    rng = np.random.default_rng(1)
    for scale in (1e-30, 0.01, 1.0, 7.0, 3e20):
        a = (rng.standard_normal((4, 64)) * scale).astype(np.float32).astype(np.float64)
        e = fp4.exponents(a)
        r = fp4.fp4_round(a)
        for i in range(4):
            for b in range(2):
                top = np.abs(a[i, 32 * b:32 * b + 32]).max()
                assert top <= 6 * 2.0 ** e[i, b] and (top > 6 * 2.0 ** (e[i, b] - 1))
            for j in range(64):
                assert r[i, j] == _nearest(a[i, j], e[i, j // 32])


def test_ties_zeros_limits_and_short_blocks():
    ties = np.zeros(32)
    ties[:16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0]
    want = [0, 1, 1, 2, 2, 4, 4, 6]
    assert np.array_equal(fp4.fp4_round(ties)[:16], np.array(want + [-w for w in want], dtype=float))
    assert np.array_equal(fp4.fp4_round(np.zeros(40)), np.zeros(40)) and fp4.exponents(np.zeros(40)).tolist() == [-126, -126]
    big = np.array([3.4e38, 6 * 2.0 ** 125, -3.4e38, 1e30])
    assert fp4.fp4_round(big).tolist() == [6 * 2.0 ** 125, 6 * 2.0 ** 125, -6 * 2.0 ** 125, 0.0]
    a = np.arange(1, 41, dtype=float)
    assert np.array_equal(fp4.fp4_round(a)[32:], fp4.fp4_round(a[32:]))     # a last block of 8
    assert np.array_equal(fp4.fp4_round(fp4.fp4_round(a)), fp4.fp4_round(a))


def test_rules_against_a_loop():
    rng = np.random.default_rng(2)
    V = 37
    for case in range(20):
        x = rng.standard_normal(V)
        hist, prompt = rng.integers(-2, V + 2, 50), int(rng.integers(0, 50))
        bias, ok = rng.standard_normal(V), rng.random(V) < (0.0 if case == 0 else 0.3)
        got, tok = fp4.process_logits(x, hist, prompt, 1.3, 0.2, 0.5, bias, ok)
        best, want_tok = -np.inf, -1
        for w in range(V):
            y = x[w]
            if w in hist.tolist():
                y = y / 1.3 if y > 0 else y * 1.3
            n = hist[prompt:].tolist().count(w)
            if n:
                y = y - 0.2 * n - 0.5
            y += bias[w]
            assert got[w] == (y if ok[w] else -np.inf) or abs(got[w] - y) < 1e-12
            if ok[w] and (want_tok < 0 or y > best):
                best, want_tok = y, w
        assert tok == want_tok
    nan = np.array([np.nan, 1.0, np.inf, -np.inf])
    assert fp4.process_logits(nan, allowed=[0, 1, 0, 1])[1] == 1
    assert fp4.process_logits(nan, allowed=[1, 0, 0, 1])[1] == 3
    assert fp4.process_logits(nan, allowed=[1, 0, 0, 0])[1] == -1
