"""Pins of the oracles of the token log probabilities and of the AdamW step (oracle/scoring.py, oracle/adamw.py) against
things that do not depend on them: loops over probabilities, closed forms, finite differences, exhaustive tables."""
import math

import numpy as np
import pytest

from oracle import adamw, scoring


def _rows(seed=0, M=4, V=11):
    return np.random.default_rng(seed).normal(0, 3, (M, V))


def test_scores_by_loops():
    z = _rows()
    z[1, 3] = z[1, 7] = -np.inf
    tokens = np.array([0, 7, -1, 10])
    lp, H, alt, alt_lp = scoring.score(z, tokens, 4)
    for m in range(4):
        e = [math.exp(v) for v in z[m]]
        p = [v / sum(e) for v in e]
        want = 0.0 if tokens[m] < 0 else math.log(p[tokens[m]]) if p[tokens[m]] else -math.inf
        assert lp[m] == pytest.approx(want, abs=1e-13)
        assert H[m] == pytest.approx(-sum(v * math.log(v) for v in p if v), abs=1e-13)
        best = sorted(range(11), key=lambda i: (-z[m, i], i))[:4]
        assert list(alt[m]) == best
        np.testing.assert_allclose(alt_lp[m], [math.log(p[i]) for i in best], atol=1e-13)


def test_scores_of_special_rows():
    z = np.zeros((5, 6))
    z[0] = -np.inf
    z[1, 2] = np.nan
    z[2, 4] = np.inf
    z[3] = [-np.inf, 1, 1, -np.inf, 1, -np.inf]
    z[4] = [0, 0, 60, 0, 0, 0]                                      # almost certain: log p = -5 e^-60
    lp, H, alt, alt_lp = scoring.score(z, np.array([1, 0, 0, 4, 2]), 4)
    assert lp[0] == -np.inf and H[0] == 0 and list(alt[0]) == [-1] * 4 and np.all(alt_lp[0] == -np.inf)
    for m in (1, 2):
        assert np.isnan(lp[m]) and np.isnan(H[m]) and list(alt[m]) == [-1] * 4 and np.isnan(alt_lp[m]).all()
    assert list(alt[3]) == [1, 2, 4, -1] and alt_lp[3, 3] == -np.inf
    assert lp[3] == pytest.approx(-math.log(3)) and H[3] == pytest.approx(math.log(3))
    assert lp[4] == pytest.approx(-5 * math.exp(-60), rel=1e-12)


def test_score_gradient_by_differences():
    z = _rows(3, 3, 9)
    z[2, 5] = -np.inf
    tokens, g, h = np.array([2, -1, 0]), np.array([0.7, 5.0, -1.1]), np.array([0.3, -0.2, 0.0])

    def value(x):
        lp, H, _, _ = scoring.score(x, tokens, 0)
        return float((g * lp + h * H).sum())

    dz = scoring.score_gradient(z, tokens, g, h)
    for m in range(3):
        for i in range(9):
            if z[m, i] == -np.inf:
                assert dz[m, i] == 0
                continue
            up, down = z.copy(), z.copy()
            up[m, i] += 1e-5
            down[m, i] -= 1e-5
            assert dz[m, i] == pytest.approx((value(up) - value(down)) / 2e-5, abs=2e-9)


def test_adamw_first_step_is_the_sign_of_the_gradient():
    g = np.array([3.0, -0.2, 1e-3])
    w, m, v = adamw.step(np.ones(3), np.zeros(3), np.zeros(3), g, lr=0.1, beta1=0.9, beta2=0.999, eps=0.0,
                         weight_decay=0.5, t=1)
    np.testing.assert_allclose(w, 1 - 0.05 - 0.1 * np.sign(g), atol=1e-14)
    np.testing.assert_allclose(m, 0.1 * g)
    np.testing.assert_allclose(v, 0.001 * g * g)


def test_adamw_constant_gradient():
    w, m, v = np.zeros(1), np.zeros(1), np.zeros(1)
    for t in range(1, 50):
        w, m, v = adamw.step(w, m, v, np.array([-2.0]), lr=0.01, beta1=0.8, beta2=0.95, eps=0.0, weight_decay=0.0, t=t)
    assert w[0] == pytest.approx(0.49) and m[0] == pytest.approx(-2 * (1 - 0.8 ** 49)) and v[0] == pytest.approx(4 * (1 - 0.95 ** 49))


def test_codes_are_e4m3():
    torch = pytest.importorskip("torch")
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    fine = ~np.isnan(want)
    assert list(codes[~fine]) == [0x7f, 0xff]
    np.testing.assert_array_equal(adamw.decode(np.where(fine, codes, 0).astype(np.uint8), np.ones(1))[fine], want[fine])


def test_scales_bring_the_largest_into_range():
    rng = np.random.default_rng(5)
    x = rng.normal(size=40 * 256) * np.repeat(10.0 ** rng.uniform(-12, 12, 40), 256)
    x[:256] = 0
    x[256:512] = 1.75 / 64                                          # the end of the range, exactly
    s = adamw.scales_of(x)
    most = np.abs(x).reshape(40, 256).max(1)
    assert s[0] == 0 and s[1] == 2.0 ** -14
    assert np.all((most[1:] / s[1:] > 224) & (most[1:] / s[1:] <= 448))
    assert np.all(np.exp2(np.round(np.log2(s[1:]))) == s[1:])


def test_rounding_keeps_the_mean_and_the_neighbours():
    # exhaustive over the 20 random bits in 64 equal steps: the mean of the decoded values is the value
    for y in (0.3, 3.1, 0.0007, 447.0, 17.03, 448.0):
        words = np.arange(64, dtype=np.uint64) * np.uint64(1 << 14) + np.uint64(1 << 13)
        codes = adamw.encode(np.full(64, y), np.ones(1), words)
        got = adamw.decode(codes, np.ones(1))
        gap = np.diff(adamw.VALUES)[np.searchsorted(adamw.VALUES, y, side="right") - 1 if y < 448 else 125]
        assert abs(got.mean() - y) <= gap / 64 and np.all(np.abs(got - y) < gap)
    assert adamw.encode(np.array([-2.0]), np.ones(1), np.array([0]))[0] == 0x80 | 0x40


def test_hash_is_even():
    r = adamw.random_words(7, 3, 0, 1 << 16).astype(np.float64)
    assert len(np.unique(r)) == 1 << 16                             # a bijection of 32-bit words
    for bits in (r % 2 ** 20 / 2 ** 20, np.floor(r / 4096) / 2 ** 20):
        # mean of 65536 uniform numbers: 0.5 within 5 / sqrt(12 * 65536)
        assert abs(bits.mean() - 0.5) < 5 / math.sqrt(12 * 65536)
        assert abs(np.corrcoef(bits[:-1], bits[1:])[0, 1]) < 5 / 256
    assert not np.array_equal(r, adamw.random_words(7, 4, 0, 1 << 16))
