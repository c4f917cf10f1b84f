"""CPU pins of the 4-bit cache's fp64 oracle: the grid and the scales by brute
force, the error bounds they promise, the attention by the plain oracle on the
same values, the choice of slots by hand."""
from fractions import Fraction

import numpy as np
import pytest

import oracle
import workloads as W
from oracle.cache import GRID


def bf16(x):
    return W.bf16_bits_to_f32(W.f32_to_bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


def rows(seed, n, d, spread=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, d))
    if spread:
        x *= 2.0 ** rng.integers(-spread, spread + 1, size=(n, 1))
    return bf16(x)


def brute(x, scale):
    """By exact fractions: the nearest of +-GRID * scale, ties to the even code."""
    best = min(range(8), key=lambda c: (abs(abs(Fraction(x)) - Fraction(GRID[c]) * Fraction(scale)),
                                        c % 2))
    return float(np.copysign(GRID[best] * scale, x))


def test_k_by_brute_force():
    x = np.concatenate([rows(1, 6, 64, 12), bf16(np.outer([1.0, 2.0 ** 20, 2.0 ** -110],
                        np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6.9], 8)))])
    got = oracle.cache_k(x)
    for r in range(len(x)):
        for b in range(2):
            blk = x[r, 32 * b:32 * b + 32]
            e = next(e for e in range(-100, 128) if np.abs(blk).max() < 7 * 2.0 ** e)
            for j in range(32):
                assert got[r, 32 * b + j] == brute(blk[j], 2.0 ** e), (r, b, j)


def test_v_by_brute_force():
    x = np.concatenate([rows(2, 6, 64, 12), bf16(np.outer([1.0, 2.0 ** 20, 2.0 ** -110],
                        np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6], 8)))])
    got = oracle.cache_v(x)
    for r in range(len(x)):
        top = Fraction(np.abs(x[r]).max())
        s = min(Fraction(m) * Fraction(2) ** p for p in range(-106, 24) for m in range(32, 64)
                if 6 * m * Fraction(2) ** p >= top and m * Fraction(2) ** p >= Fraction(2) ** -100)
        for j in range(64):
            assert got[r, j] == brute(x[r, j], float(s)), (r, j)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_values_are_bf16_and_near(d):
    """Every value is a bf16 number; K is off by at most 2^e (half the widest step, 2), V by at
    most s."""
    x = rows(3, 300, d, 30)
    for f in (oracle.cache_k, oracle.cache_v):
        y = f(x)
        assert np.array_equal(bf16(y), y)
        assert np.array_equal(f(y)[np.abs(y).max(-1) > 0] != 0, (f(y) != 0)[np.abs(y).max(-1) > 0])
    b = np.abs(x).reshape(-1, d // 32, 32).max(-1)
    err = np.abs(oracle.cache_k(x) - x).reshape(-1, d // 32, 32).max(-1)
    assert np.all(err <= b / 3.5)            # 2^e <= max / 3.5
    err = np.abs(oracle.cache_v(x) - x).max(-1)
    assert np.all(err <= np.abs(x).max(-1) / 6 * (1 + 2.0 ** -5))


def test_non_finite_values():
    x = rows(4, 4, 64)
    x[0, 3], x[1, 40], x[2, 0] = np.nan, np.inf, -np.inf
    k, v = oracle.cache_k(x), oracle.cache_v(x)
    assert np.isnan(k[0, :32]).all() and np.isfinite(k[0, 32:]).all()
    assert np.isnan(k[1, 32:]).all() and np.isfinite(k[1, :32]).all()
    assert np.isnan(v[:3]).all() and np.isfinite(v[3]).all()
    assert np.array_equal(oracle.cache_k(np.zeros((1, 64))), np.zeros((1, 64)))
    assert np.array_equal(oracle.cache_v(np.zeros((1, 64))), np.zeros((1, 64)))


@pytest.mark.parametrize("causal", [False, True])
def test_attention_is_the_plain_oracles(causal):
    rng = np.random.default_rng(5)
    q, k, v = (rng.standard_normal(s) for s in ((3, 7, 64), (50, 64), (50, 64)))
    k[44:], v[44:] = np.nan, np.nan          # behind the length: not seen
    o, a, pred, w = oracle.cache_attention(q, k, v, 44, 7, causal, 0.125)
    for g in range(3):
        ref = oracle.attention(q[None, g:g + 1], k[None, None, :44], v[None, None, :44], causal, 0.125)
        assert np.allclose(o[g], ref["O"][0, 0], rtol=1e-12, atol=1e-12)
        assert np.allclose(pred[g], ref["pred"][0, 0], rtol=1e-12, atol=1e-12)
    assert np.allclose(w.sum(), 21.0) and np.all(w[44:] == 0)
    # V = identity columns: the weights are O's column sums
    eye = np.zeros((50, 64))
    eye[:44, :44] = np.eye(44)
    o, _, _, w2 = oracle.cache_attention(q, k, eye, 44, 7, causal, 0.125)
    assert np.allclose(o.sum((0, 1))[:44], w2[:44])


def test_attention_padding_and_empty_rows():
    rng = np.random.default_rng(6)
    q, k, v = (rng.standard_normal(s) for s in ((2, 5, 64), (9, 64), (9, 64)))
    o, _, _, w = oracle.cache_attention(q, k, v, 9, 3, False, 0.125)
    assert np.all(o[:, 3:] == 0) and np.isclose(w.sum(), 6)
    o, _, _, w = oracle.cache_attention(q, k, v, 2, 4, True, 0.125)   # rows 0, 1 see nothing
    assert np.all(o[:, :2] == 0) and np.all(o[:, 2] == v[0]) and np.isclose(w.sum(), 4)
    o, _, _, w = oracle.cache_attention(q, k, v, 0, 5, False, 0.125)
    assert np.all(o == 0) and np.all(w == 0)


def test_keep():
    w = np.array([3.0, 1.0, 2.0, 2.0, 0.0, 2.0, 9.0, 1.0])
    assert oracle.cache_keep(w, 8, 8, 2).tolist() == list(range(8))
    assert oracle.cache_keep(w, 8, 4, 0).tolist() == [0, 2, 3, 6]       # of equal ones the first
    assert oracle.cache_keep(w, 8, 4, 2).tolist() == [0, 2, 6, 7]
    assert oracle.cache_keep(w, 8, 3, 3).tolist() == [5, 6, 7]
    assert oracle.cache_keep(w, 5, 3, 1).tolist() == [0, 2, 4]
    w[4], w[1] = np.nan, np.inf
    assert oracle.cache_keep(w, 8, 2, 0).tolist() == [1, 4]
    assert oracle.cache_keep(w, 8, 1, 0).tolist() == [4]
