"""The oracle of the 8-bit rows and of the token tree against other ways to the
same results: exact fractions, the causal chunk, a dense mask."""
from fractions import Fraction

import numpy as np
import pytest

import oracle


def _nearest_even(f: Fraction) -> int:
    return round(f)          # a Fraction rounds half to even


def test_quantize_by_exact_fractions():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 64)).astype(np.float32)
    x[1] *= np.float32(1e-30)
    x[2] = np.arange(64) * np.float32(0.5)      # largest 31.5: quotients on and beside ties
    x[3] = 0
    codes, scales = oracle.quantize(x)
    for r in range(6):
        s = Fraction(float(scales[r]))
        assert abs(s * 127 - Fraction(float(np.abs(x[r]).max()))) <= s * 127 * Fraction(1, 1 << 24)
        for e in range(64):
            want = _nearest_even(Fraction(float(x[r, e])) / s) if s else 0
            assert codes[r, e] == want


def test_quantize_special_rows():
    x = np.zeros((4, 64), np.float32)
    x[0, 3], x[1, 5], x[2, 7] = np.inf, np.nan, 1e-37      # 1e-37 / 127 is subnormal
    x[3, 0], x[3, 1] = np.finfo(np.float32).max, -np.finfo(np.float32).max
    codes, scales = oracle.quantize(x)
    assert np.isnan(scales[:2]).all() and not codes[:3].any() and scales[2] == 0
    assert np.isfinite(scales[3]) and codes[3, 0] == 127 and codes[3, 1] == -127


@pytest.mark.parametrize("T,M", [(1, 0), (7, 5), (12, 40)])
def test_chain_is_the_causal_chunk(T, M):
    rng = np.random.default_rng(T)
    q, kn, vn = (rng.standard_normal((2, h, T, 64)) for h in (4, 2, 2))
    kc, vc = rng.standard_normal((2, 2, M, 64)), rng.standard_normal((2, 2, M, 64))
    out, lse, wsum = oracle.sdpa_chunk(q, kc, vc, kn, vn)
    parents = np.tile(np.arange(-1, T - 1), (2, 1))
    o, l = oracle.sdpa_tree(q, kc, vc, kn, vn, parents)
    np.testing.assert_allclose(o, out, atol=1e-12)
    np.testing.assert_allclose(l, lse, atol=1e-12)
    w, ka, va = oracle.tree_accept(q, kc, kn, vn, lse, np.tile(np.arange(T), (2, 1)))
    np.testing.assert_allclose(w, wsum, atol=1e-12)
    assert np.array_equal(ka, kn) and np.array_equal(va, vn)


def test_an_accepted_path_is_the_chunk_of_its_tokens():
    rng = np.random.default_rng(9)
    T, M = 9, 20
    parents = np.array([[-1, 0, 0, 2, -1, 2, 5, 3, 6]])
    path = np.array([[0, 2, 5, 6]])
    q, kn, vn = (rng.standard_normal((1, h, T, 64)) for h in (4, 2, 2))
    kc, vc = rng.standard_normal((1, 2, M, 64)), rng.standard_normal((1, 2, M, 64))
    out, lse = oracle.sdpa_tree(q, kc, vc, kn, vn, parents)
    p = path[0]
    o, l, w = oracle.sdpa_chunk(q[:, :, p], kc, vc, kn[:, :, p], vn[:, :, p])
    np.testing.assert_allclose(out[:, :, p], o, atol=1e-12)
    np.testing.assert_allclose(lse[:, :, p], l, atol=1e-12)
    got, ka, va = oracle.tree_accept(q, kc, kn, vn, lse, path)
    np.testing.assert_allclose(got, w, atol=1e-12)
    assert np.array_equal(ka, kn[:, :, p]) and np.array_equal(va, vn[:, :, p])


def test_parents_out_of_range_are_roots():
    seen = oracle.ancestors(np.array([[0, 5, -7, 1, 2 ** 31 - 1, 4]]))[0]
    want = np.eye(6, dtype=bool)
    want[3, 1] = want[5, 4] = True
    assert np.array_equal(seen, want)
