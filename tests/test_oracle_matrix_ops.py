"""Pins of the oracle of the 8-bit products and of the matrix update: against closed forms, a search over all codes and the singular values."""
import numpy as np
import pytest

from oracle import matrix_ops as M


def test_code_values_are_those_of_the_format():
    v = M.e4m3_value(np.arange(256))
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7e] == 448.0 and np.isnan(v[0x7f]) and np.isnan(v[0xff])
    assert np.all(np.diff(v[:127]) > 0) and np.array_equal(v[128:255], -v[:127])


def test_codes_are_the_nearest_with_ties_to_even():
    grid = M.e4m3_value(np.arange(127))
    mid = (grid[1:] + grid[:-1]) / 2
    for y in (grid, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e3), np.linspace(0, 448, 3001)):
        for sign in (1, -1):
            c = M.e4m3_code(sign * y)
            near = np.abs(grid[None, :] - np.abs(y)[:, None])
            best = near.min(1)
            assert np.array_equal(np.abs(M.e4m3_value(c)) - np.abs(y) <= best, np.ones(len(y), bool))
            assert np.allclose(np.abs(np.abs(M.e4m3_value(c)) - np.abs(y)), best, rtol=0, atol=0)
    assert np.all(M.e4m3_code(mid) % 2 == 0)
    assert M.e4m3_code(np.array([np.nan]))[0] == 0x7f


def test_scales_bring_the_largest_value_to_448_at_most():
    a = np.array([0.0, 448.0, np.nextafter(448.0, 1e3), 449.0, 1.0, 1.75, 1.76, 3.4e38, 1e-45])
    e = M.scale_exponent(a)
    assert e.tolist()[:3] == [0, 0, 1] and e[3] == 1 and e[4] == -8 and e[5] == -8 and e[6] == -7 and e[-1] == -127
    nz = a[(a > 0) & (e > -127)]
    en = e[(a > 0) & (e > -127)]
    assert np.all(nz <= 448.0 * 2.0 ** en) and np.all(nz > 448.0 * 2.0 ** (en - 1))


@pytest.mark.parametrize("tile", [False, True])
def test_quantised_values_are_within_half_a_step(tile):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((150, 300)) * np.exp(rng.standard_normal((150, 1)))
    x[3, 5], x[7] = np.nan, 0.0
    q, s = M.quantize(x, tile)
    assert q.shape == (150, 384) and s.shape == (150, 3) and np.all(q[:, 300:] == 0)
    v = M.dequantize(q, s, 300)
    assert np.isnan(v[3, 5]) and np.isnan(v).sum() == 1
    ok = np.isfinite(x)
    step = 2.0 ** (s.astype(float)[:, np.arange(300) // 128] - 127) * 2.0 ** -10      # half the spacing of the smallest codes
    assert np.all(np.abs(v - x)[ok] <= np.maximum(np.abs(x) * 2.0 ** -4, step)[ok])
    if tile:
        assert np.all(s[:128] == s[0]) and np.all(s[128:] == s[128])
        assert np.array_equal(M.dequantize(*M.quantize(x.T, True), 150)[ok.T], v.T[ok.T])
    else:
        assert np.all(s[7] == 127)


@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (6, 1), (12, 30), (30, 12), (20, 20)])
@pytest.mark.parametrize("steps", [1, 5])
def test_orthogonalised_matrix_has_the_polynomial_of_the_singular_values(shape, steps):
    rng = np.random.default_rng(5)
    x = rng.standard_normal(shape)
    U, sv, Vt = np.linalg.svd(x, full_matrices=False)
    p = sv / (np.sqrt(np.sum(sv ** 2)) + 1e-7)
    a, b, c = M.DEFAULT_COEFF
    for _ in range(steps):
        p = a * p + b * p ** 3 + c * p ** 5
    assert np.allclose(M.orthogonalize(x, steps), (U * p) @ Vt, rtol=0, atol=1e-10)
    assert np.all(M.orthogonalize(np.zeros(shape), steps) == 0)


def test_emulated_roundings_shrink_with_the_numbers():
    for shape in ((40, 70), (70, 40)):
        x = np.random.default_rng(6).standard_normal(shape)
        e = M.orthogonalize(x)
        off = [np.linalg.norm(M.orthogonalize(x, numbers=n) - e) / np.linalg.norm(e) for n in (1, 2)]
        assert 1e-4 < off[0] < 4e-3 and 1e-7 < off[1] < 1e-5


def test_runs_of_steps_on_the_gram_matrix_are_the_same_polynomial():
    """The runs' own roundings apart: a few times those of the steps one by one."""
    x = np.random.default_rng(7).standard_normal((30, 90))
    e = M.orthogonalize(x)
    for runs in ((1, 1, 1, 1, 1), (2, 2, 1), (3, 2)):
        for n, most in ((1, 1e-2), (2, 1e-4)):
            off = np.linalg.norm(M.orthogonalize(x, numbers=n, runs=runs) - e) / np.linalg.norm(e)
            assert 0 < off < most


def test_update_of_one_matrix_by_hand():
    w, m, G = np.array([[1.0]]), np.array([[2.0]]), np.array([[6.0]])
    nw, nm, O = M.muon_step(w, m, G, lr=0.1, momentum=0.5, weight_decay=0.2, rms=0.0, denom=3.0, steps=1, eps=0.0)
    assert nm[0, 0] == 3.0                                   # 0.5 * 2 + 6 / 3
    assert np.isclose(O[0, 0], sum(M.DEFAULT_COEFF))           # a 1 x 1 matrix is 1 once it is divided by its norm
    assert np.isclose(nw[0, 0], 0.98 - 0.1 * O[0, 0])
    nw, _, _ = M.muon_step(np.zeros((2, 8)), np.zeros((2, 8)), np.eye(2, 8), lr=1.0, momentum=0.0, rms=0.2, steps=1)
    assert np.isclose(-nw[0, 0], 0.2 * np.sqrt(8) * M.orthogonalize(np.eye(2, 8), 1)[0, 0])
