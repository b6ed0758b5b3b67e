"""Matrices of a few strong directions with weak ones beside them, orthogonalised with 16-bit products: the weak ones grow by up to 40 in three steps, and what the
rounding of the strong ones leaves in them must not grow with them."""
import numpy as np
import pytest

from oracle import matrix_ops as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_muon import layout, tolerance, view, workspace      # noqa: E402


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_14783_amd import binding
    binding.lib()            # a missing library is a failure, not a skip
    return binding


def with_spectrum(rng, shape, strong, weak, level):
    """`strong` singular values of 1, `weak` of `level`, the rest 0."""
    k = min(shape)
    U, V = (np.linalg.qr(rng.standard_normal((n, k)))[0] for n in shape)
    s = np.zeros(k)
    s[:strong], s[strong:strong + weak] = 1.0, level
    return ((U * s) @ V.T).astype(np.float32)


@pytest.mark.parametrize("shape,count,way,most", [
    ((64, 3000), 150, 0, 1e-2), ((128, 4000), 100, 0, 1e-2), ((256, 1024), 40, 0, 5e-3), ((1024, 256), 40, 0, 5e-3), ((64, 3000), 4, 0, 1e-2), ((300, 300), 20, 0, 5e-3),
    ((90, 200), 10, 2, 1e-2), ((640, 900), 6, 0, 3e-3), ((500, 2100), 10, 1, 1e-2), ((2000, 640), 12, 1, 1e-2)])
def test_weak_directions_beside_strong_ones(hs, shape, count, way, most):
    """Within the roundings of the way that the library takes (twice the emulated error and what its spread allows, as elsewhere), and within what the header
    says to count on for so many rows."""
    rng = np.random.default_rng(shape[0] + count)
    mats, size = layout([shape] * count)
    x = rng.standard_normal(size).astype(np.float32)
    k = min(shape)
    cases = [(1, k - k // 8, 0.05), (1, k // 2, 0.1), (2, k // 2, 0.1), (1, k // 2, 0.02), (1, k // 2, 0.4)]
    for mat, case in zip(mats, cases):
        view(x, mat)[...] = with_spectrum(rng, shape, *case)
    lst = hs.make_matrices(mats)
    assert hs.hs_orthogonalize_choice(lst, 1, 0)[0] == way
    ws, n = workspace(hs, lst, 1)
    y = torch.empty(size, device="cuda")
    hs.hs_op_orthogonalize(0, torch.from_numpy(x).cuda(), y, size, lst, 1, 5, None, 1e-7, ws, n)
    got = y.cpu().double().numpy()
    for mat, case in zip(mats, cases):
        tol, e = tolerance(view(x.astype(np.float64), mat), 1, runs=(3, 2) if way == 1 else None)
        err = np.linalg.norm(view(got, mat) - e) / np.linalg.norm(e)
        assert err <= tol and err <= most, (case, err, tol)
