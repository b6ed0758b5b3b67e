"""The 8-bit products and the matrix update in every size of tile, on shapes that end inside one: each case says which tile it is for, and the library
is asked whether it takes it there."""
import numpy as np
import pytest

from oracle import matrix_ops as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_fp8 import dev, operand, product                                  # noqa: E402
from test_gpu_muon import gaussian, layout, rel, tolerance, view, workspace     # noqa: E402


@pytest.fixture(scope="module")
def hs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_14783_amd import binding
    binding.lib()            # a missing library is a failure, not a skip
    return binding


# ---- 8-bit products -----------------------------------------------------------------------------------
@pytest.mark.parametrize("m,n,k,f32,tile", [(5793, 2051, 640, 0, 256), (5793, 2051, 1100, 0, 256), (733, 5461, 200, 0, 128), (4090, 2051, 1100, 0, 128),
                                            (5793, 2051, 300, 1, 256), (2051, 5793, 200, 1, 256), (733, 5461, 200, 1, 128), (1500, 2500, 650, 1, 128)])
@pytest.mark.parametrize("aligned", [False, True])
def test_products(hs, m, n, k, f32, tile, aligned):
    """Bounds as in test_product_against_the_oracle; aligned: rows of the result start on 16 bytes, which is another way out."""
    assert hs.hs_gemm_fp8_choice(m, n, k, f32) == (tile, 1)
    rng = np.random.default_rng(m + n + k)
    a, sa = operand(rng, m, k, 3)
    b, sb = operand(rng, n, k, 3)
    bias = torch.from_numpy(rng.standard_normal(n).astype(np.float32) * 1e4).to(torch.bfloat16)
    ldc = n + 16 - n % 8 if aligned else n + 3 + n % 2
    assert (ldc % 8 == 0) == aligned
    out = torch.full((m + 1, ldc), 7.5, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    da, dsa, db, dsb = dev(a, sa, b, sb)
    product(hs, m, n, k, da, dsa, db, dsb, out, ldc, c_f32=f32, beta=-0.5 if f32 else 0.0, bias=bias.cuda())
    want, size = M.gemm_fp8(a, sa, b, sb, k, bias.double().numpy(), np.full((m, n), 7.5) if f32 else None, -0.5 if f32 else 0.0)
    got = out.cpu().double().numpy()
    bound = (k + 4) * 2.0 ** -24 * size if f32 else 2.0 ** -8 * np.abs(want) + 1.01 * (2.0 ** -9 + (k + 2) * 2.0 ** -24) * size
    assert np.all(np.abs(got[:m, :n] - want) <= bound + 1e-30)
    if not f32:      # the rounding of the values, and what is dropped (random signs)
        assert np.linalg.norm(got[:m, :n] - want) <= 2.0 ** -8 * np.linalg.norm(want) + 2.0 ** -12 * np.linalg.norm(size) / np.sqrt(k)
    assert np.all(got[m] == 7.5) and np.all(got[:, n:] == 7.5)


def test_nan_stays_in_its_row_and_column_of_large_tiles(hs):
    rng = np.random.default_rng(4)
    for m, n, k, f32 in ((5793, 2051, 640, 0), (5793, 2051, 300, 1)):
        assert hs.hs_gemm_fp8_choice(m, n, k, f32) == (256, 1)
        a, sa = operand(rng, m, k, 1)
        b, sb = operand(rng, n, k, 1)
        a[m - 1, k - 1], b[n - 1, 17], sa[1000, 1] = 0x7f, 0xff, 0xff
        out = torch.empty(m, n, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        product(hs, m, n, k, *dev(a, sa, b, sb), out, n, c_f32=f32)
        want = np.zeros((m, n), bool)
        want[m - 1], want[:, n - 1], want[1000] = True, True, True
        assert np.array_equal(~np.isfinite(out.cpu().float().numpy()), want)


# ---- matrices -------------------------------------------------------------------------------------------
# (products, shape, count, way, sides of the tiles of X X^T, of symmetric products, of S X)
LISTS = [(1, (300, 300), 58, 0, (64, 128, 64)), (1, (330, 330), 76, 0, (128, 128, 128)), (1, (430, 430), 85, 0, (256, 128, 128)),
         (1, (652, 900), 37, 0, (256, 128, 256)), (1, (900, 652), 37, 0, (256, 128, 256)), (1, (600, 1300), 11, 1, (64, 64, 256)),
         (1, (600, 1300), 29, 1, (128, 128, 128)), (1, (1500, 650), 36, 1, (256, 128, 256)),
         (0, (330, 330), 22, 0, (64, 64, 128)), (0, (330, 330), 76, 0, (128, 128, 128)), (0, (652, 900), 37, 0, (64, 128, 128)),
         (0, (900, 652), 37, 0, (64, 128, 128))]


def exact(x, eps=1e-7):
    """[count, rows, cols] in 64 bits, batched, from the definition."""
    tall = x.shape[1] > x.shape[2]
    X = (x.transpose(1, 2) if tall else x).contiguous()
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + eps)
    a, b, c = M.DEFAULT_COEFF
    for _ in range(5):
        A = torch.bmm(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.bmm(b * A + c * torch.bmm(A, A), X)
    return (X.transpose(1, 2) if tall else X).contiguous()


def matrices(flat, mats):
    return torch.stack([flat.as_strided((r, c), (ld, 1), off) for off, ld, r, c in mats])


def filled(rng, shape, count, gap, ld):
    """A buffer of Gaussian matrices, the first of low rank with noise."""
    mats, size = layout([shape] * count, gap, ld)
    x = gaussian(rng, size)
    low, r = view(x, mats[0]), min(shape) // 16
    low[...] = gaussian(rng, (shape[0], r)) @ gaussian(rng, (r, shape[1])) + 0.05 * low
    return mats, size, x


def bounds(host, mats, products, way):
    """Tolerance of each matrix: the first's own, and the others' from two of them."""
    tol = [tolerance(view(host, mats[i]), products, runs=(3, 2) if way == 1 else None) for i in (0, 1, len(mats) - 1)]
    return torch.tensor([tol[0][0]] + [max(tol[1][0], tol[2][0])] * (len(mats) - 1), dtype=torch.float64, device="cuda"), tol[1][1]


def untouched(flat, before, mats):
    rest = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
    for off, ld, r, c in mats:
        rest.as_strided((r, c), (ld, 1), off).fill_(False)
    return torch.equal(flat[rest], before[rest])


@pytest.mark.parametrize("products,shape,count,way,tiles", LISTS)
@pytest.mark.parametrize("gap,ld", [(0, 0), (3, 5)])
def test_orthogonalised_lists(hs, products, shape, count, way, tiles, gap, ld):
    mats, size, x = filled(np.random.default_rng(shape[0] + count), shape, count, gap, ld)
    lst = hs.make_matrices(mats)
    assert hs.hs_orthogonalize_choice(lst, products, count - 1) == (way, tiles)
    ws, n = workspace(hs, lst, products)
    dx = torch.from_numpy(x).cuda()
    y = torch.full_like(dx, 7.5)
    hs.hs_op_orthogonalize(0, dx, y, size, lst, products, 5, None, 1e-7, ws, n)
    want = exact(matrices(dx.double(), mats))
    tol, e = bounds(x.astype(np.float64), mats, products, way)
    assert rel(want[1].cpu().numpy(), e) <= 1e-10
    err = (matrices(y, mats).double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert bool(torch.all(err <= tol)) and untouched(y, torch.full_like(y, 7.5), mats)
    if products == 1:      # bf16 in and out, in place
        low = dx.to(torch.bfloat16)
        want = exact(matrices(low.double(), mats))
        hs.hs_op_orthogonalize(1, low, low, size, lst, products, 5, None, 1e-7, ws, n)
        err = (matrices(low, mats).double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
        assert bool(torch.all(err <= tol + 2.0 ** -8)) and untouched(low, dx.to(torch.bfloat16), mats)


@pytest.mark.parametrize("products,shape,count,way,tiles", LISTS)
@pytest.mark.parametrize("gap,ld", [(0, 0), (5, 3)])
def test_updates(hs, products, shape, count, way, tiles, gap, ld):
    """Weights, momentum and bf16 copy; bounds as in muon_tolerances of the smaller lists."""
    lr, mu, wd, rms, denom = 0.02, 0.95, 0.1, 0.2, 48.0
    mats, size, G = filled(np.random.default_rng(shape[1] + count), shape, count, gap, ld)
    rng = np.random.default_rng(1)
    w, m, G = 0.02 * gaussian(rng, size), 1e-3 * gaussian(rng, size), np.float32(denom * 1e-3) * G
    lst = hs.make_matrices(mats)
    assert hs.hs_orthogonalize_choice(lst, products, 0) == (way, tiles)
    ws, n = workspace(hs, lst, products)
    dw, dm, dG = (torch.from_numpy(a.copy()).cuda() for a in (w, m, G))
    w0, m0, low = dw.clone(), dm.clone(), torch.full((size,), 7.5, dtype=torch.bfloat16, device="cuda")
    hs.hs_muon_step(dw, dm, dG, low, size, lst, products, denom, lr, mu, 1, wd, rms, 5, None, 1e-7, ws, n)
    torch.cuda.synchronize()
    W, m64, g = (matrices(t.double(), mats) for t in (w0, m0, dG))
    g = g / denom
    mt = 4 * 2.0 ** -24 * ((mu * m64).abs() + g.abs())
    m64 = mu * m64 + g
    u = g + mu * m64
    O = exact(u)
    s = rms * np.sqrt(max(shape))
    want = (1 - lr * wd) * W - lr * s * O
    flat = torch.zeros(size, dtype=torch.float64)
    for k in (0, 1, count - 1):
        off, step, r, c = mats[k]
        flat.as_strided((r, c), (step, 1), off).copy_(u[k].cpu())
    tol, e = bounds(flat.numpy(), mats, products, way)
    assert rel(O[1].cpu().numpy(), e) <= 1e-10
    norm = lambda t: t.flatten(1).norm(dim=1)
    wt = 4 * 2.0 ** -24 * (norm(W) + norm(want)) + lr * s * 2 * tol * norm(O)
    got = matrices(dw.double(), mats)
    assert bool(torch.all(norm(got - want) <= wt)) and bool(torch.all((matrices(dm.double(), mats) - m64).abs() <= mt))
    assert untouched(dw, w0, mats) and untouched(dm, m0, mats) and torch.equal(dG.cpu(), torch.from_numpy(G))
    assert untouched(low, torch.full_like(low, 7.5), mats) and torch.equal(matrices(low, mats), matrices(dw, mats).to(torch.bfloat16))
