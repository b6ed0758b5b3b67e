"""Refusals and sizes of the 8-bit products and of the matrix update that need no GPU: every one comes back before anything is launched."""
import numpy as np
import pytest

from paper_2009_14783_amd import binding as hs

P = 1 << 20          # a stand-in for an aligned device address; no call here gets as far as using one
INVALID, SHAPE, WORKSPACE = 1, 2, 3


def refused(status, call, *args, **kw):
    with pytest.raises(hs.HsError) as e:
        call(*args, stream=0, **kw)
    assert e.value.status == status, e.value
    assert call.__name__ in str(e.value)


def quant(dtype=1, x=P, ldx=200, R=37, C=200, tile=0, q=P, ldq=256, qs=P, ldqs=4, qt=P, ldqt=128, qts=P, ldqts=4):
    return (dtype, x, ldx, R, C, tile, q, ldq, qs, ldqs, qt, ldqt, qts, ldqts)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), INVALID), (dict(R=-1), INVALID), (dict(C=-1), INVALID), (dict(tile=2), INVALID), (dict(x=None), INVALID), (dict(q=None), INVALID),
    (dict(qs=None), INVALID), (dict(qt=None), INVALID), (dict(q=None, qs=None, qt=None, qts=None), INVALID), (dict(ldx=199), SHAPE), (dict(ldq=200), SHAPE),
    (dict(ldq=128), SHAPE), (dict(ldqs=1), SHAPE), (dict(ldqt=64), SHAPE), (dict(ldqts=0), SHAPE), (dict(q=P + 8), SHAPE), (dict(qt=P + 8), SHAPE),
    (dict(x=P + 1), SHAPE), (dict(R=2 ** 31 - 1, C=2 ** 31 - 1, ldx=2 ** 31, ldq=2 ** 31, ldqs=2 ** 24, ldqt=2 ** 31, ldqts=2 ** 24), SHAPE)])
def test_quantiser_refuses(change, status):
    refused(status, hs.hs_op_quantize_fp8, *quant(**change))


def test_empty_calls_are_fine():
    hs.hs_op_quantize_fp8(*quant(R=0), stream=0)
    hs.hs_op_quantize_fp8(*quant(C=0), stream=0)
    hs.hs_op_gemm_fp8(0, 5, 7, None, 128, None, 4, None, 128, None, 4, None, 5, stream=0)
    hs.hs_op_gemm_fp8(5, 0, 7, None, 128, None, 4, None, 128, None, 4, None, 5, stream=0)
    none = hs.make_matrices([])
    hs.hs_muon_step(None, None, None, None, 0, none, 1, 0.0, 0.1, 0.9, 1, 0.0, 0.2, 5, None, 1e-7, None, 0, stream=0)
    hs.hs_op_orthogonalize(0, None, None, 0, none, 0, 5, None, 1e-7, None, 0, stream=0)


def gemm(M=5, N=6, K=200, A=P, lda=256, sa=P, ldas=4, B=P, ldb=256, sb=P, ldbs=4, C=P, ldc=6, **kw):
    return (M, N, K, A, lda, sa, ldas, B, ldb, sb, ldbs, C, ldc), kw


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), INVALID), (dict(N=-1), INVALID), (dict(K=-1), INVALID), (dict(A=None), INVALID), (dict(sa=None), INVALID), (dict(B=None), INVALID),
    (dict(sb=None), INVALID), (dict(C=None), INVALID), (dict(ldc=5), SHAPE), (dict(lda=200), SHAPE), (dict(lda=128), SHAPE), (dict(ldb=128), SHAPE),
    (dict(lda=1 << 23), SHAPE), (dict(ldas=2), SHAPE), (dict(ldbs=0), SHAPE), (dict(K=600, lda=640, ldb=640, ldbs=4), SHAPE), (dict(A=P + 8), SHAPE),
    (dict(B=P + 4), SHAPE), (dict(sa=P + 1), SHAPE), (dict(sb=P + 2), SHAPE), (dict(C=P + 2, c_f32=1), SHAPE), (dict(C=P + 1), SHAPE), (dict(bias=P + 1), SHAPE), (dict(scratch=P + 8, scratch_bytes=1 << 20), SHAPE),
    (dict(M=2 ** 31 - 1, N=2 ** 31 - 1, ldc=2 ** 31), SHAPE), (dict(ldas=1 << 23), SHAPE)])
def test_product_refuses(change, status):
    args, kw = gemm(**change)
    refused(status, hs.hs_op_gemm_fp8, *args, **kw)


LIST = [(0, 7, 5, 7), (35, 9, 3, 9)]


def ortho(mats=LIST, dtype=0, x=P, y=P, size=62, products=0, steps=5, coeff=None, eps=1e-7, ws=P, nbytes=1 << 30):
    return dtype, x, y, size, hs.make_matrices(mats), products, steps, coeff, eps, ws, nbytes


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x=P + 4), INVALID), (dict(y=P + 8), INVALID), (dict(size=61), SHAPE), (dict(products=2), INVALID), (dict(steps=0), INVALID),
    (dict(steps=65), INVALID), (dict(coeff=np.full((5, 3), np.nan)), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(ws=None), WORKSPACE), (dict(nbytes=100), WORKSPACE), (dict(ws=P + 128), INVALID),
    (dict(mats=[(0, 7, 0, 7)]), SHAPE), (dict(mats=[(0, 6, 5, 7)]), SHAPE), (dict(mats=[(-1, 7, 5, 7)]), SHAPE),
    (dict(mats=[(0, 1 << 15, 1 << 15, 1 << 15)], size=1 << 40), SHAPE), (dict(mats=[(1 << 59, 7, 5, 7)]), SHAPE),
    (dict(mats=[(0, 7, 5, 7)] * 2), INVALID), (dict(mats=[(0, 7, 5, 7), (34, 7, 2, 7)]), INVALID), (dict(mats=[(0, 10, 4, 5), (4, 10, 4, 5)]), INVALID),
    (dict(mats=[(0, 10, 4, 5), (5, 10, 3, 6)]), INVALID), (dict(mats=[(0, 10, 4, 5), (5, 9, 4, 3)]), INVALID)])
def test_orthogonalisation_refuses(change, status):
    refused(status, hs.hs_op_orthogonalize, *ortho(**change))


def muon(mats=LIST, w=P, m=P, G=P, low=None, size=62, products=0, denom=0.0, lr=0.1, momentum=0.9, nesterov=1, wd=0.0, rms=0.2, steps=5, coeff=None, eps=1e-7,
         ws=P, nbytes=1 << 30):
    return w, m, G, low, size, hs.make_matrices(mats), products, denom, lr, momentum, nesterov, wd, rms, steps, coeff, eps, ws, nbytes


@pytest.mark.parametrize("change,status", [
    (dict(w=P + 4), INVALID), (dict(m=P + 8), INVALID), (dict(G=P + 4), INVALID), (dict(low=P + 2), INVALID), (dict(w=None), INVALID), (dict(m=None), INVALID), (dict(G=None), INVALID), (dict(denom=-1.0), INVALID), (dict(denom=float("nan")), INVALID),
    (dict(denom=float("inf")), INVALID), (dict(lr=float("nan")), INVALID), (dict(momentum=1.0), INVALID), (dict(momentum=-0.1), INVALID),
    (dict(wd=float("inf")), INVALID), (dict(rms=-1.0), INVALID), (dict(rms=float("inf")), INVALID), (dict(size=61), SHAPE), (dict(nbytes=100), WORKSPACE),
    (dict(mats=[(0, 7, 5, 7)] * 2), INVALID), (dict(steps=0), INVALID)])
def test_update_refuses(change, status):
    refused(status, hs.hs_muon_step, *muon(**change))


def test_coefficients_have_the_shape_of_the_steps():
    with pytest.raises(hs.HsError):
        hs.hs_op_orthogonalize(*ortho(coeff=np.zeros((4, 3))), stream=0)


def test_workspace_sizes():
    one = hs.make_matrices([(0, 1024, 1024, 1024)])
    two = hs.make_matrices([(0, 1024, 1024, 1024), (1 << 20, 1024, 512, 1024)])
    for products in (0, 1):
        a, b = hs.hs_orthogonalize_workspace_bytes(one, products), hs.hs_orthogonalize_workspace_bytes(two, products)
        assert 8 << 20 < a < b < 64 << 20
    assert hs.hs_orthogonalize_workspace_bytes(one, 0) > hs.hs_orthogonalize_workspace_bytes(one, 1)
    wide, tall = hs.make_matrices([(0, 500, 100, 500)]), hs.make_matrices([(0, 100, 500, 100)])
    assert hs.hs_orthogonalize_workspace_bytes(wide, 1) == hs.hs_orthogonalize_workspace_bytes(tall, 1)
    for bad, products in ((hs.make_matrices([(0, 5, 0, 5)]), 1), (one, 7)):
        with pytest.raises(hs.HsError):
            hs.hs_orthogonalize_workspace_bytes(bad, products)


def test_columns_of_one_wider_matrix_are_a_fine_list():
    """What is refused for sharing elements is told apart from neighbours: the call gets as far as its workspace."""
    mats = [(0, 12, 4, 5), (5, 12, 4, 7), (48, 12, 2, 12)]
    refused(WORKSPACE, hs.hs_op_orthogonalize, *ortho(mats=mats, size=72, nbytes=100))


def test_options_of_the_workers():
    from paper_2009_14783_amd.step import MatrixUpdate
    o = MatrixUpdate.options(dict(momentum=0.9), dict(lr=1e-4))
    assert o == dict(MatrixUpdate.DEFAULTS, momentum=0.9, lr=1e-4)
    assert MatrixUpdate.options(dict(lr=1e-3), dict(lr=1e-4))["lr"] == 1e-3
    with pytest.raises(TypeError, match="momentun"):
        MatrixUpdate.options(dict(momentun=0.9), dict(lr=1e-4))
