"""Which tiles the 8-bit products and the matrix update take, asked on the host."""
import numpy as np
import pytest

from paper_2009_14783_amd import binding as hs


def stack(shapes):
    at, mats = 0, []
    for r, c in shapes:
        mats.append((at, c, r, c))
        at += r * c
    return hs.make_matrices(mats)


def test_products_of_8_bits():
    assert hs.hs_gemm_fp8_choice(1, 1024, 1024) == (64, 1) and hs.hs_gemm_fp8_choice(8192, 8192, 8192) == (256, 1)
    assert hs.hs_gemm_fp8_choice(8192, 2304, 768) == (128, 1)
    rng = np.random.default_rng(1)
    for M, N, K in rng.integers(1, 9000, (300, 3)).tolist():
        for f32 in (0, 1):
            tile, splits = hs.hs_gemm_fp8_choice(M, N, K, f32)
            assert tile in (64, 128, 256) and splits == 1                       # without scratch there is one part
            tile, splits = hs.hs_gemm_fp8_choice(M, N, K, f32, 32 << 20)
            assert splits == 1 or (splits <= 32 and 4 * splits * M * N <= 32 << 20 and 512 * (splits - 1) < K)
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 22) + 1)):
        with pytest.raises(hs.HsError):
            hs.hs_gemm_fp8_choice(*bad)


def test_lists_of_matrices():
    assert hs.hs_orthogonalize_choice(stack([(100, 300)]), 1, 0) == (2, (0, 0, 0))
    mixed = stack([(1024, 1024)] * 96 + [(4096, 1024), (1024, 4096)] * 24)
    assert [hs.hs_orthogonalize_choice(mixed, 1, i)[0] for i in (0, 95, 96, 143)] == [0, 0, 1, 1]
    assert hs.hs_orthogonalize_choice(stack([(64, 4000)] * 200), 1, 0)[0] == 0      # nor are few rows taken through A alone
    assert hs.hs_orthogonalize_choice(mixed, 0, 143)[0] == 0                     # 32-bit products go step by step
    for products in (0, 1):
        for shapes in ([(130, 190)], [(330, 330)] * 40, [(200, 2000)] * 100, [(64 + i, 400) for i in range(40)]):
            lst = stack(shapes)
            for i in (0, len(shapes) - 1):
                way, tiles = hs.hs_orthogonalize_choice(lst, products, i)
                assert all(t in ((0,) if way == 2 else (32, 64, 128) if products == 0 else (32, 64, 128, 256)) for t in tiles) and tiles[1] < 256
    one = stack([(330, 330)])
    for bad in ((one, 7, 0), (one, 1, 1), (one, 1, -1), (stack([]), 1, 0), (hs.make_matrices([(0, 5, 0, 5)]), 1, 0)):
        with pytest.raises(hs.HsError):
            hs.hs_orthogonalize_choice(*bad)
