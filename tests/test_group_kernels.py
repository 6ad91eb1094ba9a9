"""Each kernel of the products over groups of rows by name: which sizes reach it (no GPU needed)."""
import pytest

import paper_2310_03841_amd as ab
from test_group_ops import pad

FEW, FEW_WIDE, SQUARE, WIDE, TALL = (16, 16), (16, 32), (64, 64), (64, 128), (256, 256)
INT8, FLOAT = ["i8"], ["bf16", "f16"]
BOTH = INT8 + FLOAT
SEVENTY = [0] + [73 * i + 9 * (i % 5) for i in range(1, 70)] + [5200]
# (rows and columns of a tile, operands, offsets, N, K, transB); three rows behind the last group are in none.  Ragged depths, columns that end inside a tile and
# inside 16 bytes, groups without rows, left-over rows of every kind, more groups than lanes
CASES = [
    (FEW, BOTH, [0, 9, 9, 26, 27, 28], 97, 1000, True),
    (FEW, BOTH, [0, 17], 200, 1000, True),
    (FEW_WIDE, BOTH, [0, 1, 1, 3, 3, 3, 4, 5, 6, 6, 7, 7, 7, 8, 8, 9, 14], 1030, 400, True),
    (SQUARE, BOTH, [3, 20, 147, 148, 276], 130, 72, False),
    (SQUARE, BOTH, [0, 17, 100, 100, 900], 300, 713, True),
    (SQUARE, BOTH, [0, 500, 501, 1500], 600, 713, False),
    (WIDE, BOTH, [0, 2000, 2001, 4999], 1027, 136, True),
    (WIDE, BOTH, [0, 2000, 2001, 5000], 1027, 200, False),
    (TALL, BOTH, [0, 100, 1124, 1124, 2500, 6100], 2043, 384, True),
    (TALL, FLOAT, [0, 100, 1124, 1124, 2500, 6100], 2043, 448, False),
    (TALL, BOTH, [0, 4000, 4001, 9500], 2043, 640, True),
    (TALL, FLOAT, [0, 4000, 4001, 9500], 2043, 640, False),
    (TALL, BOTH, SEVENTY, 1024, 384, True),
    (TALL, FLOAT, SEVENTY, 1024, 448, False),
    (WIDE, INT8, SEVENTY, 1024, 448, False),
]


def shape_of(dtype, ends, N, K, trans_b):
    es = 1 if dtype == "i8" else 2
    return ab.make_shape(ends[-1] + 3, N, K, batch=len(ends) - 1, lda=pad(K, es), ldb=pad(K if trans_b else N, es), ldc=pad(N, 2), transB=trans_b)


@pytest.mark.parametrize("tile,dtypes,ends,N,K,trans_b", CASES)
def test_the_cases_reach_their_kernel(tile, dtypes, ends, N, K, trans_b):
    for dtype in dtypes:
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            assert ab.abft_group_tile_shape(ab.DTYPE_CODE[dtype], mode, shape_of(dtype, ends, N, K, trans_b)) == tile, (dtype, mode)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("rows,groups,N,K", [(31, 32, 4096, 1024), (15, 16, 4096, 1024), (48, 64, 2048, 768), (40, 48, 1536, 1024)])
def test_fewer_rows_than_groups_fill_the_chip_too(dtype, rows, groups, N, K):
    """A group has one row on average, rounded up as tiles are: 32 columns to a workgroup as soon as those are 512, as with a row to each group."""
    ask = lambda M: ab.abft_group_tile_shape(ab.DTYPE_CODE[dtype], ab.ABFT_DETECT, ab.make_shape(M, N, K, batch=groups))
    assert ask(rows) == ask(groups) == FEW_WIDE
    assert ask(max(1, 400 * 32 // N)) in (FEW, SQUARE)


def test_tile_shape_refuses_what_the_calls_refuse():
    ask = lambda dtype=ab.ABFT_BF16, mode=ab.ABFT_OFF, **k: ab.abft_group_tile_shape(dtype, mode, ab.make_shape(**{**dict(M=64, N=64, K=64, batch=4), **k}))
    assert ask() == FEW and ask(transB=False) == SQUARE

    def refused(code, **k):
        with pytest.raises(ab.AbftError) as e:
            ask(**k)
        assert e.value.code == code, k

    for k in (dict(dtype=7), dict(mode=ab.ABFT_DETECT_CORRECT), dict(mode=ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)):
        refused(ab.ABFT_EINVAL, **k)
    for k in (dict(M=0), dict(N=0), dict(K=0), dict(lda=60), dict(ldb=60), dict(ldc=56), dict(M=(1 << 30) + 8), dict(K=(1 << 29) + 8), dict(N=(1 << 25) + 8),
              dict(batch=65536), dict(dtype=ab.ABFT_I8, K=1 << 17)):
        refused(ab.ABFT_ESHAPE, **k)
    for k in (dict(lda=68), dict(ldb=68), dict(ldc=66), dict(strideB=-64)):
        refused(ab.ABFT_EALIGN, **k)
    # one tile more than a launch has workgroups, and one less; workgroups that pass over A
    one = dict(batch=1, K=8, ldb=8, lda=8)
    refused(ab.ABFT_ESHAPE, M=1 << 19, N=1 << 18, **one)
    assert ask(M=(1 << 19) - 64, N=1 << 18, **one) == WIDE
    refused(ab.ABFT_ESHAPE, M=1 << 30, N=1, ldc=8, mode=ab.ABFT_DETECT, **one)
    assert ask(M=1 << 28, N=1, ldc=8, mode=ab.ABFT_DETECT, **one) == SQUARE
