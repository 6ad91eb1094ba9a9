"""Each kernel of the products over groups of rows by name: which sizes reach it (no GPU needed), and on each the cases where one can go wrong without another doing
so: flips of accumulators all over its tiles, values that are not finite, offsets that are not what they should be."""
import random

import pytest
import torch

import paper_2310_03841_amd as ab
from test_group_ops import TORCH, TYPES, Group, half_step, one_flip, pad, stored_bits

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
    (FEW_WIDE, INT8, [0, 0, 0, 1, 2, 2, 3, 6, 6, 7, 8, 8, 8, 9, 10, 12, 12], 1100, 400, True),
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


def near_one(p, at, j, plain):
    """A column next to j whose sum in row `at` is of [2^-10, 1): with bit 30, the upper bit of its exponent, it becomes 2^118 or more, past every tolerance."""
    for c in list(range(j, -1, -1)) + list(range(j + 1, p.N)):
        if 2.0 ** -10 <= abs(plain[at, c].item()) < 0.99:
            return c
    raise AssertionError(at)


def places(p, plain, count, seed):
    """(group, row of the group, column): the deepest group's first and last rows and both sides of its tiles' edges, other groups' ends, corners, and some anywhere."""
    rng = random.Random(seed)
    rows = [p.ends[g + 1] - p.ends[g] for g in range(p.groups)]
    used = [g for g in range(p.groups) if rows[g]]
    deep = max(used, key=lambda g: rows[g])
    want = [(deep, rows[deep] - 1, p.N - 1), (used[0], 0, 0), (used[-1], rows[used[-1]] - 1, p.N - 1), (deep, 0, p.N - 1)]
    edges = [i for i in (15, 16, 63, 64, 127, 128, 255, 256, rows[deep] & ~255, rows[deep] & ~127) if i < rows[deep]]
    want += [(deep, i, rng.randrange(p.N)) for i in edges]
    while len(want) < count:
        g = rng.choice(used)
        want.append((g, rng.randrange(rows[g]), rng.randrange(p.N)))
    return want if p.dtype == "i8" else [(g, i, near_one(p, p.ends[g] + i, j, plain)) for g, i, j in want]


def of_types(types):
    """Cases with each of the types (operands, C) that they are for."""
    return [(tile, ends, N, K, trans_b, dtype, out) for tile, dtypes, ends, N, K, trans_b in CASES for dtype, out in types if dtype in dtypes]


@pytest.mark.gpu
@pytest.mark.parametrize("tile,ends,N,K,trans_b,dtype,out", of_types(TYPES))
def test_flips_all_over_the_tiles(tile, ends, N, K, trans_b, dtype, out):
    print(f"case {tile} {dtype} {out} {ends[:8]} {N} {K} {trans_b}", flush=True)
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1] + 3, out=out, bias=out == "f16", seed=71)
    try:
        p.run(ab.ABFT_DETECT)
        p.check()
        p.clean()
        clean = stored_bits(p)
        plain = p.plain()[0] if dtype != "i8" else None
        for n, (g, i, j) in enumerate(places(p, plain, 16, seed=N + K)):
            if n % 4 == 0:
                one_flip(p, clean, g, i, j, 30, ab.ABFT_OFF)
            # (a low bit of an integer sum need not show in a scaled C: any does in the sums)
            bit = 30 if dtype != "i8" or out else (30, 0, 31, 7)[n % 4]
            one_flip(p, clean, g, i, j, bit, ab.ABFT_DETECT)
            if out and n % 4 == 1:
                assert ab.abft_inject(p.ctx, None, p.code, p.shape, g, i, j, 0, ab.ABFT_INJECT_ACCUMULATOR) == ab.ABFT_OK
                p.run(ab.ABFT_DETECT)
                assert p.row_flag.nonzero().flatten().tolist() == [p.ends[g] + i] and p.col_flag.nonzero().flatten().tolist() == [g * N + j]
        p.run(ab.ABFT_DETECT)
        p.clean()
        assert torch.equal(stored_bits(p), clean)
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("tile,ends,N,K,trans_b,dtype,out", of_types([("bf16", None), ("f16", None)]))
def test_what_is_not_finite_stays_in_its_group(tile, ends, N, K, trans_b, dtype, out, value):
    print(f"case {tile} {dtype} {value} {ends[:8]} {N} {K} {trans_b}", flush=True)
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1] + 3, seed=72)
    try:
        want, tol = p.plain()
        rows = [p.ends[g + 1] - p.ends[g] for g in range(p.groups)]
        used = [g for g in range(p.groups) if rows[g]]
        in_a, in_b = max(used, key=lambda g: rows[g]), used[0]
        at = p.ends[in_a + 1] - 1
        p.A[at, K - 1] = value
        p.B[in_b][(N - 1, K - 1) if trans_b else (K - 1, N - 1)] = value
        p.dA, p.dB = p.A.cuda(), p.B.cuda()
        p.run(ab.ABFT_DETECT)
        got = p.C.cpu().double()[:, :N]
        bad = torch.zeros(p.M, N, dtype=torch.bool)
        bad[at], bad[p.ends[in_b]:p.ends[in_b + 1], N - 1] = True, True
        used_rows = torch.zeros(p.M, dtype=torch.bool)
        used_rows[p.ends[0]:p.ends[-1]] = True
        assert not torch.isfinite(got[bad]).any() and bool((got[~used_rows] == p.fill).all())
        fine = ~bad & used_rows[:, None]
        step = half_step(p.c_type)
        assert ((got - want).abs()[fine] <= (tol * (1 + step) + step * want.abs() + torch.finfo(p.c_type).tiny)[fine]).all()
        rf, cf = p.row_flag.cpu(), p.col_flag.cpu().view(p.groups, N)
        assert rf[at].item() == 1 and cf[in_b, N - 1].item() == 1
        for g in range(p.groups):
            if g not in (in_a, in_b):
                assert not rf[p.ends[g]:p.ends[g + 1]].any() and not cf[g].any(), g
        assert not rf[~used_rows].any()
    finally:
        p.close()


def wrong_offsets(M, groups):
    """Falling, before the first row, behind the last, and the ends of their type."""
    fall = [M - M * e // groups for e in range(groups + 1)]
    saw = [0 if e % 2 else M for e in range(groups + 1)]
    out = [-5 + e * (M + 400) // groups for e in range(groups + 1)]
    ends = [(2 ** 31 - 1, -2 ** 31, M // 2)[e % 3] for e in range(groups + 1)]
    return [fall, saw, out, ends]


def inside(n, dtype, fill):
    """(n elements, all of them with as many again on either side)."""
    whole = torch.full((3 * n,), fill, dtype=dtype, device="cuda")
    return whole[n:2 * n], whole


@pytest.mark.gpu
@pytest.mark.parametrize("tile,ends,N,K,trans_b,dtype,out", of_types([("i8", "bf16"), ("bf16", None)]))
def test_wrong_offsets_write_nothing_outside(tile, ends, N, K, trans_b, dtype, out):
    """Every kernel clamps what it reads of the offsets to [0, M]; C and the verdict lie inside larger buffers, the rest of which stays as it is."""
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1] + 3, out=out, seed=73)
    try:
        C, whole_c = inside((p.M + 256) * p.ldc, p.c_type, 5)
        p.C = C[:p.M * p.ldc].view(p.M, p.ldc)
        p.row_flag, whole_r = inside(p.M, torch.uint8, 6)
        p.col_flag, whole_f = inside(p.groups * N, torch.uint8, 7)
        for bad in wrong_offsets(p.M, p.groups):
            print(f"case {tile} {dtype} {N} {K} {trans_b} {bad[:6]}", flush=True)
            p.offsets = torch.tensor(bad, dtype=torch.int32).cuda()
            for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
                p.run(mode)
            n = C.numel()
            assert bool((whole_c[:n] == 5).all()) and bool((whole_c[n + p.M * p.ldc:] == 5).all())
            assert bool((p.C[:, N:] == 5).all())
            for whole, fill in ((whole_r, 6), (whole_f, 7)):
                n = whole.numel() // 3
                assert bool((whole[:n] == fill).all()) and bool((whole[2 * n:] == fill).all())
        # and with the right ones all is well again
        p.C.fill_(p.fill)
        p.offsets = torch.tensor(p.ends, dtype=torch.int32).cuda()
        p.run(ab.ABFT_DETECT)
        p.check()
        p.clean()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", FLOAT)
@pytest.mark.parametrize("trans_b", [True, False])
def test_gradients_on_tall_tiles_end_inside_16_bytes(dtype, trans_b):
    """Sizes that fill the chip and end inside a chunk on both sides, with NaN behind the last element of every row of both operands; a group of one row, one of none.
    Sums of at most 2600 products of whole numbers of at most 3 are exact in fp32, so one rounding is left."""
    ends, N, K = [0, 2600, 2601, 2601, 4001], 2053, 1021
    gen = torch.Generator().manual_seed(74)
    M, groups, t = ends[-1] + 3, len(ends) - 1, TORCH[dtype]

    def whole(rows, cols):
        x = torch.full((rows, pad(cols, 2)), float("nan"), dtype=t)
        x[:, :cols] = torch.randint(-3, 4, (rows, cols), generator=gen, dtype=torch.int8).to(t)
        return x.cuda()

    X, dY = whole(M, K), whole(M, N)
    rows, cols = (N, K) if trans_b else (K, N)
    dW = torch.full((groups, rows + 1, pad(cols, 2)), 77.0, dtype=t, device="cuda")
    ctx = ab.abft_create(M, groups * N, groups * 1024, groups)
    try:
        s = ab.make_shape(M, N, K, batch=groups, lda=X.shape[1], ldb=dW.shape[2], ldc=dY.shape[1], strideB=dW.stride(0), transB=trans_b)
        off = torch.tensor(ends, dtype=torch.int32).cuda()
        assert ab.abft_gemm_grouped_wgrad(ctx, X, dY, off, dW, ab.DTYPE_CODE[dtype], s) == ab.ABFT_OK
        torch.cuda.synchronize()
        assert bool((dW[:, rows] == 77).all()) and bool((dW[:, :, cols:] == 77).all()), "written outside the gradients"
        for g in range(groups):
            a, b = ends[g], ends[g + 1]
            want = torch.mm(dY[a:b, :N].float().t().contiguous(), X[a:b, :K].float())
            want = (want if trans_b else want.t()).to(t)
            assert torch.equal(dW[g, :rows, :cols], want), g
        for bad in wrong_offsets(M, groups):
            print(f"case {dtype} {trans_b} {bad}", flush=True)
            dW.fill_(77.0)
            off = torch.tensor(bad, dtype=torch.int32).cuda()
            assert ab.abft_gemm_grouped_wgrad(ctx, X, dY, off, dW, ab.DTYPE_CODE[dtype], s) == ab.ABFT_OK
            torch.cuda.synchronize()
            assert bool((dW[:, rows] == 77).all()) and bool((dW[:, :, cols:] == 77).all()), bad
    finally:
        ab.abft_destroy(ctx)
