"""4-bit rows in blocks of 32 with a power of two each, and products of them, against plain implementations in 64 bits.

Tolerances.  Quantised rows are those of exact arithmetic.  An fp32 sum of K products is off by at most K 2^-24 of the sum of their magnitudes (each of K
additions rounds once, relative to a partial sum that is no larger; the products, of 2 x 2 bits of mantissa and powers of two, are exact), the addition of a bias
by 2^-24 of the result, the rounding to a type with unit eps by eps / 2 of it."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2310_03841_amd as ab

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
U32 = 2.0 ** -24
NAN, INF = float("nan"), float("inf")
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def up(n, q):
    return (n + q - 1) // q * q


def ok(rc):
    assert rc == ab.ABFT_OK, ab.abft_strerror(rc)


def values(codes, scale, cols):
    """What packed codes and scales stand for, in 64 bits."""
    codes, scale = np.asarray(codes), np.asarray(scale)
    nib = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1)[:, :cols]
    s = np.repeat(scale, 32, axis=1)[:, :cols].astype(np.float64)
    with np.errstate(all="ignore"):
        return np.where(s == 255, NAN, LEVELS[nib & 7] * np.where(nib >= 8, -1.0, 1.0) * 2.0 ** (s - 127))


def plain_quantize(x):
    """x: float64 [rows][cols] -> (codes of elements, scales)."""
    rows, cols = x.shape
    full = np.zeros((rows, up(cols, 32)))
    full[:, :cols] = x
    b = full.reshape(rows, -1, 32)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(b).all(axis=2)
        b = np.where(bad[..., None], 0.0, b)
        top = np.abs(b).max(axis=2)
        e = np.where(top > 0, np.frexp(top)[1] - 3, -127)
        e = np.clip(e, -127, 127)
        v = np.abs(np.ldexp(b, -e[..., None]))
    far = np.abs(v[..., None] - LEVELS)
    # ties to the even code
    best = far.min(axis=-1, keepdims=True)
    code = np.where(far == best, np.where(np.arange(8) % 2 == 0, 0, 1), 9).argmin(axis=-1)
    code = np.where(v > 6, 7, code) | np.where(np.signbit(b), 8, 0)
    return np.where(bad[..., None], 0, code).reshape(rows, -1), np.where(bad, 255, e + 127)


def quantize(x, dtype, cols, order=None, topk=1, rows=None):
    tokens = x.shape[0]
    rows = tokens if order is None else rows
    q = torch.full((rows, up(cols, 32) // 2 + 16), 0x5A, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, up((cols + 31) // 32, 16) + 16), 0x77, dtype=torch.uint8, device="cuda")
    ok(ab.abft_quantize_mx4(x, ab.DTYPE_CODE[dtype], tokens, cols, x.shape[1], order, rows, topk, q, 2 * q.shape[1], s, s.shape[1]))
    return q, s


def check_quantized(x, dtype, cols):
    q, s = quantize(x, dtype, cols)
    code, scale = plain_quantize(x[:, :cols].double().cpu().numpy())
    nb, half = (cols + 31) // 32, up(cols, 32) // 2
    gq, gs = q.cpu().numpy(), s.cpu().numpy()
    assert np.array_equal(gs[:, :nb], scale) and np.all(gs[:, nb:] == 0x77)
    assert np.array_equal(gq[:, :half], code[:, 0::2] | code[:, 1::2] << 4) and np.all(gq[:, half:] == 0x5A)
    y = torch.full((x.shape[0], x.shape[1]), 77.0, dtype=TORCH[dtype], device="cuda")
    ok(ab.abft_dequantize_mx4(q, 2 * q.shape[1], s, s.shape[1], x.shape[0], cols, y, ab.DTYPE_CODE[dtype], y.shape[1]))
    want = torch.from_numpy(values(gq[:, :half], gs[:, :nb], cols)).to(TORCH[dtype])
    got = y[:, :cols].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got, nan=1.0), torch.nan_to_num(want, nan=1.0))
    assert torch.all(y[:, cols:] == 77)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 7), (3, 8), (5, 31), (4, 32), (7, 33), (197, 768), (3, 1001), (2, 2048), (5, 2049), (9, 4096), (1, 9001), (1030, 72)])
def test_rows_to_4_bits_and_back(dtype, rows, cols):
    gen = torch.Generator().manual_seed(cols)
    ld = up(cols, 8) + 8
    x = torch.randn(rows, ld, generator=gen) * torch.exp(torch.randn(rows, ld, generator=gen) * 2)
    x[:, cols:] = NAN
    check_quantized(x.to(TORCH[dtype]).cuda(), dtype, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_value_of_a_type(dtype):
    """Every bit pattern in a block of its neighbours, and next to a largest one up to sixteen times its size."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.int16).view(TORCH[dtype])
    by_size = bits[torch.sort(torch.nan_to_num(bits.double().abs(), nan=1e300, posinf=1e299, neginf=1e299), stable=True)[1]]
    check_quantized(by_size.view(-1, 64).cuda(), dtype, 64)
    finite = bits[torch.isfinite(bits)]
    for times in (1.0, 1.25, 1.5, 1.75, 2.0, 3.0, 4.0, 5.0, 8.0, 13.0, 16.0):
        pair = torch.stack([finite, (finite.double() * times).to(TORCH[dtype])], dim=1)
        rows = torch.zeros(pair.shape[0], 32, dtype=TORCH[dtype])
        rows[:, 3], rows[:, 17] = pair[:, 0], pair[:, 1]
        check_quantized(rows.cuda(), dtype, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_ties_go_to_the_even_code(dtype):
    steps = torch.arange(-32, 33).double() / 4            # multiples of 1/4 up to 8: every border and the places beside it
    for scale in (2.0 ** -10, 1.0, 2.0 ** 9):
        eps = torch.finfo(TORCH[dtype]).eps
        x = torch.cat([steps, steps * (1 + eps), steps * (1 - eps)])
        x = torch.cat([x, torch.zeros(224 - x.numel(), dtype=torch.float64)]).view(7, 32)
        x[:, 0] = 4.0
        check_quantized((x * scale).to(TORCH[dtype]).cuda(), dtype, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_blocks_that_are_not_finite(dtype):
    x = torch.randn(6, 104, generator=torch.Generator().manual_seed(1))
    x[0, 3], x[1, 40], x[2, 100], x[3], x[4, 32:64] = NAN, INF, -INF, 0.0, 0.0
    x[5] = -0.0
    check_quantized(x.to(TORCH[dtype]).cuda(), dtype, 100)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,topk,cols", [(1, 1, 8), (3, 2, 40), (9, 4, 100), (40, 3, 1024)])
def test_rows_in_the_order_of_their_groups(tokens, topk, cols):
    gen = torch.Generator().manual_seed(cols)
    x = torch.randn(tokens, up(cols, 8), generator=gen).to(torch.bfloat16).cuda()
    n = tokens * topk
    order = torch.randperm(n, generator=gen).to(torch.int32)
    for j, v in ((0, -1), (n // 2, n), (n - 1, 2 ** 31 - 1), (n // 3, -2 ** 31)):
        if n > 4:
            order[j] = v
    q, s = quantize(x, "bf16", cols, order.cuda(), topk, n)
    want, ws = quantize(x, "bf16", cols)
    for r, i in enumerate(order.tolist()):
        if 0 <= i < n:
            assert torch.equal(q[r], want[i // topk]) and torch.equal(s[r], ws[i // topk])
        else:
            assert torch.all(q[r] == 0x5A) and torch.all(s[r] == 0x77)


@pytest.mark.gpu
def test_every_scale_back():
    """All 256 scales and all 16 codes, to both types: rounded once, past the largest value to infinity."""
    q = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(256, 1)[:, :16].contiguous()
    q[:, :8] = torch.tensor([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE], dtype=torch.uint8)
    s = torch.zeros(256, 16, dtype=torch.uint8)
    s[:, 0] = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    for dtype, t in TORCH.items():
        y = torch.zeros(256, 32, dtype=t, device="cuda")
        ok(ab.abft_dequantize_mx4(q.cuda(), 32, s.cuda(), 16, 256, 32, y, ab.DTYPE_CODE[dtype], 32))
        want = torch.from_numpy(values(q.numpy(), s.numpy(), 32)).to(t)
        assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(y.cpu(), nan=1.0), torch.nan_to_num(want, nan=1.0))


# ------------------------------------------------------------------------------------------ products
def rows4(rng, rows, K, spread=3):
    """Random codes and scales; pads behind the last block that must not be used (NaN, and large elements), zeros behind K inside it."""
    nb = (K + 31) // 32
    q = rng.integers(0, 256, (rows, up(nb * 16, 16) + 16)).astype(np.uint8)
    nib = np.stack([q & 15, q >> 4], axis=-1).reshape(rows, -1)
    nib[:, K:nb * 32] = 0
    nib[:, nb * 32:] = 7
    s = rng.integers(127 - spread, 128 + spread, (rows, up(nb, 16) + 16)).astype(np.uint8)
    s[:, nb:] = 255
    return (nib[:, 0::2] | nib[:, 1::2] << 4).astype(np.uint8), s


class Product:
    def __init__(self, ends, N, K, M=None, out="bf16", bias=False, seed=0, ctx=None, dense=False):
        rng = np.random.default_rng(seed)
        self.ends, self.groups, self.N, self.K, self.out, self.t = list(ends), len(ends) - 1, N, K, out, TORCH[out]
        self.M = ends[-1] if M is None else M
        self.A, self.sA = rows4(rng, self.M, K)
        self.B, self.sB = rows4(rng, self.groups * N, K)
        self.bias = rng.normal(size=N).astype(np.float32) if bias else None
        self.own_ctx, self.dense = ctx is None, dense
        self.ctx = ctx or ab.abft_create(self.M, self.groups * N, self.groups * up(K, 128), self.groups)
        self.upload()

    def upload(self):
        dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.d = [dev(x) for x in (self.A, self.sA, self.B, self.sB, self.bias)]
        self.offsets = torch.tensor(self.ends, dtype=torch.int32).cuda()
        self.ldc = up(self.N, 8) + 8
        self.C = torch.full((self.M, self.ldc), 77.0, dtype=self.t, device="cuda")
        self.row_flag = torch.full((self.M,), 9, dtype=torch.uint8, device="cuda")
        self.col_flag = torch.full((self.groups * self.N,), 9, dtype=torch.uint8, device="cuda")
        self.counts = torch.full((8,), 55, dtype=torch.int32, device="cuda")
        A, sA, B, sB, bias = self.d
        self.shape = ab.make_shape(self.M, self.N, self.K, batch=self.groups, lda=2 * A.shape[1], ldb=2 * B.shape[1], strideB=self.N * 2 * B.shape[1], ldc=self.ldc)
        self.q = ab.make_mx4(sA, sA.shape[1], sB, sB.shape[1], self.N * sB.shape[1], bias, out=ab.DTYPE_CODE[self.out])

    def close(self):
        torch.cuda.synchronize()
        if self.own_ctx:
            ab.abft_destroy(self.ctx)

    def run(self, mode=ab.ABFT_OFF, tau=0.0, tau_cols=0.0, **kw):
        res = ab.make_result(self.row_flag, self.col_flag, self.counts, tau=tau, tau_cols=tau_cols)
        ok(ab.abft_gemm_mx4(self.ctx, self.d[0], self.d[2], None if self.dense else self.offsets, self.q, self.C, mode, self.shape, res, **kw))

    def encode(self):
        ok(ab.abft_encode_mx4(self.ctx, self.d[2], self.q, self.shape))

    def want(self):
        a, b = values(self.A, self.sA, self.K), values(self.B, self.sB, self.K).reshape(self.groups, self.N, self.K)
        c, room = np.full((self.M, self.N), 77.0), np.zeros((self.M, self.N))
        for g, (lo, hi) in enumerate(zip(self.ends, self.ends[1:])):
            c[lo:hi], room[lo:hi] = a[lo:hi] @ b[g].T, np.abs(a[lo:hi]) @ np.abs(b[g]).T
        rows = np.zeros(self.M, bool)
        rows[self.ends[0]:self.ends[-1]] = True
        if self.bias is not None:
            c[rows] += self.bias
        return c, room, rows

    def check(self, clean=True):
        c, room, rows = self.want()
        got = self.C.double().cpu().numpy()
        assert np.all(got[~rows] == 77) and np.all(got[:, self.N:] == 77)
        got, eps = got[:, :self.N], torch.finfo(self.t).eps / 2
        # (a partial sum leaves the range of fp32 only where the sum of all magnitudes does: what comes of that is not asked)
        beyond = room >= 2.0 ** 128
        got = np.where(beyond, c, got)
        assert np.array_equal(np.isnan(got), np.isnan(c))
        with np.errstate(all="ignore"):
            tol = (1 + eps) * (self.K * U32 * room + U32 * np.abs(c)) + eps * np.abs(c) + (2.0 ** -25 if self.out == "f16" else 0)
            assert np.all(np.isnan(c) | (got == c) | (np.abs(got - c) <= tol)), np.nanmax(np.abs(got - c) - tol)
        if clean:
            assert self.counts.tolist()[:3] == [0, 0, 0] and int(self.row_flag.sum()) == 0 and int(self.col_flag.sum()) == 0


PRODUCTS = [([0, 1], 1, 1), ([0, 1], 64, 64), ([0, 3], 33, 31), ([0, 16], 100, 257), ([0, 17], 130, 512), ([0, 64], 64, 256), ([0, 65], 200, 1000), ([0, 300], 140, 776), ([0, 1537], 129, 713),
            ([0, 1], 4096, 1024), ([0, 5, 5, 9], 72, 96), ([0, 1, 3, 40, 40, 41], 200, 600), ([2, 7, 30], 70, 2048), ([0, 20, 40, 43], 264, 4096), ([0, 130, 200, 290], 200, 136),
            ([3, 600, 601, 1500], 520, 384), ([0] * 40 + [3, 9], 48, 160), ([0, 3000, 3000, 5000], 1032, 512), ([0, 2, 3], 40, 9000)]


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("ends,N,K", PRODUCTS)
def test_product_matches_plain(out, ends, N, K):
    for n, bias in enumerate((False, True)):
        p = Product(ends, N, K, M=ends[-1] + 3 * n, out=out, bias=bias, seed=N + K, dense=n == 0 and len(ends) == 2)
        try:
            p.run()
            p.check(clean=False)
            p.run(ab.ABFT_DETECT)
            p.check()
            p.C.fill_(77)
            p.encode()
            p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
            p.check()
            p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
            p.check()
        finally:
            p.close()


# each kernel by name, unprotected and protected: which tiles a problem takes
KERNELS = {
    (16, 16): ([0, 1, 4, 9], 200, 520),
    (16, 32): ([0, 2, 2, 22, 24] + list(range(25, 61)), 1030, 1300),
    (64, 64): ([0, 150, 150, 1201], 200, 1000),
    (64, 128): ([0, 1000, 1530, 2311], 1100, 168),
    (256, 256): ([0, 257, 257, 2900, 3029, 5000], 1546, 768),
}
WIDE = ([0, 2, 2, 22, 24] + list(range(25, 61)), 1030, 264)     # protected by 64 columns, else by 32
DEEP = ([0, 255, 4400], 1090, 2304)                             # tiles of 256 x 256 of more slabs than three, and a last round of halves


def tile_of(ends, N, K, mode):
    up32 = up(K, 32)
    return ab.abft_mx4_tile_shape(mode, ab.make_shape(ends[-1], N, K, batch=len(ends) - 1, lda=up32, ldb=up32, strideB=N * up32, ldc=up(N, 8)))


def test_which_kernel_a_problem_takes():
    for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
        for tile, (ends, N, K) in KERNELS.items():
            assert tile_of(ends, N, K, mode) == tile, (tile, mode)
        assert tile_of(*DEEP, mode) == (256, 256)
        assert tile_of(*WIDE, mode) == (16, 64 if mode else 32)
        # not whole slabs of 256 elements (as blocks of 32 cover them), or fewer than three of them
        for K in (736, 769, 512, 3000):
            assert tile_of(KERNELS[256, 256][0], 1546, K, mode) != (256, 256)
        with pytest.raises(ab.AbftError):
            ab.abft_mx4_tile_shape(mode, ab.make_shape(4, 16, 100, lda=96, ldb=128, ldc=16))


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("ends,N,K", list(KERNELS.values()) + [WIDE, DEEP])
def test_each_kernel(out, ends, N, K):
    """Clean, with a bias; flips all over its tiles; blocks of NaN."""
    p = Product(ends, N, K, M=ends[-1] + 2, out=out, bias=True, seed=K)
    try:
        p.run()
        p.check(clean=False)
        sums = p.want()[0] - p.bias
        p.run(ab.ABFT_DETECT)
        p.check()
        rng = np.random.default_rng(K)
        sizes = np.diff(ends)
        places = [(g, r, c) for g in np.flatnonzero(sizes)[[0, -1]] for r in (0, sizes[g] - 1) for c in (0, N - 1)]
        places += [(g, rng.integers(sizes[g]), rng.integers(N)) for g in rng.choice(np.flatnonzero(sizes), 6)]
        for g, r, c in places:
            bit = 29 if abs(sums[ends[g] + r, c]) >= 2 else 30
            ok(ab.abft_inject(p.ctx, None, ab.ABFT_BF16, p.shape, int(g), int(r), int(c), bit, ab.ABFT_INJECT_ACCUMULATOR))
            p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
            assert np.flatnonzero(p.row_flag.cpu().numpy()).tolist() == [ends[g] + r], (g, r, c)
            assert np.flatnonzero(p.col_flag.cpu().numpy()).tolist() == [g * N + c], (g, r, c)
        p.run(ab.ABFT_DETECT)
        p.check()
        # a row of A and a column of B with a block of NaN, in the last group with rows
        g = int(np.flatnonzero(sizes)[-1])
        r, c = ends[g + 1] - 1, g * N + N // 2
        p.sA[r, 0], p.sB[c, (K - 1) // 32] = 255, 255
        p.upload()
        p.run(ab.ABFT_DETECT)
        p.check(clean=False)
        rf, cf = p.row_flag.cpu().numpy(), p.col_flag.cpu().numpy()
        assert rf[r] == 1 and cf[c] == 1 and rf[:ends[g]].sum() == 0 and cf[:g * N].sum() == 0
    finally:
        p.close()


# 32 columns: one piece of 512 bytes to a wave and fewer workgroups than 64 columns ask for (protected); four pieces, and more than those in turn
FEW = [([0, 2, 2, 22, 24] + list(range(25, 61)), 600, 264), ([0] + [17 * i + 4 for i in range(1, 9)], 1030, 2100), ([0] + [17 * i + 4 for i in range(1, 9)], 1030, 4480)]


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", FEW)
def test_each_kernel_of_few_rows(ends, N, K):
    assert tile_of(ends, N, K, ab.ABFT_DETECT) == (16, 32) and (K < 512 or tile_of(ends, N, K, ab.ABFT_OFF) == (16, 32))
    test_each_kernel("bf16", ends, N, K)


@pytest.mark.gpu
@pytest.mark.parametrize("spread", [3, 40])
@pytest.mark.parametrize("ends,N,K", [([0, 1], 40, 31), ([0, 5, 16], 100, 520), ([0, 3, 24, 40], 70, 1300), ([0, 2], 16, 9000), WIDE, KERNELS[16, 32]])
def test_predictions_of_few_rows_are_as_near_as_fp32(ends, N, K, spread):
    """A tile's e^T A is taken as terms of 8 bits, of which 2^-25 of a block's largest sum is left behind: as fp32 does.  With R rows to a tile, every product of a prediction or a sum is at
    most R max|A| max|B|; the additions of a wave's K / 512 MFMAs, those inside one (to some 2^-17 of its largest product), and the last ones over waves and rows stay
    below n = K / 512 + 8 steps of 2^-20 K R max|A| max|B|.  Tolerances of 1e-3 K max|A| max|B| lie 5 times and more above."""
    assert tile_of(ends, N, K, ab.ABFT_DETECT)[0] == 16
    p = Product(ends, N, K, seed=K + spread)
    try:
        rng = np.random.default_rng(1)
        p.sA[:, :(K + 31) // 32] = rng.integers(127 - spread, 128 + spread, (p.M, (K + 31) // 32))
        p.upload()
        R = min(16, int(np.diff(ends).max()))
        a, b = values(p.A, p.sA, K), values(p.B, p.sB, K)
        tau_cols = (K / 512 + 8) * 2.0 ** -20 * K * R * np.abs(a).max() * np.abs(b).max()
        p.run(ab.ABFT_DETECT, tau_cols=tau_cols)
        p.check()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", [([0, 3, 3, 8], 70, 96), ([0, 20, 21, 22, 23], 70, 600), ([0, 130, 200, 290], 200, 136), ([0, 600, 1500], 520, 384), ([0, 2500], 1100, 512)])
def test_a_flip_in_an_accumulator_is_found(ends, N, K):
    """The bit of one sum's exponent that makes it 2^64 or more times as large: its row and its column, and no others."""
    p = Product(ends, N, K, seed=3)
    try:
        sums = p.want()[0]
        for n, g in enumerate(g for g in range(p.groups) if ends[g + 1] > ends[g]):
            for row, col in {(0, 0), (ends[g + 1] - ends[g] - 1, N - 1), ((ends[g + 1] - ends[g]) // 2, N // 3)}:
                for mode in (ab.ABFT_DETECT, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED):
                    bit = 29 if abs(sums[ends[g] + row, col]) >= 2 else 30
                    ok(ab.abft_inject(p.ctx, None, ab.ABFT_BF16, p.shape, g, row, col, bit, ab.ABFT_INJECT_ACCUMULATOR))
                    p.run(mode)
                    rf, cf = p.row_flag.cpu().numpy(), p.col_flag.cpu().numpy()
                    assert np.flatnonzero(rf).tolist() == [ends[g] + row], (g, row, col)
                    assert np.flatnonzero(cf).tolist() == [g * N + col], (g, row, col)
                    assert p.counts.tolist()[:3] == [1, 1, 1]
                    p.run(mode)
                    p.check()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", [([0, 4, 9], 64, 256), ([0, 200, 400], 192, 256)])
def test_a_weight_that_changed_behind_its_encoding_shows_in_rows(ends, N, K):
    p = Product(ends, N, K, seed=5)
    try:
        p.encode()
        p.d[3][N + 7, 2] += 8                                   # a block's power of two
        p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
        rf = p.row_flag.cpu().numpy()
        assert rf[:ends[1]].sum() == 0 and rf[ends[1]:].sum() > (ends[2] - ends[1]) // 2 and int(p.col_flag.sum()) == 0
        assert p.counts.tolist()[2] == ab.ABFT_CHECKSUM_SUSPECT
        p.run(ab.ABFT_DETECT)                                    # encodes what is there
        assert p.counts.tolist()[:3] == [0, 0, 0]
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", [([0, 3, 7], 40, 200), ([0, 100, 230], 140, 400), ([0, 1500, 2600], 1040, 288)])
def test_blocks_of_nan_stay_in_their_rows_and_columns(ends, N, K):
    p = Product(ends, N, K, seed=6)
    try:
        r, c = ends[1] + 1, N + N // 2                          # a row of group 1, a column of it
        p.sA[r, 1] = 255
        p.sB[c, 2] = 255
        p.upload()
        p.run()
        p.check(clean=False)
        p.run(ab.ABFT_DETECT)
        p.check(clean=False)
        rf, cf = p.row_flag.cpu().numpy(), p.col_flag.cpu().numpy()
        assert rf[r] == 1 and cf[c] == 1 and rf[:ends[1]].sum() == 0 and cf[:N].sum() == 0
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", list(KERNELS.values()) + [WIDE, DEEP])
def test_a_nan_flags_its_own_and_all_that_meet_it_in_a_sum(ends, N, K):
    """A row of A that is NaN makes the sums of all columns of its group NaN, and no row but itself; a column of B those of all rows of its group."""
    p = Product(ends, N, K, M=ends[-1] + 2, seed=K)
    try:
        sizes = np.diff(ends)
        for g in np.flatnonzero(sizes)[[0, -1]]:
            r, c = int(ends[g] + sizes[g] // 2), int(g * N + N // 3)
            for which, at, rows, cols in ((p.sA, (r, K // 64), [r], list(range(g * N, g * N + N))), (p.sB, (c, (K - 1) // 32), list(range(ends[g], ends[g + 1])), [c])):
                kept, which[at] = which[at], 255
                p.upload()
                p.run(ab.ABFT_DETECT)
                p.check(clean=False)
                assert np.flatnonzero(p.row_flag.cpu().numpy()[:ends[-1]]).tolist() == rows
                assert np.flatnonzero(p.col_flag.cpu().numpy()).tolist() == cols
                which[at] = kept
        p.upload()
        p.run(ab.ABFT_DETECT)
        p.check()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("a,b", [(127, 127), (18, 245), (245, 18), (245, 110), (110, 245), (181, 181), (80, 80), (74, 74), (30, 140), (140, 30)])
@pytest.mark.parametrize("rows", [4, 70])
def test_checks_over_the_scales_that_they_hold_for(rows, a, b):
    """With 96 columns of depth and sums of up to 72: max|A| = 6 2^(a-127), their product and max|B| are at least 72000 2^-126, sums of either at most 72 times that, and predictions 72 96 36
    2^(a+b-254), stay below 2^127.  Clean calls are clean and a flip of an exponent is found."""
    N, K = 72, 96
    big = 6 * 2.0 ** (max(a, b) - 127), 36 * 2.0 ** (a + b - 254)
    assert 72 * big[0] < 2.0 ** 127 and K * N * big[1] < 2.0 ** 127 and min(6 * 2.0 ** (min(a, b) - 127), big[1]) >= 72000 * 2.0 ** -126
    p = Product([0, rows], N, K, seed=a)
    try:
        p.sA[:, :3], p.sB[:, :3] = a, b
        p.upload()
        p.run(ab.ABFT_DETECT)
        p.check()
        c = p.want()[0]
        i, j = np.unravel_index(np.abs(c).argmax(), c.shape)
        # (the flip makes the largest sum four times or a fourth of what it was: a change by three quarters of it at least, many times the tolerance of 0.096 max|A| max|B|)
        assert 0.75 * np.abs(c).max() > 4 * 0.096 * 36 * 2.0 ** (a + b - 254)
        ok(ab.abft_inject(p.ctx, None, ab.ABFT_BF16, p.shape, 0, int(i), int(j), 24, ab.ABFT_INJECT_ACCUMULATOR))
        p.run(ab.ABFT_DETECT)
        assert np.flatnonzero(p.row_flag.cpu().numpy()).tolist() == [i] and np.flatnonzero(p.col_flag.cpu().numpy()).tolist() == [j]
    finally:
        p.close()


@pytest.mark.gpu
def test_scales_at_the_ends_of_their_range():
    """Powers of two from 2^-127 to 2^127."""
    for a, b in ((0, 254), (254, 0), (254, 1), (127, 127), (190, 190), (64, 64), (100, 100), (183, 183), (253, 110)):
        for rows in (4, 70):
            p = Product([0, rows], 72, 96, seed=a)
            try:
                p.sA[:, :3], p.sB[:, :3] = a, b
                p.upload()
                p.run()
                p.check(clean=False)
            finally:
                p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("K", [1 << 29, (1 << 29) - 128])
def test_the_greatest_depth(K):
    """One row of A, of ones in some of its blocks and zeros else, and one of B, of ones: sums of small whole numbers, exact in fp32, and a tolerance below one block's."""
    nb = K // 32
    A, B = torch.zeros(1, K // 2, dtype=torch.uint8, device="cuda"), torch.full((1, K // 2), 0x22, dtype=torch.uint8, device="cuda")
    sA, sB = (torch.full((1, up(nb, 16)), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    blocks = torch.cat([torch.tensor([0, nb - 1]), torch.randint(0, nb, (998,), generator=torch.Generator().manual_seed(1))]).unique().cuda()
    A.view(nb, 16)[blocks] = 0x22
    C, flags = torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda"), [torch.full((n,), 9, dtype=t, device="cuda") for n, t in ((1, torch.uint8), (1, torch.uint8), (8, torch.int32))]
    ctx = ab.abft_create(1, 1, K, 1)
    try:
        shape, q = ab.make_shape(1, 1, K, lda=K, ldb=K, ldc=8), ab.make_mx4(sA, sA.shape[1], sB, sB.shape[1])
        ok(ab.abft_gemm_mx4(ctx, A, B, None, q, C, ab.ABFT_DETECT, shape, ab.make_result(*flags, tau=16.0)))
        assert float(C[0, 0]) == float(torch.tensor(32.0 * blocks.numel()).to(torch.bfloat16)) and int(torch.count_nonzero(C[0, 1:])) == 0
        assert flags[2].tolist()[:3] == [0, 0, 0] and int(flags[0]) == 0 and int(flags[1]) == 0
        # every block of the encoding: an element of A that meets one wrong there is found
        B.view(nb, 16)[int(blocks[-2]), 3] = 0x77
        ok(ab.abft_gemm_mx4(ctx, A, B, None, q, C, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED, shape, ab.make_result(*flags, tau=8.0)))
        assert int(flags[0]) == 1
    finally:
        torch.cuda.synchronize()
        ab.abft_destroy(ctx)


@pytest.mark.gpu
def test_tolerances_of_the_caller():
    """A flip of the highest bit of a sum's mantissa changes it by d, half of the power of two it begins with: tolerances below and above d, for rows and for columns.  (The sums
    themselves are off by some K 2^-24 of their magnitudes, far below a largest sum's d.)"""
    for rows in (8, 300):
        p = Product([0, rows], 96, 256, seed=9)
        try:
            c, room, _ = p.want()
            i, j = np.unravel_index(np.abs(c).argmax(), c.shape)
            d = 2.0 ** (np.floor(np.log2(abs(c[i, j]))) - 1)
            # a prediction and a sum are each of at most 256 + 96 + 300 additions one behind the other: together they stay below d / 2
            assert d / 2 > 2 * (256 + 96 + 300) * U32 * max(room.sum(axis=0).max(), room.sum(axis=1).max())
            for tau, tau_cols in ((d / 2, 2 * d), (2 * d, d / 2), (d / 2, 0.0), (2 * d, 0.0)):
                ok(ab.abft_inject(p.ctx, None, ab.ABFT_BF16, p.shape, 0, int(i), int(j), 22, ab.ABFT_INJECT_ACCUMULATOR))
                p.run(ab.ABFT_DETECT, tau=tau, tau_cols=tau_cols)
                assert np.flatnonzero(p.row_flag.cpu().numpy()).tolist() == ([i] if tau < d else [])
                assert np.flatnonzero(p.col_flag.cpu().numpy()).tolist() == ([j] if (tau_cols or tau) < d else [])
        finally:
            p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 50, 20, 64], [-5, 10, 30, 400], [2 ** 31 - 1, -2 ** 31, 64, 64], [64, 0, 0, 64]])
def test_bad_offsets_address_nothing_outside(bad):
    p = Product([0, 20, 40, 64], 72, 96, seed=10)
    try:
        whole = torch.full((64 + 512, p.ldc), 5.0, dtype=torch.bfloat16, device="cuda")
        p.C = whole[256:320]
        p.offsets = torch.tensor(bad, dtype=torch.int32).cuda()
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            p.run(mode)
        assert torch.all(whole[:256] == 5) and torch.all(whole[320:] == 5)
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N", [([40000, 40003, 69999], 24), ([10, 30000, 69990], 256)])
def test_places_past_32_bits(ends, N):
    """Rows of A 64 KB apart and of C 64 KB apart, 4.6 GB each."""
    M, K = 70000, 96
    p = Product(ends, N, K, M=M, seed=12)
    try:
        wide = torch.zeros(M, 65536, dtype=torch.uint8, device="cuda")
        wide[:, :p.A.shape[1]] = p.d[0]
        C = torch.zeros(M, 32768, dtype=torch.bfloat16, device="cuda")
        p.shape.lda, p.shape.ldc = 131072, 32768
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            C.zero_()
            ok(ab.abft_gemm_mx4(p.ctx, wide, p.d[2], p.offsets, p.q, C, mode, p.shape, ab.make_result(p.row_flag, p.col_flag, p.counts)))
            p.C[:, :N] = C[:, :N]
            p.C[:ends[0], :N], p.C[ends[-1]:, :N] = 77, 77
            p.check(clean=mode != ab.ABFT_OFF)
            assert int(torch.count_nonzero(C[:, N:])) == 0
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", [([0, 2, 2, 9], 200, 256), ([0, 100, 350], 200, 136), ([0, 1000, 2500], 1024, 256)])
def test_products_can_be_captured_in_a_graph(ends, N, K):
    """Two graphs of one context, replayed in turn with eager calls between, and offsets that change."""
    p = Product(ends, N, K, seed=14)
    try:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            p.run(ab.ABFT_DETECT)
            s.synchronize()
            graphs = []
            for mode in (ab.ABFT_DETECT, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    p.run(mode)
                graphs.append(g)
            rng = np.random.default_rng(1)
            p.run(ab.ABFT_DETECT)
            for i in range(5):
                p.ends = [0] + sorted(rng.integers(0, p.M + 1, p.groups - 1).tolist()) + [p.M]
                p.offsets.copy_(torch.tensor(p.ends, dtype=torch.int32))
                p.C.fill_(77)
                graphs[i & 1].replay()
                s.synchronize()
                p.check()
                p.run(ab.ABFT_DETECT | (ab.ABFT_B_CHECKSUM_CACHED if i & 1 else 0))
                s.synchronize()
                p.check()
    finally:
        p.close()


@pytest.mark.gpu
def test_4_bit_and_other_products_share_a_context():
    """An encoding of one kind of weights is not another's, and predictions of an earlier product are given up."""
    M, N, K = 64, 128, 256
    ctx = ab.abft_create(M, N, K, 1)
    try:
        p = Product([0, M], N, K, seed=15, ctx=ctx, dense=True)
        A, B, C = (torch.randn(*s, device="cuda").to(torch.bfloat16) for s in ((M, K), (N, K), (M, N)))
        s, res = ab.make_shape(M, N, K), ab.make_result(p.row_flag, p.col_flag, p.counts)
        ok(ab.abft_encode_b(ctx, B, ab.ABFT_BF16, s))
        cached = ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED
        assert ab.abft_gemm_mx4(ctx, p.d[0], p.d[2], None, p.q, p.C, cached, p.shape, res) == ab.ABFT_ESTATE
        p.encode()
        assert ab.abft_gemm(ctx, A, B, C, ab.ABFT_BF16, cached, s, res) == ab.ABFT_ESTATE
        ok(ab.abft_gemm(ctx, A, B, C, ab.ABFT_BF16, ab.ABFT_DETECT, s, res))
        assert p.counts.tolist()[:3] == [0, 0, 0]
        p.run(ab.ABFT_DETECT)
        p.check()
        assert ab.abft_verify(ctx, C, ab.ABFT_BF16, s, res) == ab.ABFT_ESTATE
        ok(ab.abft_gemm(ctx, A, B, C, ab.ABFT_BF16, ab.ABFT_DETECT, s, res))
        assert p.counts.tolist()[:3] == [0, 0, 0]
        p.run(ab.ABFT_OFF)
        assert ab.abft_verify(ctx, C, ab.ABFT_BF16, s, res) == ab.ABFT_ESTATE
        event = torch.cuda.Event()
        event.record()
        ok(ab.abft_gemm_done_event(ctx, event.cuda_event))
        p.run(ab.ABFT_DETECT)
        event.synchronize()
        p.check()
    finally:
        torch.cuda.synchronize()
        ab.abft_destroy(ctx)


@pytest.mark.gpu
def test_two_contexts_on_two_streams_at_once():
    ps = [Product([0, 700, 1500], 520, 512, seed=20), Product([0, 3, 9, 20], 520, 512, seed=21)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    try:
        torch.cuda.synchronize()
        for _ in range(20):
            for p, s in zip(ps, streams):
                p.run(ab.ABFT_DETECT, stream=s.cuda_stream)
        torch.cuda.synchronize()
        for p in ps:
            p.check()
    finally:
        for p in ps:
            p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [5, 300])
def test_a_layer_of_4_bit_experts(tokens):
    """From tokens to output: choices, sorted rows straight to 4 bits, the protected product, rows back."""
    E, topk, K, N = 8, 2, 264, 200
    gen = torch.Generator().manual_seed(tokens)
    x, logits = torch.randn(tokens, K, generator=gen).to(torch.bfloat16).cuda(), torch.randn(tokens, E, generator=gen).cuda()
    W = (torch.randn(E * N, K, generator=gen) * 0.1).to(torch.bfloat16).cuda()
    n, z = tokens * topk, lambda t, *s: torch.zeros(s, dtype=t, device="cuda")
    ids, w, offsets, order, place = z(torch.int32, tokens, topk), z(torch.float32, tokens, topk), z(torch.int32, E + 1), z(torch.int32, n), z(torch.int32, n)
    qw, sw = quantize(W, "bf16", K)
    q, s = z(torch.uint8, n, 144), z(torch.uint8, n, 16)
    y, out = z(torch.bfloat16, n, N), z(torch.bfloat16, tokens, N)
    flags = z(torch.uint8, n), z(torch.uint8, E * N), z(torch.int32, 8)
    ctx = ab.abft_create(n, E * N, E * 384, E)
    try:
        ok(ab.abft_route(logits, ab.ABFT_F32, ab.make_routing(tokens, E, topk), ids, w))
        ok(ab.abft_group_rows(ctx, ids, n, E, offsets, order, place))
        ok(ab.abft_quantize_mx4(x, ab.ABFT_BF16, tokens, K, K, order, n, topk, q, 288, s, 16))
        mx = ab.make_mx4(s, 16, sw, sw.shape[1], N * sw.shape[1])
        shape = ab.make_shape(n, N, K, batch=E, lda=288, ldb=2 * qw.shape[1], strideB=N * 2 * qw.shape[1], ldc=N)
        ok(ab.abft_encode_mx4(ctx, qw, mx, shape))
        ok(ab.abft_gemm_mx4(ctx, q, qw, offsets, mx, y, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED, shape, ab.make_result(*flags)))
        ok(ab.abft_combine_rows(y, ab.ABFT_BF16, n, N, N, place, w, tokens, topk, None, 0, out, N))
        qx, sx = quantize(x, "bf16", K)
        a, b = values(qx.cpu().numpy(), sx.cpu().numpy(), K), values(qw.cpu().numpy(), sw.cpu().numpy(), K).reshape(E, N, K)
        best = torch.sort(logits.cpu(), dim=1, descending=True, stable=True)[1][:, :topk].numpy()
        assert np.array_equal(ids.cpu().numpy(), best)
        p = np.exp(np.take_along_axis(logits.double().cpu().numpy(), best, axis=1))
        p /= p.sum(axis=1, keepdims=True)
        want, room = np.zeros((tokens, N)), np.zeros((tokens, N))
        for t in range(tokens):
            for j, e in enumerate(best[t]):
                want[t] += p[t, j] * (b[e] @ a[t])
                room[t] += p[t, j] * (np.abs(b[e]) @ np.abs(a[t]))
        # the product and the sum of two are each rounded to bf16; weights, products and sums in fp32
        tol = 2 * 2.0 ** -8 * 1.01 * room + (K + 64) * U32 * room
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
        assert flags[2].tolist()[:3] == [0, 0, 0]
    finally:
        torch.cuda.synchronize()
        ab.abft_destroy(ctx)


# ------------------------------------------------------------------------------------------ refusals
P = 0x1000


def test_refusals_need_no_gpu():
    E, S, A = ab.ABFT_EINVAL, ab.ABFT_ESHAPE, ab.ABFT_EALIGN

    def expect(call, good, changes):
        for change, code in changes:
            assert call(**{**good, **change}) == code, change

    expect(ab.abft_quantize_mx4, dict(X=P, dtype=ab.ABFT_BF16, tokens=4, cols=40, ldx=40, order=None, rows=4, topk=1, Q=P, ldq=64, scale=P, lds=16, stream=0),
           [(dict(dtype=ab.ABFT_I8), E), (dict(dtype=ab.ABFT_F32), E), (dict(topk=0), E), (dict(tokens=0), S), (dict(cols=0), S), (dict(rows=3), S), (dict(rows=0, order=P), S), (dict(ldx=32), S),
            (dict(ldq=32), S), (dict(lds=1), S), (dict(X=None), E), (dict(Q=None), E), (dict(scale=None), E), (dict(ldx=44), A), (dict(ldq=72), A), (dict(lds=8), A), (dict(X=P + 8), A),
            (dict(Q=P + 8), A), (dict(scale=P + 8), A), (dict(order=P + 2), A), (dict(tokens=1 << 31, rows=1 << 31), S)])
    expect(ab.abft_dequantize_mx4, dict(Q=P, ldq=64, scale=P, lds=16, rows=4, cols=40, X=P, dtype=ab.ABFT_F16, ldx=40, stream=0),
           [(dict(dtype=ab.ABFT_I8), E), (dict(rows=0), S), (dict(cols=0), S), (dict(ldq=32), S), (dict(lds=1), S), (dict(ldx=32), S), (dict(X=None), E), (dict(Q=None), E), (dict(scale=None), E),
            (dict(ldx=44), A), (dict(ldq=72), A), (dict(lds=8), A), (dict(X=P + 8), A), (dict(Q=P + 8), A), (dict(scale=P + 8), A)])
    sh = lambda **k: ab.make_shape(**{**dict(M=8, N=16, K=100, batch=2, lda=128, ldb=128, ldc=16, strideB=2048), **k})
    mx = lambda **k: ab.make_mx4(**{**dict(a=P, lda=16, b=P, ldb=16, strideB=256), **k})
    reserved = mx()
    reserved.reserved = 1
    both = [(dict(), E), (dict(mx4=reserved), E), (dict(mx4=mx(out=ab.ABFT_I8)), E), (dict(mx4=mx(b=None)), E), (dict(mx4=mx(b=P + 8)), A), (dict(mx4=mx(bias=P + 2)), A), (dict(mx4=mx(ldb=2)), S),
            (dict(mx4=mx(ldb=20)), A), (dict(mx4=mx(strideB=100)), A), (dict(shape=sh(transB=False)), E), (dict(shape=sh(M=0)), S), (dict(shape=sh(N=0)), S), (dict(shape=sh(K=0)), S),
            (dict(shape=sh(batch=0)), S), (dict(shape=sh(ldb=96)), S), (dict(shape=sh(ldb=144)), A), (dict(shape=sh(strideB=2064)), A), (dict(shape=sh(batch=1 << 16)), S)]
    expect(ab.abft_encode_mx4, dict(ctx=None, B=P, mx4=mx(), shape=sh(), stream=0), both)
    expect(ab.abft_gemm_mx4, dict(ctx=None, A=P, B=P, offsets=P, mx4=mx(), C=P, mode=ab.ABFT_OFF, shape=sh(), result=None, stream=0),
           both + [(dict(mx4=None), E), (dict(mx4=mx(a=None)), E), (dict(mx4=mx(a=P + 8)), A), (dict(mx4=mx(lda=3)), S), (dict(mx4=mx(lda=20)), A), (dict(shape=sh(lda=96)), S), (dict(shape=sh(lda=144)), A),
                   (dict(shape=sh(ldc=8)), S), (dict(shape=sh(ldc=20)), A), (dict(mode=ab.ABFT_DETECT_CORRECT), E), (dict(mode=ab.ABFT_DETECT | ab.ABFT_STORED_SUMS), E)])
    assert ctypes.sizeof(ab.abft_mx4) == 7 * 8


@pytest.mark.gpu
def test_refusals():
    """None of these calls launches anything: the pointers are never followed."""
    E, S, A, W = ab.ABFT_EINVAL, ab.ABFT_ESHAPE, ab.ABFT_EALIGN, ab.ABFT_EWORKSPACE
    ctx = ab.abft_create(64, 128, 512, 2)
    try:
        sh = lambda **k: ab.make_shape(**{**dict(M=64, N=64, K=100, batch=2, lda=128, ldb=128, ldc=64, strideB=8192), **k})
        mx, res = ab.make_mx4(P, 16, P, 16, 1024), ab.make_result(P, P, P)
        g = lambda **k: ab.abft_gemm_mx4(**{**dict(ctx=ctx, A=P, B=P, offsets=P, mx4=mx, C=P, mode=ab.ABFT_DETECT, shape=sh(), result=res), **k})
        for change, code in [(dict(A=None), E), (dict(B=None), E), (dict(C=None), E), (dict(offsets=None), E), (dict(A=P + 8), A), (dict(B=P + 8), A), (dict(C=P + 8), A), (dict(offsets=P + 2), A),
                             (dict(result=None), E), (dict(result=ab.make_result(P, None, P)), E), (dict(result=ab.make_result(P, P, P, tau=-1.0)), E), (dict(shape=sh(M=65)), W),
                             (dict(shape=sh(N=65, ldc=72)), W), (dict(shape=sh(K=500, lda=512, ldb=512)), W), (dict(shape=sh(batch=3)), W),
                             (dict(mode=ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED), ab.ABFT_ESTATE)]:
            assert g(**change) == code, change
        wide = ab.make_mx4(P, 32, P, 32, 4096)
        assert g(shape=sh(K=700, lda=704, ldb=704), mx4=wide) == W
        assert ab.abft_encode_mx4(ctx, None, mx, sh()) == E and ab.abft_encode_mx4(ctx, P + 8, mx, sh()) == A and ab.abft_encode_mx4(ctx, P, mx, sh(N=65)) == W
    finally:
        ab.abft_destroy(ctx)
