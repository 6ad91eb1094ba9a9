"""Operators of quantised layers and of mixtures of experts against plain implementations in 64 bits: rows to int8, int8 products with scales, products
grouped by expert and the gradients of their weights.

Tolerances.  A result rounded once from fp32 to a type with unit eps is off by at most eps / 2 of its size; an fp32 sum of K products
by at most K 2^-24 of the sum of their magnitudes (each of K additions rounds once, relative to a partial sum that is no larger); each
further fp32 step by 2^-24 of its result.  Integers are equal."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2310_03841_amd as ab

TORCH = {"i8": torch.int8, "bf16": torch.bfloat16, "f16": torch.float16}
U32 = 2.0 ** -24


def pad(n, es):
    q = 16 // es
    return (n + q - 1) // q * q


def rand(gen, dtype, *shape, std=1.0):
    """Values on the host; the last dimension padded to whole 16 bytes with a NaN, or a large integer, that must not be used."""
    es = 1 if dtype == "i8" else 2
    ld = pad(shape[-1], es)
    if dtype == "i8":
        x = torch.randint(-128, 128, shape[:-1] + (ld,), generator=gen, dtype=torch.int8)
        x[..., shape[-1]:] = 101
        return x
    x = (torch.randn(shape[:-1] + (ld,), generator=gen) * std).to(TORCH[dtype])
    x[..., shape[-1]:] = float("nan")
    return x


def half_step(t):
    return torch.finfo(t).eps / 2


class Group:
    """One product over groups of rows: operands on the host, what a program holds on the GPU, the plain results."""

    def __init__(self, dtype, ends, N, K, trans_b=True, M=None, out=None, bias=False, seed=0, ctx=None, dense=False):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.N, self.K, self.trans_b, self.out, self.dense = dtype, N, K, trans_b, out, dense
        self.ends, self.groups = list(ends), len(ends) - 1
        self.M = M if M is not None else ends[-1]
        self.A = rand(gen, dtype, self.M, K)
        self.B = rand(gen, dtype, self.groups, *((N, K) if trans_b else (K, N)), std=0.1)
        self.row = self.col = self.bias = None
        if out:
            self.row = torch.rand(self.M, generator=gen) * 0.03 + 0.001
            self.col = torch.rand(self.groups, N, generator=gen) * 0.001 + 0.0001
            self.bias = torch.randn(N, generator=gen) if bias else None
        self.c_type = TORCH[out] if out else (torch.int32 if dtype == "i8" else TORCH[dtype])
        self.ldc = pad(N, 4 if self.c_type == torch.int32 else 2)
        self.code = ab.DTYPE_CODE[dtype]
        self.own_ctx = ctx is None
        self.ctx = ctx or ab.abft_create(self.M, self.groups * N, self.groups * ((K + 127) // 128 * 128), self.groups)
        self.upload()

    def upload(self):
        dev = lambda x: None if x is None else x.cuda()
        self.dA, self.dB, self.dcol, self.drow, self.dbias = dev(self.A), dev(self.B), dev(self.col), dev(self.row), dev(self.bias)
        self.offsets = torch.tensor(self.ends, dtype=torch.int32).cuda()
        self.fill = 77
        self.C = torch.full((self.M, self.ldc), self.fill, dtype=self.c_type, device="cuda")
        self.row_flag = torch.full((self.M,), 9, dtype=torch.uint8, device="cuda")
        self.col_flag = torch.full((self.groups * self.N,), 9, dtype=torch.uint8, device="cuda")
        self.counts = torch.full((8,), 55, dtype=torch.int32, device="cuda")
        self.shape = ab.make_shape(self.M, self.N, self.K, batch=self.groups, lda=self.A.shape[-1], ldb=self.B.shape[-1], ldc=self.ldc,
                                   transB=self.trans_b)
        self.scales = ab.make_scales(self.drow, self.dcol, self.dbias, out=ab.DTYPE_CODE[self.out]) if self.out else None

    def close(self):
        if self.own_ctx:
            ab.abft_destroy(self.ctx)

    def call(self, mode=ab.ABFT_OFF, tau=0.0, tau_cols=0.0):
        r = None if mode == ab.ABFT_OFF else ab.make_result(self.row_flag, self.col_flag, self.counts, tau, tau_cols)
        if self.dense:
            return ab.abft_gemm_scaled(self.ctx, self.dA, self.dB, self.scales, self.C, mode, self.shape, r)
        return ab.abft_gemm_grouped(self.ctx, self.dA, self.dB, self.offsets, self.scales, self.C, self.code, mode, self.shape, r)

    def run(self, mode=ab.ABFT_OFF, **kw):
        rc = self.call(mode, **kw)
        assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
        torch.cuda.synchronize()

    def weights(self, g):
        b = self.B[g].double()
        return b[:, :self.K].t() if self.trans_b else b[:, :self.N]

    def plain(self):
        """(C in 64 bits, how far each element may be off)."""
        C = torch.zeros(self.M, self.N, dtype=torch.float64)
        tol = torch.zeros_like(C)
        for g in range(self.groups):
            a, b = self.ends[g], self.ends[g + 1]
            x, w = self.A[a:b, :self.K].double(), self.weights(g)
            p = x @ w
            t = torch.zeros_like(p)
            if self.dtype != "i8":
                t = self.K * U32 * (x.abs() @ w.abs())
            if self.out:
                p = p * self.row[a:b, None].double() * self.col[g].double()
                t = 4 * U32 * p.abs()
                if self.bias is not None:
                    p = p + self.bias.double()
                    t = t + U32 * p.abs()
            C[a:b], tol[a:b] = p, t
        return C, tol

    def check(self, C=None):
        want, tol = self.plain()
        got = (self.C if C is None else C).cpu()
        used = torch.zeros(self.M, dtype=torch.bool)
        for a, b in zip(self.ends, self.ends[1:]):
            used[a:b] = True
        assert bool((got[~used] == self.fill).all()), "rows of no group were written"
        assert bool((got[:, self.N:] == self.fill).all()), "the pad was written"
        got = got[:, :self.N].double()[used]
        want, tol = want[used], tol[used]
        if self.c_type == torch.int32:
            assert torch.equal(got, want)
            return
        step = half_step(self.c_type)
        tiny = torch.finfo(self.c_type).tiny * 2 * step                     # half a step below the normal numbers
        worst = ((got - want).abs() - (tol * (1 + step) + step * want.abs() + tiny)).max().item() if got.numel() else 0.0
        assert worst <= 0, worst

    def clean(self):
        assert not self.row_flag.any() and not self.col_flag.any()
        assert self.counts[:5].tolist() == [0, 0, 0, 0, 0]


# (offsets, N, K, transB): one row and one column upwards, edges of tiles of 16 to 256, empty groups first, last and between, rows of no group ahead
SHAPES = [
    ([0, 1], 1, 1, True),
    ([0, 1, 1, 3], 5, 9, True),
    ([0, 0, 64, 64, 129, 129], 64, 64, True),
    ([3, 20, 147, 148, 276], 130, 72, True),
    ([0, 63, 128, 193], 200, 713, True),
    ([0, 5, 9, 9, 26], 97, 264, False),
    ([0, 130, 131], 257, 136, False),
    ([0, 300, 300, 557], 300, 1000, False),
    ([2, 2, 2], 33, 40, True),                          # no rows in any group
    ([0, 600, 700], 512, 384, True),
    ([0, 257, 1100], 520, 1152, True),
    (list(range(0, 71)), 40, 128, True),                # 70 groups of a row each
    ([0] * 66 + [7, 7, 40], 64, 96, True),              # more groups than lanes, nearly all empty
    (list(range(0, 130 * 3, 3)), 72, 200, False),
]
# Tiles of every shape in both layouts of B
SHAPES += [([0, 1000, 1700, 3000], 2000, 136, True), ([0, 9000, 17000], 60, 72, False)]
# Enough for tiles of 256: left-over rows of every kind, a group without rows, columns that end inside a tile, K of the fewest slabs and of many, rows of no
# group; more than 64 groups; fewer tiles than compute units, and some rounds of them
BIG = [
    ([7, 100, 1124, 1124, 2500, 4100], 1030, 384, True),
    ([0, 256, 512, 640, 769, 4097], 1024, 1152, True),
    ([0, 1, 2, 130, 4224], 1030, 384, False),
    ([0, 1500, 1500, 4100], 1001, 448, False),
    (list(range(0, 131 * 130, 130)), 264, 384, True),
    ([0, 8192], 512, 384, True),
    ([0, 4000, 12600], 2056, 384, True),
    ([0, 5000, 5000, 12000], 1024, 448, False),
]
# Few rows to a group: one and sixteen and seventeen of them, groups of many among them, one piece of K and many, parts of a piece, and both widths of tiles
FEW = [
    ([0, 1], 4096, 1024, True),
    ([0, 16, 17, 49, 49, 50, 64], 100, 4104, True),
    ([1, 2, 3, 20, 20, 21], 33, 50, True),
    (list(range(0, 71)), 264, 136, True),
    ([0] * 40 + [170] + [171] * 23, 264, 200, True),
    ([0, 13], 1000, 713, True),
    (list(range(0, 65)), 264, 2000, True),
    (list(range(0, 33)), 2048, 1024, True),
]
TYPES = [("i8", None), ("i8", "bf16"), ("i8", "f16"), ("bf16", None), ("f16", None)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("ends,N,K,trans_b", SHAPES + BIG + FEW)
def test_grouped_matches_plain(dtype, out, ends, N, K, trans_b):
    print(f"case {dtype} {out} {ends[:8]} {N} {K} {trans_b}", flush=True)
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1] + 5, out=out, bias=bool(N % 2), seed=N + K)
    try:
        p.run()
        p.check()
        p.C.fill_(p.fill)
        p.run(ab.ABFT_DETECT)
        p.check()
        p.clean()
        # with the encoding kept, twice: what a call accumulates into starts at zero each time
        assert ab.abft_encode_b(p.ctx, p.dB, p.code, p.shape) == ab.ABFT_OK
        for _ in range(3):
            p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
            p.check()
            p.clean()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,trans_b", [(1, 64, 64, True), (1, 1000, 713, True), (7, 40, 4096, True), (16, 768, 768, True), (17, 33, 100, True),
                                           (33, 130, 200, False), (197, 768, 768, True), (300, 1001, 713, False), (1100, 520, 1152, True),
                                           (520, 600, 4224, True), (2050, 2060, 384, True)])
def test_scaled_matches_plain(out, M, N, K, trans_b):
    print(f"case {out} {M} {N} {K} {trans_b}", flush=True)
    p = Group("i8", [0, M], N, K, trans_b, out=out, bias=bool(M % 2), seed=M, dense=True)
    try:
        p.run()
        p.check()
        p.C.fill_(p.fill)
        p.run(ab.ABFT_DETECT)
        p.check()
        p.clean()
    finally:
        p.close()


@pytest.mark.gpu
def test_scales_left_out_are_ones():
    p = Group("i8", [0, 40], 70, 33, out="f16", seed=3, dense=True)
    try:
        p.scales = ab.make_scales(out=ab.ABFT_F16)
        p.B = (p.B.float() / 40).to(torch.int8)          # sums that fp16 holds
        p.A = (p.A.float() / 10).to(torch.int8)
        p.dA, p.dB = p.A.cuda(), p.B.cuda()
        p.row[:], p.col[:] = 1.0, 1.0
        p.run()
        p.check()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("ends,N,K", [([0, 7, 30], 70, 96), ([0, 100, 1124, 1124, 2500, 6100], 2043, 384), ([0, 130, 1000], 1030, 136), ([0, 8000], 520, 384)])
def test_scaled_results_are_rounded_step_by_step(out, ends, N, K):
    """fp32 behind the row's scale, fp32 behind the column's and the bias together, then C's type, in tiles inside C, at its edges, and where a flip is armed: what
    a product gives does not depend on which kernel or part of one makes it.  (Sums are below 2^24, so each is its own fp32 value; product and bias in 64 bits, 48 of
    which the product takes, are rounded to fp32 as one rounding does.)"""
    p = Group("i8", ends, N, K, M=ends[-1], out=out, bias=True, seed=17)
    try:
        group = torch.repeat_interleave(torch.arange(p.groups), torch.tensor(ends).diff())
        acc = torch.zeros(p.M, N)
        for g in range(p.groups):
            acc[ends[g]:ends[g + 1]] = (p.A[ends[g]:ends[g + 1], :K].double() @ p.weights(g)).float()
        assert acc.abs().max() < 2 ** 24
        want = ((acc * p.row[:, None]).double() * p.col[group].double() + p.bias.double()).float().to(TORCH[out])
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            p.run(mode)
            assert torch.equal(p.C.cpu()[:, :N], want), mode
        # a flip in an element whose neighbours are then made by what serves tiles at an edge
        g = max(range(p.groups), key=lambda e: ends[e + 1] - ends[e])
        s = ab.make_shape(1, N, K, batch=p.groups, lda=p.A.shape[-1], ldb=p.B.shape[-1], ldc=p.ldc, strideC=p.M * p.ldc)
        assert ab.abft_inject(p.ctx, None, p.code, s, g, 0, 1, 30, ab.ABFT_INJECT_ACCUMULATOR) == ab.ABFT_OK
        p.run()
        assert (p.C.cpu()[:, :N] != want).nonzero().tolist() == [[ends[g], 1]]
    finally:
        p.close()


# ------------------------------------------------------------------------------------------ faults
def flips(p, g, i, j, bit, mode):
    s = ab.make_shape(1 if p.M < p.groups else p.M // p.groups, p.N, p.K, batch=p.groups, lda=p.A.shape[-1], ldb=p.B.shape[-1], ldc=p.ldc,
                      strideA=0, strideC=p.M * p.ldc, transB=p.trans_b)
    rc = ab.abft_inject(p.ctx, None, p.code, s, g, i, j, bit, ab.ABFT_INJECT_ACCUMULATOR)
    assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
    p.run(mode)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("ends,N,K,trans_b", [([0, 3, 3, 8], 70, 96, True), ([0, 20, 21, 21, 22, 23], 70, 600, True), ([0, 130, 200, 290], 200, 136, False), ([0, 600, 1500], 520, 384, True),
                                               ([0, 1300, 1300, 4200], 1030, 384, True), ([0, 1300, 1300, 4200], 1030, 384, False)])
def test_a_flip_in_an_accumulator_is_found(dtype, out, ends, N, K, trans_b):
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1], out=out, seed=5)
    try:
        for g in range(p.groups):
            rows = p.ends[g + 1] - p.ends[g]
            if not rows:
                continue
            i, j = min(rows, max(1, p.M // p.groups)) - 1, N - 1
            flips(p, g, i, j, 30, ab.ABFT_DETECT)
            rf, cf = p.row_flag.nonzero().flatten().tolist(), p.col_flag.nonzero().flatten().tolist()
            assert rf == [p.ends[g] + i] and cf == [g * N + j], (g, rf, cf)
            assert p.counts[:5].tolist() == [1, 1, ab.ABFT_LOCALISED, 0, ab.ABFT_LOCALISED]
            p.run(ab.ABFT_DETECT)
            p.clean()
            p.check()
    finally:
        p.close()


def one_flip(p, clean, g, i, j, bit, mode):
    """A flip armed with the call's own shape: what differs in C, and what is flagged, is its element."""
    rc = ab.abft_inject(p.ctx, None, p.code, p.shape, g, i, j, bit, ab.ABFT_INJECT_ACCUMULATOR)
    assert rc == ab.ABFT_OK, (g, i, j, ab.abft_strerror(rc))
    p.run(mode)
    at = p.ends[g] + i
    differs = (p.C.view(torch.int16 if p.C.element_size() == 2 else torch.int32) != clean).nonzero().tolist()
    assert differs == [[at, j]], (g, i, j, bit, differs[:5])
    if mode != ab.ABFT_OFF:
        rf, cf = p.row_flag.nonzero().flatten().tolist(), p.col_flag.nonzero().flatten().tolist()
        assert rf == [at] and cf == [g * p.N + j], (g, i, j, bit, rf[:5], cf[:5])
        assert p.counts[:5].tolist() == [1, 1, ab.ABFT_LOCALISED, 0, ab.ABFT_LOCALISED]


def stored_bits(p):
    return p.C.clone().view(torch.int16 if p.C.element_size() == 2 else torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("ends,N,K,trans_b", [([0, 0, 7], 70, 96, True), ([2, 5, 290], 200, 136, False), ([0, 20, 1500, 1500], 520, 384, True)])
def test_a_flip_is_armed_with_the_shape_of_the_call(dtype, out, ends, N, K, trans_b):
    """M of a grouped call counts the rows of all groups; a context of its size takes a flip in any of a group's rows.  Bit 30 moves a floating-point sum by 2 at
    least; the tolerance is 1e-3 K max|A| max|B| < 1e-3 384 5.2 0.52 = 1.04."""
    p = Group(dtype, ends, N, K, trans_b, M=ends[-1] + 3, out=out, seed=13)
    try:
        p.run(ab.ABFT_DETECT)
        p.check()
        clean = stored_bits(p)
        g = max(range(p.groups), key=lambda e: p.ends[e + 1] - p.ends[e])
        rows = p.ends[g + 1] - p.ends[g]
        for i, j in ((0, 0), (rows - 1, N - 1), (rows // 2, N // 3)):
            for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
                one_flip(p, clean, g, i, j, 30, mode)
        # a row that the group does not have: armed, and gone with the next call
        assert ab.abft_inject(p.ctx, None, p.code, p.shape, g, rows, 0, 30, ab.ABFT_INJECT_ACCUMULATOR) == ab.ABFT_OK
        for _ in range(2):
            p.run(ab.ABFT_DETECT)
            p.clean()
            assert torch.equal(stored_bits(p), clean)
        inject = lambda *at: ab.abft_inject(p.ctx, None, p.code, p.shape, *at, 30, ab.ABFT_INJECT_ACCUMULATOR)
        for at in ((p.groups, 0, 0), (-1, 0, 0), (0, p.M, 0), (0, -1, 0), (0, 0, N), (0, 0, -1)):
            assert inject(*at) == ab.ABFT_EINVAL, at
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("i8", "bf16"), ("i8", None), ("bf16", None)])
def test_a_weight_that_changed_behind_its_encoding_shows_in_rows(dtype, out):
    p = Group(dtype, [0, 20, 20, 37, 120], 90, 160, out=out, M=125, seed=6)
    try:
        p.A[:, 5] = 3
        p.dA = p.A.cuda()
        assert ab.abft_encode_b(p.ctx, p.dB, p.code, p.shape) == ab.ABFT_OK
        p.dB[2, 11, 5] = 100
        p.B[2, 11, 5] = 100
        p.run(ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED)
        p.check()
        assert p.row_flag.nonzero().flatten().tolist() == list(range(20, 37))
        assert not p.col_flag.any() and p.counts[2].item() == ab.ABFT_CHECKSUM_SUSPECT
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("ends,N,K,trans_b", [([0, 2, 5], 40, 72, True), ([0, 20, 31], 40, 712, True), ([0, 70, 190], 136, 200, False), ([0, 300, 700], 520, 512, True), ([0, 1300, 4200], 1030, 512, True),
                                               ([0, 1300, 4200], 1030, 512, False)])
def test_values_that_are_not_finite_stay_in_their_rows_and_columns(dtype, value, ends, N, K, trans_b):
    p = Group(dtype, ends, N, K, trans_b, seed=7)
    try:
        clean, _ = p.plain()
        i = ends[1]                                           # first row of the second group
        p.A[i, K - 1] = value
        p.B[0][(N - 1, 0) if trans_b else (0, N - 1)] = value
        p.dA, p.dB = p.A.cuda(), p.B.cuda()
        p.run(ab.ABFT_DETECT)
        got = p.C.cpu().double()[:, :N]
        bad = torch.zeros(p.M, N, dtype=torch.bool)
        bad[i], bad[:ends[1], N - 1] = True, True
        assert not torch.isfinite(got[bad]).any() and torch.isfinite(got[~bad]).all()
        step = half_step(p.c_type)
        assert ((got - clean).abs()[~bad] <= step * clean.abs()[~bad] + 1e-3).all()
        # what is not finite always flags: its row, its column, and the sums that it enters
        assert p.row_flag[i].item() == 1 and p.col_flag[N - 1].item() == 1
    finally:
        p.close()


@pytest.mark.gpu
def test_tolerances_of_the_caller():
    """tau for both checks, tau_cols for the columns alone, in each kernel: a flip that the default tolerance finds and a wide one does not."""
    for ends, N, K in (([0, 3, 8], 70, 96), ([0, 100, 330], 200, 136), ([0, 1300, 4200], 1024, 384)):
        p = Group("bf16", ends, N, K, seed=8)
        try:
            for tau, tau_cols, want in ((0.0, 0.0, (1, 1)), (1e30, 0.0, (0, 0)), (1e30, 1e-3, (0, 1)), (1e-3, 1e30, (1, 0))):
                s = ab.make_shape(1, N, K, batch=p.groups, lda=p.A.shape[-1], ldb=p.B.shape[-1], ldc=p.ldc, strideA=0, strideC=p.M * p.ldc)
                assert ab.abft_inject(p.ctx, None, p.code, s, 1, 0, 5, 29, ab.ABFT_INJECT_ACCUMULATOR) == ab.ABFT_OK
                p.run(ab.ABFT_DETECT, tau=tau, tau_cols=tau_cols)
                flip = p.ends[1]
                assert (p.row_flag[flip].item(), p.col_flag[N + 5].item()) == want, (ends, tau, tau_cols)
                if tau != 1e-3 and tau_cols != 1e-3:
                    assert p.counts[:2].tolist() == list(want)
        finally:
            p.close()


# ------------------------------------------------------------------------------------------ layouts
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("i8", "bf16"), ("i8", None), ("bf16", None)])
@pytest.mark.parametrize("ends,N,K,trans_b", [([0, 2, 7], 50, 70, True), ([0, 80, 200], 130, 200, True), ([0, 80, 200], 130, 200, False),
                                              ([0, 1300, 4200], 1024, 384, True), ([0, 5000, 9000], 1024, 448, False)])
def test_wide_rows_and_matrices_far_apart(dtype, out, ends, N, K, trans_b):
    p = Group(dtype, ends, N, K, trans_b, out=out, seed=9)
    try:
        q = 16 if dtype == "i8" else 8
        wide = lambda x, more, pre: torch.nn.functional.pad(x, (0, more) + pre).cuda()
        p.dA = wide(p.A, 3 * q, ())
        whole = wide(p.B, 5 * q, (0, 3))
        p.dB = whole
        p.C = torch.full((p.M, p.ldc + 24), p.fill, dtype=p.c_type, device="cuda")
        p.shape = ab.make_shape(p.M, N, K, batch=p.groups, lda=p.dA.shape[1], ldb=whole.shape[2], ldc=p.C.shape[1], strideB=whole.stride(0), transB=trans_b)
        p.run(ab.ABFT_DETECT)
        p.check()
        p.clean()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("ends,N,K", [([40000, 40003, 69999], 24, 96), ([10, 30000, 69990], 256, 384)])
def test_places_past_32_bits(ends, N, K):
    """Rows of A and C, and matrices, more than 2^31 and 2^32 bytes from the first: those of the last group are compared."""
    M, lda, ldc = 70000, 65536, 40960
    A = torch.empty((M, lda), dtype=torch.int8, device="cuda")
    A[:, :K].random_(-128, 128)
    B = torch.empty((2, 1 << 32), dtype=torch.int8, device="cuda")
    C = torch.empty((M, ldc), dtype=torch.bfloat16, device="cuda")
    C[:, :N].fill_(7)
    W = torch.randint(-128, 128, (2, N, 384), dtype=torch.int8, device="cuda")
    for g in range(2):
        B[g, :N * 384] = W[g].flatten()
    ctx = ab.abft_create(M, 2 * N, 2 * 384, 2)
    try:
        off = torch.tensor(ends, dtype=torch.int32, device="cuda")
        rf, cf, cnt = (torch.full((n,), 3, dtype=t, device="cuda") for n, t in ((M, torch.uint8), (2 * N, torch.uint8), (8, torch.int32)))
        s = ab.make_shape(M, N, K, batch=2, lda=lda, ldb=384, ldc=ldc, strideB=1 << 32)
        row = torch.rand(M, device="cuda") * 1e-3
        sc = ab.make_scales(row, None, None, out=ab.ABFT_BF16)
        assert ab.abft_gemm_grouped(ctx, A, B, off, sc, C, ab.ABFT_I8, ab.ABFT_DETECT, s, ab.make_result(rf, cf, cnt)) == ab.ABFT_OK
        torch.cuda.synchronize()
        assert cnt[:3].tolist() == [0, 0, 0] and not rf.any() and not cf.any()
        for g in range(2):
            for a, b in ((ends[g], min(ends[g] + 100, ends[g + 1])), (max(ends[g + 1] - 100, ends[g]), ends[g + 1])):
                want = (A[a:b, :K].double() @ W[g, :, :K].double().t()) * row[a:b, None].double()
                got = C[a:b, :N].double()
                assert ((got - want).abs() <= half_step(torch.bfloat16) * want.abs() + 4 * U32 * want.abs()).all()
        assert (C[:ends[0], :N] == 7).all() and (C[ends[2]:, :N] == 7).all()
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
def test_two_contexts_on_two_streams_at_once():
    a, b = Group("bf16", [0, 900, 2500], 520, 384, seed=61), Group("i8", [0, 5, 9, 40], 300, 512, out="f16", seed=62)
    try:
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for _ in range(5):
            for p, st in zip((a, b), streams):
                with torch.cuda.stream(st):
                    assert p.call(ab.ABFT_DETECT) == ab.ABFT_OK
        torch.cuda.synchronize()
        for p in (a, b):
            p.check()
            p.clean()
    finally:
        a.close()
        b.close()


# ------------------------------------------------------------------------------------------ gradients
def wgrad(dtype, ends, N, K, trans_b, M=None, seed=0, guard=0):
    gen = torch.Generator().manual_seed(seed)
    M = M if M is not None else ends[-1]
    groups = len(ends) - 1
    X, dY = rand(gen, dtype, M, K), rand(gen, dtype, M, N, std=0.1)
    rows, cols = (N, K) if trans_b else (K, N)
    dW = torch.full((groups, rows + guard, pad(cols, 2)), 77.0, dtype=TORCH[dtype], device="cuda")
    ctx = ab.abft_create(M, groups * N, groups * ((K + 127) // 128 * 128), groups)
    s = ab.make_shape(M, N, K, batch=groups, lda=X.shape[-1], ldb=dW.shape[-1], ldc=dY.shape[-1], strideB=dW.stride(0), transB=trans_b)
    dX, ddY, off = X.cuda(), dY.cuda(), torch.tensor(ends, dtype=torch.int32).cuda()
    rc = ab.abft_gemm_grouped_wgrad(ctx, dX, ddY, off, dW, ab.DTYPE_CODE[dtype], s)
    assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
    torch.cuda.synchronize()
    ab.abft_destroy(ctx)
    got = dW.cpu()
    assert bool((got[:, rows:] == 77).all()) and bool((got[:, :, cols:] == 77).all()), "written outside the gradients"
    step = half_step(TORCH[dtype])
    for g in range(groups):
        a, b = ends[g], ends[g + 1]
        x, y = X[a:b, :K].double(), dY[a:b, :N].double()
        want, mag = y.t() @ x, y.abs().t() @ x.abs()
        if not trans_b:
            want, mag = want.t(), mag.t()
        tol = (b - a) * U32 * mag * (1 + step) + step * want.abs() + torch.finfo(TORCH[dtype]).tiny * 2 * step
        d = (got[g, :rows, :cols].double() - want).abs() - tol
        assert d.max().item() <= 0, (g, d.max().item())


WGRAD = [([0, 1], 1, 1), ([0, 0, 5, 5], 40, 72), ([3, 60, 61, 189], 130, 100), ([0, 64, 192, 200], 128, 128), ([0, 700, 701, 1500], 257, 136),
         ([0, 500, 1300], 520, 264), (list(range(0, 72)), 33, 40), ([5, 5], 16, 24), (list(range(0, 602, 2)), 60, 56),
         # enough for tiles of 256: depths of no, one and some slabs and a part of one
         ([2, 2, 3, 66, 131, 300, 1000], 1030, 520), ([0, 64, 128, 320, 1345], 1024, 1001), ([0, 700, 4001], 2056, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("trans_b", [True, False])
@pytest.mark.parametrize("ends,N,K", WGRAD)
def test_gradient_of_the_weights_matches_plain(dtype, trans_b, ends, N, K):
    print(f"case {dtype} {trans_b} {ends[:8]} {N} {K}", flush=True)
    wgrad(dtype, ends, N, K, trans_b, M=ends[-1] + 3, seed=N, guard=2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("ends,N,K", [
    # two rounds of tiles and a part of one, groups of very different depth, of the same, of none; more than three rounds
    ([0, 0, 1100, 1164, 1165, 1500, 1900, 2300, 2364, 2999, 3200], 1536, 1280), ([0, 300, 600, 900, 1200, 1500], 2568, 1928),
    ([7, 7, 7, 2500, 2500], 4096, 1288), ([0, 129, 1600, 1601, 4200], 4224, 3200), ([0] + [620 * i + 37 * (i % 7) for i in range(1, 64)] + [40000], 512, 768)])
def test_gradients_of_unequal_depths(dtype, ends, N, K):
    """Whole numbers of at most 3: a sum of 20000 products stays below 2^24, so fp32 holds it exactly and one rounding is left."""
    print(f"case {dtype} {ends[:8]} {N} {K}", flush=True)
    gen = torch.Generator().manual_seed(N + K)
    M, groups, t = ends[-1] + 5, len(ends) - 1, TORCH[dtype]
    X = torch.randint(-3, 4, (M, K), generator=gen, dtype=torch.int8).cuda().to(t)
    dY = torch.randint(-3, 4, (M, N), generator=gen, dtype=torch.int8).cuda().to(t)
    dW = torch.full((groups, N + 1, K), 77.0, dtype=t, device="cuda")
    off = torch.tensor(ends, dtype=torch.int32).cuda()
    ctx = ab.abft_create(M, groups * N, groups * ((K + 127) // 128 * 128), groups)
    try:
        s = ab.make_shape(M, N, K, batch=groups, strideB=(N + 1) * K)
        assert ab.abft_gemm_grouped_wgrad(ctx, X, dY, off, dW, ab.DTYPE_CODE[dtype], s) == ab.ABFT_OK
        torch.cuda.synchronize()
        assert bool((dW[:, N] == 77).all()), "written between the gradients"
        for g in range(groups):
            a, b = ends[g], ends[g + 1]
            want = torch.mm(dY[a:b].float().t().contiguous(), X[a:b].float()).to(t)
            assert torch.equal(dW[g, :N], want), g
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_gradients_agree_with_differences(dtype):
    """A layer's loss sum(C * G) against its differences when an element of A or of B moves by a step that the type holds exactly: the
    loss is linear in each, so a difference is the gradient up to the rounding of C."""
    ends, N, K = [0, 3, 3, 11], 24, 40
    p = Group(dtype, ends, N, K, seed=11)
    try:
        G = rand(torch.Generator().manual_seed(12), dtype, p.M, N, std=1.0)
        G[:, N:] = 0
        dG = G.cuda()
        dA = torch.zeros(p.M, p.A.shape[-1], dtype=TORCH[dtype], device="cuda")
        dW = torch.zeros_like(p.dB)
        # dA = G B: B as it lies, the other way round
        s = ab.make_shape(p.M, K, N, batch=p.groups, lda=G.shape[-1], ldb=p.B.shape[-1], ldc=dA.shape[-1], strideB=p.dB.stride(0), transB=False)
        ctx = ab.abft_create(64, 256, 4096, 8)
        assert ab.abft_gemm_grouped(ctx, dG, p.dB, p.offsets, None, dA, p.code, ab.ABFT_OFF, s) == ab.ABFT_OK
        assert ab.abft_gemm_grouped_wgrad(ctx, p.dA, dG, p.offsets, dW, p.code, p.shape) == ab.ABFT_OK
        torch.cuda.synchronize()

        def loss():
            p.upload()
            p.run()
            c = p.C.cpu().double()[:, :N]
            return (c * G.double()[:, :N]).sum().item(), (c.abs() * G.double()[:, :N].abs()).sum().item() * half_step(TORCH[dtype])

        for t, at, grad in ((p.A, (4, 7), dA), (p.B, (2, 9, 13), dW), (p.A, (0, K - 1), dA), (p.B, (0, N - 1, 0), dW), (p.B, (1, 2, 3), dW)):
            old = t[at].item()
            t[at] = 8.0
            up, e1 = loss()
            t[at] = -8.0
            down, e2 = loss()
            t[at] = old
            g = grad.cpu()[at].double().item()
            assert abs((up - down) / 16 - g) <= (e1 + e2) / 16 * 1.01 + 2 * half_step(TORCH[dtype]) * abs(g) + 1e-4, (at, up, down, g)
        ab.abft_destroy(ctx)
    finally:
        p.close()


# ------------------------------------------------------------------------------------------ rows to int8
def plain_quantize(x):
    x = x.double()
    top = x.abs().amax(dim=1)
    sound = torch.isfinite(x).all(dim=1)
    top = torch.where(sound, top, 1.0)
    q = torch.where((sound & (top > 0))[:, None], torch.round(127 * torch.where(sound[:, None], x, 0.0) / top.clamp(min=1e-300)[:, None]), 0.0)
    return q.to(torch.int8), torch.where(sound, top / 127, float("nan"))


def quantize(x, cols):
    ldq = pad(cols, 1)
    Q = torch.full((x.shape[0], ldq), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((x.shape[0],), -1.0, device="cuda")
    code = ab.ABFT_BF16 if x.dtype == torch.bfloat16 else ab.ABFT_F16
    d = x.cuda()
    rc = ab.abft_quantize_rows(d, code, x.shape[0], cols, x.shape[1], Q, ldq, scale)
    assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
    torch.cuda.synchronize()
    Q = Q.cpu()
    assert bool((Q[:, cols:] == 55).all())
    return Q[:, :cols], scale.cpu()


def check_quantize(x, cols):
    Q, scale = quantize(x, cols)
    q, s = plain_quantize(x[:, :cols])
    assert torch.equal(Q, q)
    assert torch.equal(torch.isnan(scale), torch.isnan(s))
    fine = ~torch.isnan(s)
    # one rounding of fp32; below its normal numbers half of its smallest step
    assert ((scale.double() - s).abs()[fine] <= U32 * s[fine] + 2.0 ** -150).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (197, 768), (9, 513), (4, 1000), (3, 1200), (6, 2047), (5, 2500), (7, 4096), (3, 4097), (2, 9001)])
def test_rows_to_int8(dtype, rows, cols):
    gen = torch.Generator().manual_seed(rows)
    x = rand(gen, dtype, rows, cols)
    x[:, :cols] *= torch.rand(rows, 1, generator=gen).to(x.dtype) * 4
    check_quantize(x, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_to_int8_every_value(dtype):
    """Every value of the type under the largest magnitude of its row, for many such: ties and what lies next to them among them."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(TORCH[dtype])
    bits = bits[torch.isfinite(bits.float())]
    gen = torch.Generator().manual_seed(1)
    tops = bits[torch.randint(0, len(bits), (40,), generator=gen)].abs().tolist()
    tops += [127.0, 254.0, 63.5, 1.0, 2.0, 3.0, torch.finfo(TORCH[dtype]).max, torch.finfo(TORCH[dtype]).tiny, bits.abs()[bits != 0].min().item()]
    for top in tops:
        v = bits[bits.abs() <= top]
        n = (len(v) + 4095) // 4096 * 4096
        x = torch.full((n,), 0.0, dtype=TORCH[dtype])
        x[:len(v)] = v
        x = x.view(-1, 4096)
        x[:, -1] = top
        check_quantize(x.contiguous(), 4096)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_to_int8_zeros_and_values_that_are_not_finite(dtype):
    x = rand(torch.Generator().manual_seed(2), dtype, 8, 100)
    x[0, :100] = 0
    x[1, 99] = float("inf")
    x[2, 0] = float("nan")
    x[3, 50] = float("-inf")
    x[4, :100] = -0.0
    check_quantize(x, 100)


# ------------------------------------------------------------------------------------------ together, as they are used
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantised_experts_from_tokens_to_output(dtype):
    """Tokens to int8, the first layer of their experts, its output to int8, the second layer: each step against the plain form of that step on what
    the one before it gave."""
    ends, H, F = [0, 40, 40, 111, 130], 96, 200
    M, E = 137, 4
    gen = torch.Generator().manual_seed(21)
    x = rand(gen, dtype, M, H)
    W = [torch.randint(-128, 128, (E, F, pad(H, 1)), generator=gen, dtype=torch.int8), torch.randint(-128, 128, (E, H, pad(F, 1)), generator=gen, dtype=torch.int8)]
    col = [torch.rand(E, F, generator=gen) * 0.01, torch.rand(E, H, generator=gen) * 0.01]
    off = torch.tensor(ends, dtype=torch.int32).cuda()
    ctx = ab.abft_create(M, E * F, E * 256, E)
    code, t = ab.DTYPE_CODE[dtype], TORCH[dtype]
    rf, cf, counts = (torch.zeros(n, dtype=k, device="cuda") for n, k in ((M, torch.uint8), (E * F, torch.uint8), (8, torch.int32)))
    try:
        cur, width = x.cuda(), H
        for w, c, n in zip(W, col, (F, H)):
            Q = torch.zeros(M, pad(width, 1), dtype=torch.int8, device="cuda")
            scale = torch.zeros(M, device="cuda")
            assert ab.abft_quantize_rows(cur, code, M, width, cur.shape[1], Q, Q.shape[1], scale) == ab.ABFT_OK
            out = torch.zeros(M, pad(n, 2), dtype=t, device="cuda")
            s = ab.make_shape(M, n, width, batch=E, lda=Q.shape[1], ldb=w.shape[2], ldc=out.shape[1])
            dw, dc = w.cuda(), c.cuda()
            rc = ab.abft_gemm_grouped(ctx, Q, dw, off, ab.make_scales(scale, dc, out=code), out, ab.ABFT_I8, ab.ABFT_DETECT, s,
                                      ab.make_result(rf, cf, counts))
            assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
            torch.cuda.synchronize()
            q, sc = plain_quantize(cur.cpu()[:, :width])
            assert torch.equal(Q.cpu()[:, :width], q)
            for g in range(E):
                a, b = ends[g], ends[g + 1]
                want = (q[a:b].double() @ w[g, :, :width].double().t()) * scale.cpu()[a:b, None].double() * c[g].double()
                d = (out.cpu()[a:b, :n].double() - want).abs()
                assert (d <= half_step(t) * want.abs() + 4 * U32 * want.abs() + torch.finfo(t).tiny).all()
            assert counts[:3].tolist() == [0, 0, 0]
            cur, width = out, n
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out,ends,N,K,trans_b", [("i8", "bf16", [0, 2, 2, 9], 200, 256, True), ("bf16", None, [0, 100, 350], 200, 136, False),
                                                        ("bf16", None, [0, 600, 1300], 520, 384, True)])
def test_grouped_calls_can_be_captured_in_a_graph(dtype, out, ends, N, K, trans_b):
    p = Group(dtype, ends, N, K, trans_b, out=out, seed=31)
    try:
        p.run(ab.ABFT_DETECT)
        dW = torch.zeros_like(p.dB)
        G = torch.zeros((p.M, pad(N, 2)), dtype=TORCH[dtype] if dtype != "i8" else torch.bfloat16, device="cuda").normal_()

        def calls():
            assert p.call(ab.ABFT_DETECT) == ab.ABFT_OK
            if dtype != "i8":
                s = ab.make_shape(p.M, N, K, batch=p.groups, lda=p.A.shape[-1], ldb=p.B.shape[-1], ldc=G.shape[1], transB=trans_b)
                assert ab.abft_gemm_grouped_wgrad(p.ctx, p.dA, G, p.offsets, dW, p.code, s) == ab.ABFT_OK

        calls()
        torch.cuda.synchronize()
        C0, W0 = p.C.clone(), dW.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for k in range(4):
            for x in (p.C, p.row_flag, p.col_flag, p.counts):
                x.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.C[:, :N][p.ends[0]:p.ends[-1]], C0[:, :N][p.ends[0]:p.ends[-1]]) and torch.equal(dW, W0)
            p.clean()
            if k % 2:
                p.run(ab.ABFT_DETECT)
                p.clean()
    finally:
        p.close()


@pytest.mark.gpu
def test_two_graphs_of_a_context_with_offsets_that_change():
    """Two captured calls take turns on one context, and between their replays the rows are dealt out anew where the offsets lie, as a router's kernel does."""
    splits = [[0, 0, 1300, 1301, 1700, 2600], [5, 600, 600, 600, 2590, 2595], [0, 520, 1040, 1560, 2080, 2600], [0, 0, 0, 0, 0, 0]]
    small = [[0, 3, 9, 9], [0, 0, 0, 20], [1, 17, 18, 19], [20, 20, 20, 20]]
    ctx = ab.abft_create(4096, 16384, 8192, 16)
    p = Group("bf16", splits[0], 2056, 1288, M=2600, seed=51, ctx=ctx)
    q = Group("i8", small[0], 264, 208, out="bf16", M=20, seed=52, ctx=ctx)
    whole = lambda *shape: torch.randint(-3, 4, shape, generator=torch.Generator().manual_seed(53), dtype=torch.int8).cuda().to(torch.bfloat16)
    X, dY, dW = whole(2600, 1288), whole(2600, 2056), torch.zeros(5, 2056, 1288, dtype=torch.bfloat16, device="cuda")
    s = ab.make_shape(2600, 2056, 1288, batch=5)

    def first():
        assert p.call(ab.ABFT_DETECT) == ab.ABFT_OK
        assert ab.abft_gemm_grouped_wgrad(ctx, X, dY, p.offsets, dW, ab.ABFT_BF16, s) == ab.ABFT_OK

    def second():
        assert q.call(ab.ABFT_DETECT) == ab.ABFT_OK

    try:
        graphs = []
        for f in (first, second):
            f()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                f()
            graphs.append(graph)
        for k in (0, 1, 2, 3, 1):
            for x, ends in ((p, splits[k]), (q, small[k])):
                x.ends = ends
                x.offsets.copy_(torch.tensor(ends, dtype=torch.int32))
                x.C.fill_(x.fill)
                for y in (x.row_flag, x.col_flag, x.counts):
                    y.fill_(3)
            dW.fill_(5.0)
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            for x in (p, q):
                x.check()
                x.clean()
            for g in range(5):
                a, b = splits[k][g], splits[k][g + 1]
                assert torch.equal(dW[g], torch.mm(dY[a:b].float().t().contiguous(), X[a:b].float()).to(torch.bfloat16)), (k, g)
            second()
            torch.cuda.synchronize()
            q.check()
            q.clean()
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [ab.ABFT_OFF, ab.ABFT_DETECT])
def test_the_event_of_a_context_is_recorded_behind_the_product(mode):
    p = Group("bf16", [0, 900, 2500], 520, 384, seed=63)
    try:
        begin, event, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
        event.record()
        torch.cuda.synchronize()
        assert ab.abft_gemm_done_event(p.ctx, event.cuda_event) == ab.ABFT_OK
        begin.record()
        p.run(mode)
        end.record()
        torch.cuda.synchronize()
        assert 0 < begin.elapsed_time(event) <= begin.elapsed_time(end)
        assert ab.abft_gemm_done_event(p.ctx, None) == ab.ABFT_OK
        p.check()
    finally:
        p.close()


@pytest.mark.gpu
@pytest.mark.parametrize("a,b", [(-128, -128), (-128, 127)])
@pytest.mark.parametrize("ends,N,K,trans_b", [([0, 1, 5], 200, 131071, True), ([0, 150, 300], 200, 131071, False), ([0, 2000, 2600], 1024, 1024, True), ([0, 16], 200, 2040, True)])
def test_largest_integers_at_the_greatest_depth(ends, N, K, trans_b, a, b):
    """Every product the largest in magnitude, up to K 2^14 just below 2^31: C holds the sum, the sums of sums agree in Z/2^32, and a flip of the lowest bit shows."""
    p = Group("i8", ends, N, K, trans_b, seed=64)
    try:
        p.dA.fill_(a)
        p.dB.fill_(b)
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            p.run(mode)
            assert bool((p.C[:, :N] == a * b * K).all())
        p.clean()
        one_flip(p, stored_bits(p), p.groups - 1, ends[-1] - ends[-2] - 1, N - 1, 0, ab.ABFT_DETECT)
    finally:
        p.close()


@pytest.mark.gpu
def test_grouped_and_other_calls_share_a_context():
    """Calls of other kinds between grouped ones: the regions they accumulate into are clean for each."""
    ctx = ab.abft_create(4096, 8192, 8192, 16)
    p = Group("bf16", [0, 30, 95], 136, 200, seed=41, ctx=ctx)
    q = Group("i8", [0, 7, 7, 300], 64, 128, out="f16", seed=42, ctx=ctx)
    A = torch.randn(197, 768, device="cuda").to(torch.bfloat16)
    B = (torch.randn(768, 768, device="cuda") * 0.02).to(torch.bfloat16)
    C = torch.zeros(197, 768, device="cuda", dtype=torch.bfloat16)
    rf, cf, cnt = torch.zeros(197, dtype=torch.uint8, device="cuda"), torch.zeros(768, dtype=torch.uint8, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    s = ab.make_shape(197, 768, 768)
    try:
        for _ in range(3):
            for x in (p, q):
                x.run(ab.ABFT_DETECT)
                x.check()
                x.clean()
                assert ab.abft_gemm(ctx, A, B, C, ab.ABFT_BF16, ab.ABFT_DETECT, s, ab.make_result(rf, cf, cnt)) == ab.ABFT_OK
                torch.cuda.synchronize()
                assert cnt[:3].tolist() == [0, 0, 0]
        # behind a grouped call there is nothing to verify by
        p.run(ab.ABFT_DETECT)
        assert ab.abft_verify(ctx, C, ab.ABFT_BF16, s, ab.make_result(rf, cf, cnt)) == ab.ABFT_ESTATE
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [ab.ABFT_OFF, ab.ABFT_DETECT])
@pytest.mark.parametrize("scaled", [False, True])
def test_nothing_to_verify_by_behind_a_grouped_call_of_either_mode(mode, scaled):
    """The predictions of an earlier product of the same sizes are not another's: a C that no protected product made is refused, not judged by them."""
    M, N, K = 64, 128, 64
    ctx = ab.abft_create(M, N, K, 1)
    p = Group("i8", [0, M], N, K, out="f16" if scaled else None, seed=14, ctx=ctx, dense=scaled)
    A, B = rand(torch.Generator().manual_seed(15), "i8", M, K).cuda(), rand(torch.Generator().manual_seed(16), "i8", N, K).cuda()
    C = torch.zeros(M, N, dtype=torch.int32, device="cuda")
    s = ab.make_shape(M, N, K)
    res = ab.make_result(p.row_flag, p.col_flag, p.counts)
    try:
        assert ab.abft_gemm(ctx, A, B, C, ab.ABFT_I8, ab.ABFT_DETECT, s, res) == ab.ABFT_OK
        assert ab.abft_verify(ctx, C, ab.ABFT_I8, s, res) == ab.ABFT_OK
        p.run(mode)
        assert ab.abft_verify(ctx, C, ab.ABFT_I8, s, res) == ab.ABFT_ESTATE
        assert ab.abft_correct(ctx, A, B, C, ab.ABFT_I8, s, res) == ab.ABFT_ESTATE
        assert ab.abft_correct_checksum(ctx, C, ab.ABFT_I8, s, res) == ab.ABFT_ESTATE
        p.check()
    finally:
        torch.cuda.synchronize()
        ab.abft_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 50, 20, 64], [-5, 10, 30, 400], [2 ** 31 - 1, -2 ** 31, 64, 64], [64, 0, 0, 64]])
def test_bad_offsets_address_nothing_outside(bad):
    """Offsets that fall or point outside: A and C lie inside larger buffers, whose other rows stay as they are."""
    p = Group("bf16", [0, 20, 40, 64], 72, 96, seed=51)
    try:
        whole = torch.full((64 + 2 * 256, p.ldc), 5.0, dtype=torch.bfloat16, device="cuda")
        p.C = whole[256:320]
        p.offsets = torch.tensor(bad, dtype=torch.int32).cuda()
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT):
            p.run(mode)
        assert bool((whole[:256] == 5).all()) and bool((whole[320:] == 5).all())
        dW = torch.zeros_like(p.dB)
        G = torch.zeros((64, p.ldc), dtype=torch.bfloat16, device="cuda")
        assert ab.abft_gemm_grouped_wgrad(p.ctx, p.dA, G, p.offsets, dW, p.code, p.shape) == ab.ABFT_OK
        torch.cuda.synchronize()
    finally:
        p.close()


# ------------------------------------------------------------------------------------------ refusals
def test_refusals_that_need_no_gpu():
    P = 0x1000
    q = ab.abft_quantize_rows
    ok = dict(X=P, dtype=ab.ABFT_BF16, rows=4, cols=8, ldx=8, Q=P, ldq=16, scale=P, stream=0)
    for change, code in [(dict(dtype=ab.ABFT_I8), ab.ABFT_EINVAL), (dict(dtype=9), ab.ABFT_EINVAL), (dict(rows=0), ab.ABFT_ESHAPE),
                         (dict(cols=0), ab.ABFT_ESHAPE), (dict(ldx=4), ab.ABFT_ESHAPE), (dict(ldq=4), ab.ABFT_ESHAPE), (dict(X=None), ab.ABFT_EINVAL),
                         (dict(Q=None), ab.ABFT_EINVAL), (dict(scale=None), ab.ABFT_EINVAL), (dict(X=P + 8), ab.ABFT_EALIGN), (dict(Q=P + 4), ab.ABFT_EALIGN),
                         (dict(scale=P + 2), ab.ABFT_EALIGN), (dict(ldx=12), ab.ABFT_EALIGN), (dict(ldq=24), ab.ABFT_EALIGN),
                         (dict(rows=1 << 31), ab.ABFT_ESHAPE)]:
        assert q(**{**ok, **change}) == code, change
    s = ab.make_shape(4, 16, 16, batch=2)
    one = ab.make_shape(4, 16, 16)
    sc = ab.make_scales(out=ab.ABFT_BF16)
    g = lambda **k: ab.abft_gemm_grouped(**{**dict(ctx=None, A=P, B=P, offsets=P, scales=None, C=P, dtype=ab.ABFT_BF16, mode=ab.ABFT_OFF, shape=s, stream=0), **k})
    for change, code in [(dict(), ab.ABFT_EINVAL), (dict(offsets=None), ab.ABFT_EINVAL), (dict(mode=ab.ABFT_DETECT_CORRECT), ab.ABFT_EINVAL),
                         (dict(mode=ab.ABFT_DETECT | ab.ABFT_STORED_SUMS), ab.ABFT_EINVAL), (dict(mode=ab.ABFT_DETECT | ab.ABFT_A_CHECKSUM_GIVEN), ab.ABFT_EINVAL),
                         (dict(scales=sc), ab.ABFT_EINVAL), (dict(dtype=ab.ABFT_I8, scales=ab.make_scales(out=ab.ABFT_I8)), ab.ABFT_EINVAL),
                         (dict(dtype=ab.ABFT_I8, scales=ab.make_scales(row=P + 2)), ab.ABFT_EALIGN), (dict(dtype=7), ab.ABFT_EINVAL)]:
        assert g(**change) == code, change
    assert ab.abft_gemm_scaled(None, P, P, None, P, ab.ABFT_OFF, one, stream=0) == ab.ABFT_EINVAL
    assert ab.abft_gemm_scaled(None, P, P, sc, P, ab.ABFT_OFF, s, stream=0) == ab.ABFT_ESHAPE
    assert ab.abft_gemm_scaled(None, P, P, sc, P, ab.ABFT_OFF, one, stream=0) == ab.ABFT_EINVAL
    assert ab.abft_gemm_grouped_wgrad(None, P, P, P, P, ab.ABFT_I8, s, stream=0) == ab.ABFT_EINVAL
    assert ab.abft_gemm_grouped_wgrad(None, P, P, P, P, ab.ABFT_BF16, s, stream=0) == ab.ABFT_EINVAL
    assert ctypes.sizeof(ab.abft_scales) == 4 * 8


@pytest.mark.gpu
def test_refusals():
    """None of these calls launches anything: the pointers are never followed."""
    P = 0x1000
    ctx = ab.abft_create(64, 256, 1024, 4)
    sc = ab.make_scales(out=ab.ABFT_BF16)
    shape = lambda **k: ab.make_shape(**{**dict(M=64, N=64, K=64, batch=4), **k})
    res = ab.make_result(P, P, P)
    g = lambda s=None, **k: ab.abft_gemm_grouped(**{**dict(ctx=ctx, A=P, B=P, offsets=P, scales=None, C=P, dtype=ab.ABFT_BF16, mode=ab.ABFT_DETECT,
                                                           shape=s or shape(), result=res), **k})
    try:
        for s, code in [(shape(M=65), ab.ABFT_EWORKSPACE), (shape(N=72), ab.ABFT_EWORKSPACE), (shape(K=400), ab.ABFT_EWORKSPACE),
                        (shape(batch=5), ab.ABFT_EWORKSPACE), (shape(M=0), ab.ABFT_ESHAPE), (shape(N=0), ab.ABFT_ESHAPE), (shape(K=0), ab.ABFT_ESHAPE),
                        (shape(lda=60), ab.ABFT_ESHAPE), (shape(lda=68), ab.ABFT_EALIGN), (shape(ldb=60), ab.ABFT_ESHAPE), (shape(ldc=66), ab.ABFT_EALIGN),
                        (shape(ldc=56), ab.ABFT_ESHAPE), (shape(strideB=4), ab.ABFT_EALIGN), (shape(strideB=-64), ab.ABFT_EALIGN)]:
            assert g(s) == code, code
        for change, code in [(dict(A=None), ab.ABFT_EINVAL), (dict(B=P + 8), ab.ABFT_EALIGN), (dict(offsets=P + 2), ab.ABFT_EALIGN), (dict(C=None), ab.ABFT_EINVAL),
                             (dict(result=None), ab.ABFT_EINVAL), (dict(result=ab.make_result(P, P, P, tau=-1.0)), ab.ABFT_EINVAL),
                             (dict(mode=ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED), ab.ABFT_ESTATE)]:
            assert g(**change) == code, change
        assert ab.abft_gemm_scaled(ctx, P, P, sc, P, ab.ABFT_OFF, shape(batch=1, K=1 << 17)) == ab.ABFT_ESHAPE
        w = lambda s, **k: ab.abft_gemm_grouped_wgrad(**{**dict(ctx=ctx, X=P, dY=P, offsets=P, dW=P, dtype=ab.ABFT_BF16, shape=s), **k})
        assert w(shape(strideB=64 * 32)) == ab.ABFT_ESHAPE
        assert w(shape(), offsets=None) == ab.ABFT_EINVAL
        assert w(shape(), dW=P + 8) == ab.ABFT_EALIGN
        assert w(shape(M=65)) == ab.ABFT_EWORKSPACE
        for s in (shape(K=(1 << 29) + 8), shape(N=(1 << 25) + 8), shape(M=(1 << 30) + 8), shape(batch=1, N=(1 << 27) + 8)):
            assert g(s) == ab.ABFT_ESHAPE and w(s) == ab.ABFT_ESHAPE
    finally:
        ab.abft_destroy(ctx)


@pytest.mark.gpu
def test_products_of_more_tiles_than_a_launch_are_refused_by_their_shape():
    """2^24 tiles of 64 x 128, one more than a launch has workgroups.  Nothing is launched: the pointers are never followed, and the context is as it was."""
    P = 0x1000
    ctx = ab.abft_create(1 << 19, 1 << 19, 1 << 18, 1)
    try:
        B = torch.zeros(1 << 18, 8, dtype=torch.bfloat16, device="cuda")
        s = ab.make_shape(1 << 19, 1 << 18, 8)
        assert ab.abft_encode_b(ctx, B, ab.ABFT_BF16, s) == ab.ABFT_OK
        torch.cuda.synchronize()
        for mode in (ab.ABFT_OFF, ab.ABFT_DETECT, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED):
            assert ab.abft_gemm_grouped(ctx, P, P, P, None, P, ab.ABFT_BF16, mode, s, ab.make_result(P, P, P)) == ab.ABFT_ESHAPE
        # (the encoding is still there: of a product of few rows it is asked for and found)
        small = ab.make_shape(1, 1 << 18, 8)
        A, C, off = torch.ones(1, 8, dtype=torch.bfloat16, device="cuda"), torch.ones(1, 1 << 18, dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 1], dtype=torch.int32).cuda()
        rf, cf, cnt = (torch.zeros(n, dtype=t, device="cuda") for n, t in ((1, torch.uint8), (1 << 18, torch.uint8), (8, torch.int32)))
        rc = ab.abft_gemm_grouped(ctx, A, B, off, None, C, ab.ABFT_BF16, ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED, small, ab.make_result(rf, cf, cnt))
        assert rc == ab.ABFT_OK, ab.abft_strerror(rc)
        torch.cuda.synchronize()
        assert not C.any() and cnt[:3].tolist() == [0, 0, 0]
        # gradients of 2^37 elements whose rows lie too far apart for the tiles that a launch's workgroups walk
        assert ab.abft_gemm_grouped_wgrad(ctx, P, P, P, P, ab.ABFT_BF16, ab.make_shape(8192, 1 << 19, 1 << 18)) == ab.ABFT_ESHAPE
    finally:
        ab.abft_destroy(ctx)
