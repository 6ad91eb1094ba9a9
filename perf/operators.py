"""Operators of quantised layers and of mixtures of experts, as cases that can be timed and compared.

A case is a dict of plain values.  ``prepare`` makes what a program holds before the call (operands, output and
verdict buffers, and, where ``own`` is true, a context with the weight checksum that the program encodes once),
``run`` makes one pass: the calls of libabft's operators where ``own`` is true, their plain form in elementary torch
operations otherwise.  ``exact`` is what the operators are defined as, in 64 bits.

Kinds
  quantize   rows of activations (tokens) to int8, a scale for each
  scaled     C = (A B) scaled by row and by column (+ bias), int8 operands, C in a 16-bit type
  grouped    C = A B with the weight of each row's group (expert); rows sorted by group, the last rows in none.  "i8s": int8
             operands with scales, as above
  wgrad      the gradient of such weights: for each group the product of its rows of dY and of X

Sizes are those of the layers of ViT-B/16 (197 tokens an image, hidden 768, MLP 3072) and ViT-L/16 (hidden 1024, MLP 4096), for
one expert or several; values those of such layers: activations N(0, 1), weights N(0, 0.02), gradients N(0, 0.01), quantised ones
uniform.
"""
from __future__ import annotations

import math
import random
import weakref

import torch

own = False

TORCH_TYPE = {"i8": torch.int8, "i8s": torch.int8, "bf16": torch.bfloat16, "f16": torch.float16}
ES = {"i8": 1, "i8s": 1, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------------- the cases
def _quantize(name, dtype, rows, cols):
    return dict(name=name, kind="quantize", dtype=dtype, rows=rows, cols=cols)


def _scaled(name, M, N, K, out="bf16", trans_b=True, mode="detect", bias=True):
    return dict(name=name, kind="scaled", dtype="i8s", out=out, M=M, N=N, K=K, trans_b=trans_b, mode=mode, bias=bias)


def _grouped(name, dtype, M, groups, N, K, out="", trans_b=True, mode="detect", routing=1, spare=0):
    return dict(name=name, kind="grouped", dtype=dtype, out=out, M=M, groups=groups, N=N, K=K, trans_b=trans_b, mode=mode,
                routing=routing, spare=spare)


def _wgrad(name, dtype, M, groups, N, K, trans_b=True, routing=1, spare=0):
    return dict(name=name, kind="wgrad", dtype=dtype, M=M, groups=groups, N=N, K=K, trans_b=trans_b, routing=routing,
                spare=spare)


def listed():
    return [
        # the tokens of one image ahead of a quantised layer: a call that is mostly latency
        _quantize("quantize_f16_1image", "f16", 197, 768),
        # the widest activations of a large batch: bandwidth
        _quantize("quantize_bf16_b64", "bf16", 12608, 3072),
        # one token through a quantised MLP layer: reads the weight once
        _scaled("scaled_1token", 1, 4096, 1024),
        # the quantised layer for a large batch, the weight's checksum kept
        _scaled("scaled_fc1_b64", 12608, 3072, 768),
        # odd sizes in every dimension, the right operand stored K x N, unprotected
        _scaled("scaled_odd_kn", 1537, 1001, 713, out="f16", trans_b=False, mode="off", bias=False),
        # a few tokens, each to an expert of its own among many: most of the time goes to weights
        _grouped("experts_few_tokens_bf16", "bf16", 32, 32, 4096, 1024, mode="off", routing=3),
        # the same in a small quantised model, protected
        _grouped("experts_few_tokens_i8", "i8s", 24, 8, 3072, 768, out="bf16", routing=4, spare=3),
        # experts over a large batch, protected
        _grouped("experts_fc1_bf16", "bf16", 12608, 16, 3072, 768, routing=5, spare=100),
        # the narrow, deep layer of quantised experts, protected
        _grouped("experts_fc2_i8", "i8s", 6304, 8, 768, 3072, out="bf16", routing=6),
        # the gradient of the experts' inputs: the weights read the other way round
        _grouped("experts_dx_f16", "f16", 6304, 8, 768, 3072, trans_b=False, mode="off", routing=7),
        # the gradient of the experts' weights, large batch
        _wgrad("experts_dw_bf16", "bf16", 12608, 16, 3072, 768, routing=8),
        # the same with odd sizes and few rows
        _wgrad("experts_dw_odd_f16", "f16", 1537, 5, 1001, 713, trans_b=False, routing=9, spare=37),
    ]


MOST_PRODUCTS = 12608 * 3072 * 768               # of a drawn case
MOST_WEIGHTS = 32 * 4096 * 1024


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of [lo, hi], spread over its logarithm; half of the time a multiple of 64 as layers have."""
    n = _log(rng, lo, hi)
    if hi >= 64 and rng.random() < 0.5:
        n = max(64, (n + 32) // 64 * 64)
    return min(max(n, lo), hi)


def draw(rng):
    kind = rng.choice(["quantize", "scaled", "scaled", "grouped", "grouped", "grouped", "wgrad", "wgrad"])
    if kind == "quantize":
        c = _quantize("", rng.choice(["bf16", "f16"]), _size(rng, 1, 12608), _size(rng, 64, 4096))
        while c["rows"] * c["cols"] > 12608 * 3072:
            c["cols"] = _size(rng, 64, 4096)
    else:
        dtype = rng.choice(["bf16", "f16"]) if kind == "wgrad" else rng.choice(["i8", "i8s", "i8s", "bf16", "bf16", "f16"])
        trans_b, mode = rng.random() < 0.7, rng.choice(["off", "detect", "detect"])
        while True:
            M, N, K, groups = _size(rng, 1, 12608), _size(rng, 64, 4096), _size(rng, 64, 4096), _log(rng, 1, 64)
            if kind == "scaled":
                groups = 1
            if M * N * K <= MOST_PRODUCTS and groups * N * K <= MOST_WEIGHTS:
                break
        out, routing = rng.choice(["bf16", "f16"]), rng.randint(10, 1 << 30)
        spare = rng.choice([0, 0, M // 20, M // 5])
        if kind == "scaled":
            c = _scaled("", M, N, K, out=out, trans_b=trans_b, mode=mode, bias=rng.random() < 0.5)
        elif kind == "grouped":
            c = _grouped("", dtype, M, groups, N, K, out=out if dtype == "i8s" else "", trans_b=trans_b, mode=mode,
                         routing=routing, spare=spare)
        else:
            c = _wgrad("", dtype, M, groups, N, K, trans_b=trans_b, routing=routing, spare=spare)
    del c["name"]
    return c


def _counts(c):
    """Rows of each group of a case: uneven, as routers deal them out, some groups without any."""
    rng = random.Random(c["routing"])
    weight = [0.0 if rng.random() < 0.1 else math.exp(rng.gauss(0.0, 0.7)) for _ in range(c["groups"])]
    if not any(weight):
        weight[0] = 1.0
    got = [0] * c["groups"]
    for g in rng.choices(range(c["groups"]), weight, k=c["M"] - c["spare"]):
        got[g] += 1
    return got


# ---------------------------------------------------------------------------------- what a program holds
def _pad(n, elem_bytes):
    q = 16 // elem_bytes
    return (n + q - 1) // q * q


def _values(gen, dtype, std, *shape):
    """Operand values on the GPU; the last dimension is padded to whole 16 bytes, the pad not zero."""
    full = shape[:-1] + (_pad(shape[-1], ES[dtype]),)
    if ES[dtype] == 1:
        return torch.randint(-128, 128, full, generator=gen, device="cuda", dtype=torch.int8)
    return torch.empty(full, device="cuda", dtype=torch.float32).normal_(0.0, std, generator=gen).to(TORCH_TYPE[dtype])


def _positive(gen, lo, hi, *shape):
    return torch.empty(shape, device="cuda", dtype=torch.float32).uniform_(lo, hi, generator=gen)


class _State:
    pass


def _inputs(c, seed):
    s = _State()
    s.case = c
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if c["kind"] == "quantize":
        # tokens differ in size, as those behind a layer norm's gain or an activation do
        x = _values(gen, c["dtype"], 1.0, c["rows"], c["cols"])
        s.X = (x.float() * _positive(gen, 0.1, 4.0, c["rows"], 1)).to(x.dtype)
        return s
    groups = c.get("groups", 1)
    weight = (c["N"], c["K"]) if c["trans_b"] else (c["K"], c["N"])
    if c["kind"] == "wgrad":
        s.X = _values(gen, c["dtype"], 1.0, c["M"], c["K"])
        s.dY = _values(gen, c["dtype"], 0.01, c["M"], c["N"])
        s.weight = (groups,) + weight[:1] + (_pad(weight[1], ES[c["dtype"]]),)
    else:
        s.A = _values(gen, c["dtype"], 1.0, c["M"], c["K"])
        s.B = _values(gen, c["dtype"], 0.02, groups, *weight)
    if c["dtype"] == "i8s":
        s.row = _positive(gen, 0.002, 0.03, c["M"])
        s.col = _positive(gen, 0.0001, 0.0005, groups, c["N"])
    s.bias = None
    if c.get("bias"):
        s.bias = torch.empty(c["N"], device="cuda", dtype=torch.float32).normal_(0.0, 0.1, generator=gen)
    if c["kind"] != "scaled":
        counts = _counts(c)
        random.Random(int(seed)).shuffle(counts)
        s.most = max(counts)
        ends = [0]
        for n in counts:
            ends.append(ends[-1] + n)
        s.offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    return s


def _out_type(c):
    return torch.int32 if c["dtype"] == "i8" else TORCH_TYPE[c["out"] or c["dtype"]]


def _c_shape(c):
    return c["M"], _pad(c["N"], 4 if c["dtype"] == "i8" else 2)


def _check(ab, rc, where):
    if rc != ab.ABFT_OK:
        raise ab.AbftError(rc, where)


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    if own:
        import paper_2310_03841_amd as ab
        s.ab = ab
        if c["kind"] == "quantize":
            s.Q = torch.zeros((c["rows"], _pad(c["cols"], 1)), device="cuda", dtype=torch.int8)
            s.scale = torch.zeros(c["rows"], device="cuda", dtype=torch.float32)
            return s
        groups = c.get("groups", 1)
        s.code = ab.DTYPE_CODE[c["dtype"][:2] if c["dtype"] == "i8s" else c["dtype"]]
        s.ctx = ab.abft_create(c["M"], groups * c["N"], groups * ((c["K"] + 127) // 128 * 128), groups)
        weakref.finalize(s, ab.abft_destroy, s.ctx)
        if c["kind"] == "wgrad":
            s.dW = torch.zeros(s.weight, device="cuda", dtype=TORCH_TYPE[c["dtype"]])
            s.shape = ab.make_shape(c["M"], c["N"], c["K"], batch=groups, lda=s.X.shape[-1], ldb=s.weight[-1],
                                    ldc=s.dY.shape[-1], transB=c["trans_b"])
            return s
        s.C = torch.zeros(_c_shape(c), device="cuda", dtype=_out_type(c))
        s.shape = ab.make_shape(c["M"], c["N"], c["K"], batch=groups, lda=s.A.shape[-1], ldb=s.B.shape[-1],
                                ldc=s.C.shape[-1], transB=c["trans_b"])
        s.scales = None
        if c["dtype"] == "i8s":
            s.scales = ab.make_scales(s.row, s.col, s.bias, out=ab.DTYPE_CODE[c["out"]])
        s.mode, s.result = ab.ABFT_OFF, None
        if c["mode"] == "detect":
            s.row_flag = torch.zeros(c["M"], device="cuda", dtype=torch.uint8)
            s.col_flag = torch.zeros(groups * c["N"], device="cuda", dtype=torch.uint8)
            s.counts = torch.zeros(8, device="cuda", dtype=torch.int32)
            s.result = ab.make_result(s.row_flag, s.col_flag, s.counts)
            # the weights' checksums: once, as programs do whose weights stay
            s.mode = ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED
            _check(ab, ab.abft_encode_b(s.ctx, s.B, s.code, s.shape), "abft_encode_b")
    elif c["kind"] in ("scaled", "grouped") and c["mode"] == "detect":
        wide = torch.float64 if ES[c["dtype"]] == 1 else torch.float32
        w = _stored(s.B, c).to(wide)
        s.b_sum, s.b_max = w.sum(dim=1), w.abs().amax(dim=(1, 2))
    return s


# ---------------------------------------------------------------------------------- the operators
def _stored(B, c):
    """The weights without their pad, as groups x N x K."""
    return B[..., :c["K"]] if c["trans_b"] else B[..., :c["N"]].transpose(1, 2)


def _padded(x, s):
    """Rows sorted by group, as groups x most rows of a group, with zeros behind each group's; and where each row went."""
    used = torch.arange(x.shape[0], device="cuda") < s.offsets[-1]
    group = torch.searchsorted(s.offsets[1:].contiguous(), torch.arange(x.shape[0], device="cuda"), right=True, out_int32=True).long()
    at = torch.arange(x.shape[0], device="cuda") - s.offsets[group.clamp(max=len(s.offsets) - 1)]
    groups = len(s.offsets) - 1
    # rows of no group meet in a row of their own behind all
    flat = torch.where(used, group * s.most + at, groups * s.most)
    out = torch.zeros((groups * s.most + 1, x.shape[1]), device="cuda", dtype=x.dtype)
    out[flat] = x
    return out[:-1].view(groups, s.most, x.shape[1]), flat, used


def _plain_quantize(s):
    c = s.case
    x = s.X[:, :c["cols"]].float()
    amax = x.abs().amax(dim=1, keepdim=True)
    q = torch.zeros((c["rows"], _pad(c["cols"], 1)), device="cuda", dtype=torch.int8)
    # 127 x has at most 18 bits: exact; a quotient of such values is never so near a tie that its rounding reaches one
    q[:, :c["cols"]] = torch.where(amax > 0, torch.round(x * 127.0 / amax), 0.0).to(torch.int8)
    return {"Q": q, "scale": (amax / 127.0)[:, 0]}


def _plain_product(s):
    c = s.case
    # int8: sums of up to 4096 products of 2^14 need 27 bits, checksums more; 64-bit floating point holds them exactly
    wide = torch.float64 if ES[c["dtype"]] == 1 else torch.float32
    A, w = s.A[:, :c["K"]].to(wide), _stored(s.B, c).to(wide)
    if c["kind"] == "grouped":
        rows, flat, used = _padded(A, s)
    else:
        rows = A[None]
    acc = torch.matmul(rows, w.transpose(1, 2).contiguous())
    got = {}
    if c["mode"] == "detect":
        obs_r, obs_c = acc.sum(dim=2), acc.sum(dim=1)
        pred_r = torch.matmul(rows, s.b_sum[:, :, None])[..., 0]
        pred_c = torch.matmul(w, rows.sum(dim=1)[:, :, None])[..., 0]
        tau = torch.zeros_like(s.b_max) if ES[c["dtype"]] == 1 else 1e-3 * c["K"] * rows.abs().amax(dim=(1, 2)) * s.b_max
        bad_r, bad_c = (~((obs_r - pred_r).abs() <= tau[:, None])), ~((obs_c - pred_c).abs() <= tau[:, None])
        bad_r = bad_r.reshape(-1)
        got["row_flag"] = (used & bad_r[flat.clamp(max=bad_r.numel() - 1)] if c["kind"] == "grouped" else bad_r).to(torch.uint8)
        got["col_flag"] = bad_c.reshape(-1).to(torch.uint8)
        counts = torch.zeros(8, device="cuda", dtype=torch.int32)
        counts[0], counts[1] = got["row_flag"].sum(), got["col_flag"].sum()
        counts[2] = torch.where((counts[0] > 0) & (counts[1] > 0), 1, torch.where((counts[0] > 0) | (counts[1] > 0), 2, 0))
        got["counts"] = counts
    if c["dtype"] == "i8s":
        acc = acc.float() * s.col[:, None, :]
    acc = acc.reshape(-1, c["N"])
    if c["kind"] == "grouped":
        acc = torch.where(used[:, None], acc[flat.clamp(max=acc.shape[0] - 1)], 0)
    if c["dtype"] == "i8s":
        acc = acc * s.row[:, None]
        acc = acc if s.bias is None else acc + s.bias
    got["C"] = torch.zeros(_c_shape(c), device="cuda", dtype=_out_type(c))
    got["C"][:, :c["N"]] = acc.to(_out_type(c))
    return got


def _plain_wgrad(s):
    c = s.case
    x, _, _ = _padded(s.X[:, :c["K"]].float(), s)
    dy, _, _ = _padded(s.dY[:, :c["N"]].float(), s)
    left, right = (dy, x) if c["trans_b"] else (x, dy)
    dw = torch.zeros(s.weight, device="cuda", dtype=TORCH_TYPE[c["dtype"]])
    dw[..., :right.shape[-1]] = torch.matmul(left.transpose(1, 2).contiguous(), right).to(dw.dtype)
    return {"dW": dw}


def run(state):
    s, c = state, state.case
    if not own:
        if c["kind"] == "quantize":
            return _plain_quantize(s)
        return _plain_wgrad(s) if c["kind"] == "wgrad" else _plain_product(s)
    ab = s.ab
    if c["kind"] == "quantize":
        _check(ab, ab.abft_quantize_rows(s.X, ab.DTYPE_CODE[c["dtype"]], c["rows"], c["cols"], s.X.shape[-1], s.Q,
                                         s.Q.shape[-1], s.scale), "abft_quantize_rows")
        return {"Q": s.Q, "scale": s.scale}
    if c["kind"] == "wgrad":
        _check(ab, ab.abft_gemm_grouped_wgrad(s.ctx, s.X, s.dY, s.offsets, s.dW, s.code, s.shape), "abft_gemm_grouped_wgrad")
        return {"dW": s.dW}
    if c["kind"] == "scaled":
        _check(ab, ab.abft_gemm_scaled(s.ctx, s.A, s.B, s.scales, s.C, s.mode, s.shape, s.result), "abft_gemm_scaled")
    else:
        _check(ab, ab.abft_gemm_grouped(s.ctx, s.A, s.B, s.offsets, s.scales, s.C, s.code, s.mode, s.shape, s.result),
               "abft_gemm_grouped")
    if c["mode"] != "detect":
        return {"C": s.C}
    return {"C": s.C, "row_flag": s.row_flag, "col_flag": s.col_flag, "counts": s.counts}


def exact(case, seed):
    """From the definitions, a group at a time, in 64 bits; flags and counts are whole numbers and have no such value."""
    c, s = case, _inputs(case, seed)
    if c["kind"] == "quantize":
        x = s.X[:, :c["cols"]].double()
        top = x.abs().max(dim=1).values
        q = torch.zeros((c["rows"], _pad(c["cols"], 1)), device="cuda", dtype=torch.int8)
        q[:, :c["cols"]] = (127 * x / top.clamp(min=1e-300)[:, None]).round().to(torch.int8)
        return {"Q": q, "scale": top / 127}
    ends = [0, c["M"]] if c["kind"] == "scaled" else s.offsets.tolist()
    if c["kind"] == "wgrad":
        dw = torch.zeros(s.weight, device="cuda", dtype=torch.float64)
        for g, (a, b) in enumerate(zip(ends, ends[1:])):
            d = s.dY[a:b, :c["N"]].double().t() @ s.X[a:b, :c["K"]].double()
            d = d if c["trans_b"] else d.t()
            dw[g, :, :d.shape[1]] = d
        return {"dW": dw}
    C = torch.zeros(_c_shape(c), device="cuda", dtype=torch.float64)
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        w = s.B[g].double()
        p = s.A[a:b, :c["K"]].double() @ (w[:, :c["K"]].t() if c["trans_b"] else w[:, :c["N"]])
        if c["dtype"] == "i8s":
            p = p * s.row[a:b, None].double() * s.col[g].double()
        C[a:b, :c["N"]] = p if s.bias is None else p + s.bias.double()
    got = {"C": C.to(torch.int32) if c["dtype"] == "i8" else C}
    if c["mode"] == "detect":
        got.update(row_flag=None, col_flag=None, counts=None)
    return got


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": 3.0 * n + 4 * c["rows"], "flops": 3.0 * n}
    counts = [c["M"]] if c["kind"] == "scaled" else _counts(c)
    rows, es = sum(counts), ES[c["dtype"]]
    weights = (len(counts) if c["kind"] == "wgrad" else sum(1 for n in counts if n)) * c["N"] * c["K"] * es
    flops = 2.0 * rows * c["N"] * c["K"]
    if c["kind"] == "wgrad":
        return {"bytes": float(rows * (c["N"] + c["K"]) * es + weights), "flops": flops}
    b = rows * c["K"] * es + weights + rows * c["N"] * (4 if c["dtype"] == "i8" else 2)
    if c["dtype"] == "i8s":
        b += 4 * (rows + len(counts) * c["N"])
    if c["mode"] == "detect":
        b += c["M"] + len(counts) * c["N"]
    return {"bytes": float(b), "flops": flops}
