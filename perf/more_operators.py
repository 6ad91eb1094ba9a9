"""Operators of a layer of experts from its router's scores to its output, and of 4-bit layers, as cases that can be timed and compared.

A case is a dict of plain values.  ``prepare`` makes what a program holds before the call (inputs, output buffers and, where ``own`` is
true, a context with the weight checksum that the program encodes once), ``run`` makes one pass: the calls of libabft's operators where
``own`` is true, their plain form in elementary torch operations otherwise.  ``exact`` is what the operators are defined as, in 64 bits.

Kinds
  route      scores of experts from logits, the best experts of each token with their weights; with "grad", the gradient of the logits too
  dispatch   entries (a token's choice each) sorted by expert, and the tokens' rows brought into that order
  combine    the experts' rows back to their tokens, weighted and added up; with "grad", the gradients of rows and weights too
  rows4      rows to 4-bit floating point in blocks of 32 with a power of two each, and back; with "topk", in the order of a dispatch
  product4   C = A B (+ bias) of such rows, for one matrix or one for each group of rows; C in a 16-bit type

Sizes are those of the layers of ViT-B/16 (197 tokens an image, hidden 768) and ViT-L/16 (hidden 1024, MLP 4096), for one expert or
several; values those of such layers: logits N(0, 1.5) with some experts more popular than others, activations N(0, 1), weights
N(0, 0.02), gradients N(0, 0.01).
"""
from __future__ import annotations

import math
import random
import weakref

import torch

own = False

TORCH_TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ES = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK = 32                                       # elements of a 4-bit row that share a power of two


# ---------------------------------------------------------------------------------- the cases
def _route(name, dtype, tokens, experts, topk, score="softmax", bias=False, groups=1, top_groups=1, best=1, normalise=True, scale=1.0,
           padded=0, grad=False):
    return dict(name=name, kind="route", dtype=dtype, tokens=tokens, experts=experts, topk=topk, score=score, bias=bias, groups=groups,
                top_groups=top_groups, best=best, normalise=normalise, scale=scale, padded=padded, grad=grad)


def _dispatch(name, dtype, tokens, experts, topk, cols, padded=0):
    return dict(name=name, kind="dispatch", dtype=dtype, tokens=tokens, experts=experts, topk=topk, cols=cols, padded=padded)


def _combine(name, dtype, tokens, topk, cols, base=False, padded=0, grad=False):
    return dict(name=name, kind="combine", dtype=dtype, tokens=tokens, topk=topk, cols=cols, base=base, padded=padded, grad=grad)


def _rows4(name, dtype, tokens, cols, topk=0, padded=0):
    return dict(name=name, kind="rows4", dtype=dtype, tokens=tokens, cols=cols, topk=topk, padded=padded)


def _product4(name, M, groups, N, K, out="bf16", mode="detect", bias=False, routing=0, spare=0):
    return dict(name=name, kind="product4", out=out, M=M, groups=groups, N=N, K=K, mode=mode, bias=bias, routing=routing, spare=spare)


def listed():
    return [
        # a few tokens in flight, sigmoid scores with a bias for balance, only the best groups of experts: latency
        _route("route_few_bf16", "bf16", 16, 64, 8, score="sigmoid", bias=True, groups=8, top_groups=4, best=2, scale=2.5),
        # training on a large batch, forward and backward
        _route("route_train_f32", "f32", 12608, 128, 8, padded=100, grad=True),
        # rows of a few tokens for their experts: latency
        _dispatch("dispatch_few_bf16", "bf16", 16, 32, 4, 1024),
        # the same for a large batch: bandwidth
        _dispatch("dispatch_b64_bf16", "bf16", 12608, 64, 4, 1024, padded=100),
        # the experts' rows of a few tokens back: latency
        _combine("combine_few_bf16", "bf16", 16, 4, 1024),
        # training on a large batch with a residual, forward and backward, a width that is no whole number of blocks
        _combine("combine_train_f16", "f16", 12608, 2, 1001, base=True, padded=37, grad=True),
        # one image's tokens to 4 bits and back: latency
        _rows4("rows4_f16_1image", "f16", 197, 768),
        # sorted rows of a large batch straight to 4 bits, and back: bandwidth
        _rows4("rows4_b64_bf16", "bf16", 6304, 4096, topk=2, padded=50),
        # one token through a 4-bit layer: reads the weight once
        _product4("product4_1token", 1, 1, 4096, 1024, mode="off", bias=True),
        # a few tokens, each to an expert of its own among many, protected: most of the time goes to weights
        _product4("product4_experts_few", 32, 32, 4096, 1024, routing=3),
        # odd sizes in every dimension, one matrix, unprotected
        _product4("product4_odd_f16", 1537, 1, 1001, 713, out="f16", mode="off"),
        # experts over a large batch, protected, the weights' checksums kept
        _product4("product4_experts_b64", 12608, 16, 4096, 1024, routing=5, spare=100),
    ]


MOST_LOGITS = 12608 * 256
MOST_ELEMENTS = 12608 * 4 * 1024                 # of rows
MOST_PRODUCTS = 12608 * 4096 * 1024
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
    kind = rng.choice(["route", "route", "dispatch", "combine", "combine", "rows4", "product4", "product4", "product4"])
    tokens = _size(rng, 1, 12608)
    padded = rng.choice([0, 0, tokens // 20, tokens // 3])
    if kind == "route":
        while True:
            tokens, experts = _size(rng, 1, 12608), rng.choice([_log(rng, 2, 512), 1 << rng.randint(2, 9)])
            if tokens * experts <= MOST_LOGITS:
                break
        padded = rng.choice([0, 0, tokens // 20, tokens // 3])
        topk = min(experts, rng.choice([1, 2, 4, 6, 8, 10]))
        groups = rng.choice([g for g in (1, 1, 2, 3, 4, 8, 16) if experts % g == 0 and (g == 1 or experts // g >= 2)])
        least = (topk + experts // groups - 1) // (experts // groups)
        c = _route("", rng.choice(["bf16", "f16", "f32"]), tokens, experts, topk, score=rng.choice(["softmax", "sigmoid"]),
                   bias=rng.random() < 0.5, groups=groups, top_groups=rng.randint(least, groups), best=rng.choice([1, 2]),
                   normalise=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]), padded=padded, grad=rng.random() < 0.5)
    elif kind == "product4":
        mode = rng.choice(["off", "detect"])
        while True:
            M, N, K, groups = _size(rng, 1, 12608), _size(rng, 64, 4096), _size(rng, 64, 4096), rng.choice([1, _log(rng, 1, 64)])
            if M * N * K <= MOST_PRODUCTS and groups * N * K <= MOST_WEIGHTS:
                break
        c = _product4("", M, groups, N, K, out=rng.choice(["bf16", "f16"]), mode=mode, bias=rng.random() < 0.3,
                      routing=rng.randint(10, 1 << 30), spare=0 if groups == 1 else rng.choice([0, 0, M // 20, M // 5]))
    else:
        cols, topk = _size(rng, 32, 4096), rng.choice([1, 2, 4, 6, 8])
        while tokens * topk * cols > MOST_ELEMENTS:
            cols, topk = _size(rng, 32, 4096), rng.choice([1, 2, 4, 6, 8])
        dtype = rng.choice(["bf16", "f16"])
        if kind == "dispatch":
            c = _dispatch("", dtype, tokens, max(topk, _log(rng, 2, 256)), topk, cols, padded=padded)
        elif kind == "combine":
            c = _combine("", dtype, tokens, topk, cols, base=rng.random() < 0.5, padded=padded, grad=rng.random() < 0.5)
        else:
            c = _rows4("", dtype, tokens, cols, topk=rng.choice([0, topk]), padded=0)
            c["padded"] = padded if c["topk"] else 0
    del c["name"]
    return c


def _counts(c):
    """Rows of each group of a case: uneven, as routers deal them out, some groups without any."""
    if c["groups"] == 1:
        return [c["M"] - c["spare"]]
    rng = random.Random(c["routing"])
    weight = [0.0 if rng.random() < 0.1 else math.exp(rng.gauss(0.0, 0.7)) for _ in range(c["groups"])]
    if not any(weight):
        weight[0] = 1.0
    got = [0] * c["groups"]
    for g in rng.choices(range(c["groups"]), weight, k=c["M"] - c["spare"]):
        got[g] += 1
    return got


# ---------------------------------------------------------------------------------- what a program holds
def _up(n, q):
    return (n + q - 1) // q * q


def _pad(n, elem_bytes):
    return _up(n, 16 // elem_bytes)


def _normal(gen, std, *shape):
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, std, generator=gen)


def _rows(gen, dtype, std, rows, cols):
    """Rows padded to whole 16 bytes, the pad not zero."""
    return _normal(gen, std, rows, _pad(cols, ES[dtype])).to(TORCH_TYPE[dtype])


def _choices(gen, tokens, experts, topk, padded):
    """Experts of each token, different ones, some experts more popular; -1 for the tokens that pad a batch, anywhere in it."""
    liking = _normal(gen, 1.0, tokens, experts) + _normal(gen, 0.7, experts)
    ids = torch.argsort(liking, dim=1, descending=True)[:, :topk].to(torch.int32)
    out = torch.randperm(tokens, generator=gen, device="cuda")[:padded]
    ids[out] = -1
    return ids.contiguous()


def _order(gen, tokens, topk, padded):
    """The entries of all tokens but the padded ones in an order of their rows, -1 behind them; and the row of each entry."""
    n = tokens * topk
    keep = torch.ones(tokens, dtype=torch.bool, device="cuda")
    keep[torch.randperm(tokens, generator=gen, device="cuda")[:padded]] = False
    mixed = torch.randperm(n, generator=gen, device="cuda")
    mixed = mixed[keep[mixed // topk]]
    order = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    order[:mixed.numel()] = mixed.to(torch.int32)
    place = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    place[mixed] = torch.arange(mixed.numel(), dtype=torch.int32, device="cuda")
    return order, place.view(tokens, topk)


def _codes(gen, std, rows, cols):
    """4-bit rows as a quantised tensor has them: two elements to a byte, the first in its low half, zeros behind the last, and the
    biased exponents of their blocks.  Rows lie whole 16 bytes apart."""
    blocks = (cols + BLOCK - 1) // BLOCK
    x = _normal(gen, std, rows, blocks * BLOCK)
    x[:, cols:] = 0
    return _to4(x.view(rows, blocks, BLOCK))


class _State:
    pass


def _inputs(c, seed):
    s = _State()
    s.case = c
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if c["kind"] == "route":
        x = _normal(gen, 1.5, c["tokens"], _pad(c["experts"], ES[c["dtype"]]))
        x[:, :c["experts"]] += _normal(gen, 0.5, c["experts"])
        x[torch.randperm(c["tokens"], generator=gen, device="cuda")[:c["padded"]]] = -math.inf
        s.logits = x.to(TORCH_TYPE[c["dtype"]])
        s.bias = _normal(gen, 0.05, c["experts"]) if c["bias"] else None
        s.dweight = _normal(gen, 0.01, c["tokens"], c["topk"]) if c["grad"] else None
    elif c["kind"] == "dispatch":
        s.expert = _choices(gen, c["tokens"], c["experts"], c["topk"], c["padded"])
        s.X = _rows(gen, c["dtype"], 1.0, c["tokens"], c["cols"])
    elif c["kind"] == "combine":
        s.order, s.place = _order(gen, c["tokens"], c["topk"], c["padded"])
        s.Y = _rows(gen, c["dtype"], 1.0, c["tokens"] * c["topk"], c["cols"])
        s.weight = torch.softmax(_normal(gen, 1.0, c["tokens"], c["topk"]), dim=1)
        s.base = _rows(gen, c["dtype"], 1.0, c["tokens"], c["cols"]) if c["base"] else None
        s.dout = _rows(gen, c["dtype"], 0.01, c["tokens"], c["cols"]) if c["grad"] else None
    elif c["kind"] == "rows4":
        # tokens differ in size, as those behind a layer norm's gain or an activation do
        x = _rows(gen, c["dtype"], 1.0, c["tokens"], c["cols"])
        s.X = (x.float() * torch.exp(_normal(gen, 1.0, c["tokens"], 1))).to(x.dtype)
        s.order = _order(gen, c["tokens"], c["topk"], c["padded"])[0] if c["topk"] else None
    else:
        s.A, s.a_scale = _codes(gen, 1.0, c["M"], c["K"])
        s.B, s.b_scale = _codes(gen, 0.02, c["groups"] * c["N"], c["K"])
        s.bias = _normal(gen, 0.1, c["N"]) if c["bias"] else None
        counts = _counts(c)
        random.Random(int(seed)).shuffle(counts)
        s.most = max(counts)
        ends = [0]
        for n in counts:
            ends.append(ends[-1] + n)
        s.offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    return s


def _zeros(dtype, *shape):
    return torch.zeros(shape, device="cuda", dtype=dtype)


def _check(ab, rc, where):
    if rc != ab.ABFT_OK:
        raise ab.AbftError(rc, where)


def _prepare_own(s):
    import paper_2310_03841_amd as ab
    c = s.case
    s.ab = ab
    if c["kind"] != "product4":
        s.code = ab.DTYPE_CODE[c["dtype"]]
        s.type = TORCH_TYPE[c["dtype"]]
    if c["kind"] == "route":
        s.routing = ab.make_routing(c["tokens"], c["experts"], c["topk"], ld=s.logits.shape[1],
                                    score=ab.ABFT_SIGMOID if c["score"] == "sigmoid" else ab.ABFT_SOFTMAX, normalise=c["normalise"],
                                    scale=c["scale"], bias=s.bias, groups=c["groups"], top_groups=c["top_groups"], group_best=c["best"])
        s.expert, s.weight = _zeros(torch.int32, c["tokens"], c["topk"]), _zeros(torch.float32, c["tokens"], c["topk"])
        s.dlogits = _zeros(s.type, *s.logits.shape) if c["grad"] else None
    elif c["kind"] == "dispatch":
        n = c["tokens"] * c["topk"]
        s.ctx = ab.abft_create(n, c["experts"], 1, c["experts"])
        weakref.finalize(s, ab.abft_destroy, s.ctx)
        s.offsets, s.order, s.place = _zeros(torch.int32, c["experts"] + 1), _zeros(torch.int32, n), _zeros(torch.int32, c["tokens"], c["topk"])
        s.Y = _zeros(s.type, n, s.X.shape[1])
    elif c["kind"] == "combine":
        s.out = _zeros(s.type, c["tokens"], s.Y.shape[1])
        if c["grad"]:
            s.dY, s.dweight = _zeros(s.type, *s.Y.shape), _zeros(torch.float32, c["tokens"], c["topk"])
    elif c["kind"] == "rows4":
        n = c["tokens"] * (c["topk"] or 1)
        s.Q = _zeros(torch.uint8, n, _up(c["cols"], BLOCK) // 2)
        s.scale = _zeros(torch.uint8, n, _up((c["cols"] + BLOCK - 1) // BLOCK, 16))
        s.back = _zeros(s.type, n, s.X.shape[1])
    else:
        G, N = c["groups"], c["N"]
        s.ctx = ab.abft_create(c["M"], G * N, G * _up(c["K"], 128), G)
        weakref.finalize(s, ab.abft_destroy, s.ctx)
        s.C = _zeros(TORCH_TYPE[c["out"]], c["M"], _pad(N, 2))
        s.shape = ab.make_shape(c["M"], N, c["K"], batch=G, lda=2 * s.A.shape[1], ldb=2 * s.B.shape[1], ldc=s.C.shape[1])
        s.scales = ab.make_mx4(s.a_scale, s.a_scale.shape[1], s.b_scale, s.b_scale.shape[1], N * s.b_scale.shape[1], s.bias,
                               out=ab.DTYPE_CODE[c["out"]])
        s.mode, s.result = ab.ABFT_OFF, None
        if c["mode"] == "detect":
            s.row_flag, s.col_flag = _zeros(torch.uint8, c["M"]), _zeros(torch.uint8, G * N)
            s.counts = _zeros(torch.int32, 8)
            s.result = ab.make_result(s.row_flag, s.col_flag, s.counts)
            # the weights' checksums: once, as programs do whose weights stay
            s.mode = ab.ABFT_DETECT | ab.ABFT_B_CHECKSUM_CACHED
            _check(ab, ab.abft_encode_mx4(s.ctx, s.B, s.scales, s.shape), "abft_encode_mx4")


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _prepare_own(s)
    elif case["kind"] == "product4" and case["mode"] == "detect":
        w = _from4(s.B, s.b_scale, case["K"]).view(case["groups"], case["N"], case["K"])
        s.b_sum, s.b_max = w.sum(dim=1), w.abs().amax(dim=(1, 2))
    return s


# ---------------------------------------------------------------------------------- the operators
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _to4(x):
    """Blocks [rows][blocks][32] of fp32 to packed codes and biased exponents, both with rows of whole 16 bytes."""
    rows, blocks = x.shape[:2]
    top = x.abs().amax(dim=2)
    # the exponent of the largest, as frexp gives it (a mantissa of [0.5, 1)), less that of 6
    e = torch.where(top > 0, torch.frexp(top)[1] - 1 - 2, -127).clamp(-127, 127)
    # (in two steps: a single power of two may be out of range)
    half = torch.div(-e, 2, rounding_mode="floor")
    v = torch.ldexp(torch.ldexp(x, half[..., None]), (-e - half)[..., None])
    a = v.abs()
    # steps of 1/2 below 2, of 1 below 4, of 2 above
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.clamp(torch.round(a / step) * step, max=6.0)
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, value in enumerate(_E2M1):
        code = torch.where(a == value, i, code).to(torch.uint8)
    code = code | torch.where(torch.signbit(x), 8, 0).to(torch.uint8)
    code = code.view(rows, blocks * BLOCK)
    scale = torch.zeros((rows, _up(blocks, 16)), device=x.device, dtype=torch.uint8)
    scale[:, :blocks] = (e + 127).to(torch.uint8)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scale


def _from4(codes, scale, cols, wide=torch.float32):
    """The values that packed codes and exponents stand for."""
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device, dtype=wide)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=2).view(codes.shape[0], -1)
    e = scale[:, :v.shape[1] // BLOCK].to(torch.int32) - 127
    v = torch.ldexp(v.view(v.shape[0], -1, BLOCK), e[..., None].to(wide if wide == torch.float64 else torch.int32))
    return v.view(v.shape[0], -1)[:, :cols]


def _plain_route(s):
    c = s.case
    T, E, k, G = c["tokens"], c["experts"], c["topk"], c["groups"]
    x = s.logits[:, :E].double()                   # scores of far and near logits meet at a border: 64 bits
    masked = x == -math.inf
    if c["score"] == "softmax":
        top = x.amax(dim=1, keepdim=True)
        e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        score = e / e.sum(dim=1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    key = score if s.bias is None else score + s.bias.double()
    key = torch.where(masked, -math.inf, key)
    if G > 1:
        per = key.view(T, G, E // G)
        value = torch.sort(per, dim=2, descending=True)[0][:, :, :c["best"]].sum(dim=2)
        at = torch.sort(value, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        stay = torch.zeros((T, G), dtype=torch.bool, device="cuda")
        stay.scatter_(1, at, True)
        key = torch.where(stay[:, :, None], per, -math.inf).view(T, E)
    best, at = torch.sort(key, dim=1, descending=True, stable=True)
    at, there = at[:, :k], best[:, :k] > -math.inf
    chosen = torch.where(there, torch.gather(score, 1, at), 0.0)
    total = chosen.sum(dim=1, keepdim=True).clamp(min=1e-300) if c["normalise"] else 1.0
    share = chosen / total
    got = {"expert": torch.where(there, at, -1).to(torch.int32), "weight": (share * c["scale"]).float()}
    if c["grad"]:
        dw = torch.where(there, s.dweight.double(), 0.0) * c["scale"]
        if c["normalise"]:
            dw = (dw - (dw * share).sum(dim=1, keepdim=True)) / total
        ds = torch.zeros_like(score).scatter_add_(1, at, torch.where(there, dw, 0.0))
        if c["score"] == "softmax":
            dx = score * (ds - (ds * score).sum(dim=1, keepdim=True))
        else:
            dx = ds * score * (1.0 - score)
        got["dlogits"] = torch.zeros_like(s.logits)
        got["dlogits"][:, :E] = dx.to(s.logits.dtype)
    return got


def _plain_dispatch(s):
    c = s.case
    e = s.expert.reshape(-1).long()
    n, E = e.numel(), c["experts"]
    order = torch.sort(torch.where(e < 0, E, e), stable=True)[1]
    used = (e >= 0).sum()
    there = torch.arange(n, device="cuda") < used
    offsets = torch.zeros(E + 1, device="cuda", dtype=torch.int32)
    offsets[1:] = torch.cumsum(torch.bincount(torch.where(e < 0, E, e), minlength=E + 1)[:E], dim=0)
    place = torch.zeros(n, device="cuda", dtype=torch.int32)
    place[order] = torch.where(there, torch.arange(n, device="cuda"), -1).to(torch.int32)
    y = torch.where(there[:, None], s.X[order // c["topk"]], 0.0)
    y[:, c["cols"]:] = 0
    return {"offsets": offsets, "order": torch.where(there, order, -1).to(torch.int32), "place": place.view(-1, c["topk"]), "Y": y}


def _plain_combine(s):
    c = s.case
    cols, there = c["cols"], s.place >= 0
    at = s.place.clamp(min=0).long()
    out = _zeros(torch.float32, c["tokens"], s.Y.shape[1])
    if c["base"]:
        out[:, :cols] = s.base[:, :cols].float()
    for j in range(c["topk"]):
        out[:, :cols] += torch.where(there[:, j, None], s.weight[:, j, None] * s.Y[at[:, j], :cols].float(), 0.0)
    got = {"out": out.to(s.Y.dtype)}
    if c["grad"]:
        dout, used = s.dout[:, :cols].float(), s.order >= 0
        of = s.order.clamp(min=0).long()
        dy = torch.zeros_like(s.Y)
        dy[:, :cols] = torch.where(used[:, None], s.weight.reshape(-1)[of, None] * dout[of // c["topk"]], 0.0).to(s.Y.dtype)
        dw = _zeros(torch.float32, c["tokens"], c["topk"])
        for j in range(c["topk"]):
            dw[:, j] = torch.where(there[:, j], (s.Y[at[:, j], :cols].double() * dout.double()).sum(dim=1), 0.0).float()
        got.update(dY=dy, dweight=dw)
    return got


def _plain_rows4(s):
    c = s.case
    x = s.X[:, :c["cols"]].float()
    if c["topk"]:
        x = torch.where(s.order[:, None] >= 0, x[s.order.clamp(min=0).long() // c["topk"]], 0.0)
    full = _zeros(torch.float32, x.shape[0], _up(c["cols"], BLOCK))
    full[:, :c["cols"]] = x
    codes, scale = _to4(full.view(x.shape[0], -1, BLOCK))
    back = _zeros(s.X.dtype, x.shape[0], s.X.shape[1])
    back[:, :c["cols"]] = _from4(codes, scale, c["cols"]).to(s.X.dtype)
    return {"values": back}


def _plain_product4(s):
    c = s.case
    G, N, K, M = c["groups"], c["N"], c["K"], c["M"]
    a = _from4(s.A, s.a_scale, K)
    w = _from4(s.B, s.b_scale, K).view(G, N, K)
    used = torch.arange(M, device="cuda") < s.offsets[-1]
    if G == 1:
        rows, flat = a[None], torch.arange(M, device="cuda")
    else:
        # rows sorted by group, as groups x most rows of a group, with zeros behind each group's; rows of no group meet in one behind all
        group = torch.searchsorted(s.offsets[1:].contiguous(), torch.arange(M, device="cuda"), right=True, out_int32=True).long()
        at = torch.arange(M, device="cuda") - s.offsets[group.clamp(max=G)]
        flat = torch.where(used, group * s.most + at, G * s.most)
        rows = _zeros(torch.float32, G * s.most + 1, K)
        rows[flat] = a
        rows = rows[:-1].view(G, s.most, K)
        flat = flat.clamp(max=G * s.most - 1)
    acc = torch.matmul(rows, w.transpose(1, 2).contiguous())
    if c["bias"]:
        acc = acc + s.bias
    got = {"C": _zeros(TORCH_TYPE[c["out"]], M, _pad(N, 2))}
    got["C"][:, :N] = torch.where(used[:, None], acc.reshape(-1, N)[flat], 0.0).to(got["C"].dtype)
    if c["mode"] == "detect":
        if c["bias"]:
            acc = acc - s.bias                     # the sums ahead of the bias are what is checked
        obs_r, obs_c = acc.sum(dim=2), acc.sum(dim=1)
        pred_r = torch.matmul(rows, s.b_sum[:, :, None])[..., 0]
        pred_c = torch.matmul(w, rows.sum(dim=1)[:, :, None])[..., 0]
        tau = 1e-3 * K * rows.abs().amax(dim=(1, 2)) * s.b_max
        bad_r, bad_c = ~((obs_r - pred_r).abs() <= tau[:, None]), ~((obs_c - pred_c).abs() <= tau[:, None])
        got["row_flag"] = (used & bad_r.reshape(-1)[flat]).to(torch.uint8)
        got["col_flag"] = bad_c.reshape(-1).to(torch.uint8)
        counts = _zeros(torch.int32, 8)
        counts[0], counts[1] = got["row_flag"].sum(), got["col_flag"].sum()
        counts[2] = torch.where((counts[0] > 0) & (counts[1] > 0), 1, torch.where((counts[0] > 0) | (counts[1] > 0), 2, 0))
        got["counts"] = counts
    return got


_PLAIN = {"route": _plain_route, "dispatch": _plain_dispatch, "combine": _plain_combine, "rows4": _plain_rows4, "product4": _plain_product4}


def run(state):
    s, c = state, state.case
    if not own:
        return _PLAIN[c["kind"]](s)
    ab = s.ab
    if c["kind"] == "route":
        _check(ab, ab.abft_route(s.logits, s.code, s.routing, s.expert, s.weight), "abft_route")
        got = {"expert": s.expert, "weight": s.weight}
        if c["grad"]:
            _check(ab, ab.abft_route_grad(s.logits, s.code, s.routing, s.expert, s.dweight, s.dlogits, s.dlogits.shape[1]), "abft_route_grad")
            got["dlogits"] = s.dlogits
        return got
    if c["kind"] == "dispatch":
        n = c["tokens"] * c["topk"]
        _check(ab, ab.abft_group_rows(s.ctx, s.expert, n, c["experts"], s.offsets, s.order, s.place), "abft_group_rows")
        _check(ab, ab.abft_gather_rows(s.X, s.code, c["tokens"], c["cols"], s.X.shape[1], s.order, n, c["topk"], s.Y, s.Y.shape[1]),
               "abft_gather_rows")
        return {"offsets": s.offsets, "order": s.order, "place": s.place, "Y": s.Y}
    if c["kind"] == "combine":
        n, ld = c["tokens"] * c["topk"], s.Y.shape[1]
        _check(ab, ab.abft_combine_rows(s.Y, s.code, n, c["cols"], ld, s.place, s.weight, c["tokens"], c["topk"], s.base, ld, s.out, ld),
               "abft_combine_rows")
        if not c["grad"]:
            return {"out": s.out}
        _check(ab, ab.abft_combine_rows_grad(s.dout, s.code, c["tokens"], c["cols"], ld, s.place, s.weight, c["topk"], s.Y, n, ld, s.dY, ld,
                                             s.dweight), "abft_combine_rows_grad")
        return {"out": s.out, "dY": s.dY, "dweight": s.dweight}
    if c["kind"] == "rows4":
        n = s.Q.shape[0]
        _check(ab, ab.abft_quantize_mx4(s.X, s.code, c["tokens"], c["cols"], s.X.shape[1], s.order, n, c["topk"] or 1, s.Q, 2 * s.Q.shape[1],
                                        s.scale, s.scale.shape[1]), "abft_quantize_mx4")
        _check(ab, ab.abft_dequantize_mx4(s.Q, 2 * s.Q.shape[1], s.scale, s.scale.shape[1], n, c["cols"], s.back, s.code, s.back.shape[1]),
               "abft_dequantize_mx4")
        return {"values": s.back}
    offsets = s.offsets if c["groups"] > 1 else None
    _check(ab, ab.abft_gemm_mx4(s.ctx, s.A, s.B, offsets, s.scales, s.C, s.mode, s.shape, s.result), "abft_gemm_mx4")
    if c["mode"] != "detect":
        return {"C": s.C}
    return {"C": s.C, "row_flag": s.row_flag, "col_flag": s.col_flag, "counts": s.counts}


# ---------------------------------------------------------------------------------- the definitions
def _exact_route(s):
    c = s.case
    T, E, k, G = c["tokens"], c["experts"], c["topk"], c["groups"]
    x = s.logits[:, :E].double()
    score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(x, dim=1), nan=0.0)
    key = score + (0.0 if s.bias is None else s.bias.double())
    key[torch.isinf(x)] = -math.inf
    if G > 1:
        size = E // G
        # rounds of the best that is left, first ones first, as the choice is defined
        left, value = key.clone(), torch.zeros(T, G, device="cuda", dtype=torch.float64)
        for _ in range(c["best"]):
            at = left.view(T, G, size).argmax(dim=2, keepdim=True)
            value += left.view(T, G, size).gather(2, at)[..., 0]
            left.view(T, G, size).scatter_(2, at, -math.inf)
        rank = (value[:, None, :] > value[:, :, None]).sum(dim=2)
        equal = value[:, None, :] == value[:, :, None]
        rank += (equal & torch.ones(G, G, dtype=torch.bool, device="cuda").tril(-1)).sum(dim=2)
        key = key.masked_fill((rank >= c["top_groups"]).repeat_interleave(size, dim=1), -math.inf)
    expert, weight = torch.full((T, k), -1, device="cuda", dtype=torch.int32), _zeros(torch.float64, T, k)
    leaf = x.clone()
    for j in range(k):
        best = key.amax(dim=1, keepdim=True)
        first = torch.where(key == best, torch.arange(E, device="cuda"), E).amin(dim=1, keepdim=True)
        there = best > -math.inf
        expert[:, j] = torch.where(there, first, -1)[:, 0].to(torch.int32)
        weight[:, j] = torch.where(there, score.gather(1, first), 0.0)[:, 0]
        key.scatter_(1, first, -math.inf)
    got = {"expert": expert}
    total = weight.sum(dim=1, keepdim=True)
    got["weight"] = c["scale"] * (torch.where(total > 0, weight / total, 0.0) if c["normalise"] else weight)
    if c["grad"]:
        leaf = torch.where(torch.isinf(leaf), -1e4, leaf).requires_grad_()
        sc = torch.sigmoid(leaf) if c["score"] == "sigmoid" else torch.softmax(leaf, dim=1)
        w = sc.gather(1, expert.clamp(min=0).long()) * (expert >= 0)
        if c["normalise"]:
            w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
        (c["scale"] * w * s.dweight.double()).sum().backward()
        dx = _zeros(torch.float64, *s.logits.shape)
        dx[:, :E] = leaf.grad * (expert[:, :1] >= 0)
        got["dlogits"] = dx
    return got


def _exact_product4(s):
    c = s.case
    a, w = _values4(s.A, s.a_scale, c["K"]), _values4(s.B, s.b_scale, c["K"]).view(c["groups"], c["N"], c["K"])
    C = _zeros(torch.float64, c["M"], _pad(c["N"], 2))
    ends = s.offsets.tolist()
    for g, (lo, hi) in enumerate(zip(ends, ends[1:])):
        p = a[lo:hi] @ w[g].t()
        C[lo:hi, :c["N"]] = p if s.bias is None else p + s.bias.double()
    got = {"C": C}
    if c["mode"] == "detect":
        got.update(row_flag=None, col_flag=None, counts=None)
    return got


def _values4(codes, scale, cols):
    """Sign, exponent and mantissa of each element, and its block's power of two, in 64 bits."""
    nib = torch.stack([codes % 16, codes // 16], dim=2).view(codes.shape[0], -1)[:, :cols].double()
    sign, mag = torch.where(nib >= 8, -1.0, 1.0), torch.remainder(nib, 8)
    e, m = torch.div(mag, 2, rounding_mode="floor"), torch.remainder(mag, 2)
    v = torch.where(e > 0, (1 + m / 2) * torch.exp2(e - 1), m / 2)
    return sign * v * torch.exp2(scale.double().repeat_interleave(BLOCK, dim=1)[:, :cols] - 127)


def exact(case, seed):
    """From the definitions, in 64 bits; flags and counts are whole numbers and have no such value."""
    c, s = case, _inputs(case, seed)
    if c["kind"] == "route":
        return _exact_route(s)
    if c["kind"] == "product4":
        return _exact_product4(s)
    cols = c["cols"]
    if c["kind"] == "dispatch":
        e = s.expert.reshape(-1).tolist()
        by = [[] for _ in range(c["experts"])]
        for i, g in enumerate(e):
            if g >= 0:
                by[g].append(i)
        order = [i for g in by for i in g]
        y = _zeros(torch.float64, len(e), s.X.shape[1])
        y[:len(order), :cols] = s.X[torch.tensor(order, dtype=torch.long, device="cuda") // c["topk"], :cols].double()
        return {"offsets": None, "order": None, "place": None, "Y": y}
    if c["kind"] == "combine":
        n = c["tokens"] * c["topk"]
        y = torch.cat([s.Y[:, :cols].double(), _zeros(torch.float64, 1, cols)])
        mine = y[torch.where(s.place < 0, n, s.place).long()]                    # tokens x topk x cols
        out = _zeros(torch.float64, c["tokens"], s.Y.shape[1])
        out[:, :cols] = torch.matmul(s.weight.double()[:, None, :], mine)[:, 0]
        if c["base"]:
            out[:, :cols] += s.base[:, :cols].double()
        got = {"out": out}
        if c["grad"]:
            d = s.dout[:, :cols].double()
            dy = _zeros(torch.float64, n + 1, s.Y.shape[1])
            dy[torch.where(s.place < 0, n, s.place).long().reshape(-1), :cols] = (s.weight.double()[:, :, None] * d[:, None, :]).reshape(-1, cols)
            got.update(dY=dy[:-1], dweight=torch.matmul(mine, d[:, :, None])[..., 0])
        return got
    x = s.X[:, :cols].double()
    n = c["tokens"] * (c["topk"] or 1)
    if c["topk"]:
        x = torch.cat([x, _zeros(torch.float64, 1, cols)])[torch.where(s.order < 0, c["tokens"], torch.div(s.order, c["topk"], rounding_mode="floor")).long()]
    back = _zeros(torch.float64, n, s.X.shape[1])
    levels = torch.tensor(_E2M1, device="cuda", dtype=torch.float64)
    # an even code wins where two levels are equally far
    handicap = torch.tensor([0.0, 1e-9] * 4, device="cuda", dtype=torch.float64)
    for lo in range(0, cols, BLOCK):
        b = x[:, lo:lo + BLOCK]
        top = b.abs().amax(dim=1, keepdim=True)
        unit = torch.exp2((torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 2).clamp(-127, 127))
        best, at = torch.full_like(b, math.inf), torch.zeros_like(b)
        for i in range(8):
            far = (b.abs() / unit - levels[i]).abs() + handicap[i]
            at = torch.where(far < best, levels[i], at)
            best = torch.minimum(far, best)
        back[:, lo:lo + BLOCK] = at * unit * torch.sign(b)
    return {"values": back}


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "route":
        n = c["tokens"] * c["experts"]
        grad = c["grad"]
        return {"bytes": float(n * ES[c["dtype"]] * (2 if grad else 1) + c["tokens"] * c["topk"] * (12 if grad else 8)),
                "flops": float(n * (8 if grad else 4))}
    if c["kind"] == "product4":
        counts = _counts(c)
        rows, busy = sum(counts), sum(1 for n in counts if n)
        b = (rows + busy * c["N"]) * (c["K"] / 2 + c["K"] / BLOCK) + 2 * rows * c["N"]
        if c["mode"] == "detect":
            b += c["M"] + c["groups"] * c["N"]
        return {"bytes": float(b), "flops": 2.0 * rows * c["N"] * c["K"]}
    tokens = c["tokens"] - c["padded"]
    n, es = tokens * (c["topk"] or 1), ES[c["dtype"]]
    if c["kind"] == "dispatch":
        return {"bytes": float((tokens + n) * c["cols"] * es + 12 * c["tokens"] * c["topk"] + 4 * c["experts"]), "flops": float(n)}
    if c["kind"] == "combine":
        b = n * c["cols"] * es + c["tokens"] * c["cols"] * es * (2 if c["base"] else 1) + 8 * c["tokens"] * c["topk"]
        f = 2.0 * n * c["cols"]
        if c["grad"]:
            b += (n + tokens) * c["cols"] * es + 4 * c["tokens"] * c["topk"]
            f *= 2.5
        return {"bytes": float(b), "flops": f}
    return {"bytes": float((tokens + n) * c["cols"] * es + n * c["cols"] * (1 + 1 / 16)), "flops": 4.0 * n * c["cols"]}
