"""Layer norm, dropout and the residual tail that joins them, as the learned prior of an unrolled network calls them.

Every array is viewed as (outer, features, inner) with the statistics over the features: inner = 1 are rows of features
(tokens, or maps stored with the features last), inner > 1 are feature maps with the features in front of the voxels.  A case
with kind "forward" is one forward call; "train" is the forward call and its vector-Jacobian product for a given cotangent,
the pair that one training step makes of the operator.

Dropout is defined without a stored mask: element i in memory order takes word i mod 4 of Philox4x32-10 (Salmon et al.,
"Parallel random numbers: as easy as 1, 2, 3", 2011) with the counter offset + i div 4 and the seed as key, and is dropped
where that word is below floor(p 2^32).  What is kept is multiplied by 1 / (1 - p), a number of 32 bits.
"""
import math
import struct

import torch

own = False

EPS = 1e-5
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}
LARGEST = 4 * 100 * 640 * 368                  # elements of the largest listed maps


def _scale(p):
    return struct.unpack("f", struct.pack("f", 1.0 / (1.0 - p)))[0]


def listed():
    def case(name, op, kind, dtype, outer, features, inner, wtype="float32", p=0.0, residual=False):
        return {"name": name, "op": op, "kind": kind, "dtype": dtype, "wtype": wtype, "outer": outer, "features": features,
                "inner": inner, "p": p, "residual": residual}
    return [
        # one vector of 160 features for each of the 20 frames of a cine: a conditioning path, launch latency only
        case("norm frame vectors", "norm", "forward", "bfloat16", 20, 160, 1),
        # patches of 8 x 8 x 8 voxels of a 320 x 320 x 256 knee volume as rows of 1024 features
        case("norm patch rows", "norm", "train", "bfloat16", 51200, 1024, 1),
        # 60 features of 20 frames of 192 x 160, single precision as the paper's networks
        case("norm cine maps", "norm", "train", "float32", 20, 60, 192 * 160),
        # 70 features of three frames with an odd number of voxels (209 x 187), inference in half precision
        case("norm odd maps", "norm", "forward", "float16", 3, 70, 209 * 187, wtype="float16"),
        # wide rows of odd length: a row starts at any element of a 16-byte piece
        case("norm odd wide rows", "norm", "train", "float32", 2049, 4099, 1),
        # the conditioning vectors again: dropout alone, launch latency only
        case("dropout frame vectors", "dropout", "forward", "bfloat16", 20, 160, 1, p=0.1),
        # the residual add of a block without normalisation: 100 features of four knee slices of 640 x 368
        case("dropout knee maps", "dropout", "train", "bfloat16", 4, 100, 640 * 368, p=0.1, residual=True),
        # an odd number of elements in single precision
        case("dropout odd size", "dropout", "train", "float32", 37, 101, 2049, p=0.25),
        # tail of a block on the conditioning vectors: forward and backward, launch latency only
        case("tail frame vectors", "tail", "train", "bfloat16", 20, 160, 1, p=0.1),
        # tail of a residual block on 100 features of four knee slices, mixed precision
        case("tail knee maps", "tail", "train", "bfloat16", 4, 100, 640 * 368, p=0.1),
        # tail of a residual block on 50 features of a cine, single precision
        case("tail cine maps", "tail", "train", "float32", 20, 50, 192 * 160, p=0.05),
        # tail of a block on rows of 1000 features in half precision
        case("tail patch rows", "tail", "train", "float16", 12801, 1000, 1, wtype="float16", p=0.2),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    op = rng.choice(["norm", "dropout", "tail"])
    if rng.random() < 0.5:
        features, inner = log(8, 8000), 1
        outer = log(1, max(1, LARGEST // 4 // features))
    else:
        outer, features = log(1, 32), log(8, 640)
        inner = log(2, max(2, LARGEST // 4 // (outer * features)))
        if rng.random() < 0.5:
            inner = (inner + 7) // 8 * 8
    dtype = rng.choice(list(TYPES))
    return {"op": op, "kind": rng.choice(["forward", "train"]), "dtype": dtype,
            "wtype": rng.choice(["float32", dtype]), "outer": outer, "features": features, "inner": inner,
            "p": 0.0 if op == "norm" else round(rng.uniform(0.02, 0.6), 3),
            "residual": op == "dropout" and rng.random() < 0.5}


def prepare(case, seed):
    """Feature maps with a mean and a spread of their own for every feature, as convolutions leave them; cotangents that are
    small against them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1 + seed)
    dtype, wtype = TYPES[case["dtype"]], TYPES[case["wtype"]]
    shape = (case["outer"], case["features"], case["inner"])

    def normal(size, spread=1.0, mean=0.0):
        return torch.randn(size, generator=gen, device="cuda").mul_(spread).add_(mean)

    def maps():
        spread, mean = normal((1, shape[1], 1), 0.2, 1.0), normal((1, shape[1], 1), 0.5)
        return torch.randn(shape, generator=gen, device="cuda").mul_(spread).add_(mean).to(dtype)

    s = {"op": case["op"], "kind": case["kind"], "p": float(case["p"]), "x": maps(),
         "seed": (1 << 40) + 977 * int(seed), "offset": 1000003 * (int(seed) % 4096)}
    if case["op"] == "tail" or case["residual"]:
        s["residual"] = maps()
    if case["op"] != "dropout":
        s["weight"], s["bias"] = normal(shape[1], 0.1, 1.0).to(wtype), normal(shape[1], 0.1).to(wtype)
    if case["kind"] == "train":
        s["grad"] = normal(shape, 0.1).to(dtype)
        if case["op"] == "tail":
            s["grad_sum"] = normal(shape, 0.1).to(dtype)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _kept(state, n):
    """Truth values of the elements that dropout keeps.  64-bit products hold all bits of two 32-bit factors."""
    low = 0xFFFFFFFF
    c = torch.arange((n + 3) // 4, device="cuda", dtype=torch.int64) + state["offset"]
    a, b = c & low, (c >> 32) & low
    c = d = torch.zeros_like(a)
    k0, k1 = state["seed"] & low, (state["seed"] >> 32) & low
    for _ in range(10):
        p0, p1 = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((p1 >> 32) & low) ^ b ^ k0, p1 & low, ((p0 >> 32) & low) ^ d ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((a, b, c, d), 1).reshape(-1)[:n]
    return words >= int(math.floor(state["p"] * 4294967296.0))


def _dropped(v, kept, p):
    return torch.where(kept, v * _scale(p), 0.0)


def _sum(x, kept, p, residual):
    """residual + dropout(x) with one rounding: kept values times the scale and the sum are exact in 64 bits, and a norm that
    follows would show every element that a rounding in between moves over a border of the arrays' type."""
    return (residual.double() + _dropped(x.double(), kept, p)).float().to(x.dtype)


def _norm(x, weight, bias):
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd * weight + bias, mean, rstd


def _norm_vjp(grad, x, weight, mean, rstd):
    h = (x - mean) * rstd
    g = grad * weight
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx, (grad * h).sum((0, 2)), grad.sum((0, 2))


def _plain(s):
    x, p, dtype = s["x"], s["p"], s["x"].dtype
    kept = _kept(s, x.numel()).view(x.shape) if s["op"] != "norm" else None
    grad = s["grad"].float() if s["kind"] == "train" else None
    if s["op"] == "dropout":
        out = [_sum(x, kept, p, s["residual"]) if "residual" in s else _dropped(x.float(), kept, p).to(dtype)]
        return out if grad is None else out + [_dropped(grad, kept, p).to(dtype)]
    weight, bias = (s[k].float().view(1, -1, 1) for k in ("weight", "bias"))
    wtype = s["weight"].dtype
    if s["op"] == "norm":
        v, stored = x.float(), []
    else:
        total = _sum(x, kept, p, s["residual"])              # the residual stream, as it is stored
        v, stored = total.float(), [total]
    y, mean, rstd = _norm(v, weight, bias)
    out = [y.to(dtype), mean.squeeze(1), rstd.squeeze(1)] + stored
    if grad is None:
        return out
    dx, dw, db = _norm_vjp(grad, v, weight, mean, rstd)
    if s["op"] == "norm":
        return out + [dx.to(dtype), dw.to(wtype), db.to(wtype)]
    ds = s["grad_sum"].float() + dx
    return out + [_dropped(ds, kept, p).to(dtype), ds.to(dtype), dw.to(wtype), db.to(wtype)]


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _own(s):
    import paper_2207_08393_b200 as g
    x, train = s["x"], s["kind"] == "train"
    if s["op"] == "dropout":
        out = [g.dropout_forward(x, s["p"], s["seed"], s["offset"], residual=s.get("residual"))]
        return out + [g.dropout_vjp(s["grad"], s["p"], s["seed"], s["offset"])] if train else out
    if s["op"] == "norm":
        y, mean, rstd = g.layer_norm_forward(x, s["weight"], s["bias"], EPS, dim=1)
        out = [y, mean, rstd]
        return out + list(g.layer_norm_vjp(s["grad"], x, s["weight"], mean, rstd, dim=1)) if train else out
    y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, s["residual"], s["weight"], s["bias"], s["p"], s["seed"],
                                                            s["offset"], EPS, dim=1)
    out = [y, mean, rstd, total]
    if not train:
        return out
    return out + list(g.dropout_add_layer_norm_vjp(s["grad"], s["grad_sum"], total, s["weight"], mean, rstd, s["p"],
                                                   s["seed"], s["offset"], dim=1))


def run(state):
    return _own(state) if own else _plain(state)


# ---- work and definition ---------------------------------------------------------------------------------------------

def work(case):
    """Every input once and every output once: activations, statistics and weights.  (A training step's forward and
    backward calls both read the normalised array; it is counted once.)"""
    n = case["outer"] * case["features"] * case["inner"]
    b, rows = BYTES[case["dtype"]], case["outer"] * case["inner"]
    train = case["kind"] == "train"
    weights = 2 * case["features"] * BYTES[case["wtype"]]
    if case["op"] == "dropout":
        arrays, small, flops = 2 + bool(case["residual"]) + 2 * train, 0, 1 + bool(case["residual"]) + train
    elif case["op"] == "norm":
        arrays, small, flops = 2 + 2 * train, 8 * rows + weights * (1 + train), 7 + 13 * train
    else:
        arrays, small, flops = 4 + 4 * train, 8 * rows + weights * (1 + train), 9 + 15 * train
    return {"bytes": arrays * n * b + small, "flops": flops * n}


def exact(case, seed):
    """The definition in 64 bits.  The mask's words come from 16-bit limbs here."""
    s = prepare(case, seed)
    x, p = s["x"].double(), s["p"]
    n = x.numel()
    keep = None
    if s["op"] != "norm":
        def high_low(word, factor):
            w0, w1, f0, f1 = word & 0xFFFF, word >> 16, factor & 0xFFFF, factor >> 16
            mid = w1 * f0 + (w0 * f0 >> 16)
            mid2 = w0 * f1 + (mid & 0xFFFF)
            return w1 * f1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (w0 * f0 & 0xFFFF)
        index = torch.arange(s["offset"], s["offset"] + -(-n // 4), device="cuda")
        ctr = [index % 2 ** 32, index // 2 ** 32, torch.zeros_like(index), torch.zeros_like(index)]
        for turn in range(10):
            key = [(s["seed"] % 2 ** 32 + turn * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32]
            h0, l0 = high_low(ctr[0], 0xD2511F53)
            h1, l1 = high_low(ctr[2], 0xCD9E8D57)
            ctr = [h1 ^ ctr[1] ^ key[0], l1, h0 ^ ctr[3] ^ key[1], l0]
        keep = torch.empty(4 * index.numel(), dtype=torch.float64, device="cuda")
        limit = math.floor(p * 2 ** 32)
        for k in range(4):
            keep[k::4] = (ctr[k] >= limit).double()
        keep = keep[:n].view(x.shape) * _scale(p)
        del ctr, index
    if s["op"] == "dropout":
        out = [s["residual"].double().addcmul_(x, keep) if "residual" in s else x * keep]
        return out + [s["grad"].double().mul_(keep)] if s["kind"] == "train" else out
    stored = []
    if s["op"] == "tail":                       # what the norm sees is the stored sum, in the arrays' type
        x = s["residual"].double().addcmul_(x, keep).float().to(s["x"].dtype).double()
        stored = [x]
    w = s["weight"].double()[None, :, None]
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    sd = (var + EPS).sqrt()
    h = (x - mean) / sd
    out = [h * w + s["bias"].double()[None, :, None], mean[:, 0], sd.reciprocal()[:, 0]] + stored
    if s["kind"] != "train":
        return out
    dy = s["grad"].double()
    dw, db = torch.einsum("odi,odi->d", dy, h), torch.einsum("odi->d", dy)
    g = dy * w
    g -= g.mean(1, keepdim=True)
    g -= h * torch.einsum("odi,odi->oi", g, h)[:, None] / case["features"]
    g /= sd
    if s["op"] == "norm":
        return out + [g, dw, db]
    g += s["grad_sum"].double()
    return out + [g * keep, g, dw, db]
