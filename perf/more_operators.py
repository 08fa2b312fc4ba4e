"""The gated recurrence of a prior that looks along frames, slices or tokens, its form for one new frame, and the matrix-orthogonal
update that trains such a prior's weights.

scan    h_t = f_t h_(t-1) + (1 - f_t) x_t with f_t = 1 / (1 + exp(-gate_t)) along axis 2 of arrays (batch, channels, steps, inner); inner
        = 1 are series with the steps last in memory, channels = 1 rows of features one step after the other.  "lengths" gives each
        example a number of valid steps: behind it h is 0 and the state stays.  "reverse" runs from the last valid step to the
        first.  kind "train" is the forward call and its vector-Jacobian product.
step    one step with the state updated in place: a live frame.
orthogonalise
        X_0 = X / (|X| + 1e-7) (Frobenius norm), five times X <- a X + (b A + c A A) X with A = X X^T over the shorter side.
muon    momentum <- 0.95 momentum + grad, X = grad + 0.95 momentum, weight <- (1 - lr wd) weight - lr s orthogonalise(X),
        s = 0.2 sqrt(max(rows, columns)), for a list of matrices of one shape (K. Jordan et al., "Muon: an optimizer for hidden layers
        in neural networks", 2024; the scale is that of J. Liu et al., "Muon is scalable for LLM training", 2025).
"""
import math

import torch

own = False

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}
A, B, C = 3.4445, -4.7750, 2.0315            # the published coefficients
TURNS, EPS = 5, 1e-7
LR, WD, MOMENTUM = 0.02, 0.01, 0.95
MOST_SCAN, MOST_FLOPS = 4 * 160 * 81920, 5 * (3 * 1024 * 1024 * 9216 + 1024 ** 3)


def _scan_case(name, kind, dtype, batch, channels, steps, inner, ragged=False, reverse=False, state=False, joint=False):
    return {"name": name, "op": "scan", "kind": kind, "dtype": dtype, "batch": batch, "channels": channels, "steps": steps, "inner": inner,
            "ragged": ragged, "reverse": reverse, "state": state, "joint": joint}


def _matrix_case(name, op, dtype, count, rows, columns):
    return {"name": name, "op": op, "dtype": dtype, "count": count, "rows": rows, "columns": columns}


def listed():
    return [
        # 60 features of 20 frames of 192 x 160 along the frames, single precision as the paper's networks
        _scan_case("scan cine maps", "train", "float32", 1, 60, 20, 192 * 160),
        # 4 features of 160 sections of 320 x 256 of a knee volume, from section to section, mixed precision
        _scan_case("scan knee sections", "train", "bfloat16", 1, 4, 160, 320 * 256),
        # patches of a knee volume as one sequence of 51200 tokens of 1024 features: few columns, a long axis
        _scan_case("scan patch tokens", "train", "bfloat16", 1, 1, 51200, 1024, state=True),
        # three cines of odd size and unequal length (at most 21 frames), backwards in time, both inputs halves of one array
        _scan_case("scan ragged cines", "train", "float16", 3, 35, 21, 145 * 187, ragged=True, reverse=True, state=True, joint=True),
        # series of 20 frames for every voxel, the frames last in memory, inference
        _scan_case("scan voxel series", "forward", "bfloat16", 1, 60 * 192 * 160, 20, 1),
        # sixteen long traces of an odd number of samples: nearly no rows
        _scan_case("scan long traces", "train", "float32", 1, 16, 262145, 1),
        # one vector of 160 features for each of 20 frames: a conditioning path, launch latency only
        {"name": "step frame vectors", "op": "step", "dtype": "bfloat16", "batch": 20, "inner": 160},
        # 60 features of one live frame of 192 x 160
        {"name": "step live frame", "op": "step", "dtype": "bfloat16", "batch": 60, "inner": 192 * 160},
        # the convolutions of eight priors of two blocks with 100 features, 3 x 3, as matrices
        _matrix_case("orthogonalise convolutions", "orthogonalise", "float32", 32, 100, 900),
        # wide convolutions of 512 features in mixed precision
        _matrix_case("orthogonalise wide", "orthogonalise", "bfloat16", 4, 512, 4608),
        # the volumetric convolutions of four priors with 60 features, 3 x 3 x 3, updated
        _matrix_case("muon volumetric", "muon", "float32", 16, 60, 1620),
        # one large matrix, taller than wide
        _matrix_case("muon tall", "muon", "float32", 1, 9216, 1024),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))
    op = rng.choice(["scan", "scan", "step", "orthogonalise", "muon"])
    dtype = rng.choice(list(TYPES))
    if op == "step":
        batch = log(1, 256)
        return {"op": op, "dtype": dtype, "batch": batch, "inner": log(1, 4000000 // batch)}
    if op == "scan":
        most = log(2000, MOST_SCAN // 2)
        form = rng.choice(["maps", "tokens", "series"])
        steps = min(log(1, 512) if form == "maps" else log(1, 60000), most)
        batch = log(1, max(1, min(16, most // steps)))
        inner = 1 if form == "series" else log(1, max(1, min(2048 if form == "tokens" else 90000, most // (steps * batch))))
        if inner > 8 and rng.random() < 0.5:
            inner = inner // 8 * 8
        channels = 1 if form == "tokens" else log(1, max(1, most // (steps * batch * inner)))
        case = _scan_case("", rng.choice(["forward", "train"]), dtype, batch, channels, steps, inner, rng.random() < 0.3,
                          rng.random() < 0.4, rng.random() < 0.4, rng.random() < 0.3)
        del case["name"]
        return case
    small = log(1, 640)
    large = log(small, max(small, min(12000, 16 * small + 64)))
    most = MOST_FLOPS // (5 * (3 * small * small * large + small ** 3))
    count = log(1, max(1, min(32, most)))
    rows, columns = (small, large) if rng.random() < 0.7 else (large, small)
    return {"op": op, "dtype": dtype, "count": count, "rows": rows, "columns": columns}


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1 + seed)
    return gen


def prepare(case, seed):
    """Features of unit spread; gates with a mean of their own for each channel (inner > 1 and one channel: each feature), so that some
    forget within a step and some keep for a hundred; gradients whose singular values fall off as those of convolutions do."""
    gen, dtype = _generator(int(seed)), TYPES[case["dtype"]]

    def normal(size, spread=1.0, mean=0.0):
        return torch.randn(size, generator=gen, device="cuda").mul_(spread).add_(mean)

    if case["op"] == "step":
        shape = (case["batch"], case["inner"])
        return {"op": "step", "x": normal(shape).to(dtype), "gate": normal(shape, 1.5, 1.0).to(dtype), "state": normal(shape)}
    if case["op"] == "scan":
        b, c, t, n = (case[k] for k in ("batch", "channels", "steps", "inner"))
        shape = (b, c, t, n)
        bias = normal((1, c, 1, 1) if c > 1 else (1, 1, 1, n), 1.5, 1.5)
        s = {"op": "scan", "kind": case["kind"], "reverse": case["reverse"], "state": None, "lengths": None, "grad_last": None}
        if case["joint"]:
            both = torch.empty((b, 2 * c, t, n), dtype=dtype, device="cuda")
            both[:, :c], both[:, c:] = normal(shape), normal(shape).add_(bias)
            s["x"], s["gate"] = both[:, :c], both[:, c:]
        else:
            s["x"], s["gate"] = normal(shape).to(dtype), normal(shape).add_(bias).to(dtype)
        if case["state"]:
            s["state"] = normal((b, c, n))
        if case["ragged"]:
            s["lengths"] = torch.randint(0, t + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
        if case["kind"] == "train":
            s["grad"] = normal(shape, 0.1).to(dtype)
            if case["state"]:
                s["grad_last"] = normal((b, c, n), 0.1)
        return s
    k, m, n = case["count"], case["rows"], case["columns"]
    low = min(m, n)
    falls = 1.0 / (1.0 + torch.arange(low, device="cuda", dtype=torch.float32))
    grads = (normal((k, m, low)) * falls) @ normal((k, low, n)) * (1e-3 / math.sqrt(low))
    s = {"op": case["op"], "x": grads.to(dtype)}
    if case["op"] == "muon":
        s["weights"] = list(normal((k, m, n), 1.0 / math.sqrt(n)).to(dtype).unbind(0))
        s["momenta"] = list(((normal((k, m, low)) * falls) @ normal((k, low, n)) * (1e-2 / math.sqrt(low))).unbind(0))
        s["grads"] = list(s.pop("x").unbind(0))
        s["scale"] = 0.2 * math.sqrt(max(m, n))
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _recur(f, u):
    """h_t = f_t h_(t-1) + u_t from a state of zero along axis 2, by doubling: after each turn h holds the sum of twice as many steps."""
    n = 1
    while n < f.shape[2]:
        u = torch.cat((u[:, :, :n], u[:, :, n:] + f[:, :, n:] * u[:, :, :-n]), 2)
        f = torch.cat((f[:, :, :n], f[:, :, n:] * f[:, :, :-n]), 2)
        n *= 2
    return u


def _back(v, s):
    return v.flip(2) if s["reverse"] else v


def _plain_scan(s):
    dtype = s["x"].dtype
    x, gate = s["x"].float(), s["gate"].float()
    b, c, t, n = x.shape
    f, rest = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    zero = torch.zeros((b, c, 1, n), device="cuda")
    there = None
    if s["lengths"] is not None:
        there = torch.arange(t, device="cuda").view(1, 1, t, 1) < s["lengths"].view(b, 1, 1, 1)
        keep, take = torch.where(there, f, 1.0), torch.where(there, rest * x, 0.0)
    else:
        keep, take = f, rest * x
    first = zero if s["state"] is None else s["state"].unsqueeze(2)
    keep, take = _back(keep, s), _back(take, s)
    h = _recur(keep, torch.cat((take[:, :, :1] + keep[:, :, :1] * first, take[:, :, 1:]), 2))
    last = h[:, :, -1]
    y = _back(h, s)
    out = [(y if there is None else torch.where(there, y, 0.0)).to(dtype), last]
    if s["kind"] != "train":
        return out
    grad = s["grad"].float()
    if there is not None:
        grad = torch.where(there, grad, 0.0)
    grad = _back(grad, s)
    if s["grad_last"] is not None:
        grad = torch.cat((grad[:, :, :-1], grad[:, :, -1:] + s["grad_last"].unsqueeze(2)), 2)
    # the cotangent of h runs the other way, through the gate of the step behind
    d = _recur(torch.cat((keep[:, :, 1:], zero), 2).flip(2), grad.flip(2)).flip(2)
    before = torch.cat((first, h[:, :, :-1]), 2)
    d_state = d[:, :, 0] * keep[:, :, 0]
    d, before = _back(d, s), _back(before, s)
    dx, dg = d * rest, d * (before - x) * f * rest
    if there is not None:
        dx, dg = torch.where(there, dx, 0.0), torch.where(there, dg, 0.0)
    return out + [dx.to(dtype), dg.to(dtype)] + ([] if s["state"] is None else [d_state])


def _plain_step(s):
    x, f = s["x"].float(), 1.0 / (1.0 + torch.exp(-s["gate"].float()))
    rest = 1.0 / (1.0 + torch.exp(s["gate"].float()))
    s["state"].mul_(f).add_(rest * x)
    return [s["state"].to(s["x"].dtype), s["state"]]


def _orthogonal(x):
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-1, -2) if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(TURNS):
        a = x @ x.transpose(-1, -2)
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.transpose(-1, -2) if tall else x


def _plain_muon(s):
    grads, momenta, weights = (torch.stack(s[k]).float() for k in ("grads", "momenta", "weights"))
    momenta = MOMENTUM * momenta + grads
    weights = (1.0 - LR * WD) * weights - LR * s["scale"] * _orthogonal(grads + MOMENTUM * momenta)
    torch._foreach_copy_(s["momenta"], list(momenta.unbind(0)))
    torch._foreach_copy_(s["weights"], list(weights.to(s["weights"][0].dtype).unbind(0)))
    return s["weights"] + s["momenta"]


def _plain(s):
    if s["op"] == "scan":
        return _plain_scan(s)
    if s["op"] == "step":
        return _plain_step(s)
    if s["op"] == "orthogonalise":
        return [_orthogonal(s["x"].float()).to(s["x"].dtype)]
    return _plain_muon(s)


# ---- the framework's calls -------------------------------------------------------------------------------------------

def _own(s):
    import paper_2207_08393_b200 as g
    if s["op"] == "scan":
        y, last, saved = g.gated_scan_forward(s["x"], s["gate"], s["state"], s["lengths"], dim=2, reverse=s["reverse"],
                                              save=s["kind"] == "train")
        if s["kind"] != "train":
            return [y, last]
        dx, dg, d_state = g.gated_scan_vjp(s["grad"], s["grad_last"], s["x"], s["gate"], saved, s["lengths"], dim=2,
                                           reverse=s["reverse"], state_grad=s["state"] is not None)
        return [y, last, dx, dg] + ([] if d_state is None else [d_state])
    if s["op"] == "step":
        return [g.gated_step(s["x"], s["gate"], s["state"]), s["state"]]
    if s["op"] == "orthogonalise":
        return [g.orthogonalise(s["x"], TURNS, (A, B, C), EPS)]
    g.muon_step(s["weights"], s["grads"], s["momenta"], LR, MOMENTUM, nesterov=True, weight_decay=WD, scale=s["scale"], steps=TURNS,
                coefficients=(A, B, C), eps=EPS)
    return s["weights"] + s["momenta"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- work and definition ---------------------------------------------------------------------------------------------

def work(case):
    """Every input once and every output once; the products of symmetric results by their half."""
    b = BYTES[case["dtype"]]
    if case["op"] == "step":
        n = case["batch"] * case["inner"]
        return {"bytes": n * (3 * b + 8), "flops": 8 * n}
    if case["op"] == "scan":
        rows = case["batch"] * case["channels"] * case["inner"]
        n, train = rows * case["steps"], case["kind"] == "train"
        small = 4 * rows * (1 + case["state"] * (1 + 2 * train))
        return {"bytes": n * b * (6 if train else 3) + small, "flops": n * (22 if train else 8)}
    n, s, t = case["count"] * case["rows"] * case["columns"], min(case["rows"], case["columns"]), max(case["rows"], case["columns"])
    flops = case["count"] * TURNS * (s * s * t + s ** 3 + 2 * s * s * t)
    return {"bytes": n * (2 * b if case["op"] == "orthogonalise" else 3 * b + 8), "flops": flops}


def _exact_recur(f, u, state):
    """The recurrence in 64 bits, one step after the other in blocks of about sqrt(steps) side by side, joined by the blocks' last
    values and the products of their factors."""
    b, c, t, n = f.shape
    size = max(1, math.isqrt(t))
    blocks = -(-t // size)
    over = blocks * size - t

    def cut(v, fill):
        tail = torch.full((b, c, over, n), fill, dtype=torch.float64, device="cuda")
        return torch.cat((v, tail), 2).view(b, c, blocks, size, n)

    f, u = cut(f, 1.0), cut(u, 0.0)
    h, prod = torch.empty_like(u), torch.empty_like(f)
    now, p = torch.zeros_like(u[:, :, :, 0]), torch.ones_like(f[:, :, :, 0])
    for k in range(size):
        now, p = torch.addcmul(u[:, :, :, k], f[:, :, :, k], now), p * f[:, :, :, k]
        h[:, :, :, k], prod[:, :, :, k] = now, p
    for k in range(blocks):
        h[:, :, k].addcmul_(prod[:, :, k], state.unsqueeze(2))
        state = h[:, :, k, -1].clone()
    return h.view(b, c, blocks * size, n)[:, :, :t]


def _exact_scan(case, s):
    x, g = s["x"].double(), s["gate"].double()
    b, c, t, n = x.shape
    state = torch.zeros((b, c, n), dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    f = torch.sigmoid(g)
    rest = torch.sigmoid(-g)
    valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(t, device="cuda")[None, :] < s["lengths"][:, None]).double()[:, None, :, None]
    hold = f if valid is None else f * valid + (1 - valid)
    feed = rest * x if valid is None else rest * x * valid
    order = (lambda v: torch.flip(v, (2,))) if case["reverse"] else (lambda v: v)
    h = _exact_recur(order(hold), order(feed), state)
    y = order(h)
    out = [y if valid is None else y * valid, h[:, :, -1]]
    if case["kind"] != "train":
        return out
    dy = s["grad"].double()
    dy = order(dy if valid is None else dy * valid)
    end = torch.zeros((b, c, n), dtype=torch.float64, device="cuda") if s["grad_last"] is None else s["grad_last"].double()
    fo = order(hold)
    through = torch.ones_like(fo)
    through[:, :, :-1] = fo[:, :, 1:]
    back = _exact_recur(torch.flip(through, (2,)), torch.flip(dy, (2,)), end)
    d = order(torch.flip(back, (2,)))
    past = order(torch.cat((state.unsqueeze(2), h[:, :, :-1]), 2))
    dx = d * rest
    dg = dx * f * (past - x)
    if valid is not None:
        dx, dg = dx * valid, dg * valid
    return out + [dx, dg] + ([] if s["state"] is None else [back[:, :, -1] * fo[:, :, 0]])


def _exact_orthogonal(x):
    """From the eigenvalues of the Gram matrix: every turn multiplies a singular value v by a + b v^2 + c v^4."""
    x = x.double()
    if x.shape[-2] > x.shape[-1]:
        return _exact_orthogonal(x.transpose(-1, -2)).transpose(-1, -2)
    x = x / (torch.linalg.matrix_norm(x)[..., None, None] + EPS)
    squares, vectors = torch.linalg.eigh(x @ x.mT)
    total = torch.ones_like(squares)
    for _ in range(TURNS):
        factor = A + squares * (B + C * squares)
        total, squares = total * factor, squares * factor * factor
    return (vectors * total[..., None, :]) @ (vectors.mT @ x)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "scan":
        return _exact_scan(case, s)
    if case["op"] == "step":
        state = torch.lerp(s["x"].double(), s["state"].double(), torch.sigmoid(s["gate"].double()))
        return [state, state]
    if case["op"] == "orthogonalise":
        return [_exact_orthogonal(s["x"])]
    momenta = [MOMENTUM * m.double() + g.double() for m, g in zip(s["momenta"], s["grads"])]
    moves = _exact_orthogonal(torch.stack([g.double() + MOMENTUM * m for m, g in zip(momenta, s["grads"])]))
    return [(1 - LR * WD) * w.double() - LR * s["scale"] * o for w, o in zip(s["weights"], moves)] + momenta
