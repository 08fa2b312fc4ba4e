"""Layer norm, dropout and the residual tail on the GPU against the 64-bit definitions.

Tolerances.  u = 2^-24 is the largest relative error of a 32-bit operation and half the step of the stored type (f32 2^-24,
f16 2^-11, bf16 2^-8) that of the last rounding.  A sum of n terms that is formed as chains of at most m terms and a tree is off by
at most (m + tree) u times the sum of the magnitudes; no kernel has chains longer than chain(n) with the tree counted in.  What
follows from a mean is off by its error divided by the standard deviation, hence the factors rstd max|x|.
"""
import numpy as np
import pytest

from oracle import prior_oracle as po

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 0.0, "float16": 2.0 ** -25, "bfloat16": 0.0}         # half of the smallest step
EPS = 1e-5


def chain(n):
    return 96 + n / 32


def dt(name):
    return getattr(torch, name)


def as64(t):
    return t.detach().double().cpu().numpy()


def make(shape, dtype, seed, mean=0.3, spread=1.0):
    """Values of the type, as a CUDA tensor and in 64 bits."""
    rng = np.random.default_rng(seed)
    t = torch.from_numpy((rng.normal(size=shape) * spread + mean).astype(np.float32)).to("cuda").to(dt(dtype))
    return t, as64(t)


def near(got, ref, tol, what):
    got = as64(got)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g against %.3g" % (
        what, bad.sum(), bad.size, np.abs(got - ref)[bad].max(), np.broadcast_to(tol, ref.shape)[bad].max())


def norm_tolerances(x, weight, mean, rstd, ref_y, dtype):
    """(of y, mean, rstd) for the arrays of a forward call, shapes (o, d, i), (d,), (o, i)."""
    k = chain(x.shape[1]) * U
    big = np.abs(x).max(1)
    tm = k * big
    # the deviations: each is off by the mean's error and its own rounding
    th = (tm + 2 * U * big) * rstd
    tr = rstd * (th + k)                            # sum of squares: relative error 2 (th + k), halved by the root
    h = np.abs(x - mean[:, None]) * rstd[:, None]
    ty = np.abs(weight)[None, :, None] * ((th + 4 * U)[:, None] + h * (tr / rstd + 2 * U)[:, None])
    return ty + HALF[dtype] * np.abs(ref_y) + 2 * U * np.abs(ref_y) + TINY[dtype], tm, tr


def vjp_tolerances(dy, x, weight, mean, rstd, dtype, wtype):
    """(of grad_x before its rounding, grad_weight, grad_bias); mean and rstd are the given 32-bit ones."""
    k = chain(x.shape[1]) * U
    h = np.abs(x - mean[:, None]) * rstd[:, None]
    eh = 4 * U * (h + (np.abs(x).max(1) * rstd)[:, None])
    gm = np.abs(dy * weight[None, :, None])
    c1, c2 = gm.mean(1), (gm * h).mean(1)
    t1, t2 = (k + 2 * U) * c1, (k + 2 * U) * c2 + (gm * eh).mean(1)
    td = rstd[:, None] * (4 * U * gm + t1[:, None] + t2[:, None] * h + c2[:, None] * eh + 6 * U * (c1[:, None] + h * c2[:, None]))
    n = x.shape[0] * x.shape[2]
    kp = chain(n) * U
    tw = kp * np.abs(dy * h).sum((0, 2)) + (np.abs(dy) * eh).sum((0, 2))
    tb = kp * np.abs(dy).sum((0, 2))
    return td, tw, tb


ROWS = [(1, 1, 1), (5, 1, 1), (3, 2, 1), (33, 3, 1), (20, 7, 1), (9, 8, 1), (150, 31, 1), (64, 32, 1), (7, 33, 1), (40, 64, 1),
        (13, 100, 1), (300, 127, 1), (11, 128, 1), (20, 160, 1), (17, 255, 1), (8, 257, 1), (31, 367, 1), (10, 513, 1), (6, 1000, 1),
        (9, 1001, 1), (1, 1024, 1), (700, 1024, 1), (5, 2049, 1), (41, 4099, 1), (3, 8190, 1), (3, 8191, 1), (4, 8192, 1),
        (2, 8193, 1), (2, 20011, 1), (5000, 24, 1), (2500, 96, 1)]
MAPS = [(1, 1, 2), (2, 5, 3), (1, 3, 31), (3, 16, 64), (1, 60, 33), (2, 100, 132), (2, 70, 391), (1, 100, 4096), (4, 50, 1000), (1, 128, 257),
        (2, 129, 72), (1, 257, 40), (1, 300, 515), (1, 513, 64), (2, 640, 96), (1, 700, 1023), (5, 8, 1023), (1, 1025, 36), (40, 6, 5),
        (1, 2000, 33), (3, 2, 10007)]
TYPES = [("float32", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32")]
TAILS = [(s, p) for s in ROWS[:-2] + MAPS[:-1] for p in (0.1, 0.5)] + [(s, p) for s in ROWS[::4] + MAPS[::3] for p in (0.0, 1.0)]


def weights(d, wtype, seed):
    w, w64 = make((d,), wtype, seed + 1, 1.0, 0.2)
    b, b64 = make((d,), wtype, seed + 2, 0.0, 0.2)
    return w, w64, b, b64


def check_norm_vjp(got, dy, v, w64, mean, rstd, dtype, wtype, extra=None, what=""):
    """grad_x (or the tail's grad_residual, with ``extra`` the cotangent added to it) and the weights' gradients."""
    gx, gw, gb = got
    ref = po.layer_norm_vjp(dy, v, w64, mean, rstd)
    td, tw, tb = vjp_tolerances(dy, v, w64, mean, rstd, dtype, wtype)
    rx = ref[0] if extra is None else ref[0] + extra
    if extra is not None:
        td = td + U * (np.abs(extra) + np.abs(rx))
    near(gx, rx, td + HALF[dtype] * np.abs(rx) * 1.01 + TINY[dtype], what + " grad_x")
    near(gw, ref[1], tw + HALF[wtype] * np.abs(ref[1]) * 1.01 + TINY[wtype], what + " grad_weight")
    near(gb, ref[2], tb + HALF[wtype] * np.abs(ref[2]) * 1.01 + TINY[wtype], what + " grad_bias")
    return rx, td


@pytest.mark.parametrize("dtype,wtype", TYPES)
@pytest.mark.parametrize("shape", ROWS + MAPS)
def test_layer_norm(shape, dtype, wtype):
    import paper_2207_08393_b200 as g
    seed = sum(shape) * 7 + len(dtype)
    x, x64 = make(shape, dtype, seed)
    dy, dy64 = make(shape, dtype, seed + 3, 0.1, 0.5)
    w, w64, b, b64 = weights(shape[1], wtype, seed)
    y, mean, rstd = g.layer_norm_forward(x, w, b, EPS, dim=1)
    ry, rm, rr = po.layer_norm(x64, w64, b64, EPS)
    ty, tm, tr = norm_tolerances(x64, w64, rm, rr, ry, dtype)
    near(mean, rm, tm, "mean")
    near(rstd, rr, tr, "rstd")
    near(y, ry, ty + U * np.abs(b64)[None, :, None], "y")
    got = g.layer_norm_vjp(dy, x, w, mean, rstd, dim=1)
    check_norm_vjp(got, dy64, x64, w64, as64(mean), as64(rstd), dtype, wtype)


@pytest.mark.parametrize("dtype,wtype", TYPES)
@pytest.mark.parametrize("shape,p", TAILS)
def test_tail(shape, p, dtype, wtype):
    """The sum bit for bit where its arithmetic has one rounding, the norm of the stored sum, and the VJP."""
    import paper_2207_08393_b200 as g
    seed, offset = 5 + sum(shape) * 11 + len(dtype), 2 ** 32 - 3
    x, x64 = make(shape, dtype, seed)
    res, res64 = make(shape, dtype, seed + 9, -0.2)
    dy, dy64 = make(shape, dtype, seed + 3, 0.1, 0.5)
    ds, ds64 = make(shape, dtype, seed + 4, 0.0, 0.5)
    w, w64, b, b64 = weights(shape[1], wtype, seed)
    y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, res, w, b, p, seed, offset, EPS, dim=1)
    dropped = po.dropout(x64, p, seed, offset)
    # residual + x scale in 64 bits is exact or within 2^-53 of it, so its 32-bit rounding is that of a fused multiply-add
    expect = torch.from_numpy((res64 + dropped).astype(np.float32)).to(dt(dtype))
    assert torch.equal(total.cpu(), expect)
    t64 = as64(total)
    ry, rm, rr = po.layer_norm(t64, w64, b64, EPS)
    ty, tm, tr = norm_tolerances(t64, w64, rm, rr, ry, dtype)
    near(mean, rm, tm, "mean")
    near(rstd, rr, tr, "rstd")
    near(y, ry, ty + U * np.abs(b64)[None, :, None], "y")
    for given in (True, False):
        gx, gr, gw, gb = g.dropout_add_layer_norm_vjp(dy, ds if given else None, total, w, mean, rstd, p, seed, offset, dim=1)
        rx, td = check_norm_vjp((gr, gw, gb), dy64, t64, w64, as64(mean), as64(rstd), dtype, wtype,
                                ds64 if given else np.zeros_like(ds64))
        keep = po.kept(shape, p, seed, offset) * po.scale(p)
        near(gx, rx * keep, (td + 2 * U * np.abs(rx)) * keep + HALF[dtype] * np.abs(rx * keep) * 1.01 + TINY[dtype], "grad_x")


@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 0.05, 0.3, 0.999, 1.0])
@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("n", [1, 3, 4, 5, 8, 63, 1000, 4097, 100003])
def test_dropout(n, dtype, p):
    import paper_2207_08393_b200 as g
    seed, offset = (n << 33) + 12345, 2 ** 64 - 2 if n % 2 else n
    x, x64 = make((n,), dtype, n)
    res, res64 = make((n,), dtype, n + 1)
    # both have one rounding to 32 bits and one to the type
    ref = po.dropout(x64, p, seed, offset)
    assert torch.equal(g.dropout_forward(x, p, seed, offset).cpu(), torch.from_numpy(ref.astype(np.float32)).to(dt(dtype)))
    assert torch.equal(g.dropout_vjp(x, p, seed, offset).cpu(), torch.from_numpy(ref.astype(np.float32)).to(dt(dtype)))
    got = g.dropout_forward(x, p, seed, offset, residual=res)
    assert torch.equal(got.cpu(), torch.from_numpy((res64 + ref).astype(np.float32)).to(dt(dtype)))
    step = torch.tensor([2 ** 35 + 7], device="cuda")
    ref = po.dropout(x64, p, seed, offset, 2 ** 35 + 7)
    assert torch.equal(g.dropout_forward(x, p, seed, offset, step=step).cpu(), torch.from_numpy(ref.astype(np.float32)).to(dt(dtype)))


def test_share_of_dropped_elements():
    """2^22 independent words: the share is within six standard deviations of p, and neighbouring ranges and steps differ."""
    import paper_2207_08393_b200 as g
    n = 1 << 22
    x = torch.ones(n, device="cuda")
    for p in (0.02, 0.5, 0.9):
        gone = float((g.dropout_forward(x, p, 7, 0) == 0).double().mean())
        assert abs(gone - p) < 6 * (p * (1 - p) / n) ** 0.5
    a, b = g.dropout_forward(x, 0.5, 7, 0) == 0, g.dropout_forward(x, 0.5, 7, n // 4) == 0
    assert abs(float((a == b).double().mean()) - 0.5) < 6 * 0.5 / n ** 0.5
    c = g.dropout_forward(x, 0.5, 7, 0, step=torch.ones(1, dtype=torch.int64, device="cuda")) == 0
    assert abs(float((a == c).double().mean()) - 0.5) < 6 * 0.5 / n ** 0.5


@pytest.mark.parametrize("shape", [(6, 33, 1), (3, 1000, 1), (2, 20, 36), (2, 300, 33), (2, 9000, 1)])
def test_dropped_elements_may_hold_anything(shape):
    """Infinities and NaN where the mask drops: selected away, forward and backward."""
    import paper_2207_08393_b200 as g
    p, seed, offset = 0.4, 21, 4
    keep = torch.from_numpy(po.kept(shape, p, seed, offset)).cuda()
    x = make(shape, "float32", 1)[0]
    res = make(shape, "float32", 2)[0]
    bad = torch.where(keep, x, torch.tensor(float("nan"), device="cuda"))
    bad.view(-1)[::2] = torch.where(keep.view(-1)[::2], x.view(-1)[::2], torch.tensor(float("-inf"), device="cuda"))
    assert torch.equal(g.dropout_forward(bad, p, seed, offset), g.dropout_forward(x, p, seed, offset))
    assert torch.equal(g.dropout_forward(bad, p, seed, offset, residual=res), g.dropout_forward(x, p, seed, offset, residual=res))
    for a, b in zip(g.dropout_add_layer_norm_forward(bad, res, None, None, p, seed, offset, dim=1),
                    g.dropout_add_layer_norm_forward(x, res, None, None, p, seed, offset, dim=1)):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("shape", [(7, 65, 1), (5, 520, 1), (2, 24, 40), (1, 40, 33), (3, 8193, 1)])
def test_a_bad_value_stays_in_its_position(shape):
    """NaN and infinities spoil the statistics of their own position and nothing else."""
    import paper_2207_08393_b200 as g
    x = make(shape, "float32", 3)[0]
    y, mean, rstd = g.layer_norm_forward(x, dim=1)
    worse = x.clone()
    worse[-1, 2, -1], worse[0, 1, 0] = float("nan"), float("inf")
    y2, mean2, rstd2 = g.layer_norm_forward(worse, dim=1)
    hit = torch.zeros(shape, dtype=torch.bool, device="cuda")
    hit[-1, :, -1] = hit[0, :, 0] = True
    assert torch.equal(torch.where(hit, 0, y), torch.where(hit, 0, y2)) and bool(torch.isnan(y2[hit]).all())
    assert bool(torch.isnan(rstd2[-1, -1])) and bool(torch.isnan(rstd2[0, 0]))


@pytest.mark.parametrize("shape", [(9, 48, 1), (5, 4099, 1), (2, 31, 40), (1, 64, 37), (2, 9001, 1)])
@pytest.mark.parametrize("dtype", list(HALF))
def test_constant_features_and_far_means(shape, dtype):
    """Equal features have variance zero: y is the bias and the gradient finite.  A mean far from zero costs no digits of the
    variance: the features are whole numbers around 2048 (exact in every type up to bf16's 8 bits: multiples of 16)."""
    import paper_2207_08393_b200 as g
    w, w64, b, b64 = weights(shape[1], "float32", 1)
    x = torch.full(shape, 1.5, dtype=dt(dtype), device="cuda")
    y, mean, rstd = g.layer_norm_forward(x, w, b, EPS, dim=1)
    assert torch.equal(mean, torch.full_like(mean, 1.5))
    near(rstd, np.full(rstd.shape, EPS ** -0.5), EPS ** -0.5 * 4 * U, "rstd")      # eps itself is rounded
    near(y, np.broadcast_to(b64[None, :, None], shape), HALF[dtype] * np.abs(b64)[None, :, None] + TINY[dtype], "y")
    gx, gw, gb = g.layer_norm_vjp(y, x, w, mean, rstd, dim=1)
    assert bool(torch.isfinite(gx).all()) and torch.equal(gw, torch.zeros_like(gw))
    rng = np.random.default_rng(2)
    x64 = 2048.0 + 16.0 * rng.integers(-3, 4, size=shape)
    x = torch.from_numpy(x64).cuda().to(dt(dtype))
    assert np.array_equal(as64(x), x64)
    y, mean, rstd = g.layer_norm_forward(x, w, b, EPS, dim=1)
    ry, rm, rr = po.layer_norm(x64, w64, b64, EPS)
    ty, tm, tr = norm_tolerances(x64, w64, rm, rr, ry, dtype)
    near(y, ry, ty, "y")
    near(rstd, rr, tr, "rstd")


@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("shape,wide,dim", [
    ((5, 24, 1), (5, 40, 1), 1), ((4, 24, 12), (4, 56, 12), 1), ((3, 24, 13), (3, 31, 13), 1), ((6, 33, 1), (6, 50, 1), 1), ((3, 300, 64), (3, 320, 64), 1),
    ((6, 1000, 1), (6, 1024, 1), 1), ((3, 9000, 1), (3, 9008, 1), 1)])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_slices_of_wider_arrays(shape, wide, dim, dtype, shift):
    """Inputs with a pitch and any alignment give what contiguous ones give; outputs written between canaries."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding, prior_ops
    o, d, i = shape
    p, seed, offset = 0.3, 77, 5

    def widened(t):
        big = torch.full((wide[0] * wide[1] * wide[2] + 16,), -7.0, dtype=t.dtype, device="cuda")
        s = big[shift:shift + wide[0] * wide[1] * wide[2]].view(wide)[:, :d]
        s.copy_(t)
        return big, s

    x, res, dy, ds = (make(shape, dtype, k)[0] for k in range(4))
    (xb, xs), (rb, rs), (yb, ys), (sb, ss) = (widened(t) for t in (x, res, dy, ds))
    w, _, b, _ = weights(d, "float32", 4)
    sliced = g.layer_norm_forward(xs, w, b, dim=1)
    x64 = as64(x)
    ry, rm, rr = po.layer_norm(x64, as64(w), as64(b), EPS)
    ty, tm, tr = norm_tolerances(x64, as64(w), rm, rr, ry, dtype)
    near(sliced[0], ry, ty + U, "y")
    near(sliced[1], rm, tm, "mean")
    near(sliced[2], rr, tr, "rstd")
    got = g.layer_norm_vjp(ys, xs, w, sliced[1], sliced[2], dim=1)
    check_norm_vjp(got, as64(dy), x64, as64(w), as64(sliced[1]), as64(sliced[2]), dtype, "float32")
    assert torch.equal(g.dropout_forward(xs, p, seed, offset, residual=rs), g.dropout_forward(x, p, seed, offset, residual=res))
    a, c = g.dropout_add_layer_norm_forward(x, res, w, b, p, seed, offset, dim=1), g.dropout_add_layer_norm_forward(xs, rs, w, b, p, seed, offset, dim=1)
    assert torch.equal(a[1], c[1])
    # outputs with a pitch: what lies between the slices stays as it was
    ob, os_ = widened(torch.zeros_like(x))
    tb, ts = widened(torch.zeros_like(x))
    pitch = [wide[1] * wide[2]] * 4
    mean, rstd = torch.empty_like(sliced[1]), torch.empty_like(sliced[2])
    dims = binding.make_feature_dims(prior_ops._DTYPES[x.dtype], 0, o, d, i, EPS, pitch, torch.cuda.current_stream())
    g.gleam_dropout_add_layer_norm_forward(xs, rs, w, b, ts, os_, mean, rstd, g.make_dropout_args(p, seed, offset), dims)
    assert torch.equal(ts, c[1])
    t64 = as64(ts)
    ry, rm, rr = po.layer_norm(t64, as64(w), as64(b), EPS)
    near(os_, ry, norm_tolerances(t64, as64(w), rm, rr, ry, dtype)[0] + U, "y")
    gxb, gxs = widened(torch.zeros_like(x))
    grb, grs = widened(torch.zeros_like(x))
    gw, gb = torch.empty_like(w), torch.empty_like(w)
    dims = binding.make_feature_dims(prior_ops._DTYPES[x.dtype], 0, o, d, i, EPS, pitch + pitch[:1], torch.cuda.current_stream())
    ws = torch.empty(g.gleam_layer_norm_workspace_size(dims) + 256, dtype=torch.uint8, device="cuda")
    dims.workspace, dims.workspace_bytes = ws.data_ptr(), ws.numel()
    g.gleam_dropout_add_layer_norm_vjp(ys, ss, ts, w, mean, rstd, gxs, grs, gw, gb, g.make_dropout_args(p, seed, offset), dims)
    check_norm_vjp((grs, gw, gb), as64(dy), t64, as64(w), as64(mean), as64(rstd), dtype, "float32", as64(ds))
    for big, s in ((ob, os_), (tb, ts), (gxb, gxs), (grb, grs)):
        s.fill_(-7.0)
        assert bool((big == -7.0).all())
    db, dsl = widened(torch.zeros_like(x))
    dims = binding.make_feature_dims(prior_ops._DTYPES[x.dtype], 0, o, d, i, EPS, pitch, torch.cuda.current_stream())
    g.gleam_dropout_forward(xs, rs, dsl, g.make_dropout_args(p, seed, offset), dims)
    assert torch.equal(dsl, a[1])
    dsl.fill_(-7.0)
    assert bool((db == -7.0).all())


@pytest.mark.parametrize("shape", [(2, 12, 5, 7), (3, 64, 4, 8), (1, 5, 1, 9)])
def test_features_last_in_memory(shape):
    """channels_last maps are rows of features; the results agree with those of the other order."""
    import paper_2207_08393_b200 as g
    x = make(shape, "float32", 1)[0]
    last = x.to(memory_format=torch.channels_last)
    w, _, b, _ = weights(shape[1], "float32", 4)
    dy = make(shape, "float32", 6)[0]
    a, c = g.layer_norm_forward(x, w, b, dim=1), g.layer_norm_forward(last, w, b, dim=1)
    assert c[0].stride() == last.stride() and a[0].stride() == x.stride()
    for s, t in zip(a, c):
        near(s, as64(t), 1e-5, "order")
    va = g.layer_norm_vjp(dy, x, w, a[1], a[2], dim=1)
    vc = g.layer_norm_vjp(dy.to(memory_format=torch.channels_last), last, w, c[1], c[2], dim=1)
    for s, t in zip(va, vc):
        near(s, as64(t), 1e-4, "order")
    if shape[2] > 1:
        with pytest.raises(ValueError, match="another order"):
            g.layer_norm_vjp(dy, last, w, c[1], c[2], dim=1)
    d = g.dropout_forward(last, 0.5, 3, 0)
    assert d.stride() == last.stride()
    assert torch.equal(d.permute(0, 2, 3, 1).contiguous(), g.dropout_forward(last.permute(0, 2, 3, 1).contiguous(), 0.5, 3, 0))


@pytest.mark.parametrize("shape", [(6, 40, 1), (3, 517, 1), (2, 24, 48), (1, 33, 35), (2, 9000, 1), (1, 700, 64)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_outputs_in_place_of_inputs(shape, dtype):
    """An output that is exactly an input gives the bits of a call with memory of its own."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding, prior_ops
    x, res, dy, ds = (make(shape, dtype, k)[0] for k in range(4))
    w, _, b, _ = weights(shape[1], "float32", 4)
    m = g.make_dropout_args(0.3, 9, 2)
    o, d, i = shape
    dims = lambda: binding.make_feature_dims(prior_ops._DTYPES[x.dtype], 0, o, d, i, EPS, stream=torch.cuda.current_stream())
    y, mean, rstd = g.layer_norm_forward(x, w, b, dim=1)
    t = x.clone()
    g.gleam_layer_norm_forward(t, w, b, t, None, None, dims())
    assert torch.equal(t, y)
    gx, gw, gb = g.layer_norm_vjp(dy, x, w, mean, rstd, dim=1)
    for which in (0, 1):
        pair = [dy.clone(), x.clone()]
        gw2, gb2, dd = torch.empty_like(gw), torch.empty_like(gb), dims()
        ws = torch.empty(g.gleam_layer_norm_workspace_size(dd), dtype=torch.uint8, device="cuda")
        dd.workspace, dd.workspace_bytes = ws.data_ptr(), ws.numel()
        g.gleam_layer_norm_vjp(pair[0], pair[1], w, mean, rstd, pair[which], gw2, gb2, dd)
        assert torch.equal(pair[which], gx) and torch.equal(gw2, gw) and torch.equal(gb2, gb)
    out = g.dropout_forward(x, 0.3, 9, 2, residual=res)
    t = res.clone()
    g.gleam_dropout_forward(x, t, t, m, dims())
    assert torch.equal(t, out)
    y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, res, w, b, 0.3, 9, 2, dim=1)
    tx, tr = x.clone(), res.clone()
    g.gleam_dropout_add_layer_norm_forward(tx, tr, w, b, tr, tx, None, None, m, dims())      # the residual stream updated in place
    assert torch.equal(tr, total) and torch.equal(tx, y)
    gx, gr, gw, gb = g.dropout_add_layer_norm_vjp(dy, ds, total, w, mean, rstd, 0.3, 9, 2, dim=1)
    ty, ts = dy.clone(), ds.clone()
    g.gleam_dropout_add_layer_norm_vjp(ty, ts, total, w, mean, rstd, ty, ts, None, None, m, dims())
    assert torch.equal(ty, gx) and torch.equal(ts, gr)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("features,inner", [(16, 1), (32, 1), (64, 1), (100, 1), (128, 1), (512, 1), (1000, 1), (1024, 1), (4096, 1), (24, 20), (60, 33), (100, 512)])
@pytest.mark.parametrize("outer", [1, 3, 5, 37])
def test_what_lies_behind_the_last_slice_stays(outer, features, inner, dtype):
    """Every output in a buffer of its own that goes on behind the last slice: the canary there stays, whatever part of a warp
    or block the last rows fill."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding, prior_ops
    shape, n, room = (outer, features, inner), outer * features * inner, 8192
    x, res, dy, ds = (make(shape, dtype, k)[0] for k in range(4))
    w, _, b, _ = weights(features, "float32", 4)
    bufs = [torch.full((n + room,), -7.0, dtype=x.dtype, device="cuda") for _ in range(5)]
    total, y, gx, gr, drop = (t[:n].view(shape) for t in bufs)
    stats = [torch.full((outer * inner + room,), -7.0, device="cuda") for _ in range(2)]
    mean, rstd = (t[:outer * inner].view(outer, inner) for t in stats)
    grads = [torch.full((features + room,), -7.0, device="cuda") for _ in range(2)]
    m = g.make_dropout_args(0.3, 5, 1)
    dims = lambda: binding.make_feature_dims(prior_ops._DTYPES[x.dtype], 0, outer, features, inner, EPS, stream=torch.cuda.current_stream())
    g.gleam_dropout_add_layer_norm_forward(x, res, w, b, total, y, mean, rstd, m, dims())
    dd = dims()
    size = g.gleam_layer_norm_workspace_size(dd)
    ws = torch.full((size + room,), 77, dtype=torch.uint8, device="cuda")
    dd.workspace, dd.workspace_bytes = ws.data_ptr(), size
    g.gleam_dropout_add_layer_norm_vjp(dy, ds, total, w, mean, rstd, gx, gr, grads[0], grads[1], m, dd)
    g.gleam_dropout_forward(x, res, drop, m, dims())
    ref = g.dropout_add_layer_norm_forward(x, res, w, b, 0.3, 5, 1, EPS, dim=1)
    back = g.dropout_add_layer_norm_vjp(dy, ds, ref[1], w, ref[2], ref[3], 0.3, 5, 1, dim=1)
    for t, c in ((total, ref[1]), (y, ref[0]), (mean, ref[2]), (rstd, ref[3]), (gx, back[0]), (gr, back[1]),
                 (grads[0][:features], back[2]), (grads[1][:features], back[3]), (drop, ref[1])):
        assert torch.equal(t, c)
    for t, k in [(t, n) for t in bufs] + [(t, outer * inner) for t in stats] + [(t, features) for t in grads]:
        assert bool((t[k:] == -7.0).all())
    assert bool((ws[size:] == 77).all())


def test_overlaps_are_refused():
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding
    buf = torch.zeros(4096, device="cuda")
    at = lambda k: buf[k:]
    d = binding.make_feature_dims(0, 0, 4, 32, 1, EPS)
    m = g.make_dropout_args(0.5)

    def refused(call, *args):
        with pytest.raises(g.GleamError) as e:
            call(*args)
        assert e.value.status == binding.GLEAM_ERR_ALIAS

    refused(g.gleam_layer_norm_forward, at(0), None, None, at(64), None, None, d)            # y inside x
    refused(g.gleam_layer_norm_forward, at(0), at(600), None, at(500), None, None, d)        # y over weight
    refused(g.gleam_layer_norm_forward, at(0), None, None, at(512), at(512), None, d)        # mean inside y
    refused(g.gleam_layer_norm_forward, at(0), None, None, at(512), at(1024), at(1026), d)   # mean and rstd
    refused(g.gleam_dropout_forward, at(0), at(256), at(300), m, d)
    refused(g.gleam_dropout_add_layer_norm_forward, at(0), at(256), None, None, at(512), at(512), None, None, m, d)  # sum and y are one
    pitched = binding.make_feature_dims(0, 0, 4, 32, 1, EPS, [64, 64])
    g.gleam_layer_norm_forward(at(0), None, None, at(32), None, None, pitched)               # halves of rows of 64
    refused(g.gleam_layer_norm_forward, at(0), None, None, at(31), None, None, pitched)
    refused(g.gleam_layer_norm_forward, at(0), None, None, at(33), None, None, pitched)
    host = torch.zeros(256).pin_memory()
    with pytest.raises(g.GleamError) as e:
        g.gleam_layer_norm_forward(host, None, None, at(0), None, None, d)
    assert e.value.status == binding.GLEAM_ERR_NOT_DEVICE_POINTER


def test_torch_layer_refusals():
    import paper_2207_08393_b200 as g
    x = torch.randn(4, 8, 6, device="cuda")
    w = torch.ones(8, device="cuda")
    y, mean, rstd = g.layer_norm_forward(x, w, dim=1)
    for call in (lambda: g.layer_norm_forward(x.double(), dim=1), lambda: g.layer_norm_forward(x, w.half(), dim=1),
                 lambda: g.layer_norm_forward(x, torch.ones(7, device="cuda"), dim=1), lambda: g.layer_norm_forward(x, w, w.cpu(), dim=1),
                 lambda: g.layer_norm_forward(x, dim=3), lambda: g.layer_norm_forward(torch.empty(3, 0, device="cuda")),
                 lambda: g.layer_norm_vjp(y.half(), x, w, mean, rstd, dim=1), lambda: g.layer_norm_vjp(y, x, w, mean[:2], rstd, dim=1),
                 lambda: g.layer_norm_vjp(y, x, w, mean.half(), rstd, dim=1), lambda: g.dropout_forward(x, 1.5, 0, 0),
                 lambda: g.dropout_forward(x, 0.5, 0, 0, residual=x[:2]), lambda: g.dropout_forward(x, 0.5, 0, 0, step=torch.zeros(1, device="cuda")),
                 lambda: g.dropout_forward(x, 0.5, 0, 0, residual=x.transpose(0, 2).contiguous().transpose(0, 2)),
                 lambda: g.dropout_add_layer_norm(x, x, w, w, 0.5)):
        with pytest.raises(ValueError):
            call()
    for eps in (-1.0, float("nan")):
        with pytest.raises(g.GleamError):
            g.layer_norm_forward(x, eps=eps, dim=1)


def test_calls_on_nothing():
    import paper_2207_08393_b200 as g
    for shape in ((0, 8, 6), (4, 8, 0)):
        x = torch.empty(shape, device="cuda")
        w = torch.ones(8, device="cuda")
        y, mean, rstd = g.layer_norm_forward(x, w, w, dim=1)
        assert y.shape == x.shape and mean.numel() == 0
        gx, gw, gb = g.layer_norm_vjp(y, x, w, mean, rstd, dim=1)
        assert not gw.any() and not gb.any()
        assert g.dropout_forward(x, 0.5, 0, 0, residual=x).shape == x.shape
        y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, x, w, w, 0.5, 0, 0, dim=1)
        gx, gr, gw, gb = g.dropout_add_layer_norm_vjp(y, None, total, w, mean, rstd, 0.5, 0, 0, dim=1)
        assert gx.shape == x.shape and not gw.any() and not gb.any()


def test_missing_weights_and_unwanted_outputs():
    import paper_2207_08393_b200 as g
    for shape in ((9, 70, 1), (2, 30, 44), (2, 8200, 1)):
        x, dy = make(shape, "float32", 1)[0], make(shape, "float32", 2)[0]
        one, zero = torch.ones(shape[1], device="cuda"), torch.zeros(shape[1], device="cuda")
        a, c = g.layer_norm_forward(x, dim=1), g.layer_norm_forward(x, one, zero, dim=1)
        assert all(torch.equal(s, t) for s, t in zip(a, c))
        full = g.layer_norm_vjp(dy, x, one, a[1], a[2], dim=1)
        bare = g.layer_norm_vjp(dy, x, None, a[1], a[2], dim=1, weight_grad=False, bias_grad=False)
        only = g.layer_norm_vjp(dy, x, None, a[1], a[2], dim=1, weight_grad=False)
        assert torch.equal(full[0], bare[0]) and bare[1] is None and bare[2] is None
        assert torch.equal(full[0], only[0]) and only[1] is None and torch.equal(only[2], full[2])


@pytest.mark.parametrize("shape", [(3000, 160, 1), (700, 1003, 1), (4, 60, 4096), (3, 70, 1001), (40, 9001, 1)])
def test_repeated_calls_give_the_same_bits(shape):
    import paper_2207_08393_b200 as g
    x, res, dy, ds = (make(shape, "bfloat16", k)[0] for k in range(4))
    w, _, b, _ = weights(shape[1], "float32", 4)

    def once():
        y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, res, w, b, 0.2, 1, 0, dim=1)
        return (y, total, mean, rstd) + g.dropout_add_layer_norm_vjp(dy, ds, total, w, mean, rstd, 0.2, 1, 0, dim=1)
    first = once()
    for _ in range(5):
        assert all(torch.equal(a, c) for a, c in zip(first, once()))


def test_beyond_32_bits():
    """Element numbers and offsets beyond 2^32, at both ends of the array: a bf16 array of 4.3e9 elements in place."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding
    n = (1 << 32) + 4096
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    dims = binding.make_feature_dims(binding.GLEAM_BF16, 0, 1, 1, n, stream=torch.cuda.current_stream())
    g.gleam_dropout_forward(x, None, x, g.make_dropout_args(0.5, 3, 1), dims)
    for start in (0, (1 << 31) - 64, (1 << 32) - 64, n - 4096):
        piece = as64(x[start:start + 128])
        assert np.array_equal(piece != 0, po.words(128, 3, 1 + start // 4) >= 2 ** 31)
    for shape in ((n // 4096, 4096, 1), (1, 64, n // 64)):
        x = x.view(shape)
        x.fill_(1.0)
        x[-1, 1::2] = 3.0                                       # features 1, 3, 1, 3: mean 2, variance 1
        if shape[2] > 1:
            x[:, 1::2] = 3.0
        dims = binding.make_feature_dims(binding.GLEAM_BF16, 0, *shape, eps=0.0 if shape[2] > 1 else 1.0, stream=torch.cuda.current_stream())
        g.gleam_layer_norm_forward(x, None, None, x, None, None, dims)
        h = 1.0 if shape[2] > 1 else 2 ** -0.5
        last = as64(x[-1, :, -1])
        assert np.abs(last[0::2] + h).max() <= 2 ** -8 and np.abs(last[1::2] - h).max() <= 2 ** -8
        first = as64(x[0, :, 0])
        assert np.abs(np.abs(first) - (1.0 if shape[2] > 1 else 0.0)).max() <= 2 ** -8


def test_another_stream_and_two_at_once():
    """Calls on side streams, concurrently, each with scratch of its own, give what the calls one after another give."""
    import paper_2207_08393_b200 as g
    sets = []
    for k, shape in enumerate([(2000, 513, 1), (3, 60, 3001), (2000, 512, 1), (2, 100, 4096)]):
        x, res, dy, ds = (make(shape, "float32", 10 * k + j)[0] for j in range(4))
        w, _, b, _ = weights(shape[1], "float32", k)
        sets.append((x, res, dy, ds, w, b))

    def work(s):
        x, res, dy, ds, w, b = s
        y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, res, w, b, 0.2, 1, 0, dim=1)
        return (y, total) + g.dropout_add_layer_norm_vjp(dy, ds, total, w, mean, rstd, 0.2, 1, 0, dim=1)
    one = [work(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        many = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                many.append(work(s))
        torch.cuda.synchronize()
        for a, c in zip(one, many):
            assert all(torch.equal(u, v) for u, v in zip(a, c))


def test_captured_calls_draw_anew_at_every_replay():
    """A captured forward and backward with the device counter: each replay's mask is that of its step, and a second captured
    graph is independent of the first."""
    import paper_2207_08393_b200 as g
    shape = (64, 96, 1)
    x, res, dy = (make(shape, "float32", k)[0] for k in range(3))
    w, _, b, _ = weights(shape[1], "float32", 4)
    graphs = []
    for k in range(2):
        step = torch.zeros(1, dtype=torch.int64, device="cuda")

        def work():
            y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, res, w, b, 0.5, k, 8, dim=1, step=step)
            grads = g.dropout_add_layer_norm_vjp(dy, None, total, w, mean, rstd, 0.5, k, 8, dim=1, step=step)
            out = total.clone()
            step.add_(1)
            return (out,) + grads
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work()
        torch.cuda.current_stream().wait_stream(side)
        step.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = work()
        graphs.append((graph, outs, k, step))                  # the counter lives as long as the graph that reads it
    for turn in range(3):
        for graph, outs, k, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph, outs, k, _ in graphs:
            keep = torch.from_numpy(po.kept(shape, 0.5, k, 8, turn)).cuda()
            same = torch.equal(outs[0], torch.where(keep, torch.addcmul(res, x, torch.full_like(x, 2.0)), res))
            assert same, (turn, k)
            assert bool((outs[1][~keep] == 0).all()) and bool((outs[1][keep] != 0).any())


def test_autograd_matches_differences():
    """The autograd nodes against central differences of the 64-bit definitions, a run of them as a block uses them:
    norm, dropout with residual, tail; the loss touches both outputs of the tail."""
    import paper_2207_08393_b200 as g
    rng = np.random.default_rng(4)
    shape, p = (2, 6, 5), 0.4
    vals = [rng.normal(size=shape).astype(np.float32), rng.normal(size=shape).astype(np.float32)] + \
           [(1 + 0.2 * rng.normal(size=6)).astype(np.float32) for _ in range(4)]
    cy, cs = rng.normal(size=shape), rng.normal(size=shape)
    offsets = []

    def ours(x, r, w1, b1, w2, b2):
        gen = g.DropoutGenerator(11)
        n = g.layer_norm(x, w1, b1, EPS, dim=1)
        u = g.dropout(n, p, gen, residual=r)
        y, total = g.dropout_add_layer_norm(x, u, w2, b2, p, gen, EPS, dim=1)
        offsets.append(gen.offset)
        return (y * torch.from_numpy(cy).cuda().float()).sum() + (total * torch.from_numpy(cs).cuda().float()).sum()

    def ref(x, r, w1, b1, w2, b2):
        n = po.layer_norm(x, w1, b1, EPS)[0]
        u = r + po.dropout(n, p, 11, 0)
        total = u + po.dropout(x, p, 11, 15)
        return float((po.layer_norm(total, w2, b2, EPS)[0] * cy).sum() + (total * cs).sum())

    leaves = [torch.from_numpy(v).cuda().requires_grad_(True) for v in vals]
    loss = ours(*leaves)
    assert offsets[-1] == 30
    loss.backward()
    v64 = [v.astype(np.float64) for v in vals]
    base = ref(*v64)
    size = np.abs(cy).sum() * 3 + np.abs(cs).sum() * 3
    assert abs(float(loss.detach()) - base) <= 64 * U * size
    for which, leaf in enumerate(leaves):
        grad = as64(leaf.grad)
        biggest = np.abs(grad).max() + 1.0
        for at in np.ndindex(grad.shape):
            up, down = [v.copy() for v in v64], [v.copy() for v in v64]
            up[which][at] += 1e-5
            down[which][at] -= 1e-5
            # differences of 64-bit values: truncation about 1e-10, cancellation about 1e-11 / 1e-5
            assert abs((ref(*up) - ref(*down)) / 2e-5 - grad[at]) <= 512 * U * biggest * 8 + 1e-5, (which, at)


def test_autograd_in_other_orders_and_partial_gradients():
    """Cotangents arrive expanded, transposed or not at all; gradients only where they are asked for."""
    import paper_2207_08393_b200 as g
    x = torch.randn(3, 8, 4, 5, device="cuda").to(memory_format=torch.channels_last).requires_grad_(True)
    w = torch.ones(8, device="cuda", requires_grad=True)
    y = g.layer_norm(x, w, None, EPS, dim=1)
    y.sum().backward()                                   # an expanded cotangent
    assert x.grad.shape == x.shape and float(x.grad.abs().max()) < 1e-5
    gen = g.DropoutGenerator(1)
    xd = x.detach().requires_grad_(True)
    out = g.dropout(xd, 0.5, gen)
    (out * 3.0).sum().backward()
    assert torch.equal(xd.grad, torch.where(out.detach() == 0, 0.0, 6.0))
    frozen = torch.randn(3, 8, 4, 5, device="cuda")
    t = torch.randn(3, 8, 4, 5, device="cuda", requires_grad=True)
    y, total = g.dropout_add_layer_norm(frozen, t, w.detach(), None, 0.5, gen, dim=1)
    total.sum().backward()                               # y is not used
    assert torch.equal(t.grad, torch.ones_like(t))
    t.grad = None
    y, total = g.dropout_add_layer_norm(frozen, t, w.detach(), None, 0.0, dim=1)
    (y.transpose(1, 3) * torch.randn(3, 5, 4, 8, device="cuda")).sum().backward()
    assert bool(torch.isfinite(t.grad).all()) and w.grad is not None
    step = g.DropoutGenerator(1, capturable=True)
    z = g.dropout(t, 0.5, step)
    step.advance()
    with pytest.raises(RuntimeError, match="inplace"):   # the counter moved before the backward pass
        z.sum().backward()


def test_calls_from_several_threads():
    """The calls release the interpreter's lock; threads on streams of their own get the bits of calls in turn."""
    import threading
    import paper_2207_08393_b200 as g
    shapes = [(50, 96, 1), (3, 24, 260), (20, 1003, 1), (2, 33, 129)]
    data = []
    for k, shape in enumerate(shapes):
        torch.manual_seed(k)
        data.append([torch.randn(shape, device="cuda") for _ in range(4)] + [torch.rand(shape[1], device="cuda")])

    def run(k):
        x, r, dy, ds, w = data[k]
        y, total, mean, rstd = g.dropout_add_layer_norm_forward(x, r, w, None, 0.3, 11, 4 * k, dim=1)
        return (y, total) + g.dropout_add_layer_norm_vjp(dy, ds, total, w, mean, rstd, 0.3, 11, 4 * k, dim=1)

    want = [run(k) for k in range(len(shapes))]
    torch.cuda.synchronize()
    got = [None] * len(shapes)

    def work(k):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                got[k] = run(k)
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(shapes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(want, got):
        for u, v in zip(a, b):
            assert torch.equal(u, v)


@pytest.mark.parametrize("p", [0.0, 0.5])
def test_dropout_takes_a_residual_in_any_order(p):
    """As the tail does: a residual (or x) in another memory order gives the values and gradients of x's order."""
    import paper_2207_08393_b200 as g
    x, r, c = (make((2, 6, 4, 5), "float32", k)[0] for k in range(3))
    last = lambda t: t.to(memory_format=torch.channels_last)
    for xo, ro in ((x, last(r)), (last(x), r), (last(x), r.transpose(2, 3).contiguous().transpose(2, 3)), (x, r[:1].expand(2, 6, 4, 5))):
        got, want = [], []
        for res, out in ((ro, got), (torch.empty_like(xo).copy_(ro), want)):
            leaves = [xo.detach().requires_grad_(), res.detach().requires_grad_()]
            y = g.dropout(leaves[0], p, g.DropoutGenerator(5), residual=leaves[1])
            (y * c).sum().backward()
            out += [y.detach()] + [t.grad for t in leaves]
        for a, b in zip(got, want):
            assert a.shape == b.shape and torch.equal(a, b)
        assert got[0].stride() == xo.stride()


@pytest.mark.parametrize("n", [1, 7])
def test_numbers_that_torch_negates_when_it_reads_them(n):
    """The imaginary part of a conjugate is memory with a negative bit: refused by the calls, resolved by the autograd nodes."""
    import paper_2207_08393_b200 as g
    lazy = torch.randn(n, 1, dtype=torch.complex64, device="cuda").conj().imag
    plain = lazy.clone()
    w = torch.randn(1, dtype=torch.complex64, device="cuda").conj().imag
    assert lazy.is_neg() and w.is_neg() and not plain.is_neg()
    y, mean, rstd = g.layer_norm_forward(plain)
    for call in (lambda: g.dropout_forward(lazy, 0.5, 1, 0), lambda: g.dropout_forward(plain, 0.5, 1, 0, residual=lazy),
                 lambda: g.layer_norm_forward(lazy), lambda: g.layer_norm_forward(plain, w), lambda: g.layer_norm_forward(plain, None, w),
                 lambda: g.layer_norm_vjp(lazy, plain, None, mean, rstd), lambda: g.layer_norm_vjp(plain, plain, w, mean, rstd),
                 lambda: g.dropout_add_layer_norm_forward(plain, lazy, None, None, 0.5, 1, 0)):
        with pytest.raises(ValueError, match="resolve_neg"):
            call()
    for f in (lambda x, r: g.dropout(x, 0.5, g.DropoutGenerator(5), residual=r), lambda x, r: g.dropout_add_layer_norm(x, r, None, None, 0.5, g.DropoutGenerator(5))[1]):
        assert torch.equal(f(plain, lazy), f(plain, plain))
    leaf = plain.clone().requires_grad_()
    want = torch.autograd.grad(g.dropout(leaf, 0.5, g.DropoutGenerator(5)), leaf, plain)[0]
    assert torch.equal(torch.autograd.grad(g.dropout(leaf, 0.5, g.DropoutGenerator(5)), leaf, lazy)[0], want)
    y, total = g.dropout_add_layer_norm(leaf, plain, None, None, 0.0)
    assert torch.equal(torch.autograd.grad(total, leaf, lazy)[0], plain)


# Slices that begin anywhere: maps of 128 positions or more whose inner length is odd or whose memory begins between pieces.

@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("shape,wide", [((3, 24, 133), (3, 31, 133)), ((2, 70, 391), (2, 73, 391)), ((2, 300, 129), (2, 301, 129)), ((3, 24, 256), (3, 25, 256))])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_slices_of_wider_arrays_that_begin_anywhere(shape, wide, dtype, shift):
    test_slices_of_wider_arrays(shape, wide, 1, dtype, shift)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("features,inner", [(16, 131), (60, 133), (100, 515), (300, 129), (600, 131)])
@pytest.mark.parametrize("outer", [1, 5])
def test_what_lies_behind_slices_that_begin_anywhere_stays(outer, features, inner, dtype):
    test_what_lies_behind_the_last_slice_stays(outer, features, inner, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(2, 24, 133), (1, 70, 391), (2, 300, 129)])
def test_outputs_in_place_of_slices_that_begin_anywhere(shape, dtype):
    test_outputs_in_place_of_inputs(shape, dtype)


@pytest.mark.parametrize("shape", [(2, 20, 133), (1, 300, 391), (3, 16, 1023)])
def test_bad_values_in_slices_that_begin_anywhere(shape):
    test_dropped_elements_may_hold_anything(shape)
    test_a_bad_value_stays_in_its_position(shape)


# Variances.  The features are whole numbers whose sums are exact in 32 bits in any order, so a mean (of all, or of a part that is
# joined to the others) is off by at most two roundings, 2 U max|x|.  Squares of deviations from a mean that is off by e give var +
# e^2; a join of parts with means m_w gives further 2 (m_w - m) e_w, summed over the parts at most 4 sd e.  A part whose squares
# are taken about its first feature, k numbers d, leaves sum d^2 - (sum d)^2 / k, which is at least 1 / (k + 1) of sum d^2: with 1.5
# roundings of the product and parts of at most 40 features that is 62 U of what is left.  With R = max|x| / sd the variance is
# thus off by at most (8 R + chain + 64) U + (2 R U)^2 of itself.

def variance_tolerance(x, rstd):
    r = np.abs(x).max(1) * rstd
    return (8 * r + chain(x.shape[1]) + 64) * U + (2 * r * U) ** 2


def check_variance(x64, dtype):
    import paper_2207_08393_b200 as g
    x = torch.from_numpy(x64).cuda().to(dt(dtype))
    assert np.array_equal(as64(x), x64) and np.abs(x64).sum(1).max() < 2 ** 24
    y, mean, rstd = g.layer_norm_forward(x, None, None, EPS, dim=1)
    ones = np.ones(x64.shape[1])
    ry, rm, rr = po.layer_norm(x64, ones, 0 * ones, EPS)
    t = variance_tolerance(x64, rr)
    big = np.abs(x64).max(1)
    near(mean, rm, 2 * U * big, "mean")
    near(rstd, rr, t * rr, "rstd")
    h = np.abs(ry)
    near(y, ry, (2 * U * big * rr)[:, None] + h * (t[:, None] + 4 * U) + HALF[dtype] * h * 1.01 + TINY[dtype], "y")
    return rr, t


@pytest.mark.parametrize("dtype,base,step", [("float32", None, 1), ("float16", 2048, 2), ("bfloat16", 255, 1)])
@pytest.mark.parametrize("shape", [(90, 31, 1), (40, 160, 1), (12, 513, 1), (9, 4099, 1), (2, 9001, 1), (2, 31, 40), (1, 60, 391), (1, 200, 64), (1, 300, 72),
                                   (1, 640, 40), (1, 1500, 33)])
def test_a_far_mean_costs_no_digits_of_the_variance(shape, dtype, base, step):
    """Whole numbers around a mean of 100 to 10^5 standard deviations, as far as their sums stay exact.  The mean of the squares
    less the square of the mean, in 32 bits, is beyond the tolerance on the same numbers."""
    d = shape[1]
    base = min(base, 2 ** 23 // d // step * step) if base else 2 ** 23 // d
    x64 = base + step * np.random.default_rng(d).integers(-1, 2, size=shape).astype(np.float64)
    rr, t = check_variance(x64, dtype)
    x32 = x64.astype(np.float32)
    m, s = x32.sum(1, dtype=np.float32) / np.float32(d), (x32 * x32).sum(1, dtype=np.float32) / np.float32(d)
    bad = 1.0 / np.sqrt(np.maximum(s - m * m, 0).astype(np.float64) + EPS)
    assert (np.abs(bad - rr) > t * rr).any()


@pytest.mark.parametrize("dtype", list(HALF))
@pytest.mark.parametrize("part", [8, 16, 32, 40])
@pytest.mark.parametrize("shape", [(5, 31, 1), (3, 1003, 1), (2, 60, 40), (1, 128, 391), (1, 200, 64), (1, 300, 72), (2, 640, 40), (1, 700, 64)])
def test_features_that_stand_out(shape, part, dtype):
    """Every part's first feature thirty standard deviations from the others."""
    x64 = np.random.default_rng(part).integers(-3, 4, size=shape).astype(np.float64)
    x64[:, ::part] += 64
    check_variance(x64, dtype)


def kept_at(start, count, p, seed, offset):
    return po.words(count + 3, seed, offset + start // 4)[start % 4:][:count] >= np.uint64(int(p * 2 ** 32))


@pytest.mark.parametrize("features,inner", [(4096, 1), (4099, 1), (24, 1), (9001, 1), (64, 2 ** 26 + 64), (64, 2 ** 26 + 65), (700, 2 ** 23)])
def test_tails_beyond_32_bits(features, inner):
    """The residual tail and its VJP on more than 2^32 elements in bf16, outputs in place of inputs, against the definition at
    positions whose elements lie at both ends of the array and around the powers of two."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import binding
    outer = 2 ** 32 // features + 3 if inner == 1 else 1
    shape, p, seed, offset = (outer, features, inner), 0.5, 9, 2 ** 33 + 1
    assert outer * features * inner > 2 ** 32
    gen = torch.Generator("cuda").manual_seed(features)
    x, res = (torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    w, w64, b, b64 = weights(features, "float32", 1)
    if inner == 1:
        at = sorted({0, 1, 2 ** 31 // features, 2 ** 32 // features - 1, 2 ** 32 // features, outer - 1})
        pick = lambda t: t[at]
        keep = np.stack([kept_at(r * features, features, p, seed, offset) for r in at])[:, :, None]
        stats = lambda t: as64(t[at])
    else:
        runs = ((0, 64), (2 ** 31 % inner // 2 + 64, 8), (inner // 2, 8), (inner - 64, 64))
        at = torch.cat([torch.arange(k, k + n) for k, n in runs]).cuda()
        pick = lambda t: t[:, :, at]
        keep = np.stack([np.concatenate([kept_at(c * inner + k, n, p, seed, offset) for k, n in runs]) for c in range(features)])[None]
        stats = lambda t: as64(t[:, at])
    x64, r64 = as64(pick(x)), as64(pick(res))
    mean, rstd = (torch.empty((outer, inner), device="cuda") for _ in range(2))
    m = g.make_dropout_args(p, seed, offset)
    dims = binding.make_feature_dims(binding.GLEAM_BF16, 0, *shape, eps=EPS, stream=torch.cuda.current_stream())
    g.gleam_dropout_add_layer_norm_forward(x, res, w, b, res, x, mean, rstd, m, dims)
    want = torch.from_numpy((r64 + x64 * keep * 2.0).astype(np.float32)).to(torch.bfloat16)
    assert torch.equal(pick(res).cpu(), want)
    t64 = as64(want)
    ry, rm, rr = po.layer_norm(t64, w64, b64, EPS)
    ty, tm, tr = norm_tolerances(t64, w64, rm, rr, ry, "bfloat16")
    near(pick(x), ry, ty + U * np.abs(b64)[None, :, None], "y")
    near(torch.from_numpy(stats(mean)), rm, tm, "mean")
    near(torch.from_numpy(stats(rstd)), rr, tr, "rstd")
    x.normal_(generator=gen)                                   # the cotangent of y
    dy64, m64, s64 = as64(pick(x)), stats(mean), stats(rstd)
    g.gleam_dropout_add_layer_norm_vjp(x, None, res, w, mean, rstd, x, res, None, None, m, dims)
    rx = po.layer_norm_vjp(dy64, t64, w64, m64, s64)[0]
    td = vjp_tolerances(dy64, t64, w64, m64, s64, "bfloat16", "float32")[0]
    near(pick(res), rx, td + HALF["bfloat16"] * np.abs(rx) * 1.01, "grad_residual")
    rx = rx * keep * 2.0
    near(pick(x), rx, 2 * td + HALF["bfloat16"] * np.abs(rx) * 1.01, "grad_x")
