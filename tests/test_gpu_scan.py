"""The gated recurrence on the GPU against its definition in 64 bits.

Tolerances.  Gates are at most 4 here, so a state forgets an error within 1 + e^4 < 56 steps on average.  A step rounds once (2^-24 of the
largest value M there is) and its gate is off by at most 16 * 2^-24 of itself (exponential 2^-22 + 4 * 2^-23 of the argument's rounding,
division 2^-22), which moves the state by as much of M.  The sum is 56 * 17 * 2^-24 M < 6e-5 M, and storing rounds by half a step of the
type.  Cotangents go through the same chain; the gate's has one more factor of at most 2 M.
"""
import numpy as np
import pytest

from oracle import scan_oracle as so

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CHAIN = 6e-5
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, dtype, scale, what):
    got = host(got)
    assert got.shape == ref.shape, what
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal
    off = np.abs(got - ref) - (CHAIN * scale + (0 if dtype == torch.float32 else half) * np.abs(ref) + tiny)
    assert np.isfinite(got).all() and (off <= 0).all(), "%s: %g over the tolerance at %s" % (what, off.max(), np.unravel_index(np.argmax(off), off.shape))


def inputs(shape, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda s: torch.randn(s, generator=gen, device="cuda")
    b, c, t, n = shape
    x, gate, dy = normal(shape).to(dtype), (1.5 * normal(shape) + 1.0).clamp(-9, 4).to(dtype), normal(shape).to(dtype)
    return x, gate, dy, normal((b, c, n)), normal((b, c, n))


def check(x, gate, dy, state, dlast, lengths=None, reverse=False, dim=2):
    """All outputs of the two calls on (batch, channels, steps, inner) views."""
    import paper_2207_08393_b200 as g
    before = [t.clone() for t in (x, gate, dy)]
    y, last, saved = g.gated_scan_forward(x, gate, state, lengths, dim, reverse)
    dx, dg, ds = g.gated_scan_vjp(dy, dlast, x, gate, saved, lengths, dim, reverse)
    for t, u in zip((x, gate, dy), before):
        assert torch.equal(torch.nan_to_num(t, 7.0), torch.nan_to_num(u, 7.0))
    n = None if lengths is None else np.clip(lengths.cpu().numpy(), 0, x.shape[2])
    opt = lambda t: None if t is None else host(t)
    clean = lambda t: np.nan_to_num(host(t), nan=0.0, posinf=0.0, neginf=0.0) if lengths is not None else host(t)
    hx, hg, hy = clean(x), clean(gate), clean(dy)
    ry, rlast, rbefore = so.forward(hx, hg, opt(state), n, reverse)
    rdx, rdg, rds = so.vjp(hy, opt(dlast), hx, hg, rbefore, n, reverse)
    m = max(np.abs(hx).max(initial=0), np.abs(rbefore).max(initial=0), 1)
    d = 56 * max(np.abs(hy).max(initial=0), 1) + (0 if dlast is None else np.abs(host(dlast)).max())
    close(y, ry, x.dtype, m, "y")
    close(last, rlast, torch.float32, m, "last")
    close(dx, rdx, x.dtype, d, "grad_x")
    close(dg, rdg, x.dtype, 2 * m * d, "grad_gate")
    close(ds, rds, torch.float32, d, "grad_state")
    return y, last, saved, dx, dg, ds


# inner > 1: chunks of 16 steps; pieces of 8 bytes, or single chains where sizes are odd; parts where chains are few and long
MAPS = [(1, 2, 21, 1025), (2, 1, 40, 259), (1, 1, 3000, 131), (3, 2, 9, 128), (1, 1, 1, 2), (1, 3, 20, 64), (2, 5, 16, 8), (2, 5, 17, 12), (3, 2, 33, 7), (1, 4, 21, 145), (2, 1, 1000, 6), (1, 1, 2049, 33),
        (2, 3, 65, 1026), (5, 1, 2, 2), (1, 40, 48, 1024)]
# inner = 1: chains that share tiles, that fill some, that are cut into parts
SERIES = [(1, 1, 1, 1), (1, 7, 1, 1), (1, 16, 20, 1), (3, 11, 21, 1), (2, 300, 64, 1), (1, 9, 255, 1), (1, 10, 256, 1), (2, 5, 257, 1), (1, 3, 4097, 1),
          (1, 2, 20000, 1), (4, 1, 8192, 1), (2, 5000, 3, 1), (1, 1, 40001, 1), (1, 70, 600, 1), (1, 5, 33, 1), (3, 1, 65, 1), (2, 3, 1000, 1), (1, 33, 70, 1)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape", MAPS + SERIES)
def test_forward_and_vjp(shape, reverse, dtype):
    x, gate, dy, state, dlast = inputs(shape, TYPES[dtype])
    check(x, gate, dy, state, dlast, None, reverse)
    check(x, gate, dy, None, None, None, reverse)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape,lengths", [
    ((3, 5, 21, 24), [21, 0, 7]), ((4, 2, 40, 9), [1, 40, 39, -5]), ((2, 1, 1000, 6), [999, 3]), ((3, 11, 21, 1), [20, 0, 21]), ((4, 3, 700, 1), [0, 699, 255, 1]),
    ((2, 2, 9000, 1), [8999, 4097]), ((3, 40, 5, 1), [9, 2, 0]), ((3, 2, 37, 257), [37, 8, 0]), ((2, 20, 70, 1), [69, 1]), ((2, 1, 77, 1), [0, 70])])
def test_lengths(shape, lengths, reverse, dtype):
    """What is behind a length is not read: it holds NaN and infinities here."""
    x, gate, dy, state, dlast = inputs(shape, TYPES[dtype], 1)
    for i, n in enumerate(lengths):
        n = min(max(n, 0), shape[2])
        x[i, :, n:], gate[i, :, n:], dy[i, :, n:] = float("nan"), float("inf"), float("nan")
    got = check(x, gate, dy, state, dlast, torch.tensor(lengths, dtype=torch.int32, device="cuda"), reverse)
    for i, n in enumerate(lengths):
        n = min(max(n, 0), shape[2])
        assert all(int(torch.count_nonzero(t[i, :, n:])) == 0 for t in (got[0], got[3], got[4]))
        if n == 0:
            assert torch.equal(got[1][i], state[i]) and torch.equal(got[5][i], dlast[i])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape", [(2, 3, 20, 64), (2, 3, 37, 9), (3, 4, 300, 1), (2, 8, 21, 1)])
def test_slices_and_orders(shape, reverse, dtype):
    """Halves of one array, slices along the steps, arrays that begin anywhere, steps before channels in memory."""
    b, c, t, n = shape
    x, gate, dy, state, dlast = inputs(shape, TYPES[dtype], 2)
    both = torch.cat((x, gate), 1)
    longer = torch.zeros((b, c, t + 3, n), dtype=x.dtype, device="cuda")
    longer[:, :, 1:t + 1] = dy
    check(both[:, :c], both[:, c:], longer[:, :, 1:t + 1], state, dlast, None, reverse)
    shifted = torch.zeros(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(shape).copy_(x)
    check(shifted, gate, dy, state, dlast, None, reverse)
    turned = [v.transpose(1, 2).contiguous().transpose(1, 2) for v in (x, gate)]
    check(turned[0], turned[1], dy, state, dlast, None, reverse)


@pytest.mark.parametrize("shape,dim", [((20,), 0), ((20, 6), 0), ((3, 20), 1), ((3, 20), -1), ((3, 20, 6), -2), ((2, 3, 4, 5, 6), 2), ((2, 3, 4, 5, 6), 3),
                                       ((2, 3, 4, 5, 6), 4)])
def test_axes(shape, dim):
    import paper_2207_08393_b200 as g
    x, gate = torch.randn(shape, device="cuda"), torch.randn(shape, device="cuda")
    d = dim % len(shape)
    numel = lambda s: int(np.prod(s))
    four = (1 if d == 0 else shape[0], numel(shape[1:d]) if d else 1, shape[d], numel(shape[d + 1:]))
    y, last, _ = g.gated_scan_forward(x, gate, dim=dim)
    ry, rlast, _ = so.forward(host(x).reshape(four), host(gate).reshape(four))
    assert last.shape == shape[:d] + shape[d + 1:]
    close(y, ry.reshape(shape), torch.float32, 4.0, "y")
    close(last, rlast.reshape(last.shape), torch.float32, 4.0, "last")


def test_nothing_to_do():
    import paper_2207_08393_b200 as g
    state, dlast = torch.randn(2, 3, 4, device="cuda"), torch.randn(2, 3, 4, device="cuda")
    x = torch.empty(2, 3, 0, 4, device="cuda")
    y, last, saved = g.gated_scan_forward(x, x, state)
    assert y.shape == x.shape and torch.equal(last, state)
    assert torch.equal(g.gated_scan_vjp(x, dlast, x, x, saved)[2], dlast)
    assert int(torch.count_nonzero(g.gated_scan_forward(x, x)[1])) == 0
    x = torch.empty(0, 3, 5, 4, device="cuda")
    y, last, saved = g.gated_scan_forward(x, x)
    assert g.gated_scan_vjp(y, None, x, x, saved)[0].shape == x.shape


@pytest.mark.parametrize("shape", [(2, 3, 40, 8), (2, 30, 20, 1), (1, 1, 3000, 1)])
def test_infinite_gates_keep_and_forget(shape):
    import paper_2207_08393_b200 as g
    x, gate, dy, state, _ = inputs(shape, torch.float32, 3)
    gate[:] = float("inf")
    y, last, saved = g.gated_scan_forward(x, gate, state)
    assert torch.equal(last, state) and torch.equal(y, state.unsqueeze(2).expand_as(y))
    dx, dg, ds = g.gated_scan_vjp(dy, None, x, gate, saved)
    assert int(torch.count_nonzero(dx)) == int(torch.count_nonzero(dg)) == 0
    gate[:] = -float("inf")
    y, last, saved = g.gated_scan_forward(x, gate, state)
    assert torch.equal(y, x) and torch.equal(last, x[:, :, -1])
    dx, dg, ds = g.gated_scan_vjp(dy, None, x, gate, saved)
    assert torch.equal(dx, dy) and int(torch.count_nonzero(dg)) == int(torch.count_nonzero(ds)) == 0
    # far gates: 1 - f keeps its digits where f is 1 to 32 bits
    gate[:] = 30.0
    dx = g.gated_scan_vjp(dy, None, x, gate, g.gated_scan_forward(x, gate)[2])[0]
    tail = dx[:, :, -1] / dy[:, :, -1]
    assert float((tail / np.exp(-30.0) - 1).abs().max()) < 1e-5


@pytest.mark.parametrize("shape", [(2, 3, 20, 16), (1, 2, 5000, 1), (1, 1, 4000, 64), (1, 64, 21, 1)])
def test_a_nan_stays_in_its_chain(shape):
    import paper_2207_08393_b200 as g
    x, gate, *_ = inputs(shape, torch.float32, 4)
    x[0, 0, 7, 0] = float("nan")
    y, last, _ = g.gated_scan_forward(x, gate)
    bad = torch.isnan(y)
    want = torch.zeros_like(bad)
    want[0, 0, 7:, 0] = True
    assert torch.equal(bad, want) and int(torch.isnan(last).sum()) == 1


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(1,), (7,), (20, 160), (3, 5, 33), (60, 12, 16)])
def test_steps_are_the_scan(shape, dtype):
    """Frames one at a time give the bits of the scan over them."""
    import paper_2207_08393_b200 as g
    gen = torch.Generator(device="cuda").manual_seed(5)
    frames = [(torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype]), torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype])) for _ in range(6)]
    state = torch.randn(shape, generator=gen, device="cuda")
    first = state.clone()
    ys = [g.gated_step(x, gate, state) for x, gate in frames]
    x, gate = (torch.stack([f[k] for f in frames]).unsqueeze(-1) for k in (0, 1))
    ry, rlast, _ = so.forward(host(x).reshape(1, 1, 6, -1), host(gate).reshape(1, 1, 6, -1), host(first).reshape(1, 1, -1))
    close(torch.stack(ys).reshape(1, 1, 6, -1), ry, TYPES[dtype], 4.0, "y")
    close(state.reshape(1, 1, -1), rlast, torch.float32, 4.0, "state")
    if state.numel() > 1:
        y, last, _ = g.gated_scan_forward(torch.stack([f[0] for f in frames]), torch.stack([f[1] for f in frames]), first, dim=0)
        assert torch.equal(last, state) and all(torch.equal(a, b) for a, b in zip(y, ys))


def test_a_step_on_halves_of_one_array():
    import paper_2207_08393_b200 as g
    u = torch.randn(4, 12, 5, 8, device="cuda")
    state = torch.randn(4, 6, 5, 8, device="cuda")
    ref = so.forward(host(u[:, :6]).reshape(4, 1, 1, -1), host(u[:, 6:]).reshape(4, 1, 1, -1), host(state).reshape(4, 1, -1))[1]
    g.gated_step(u[:, :6], u[:, 6:], state)
    close(state.reshape(4, 1, -1), ref, torch.float32, 4.0, "state")


def test_refusals():
    import paper_2207_08393_b200 as g
    x = torch.randn(2, 3, 5, 8, device="cuda")
    s = torch.zeros(2, 3, 8, device="cuda")
    n = torch.ones(2, dtype=torch.int32, device="cuda")
    bad = [dict(gate=x[:, :2]), dict(gate=x.half()), dict(gate=x.cpu()), dict(x=x.double(), gate=x.double()), dict(state=s.half()), dict(state=s[:, :, :4]),
           dict(state=s.transpose(0, 1).contiguous().transpose(0, 1)), dict(lengths=n.long()), dict(lengths=n[:1]), dict(lengths=n.cpu()), dict(lengths=n, dim=0),
           dict(dim=4), dict(dim=-5), dict(x=x.transpose(2, 3), gate=x.transpose(2, 3)), dict(x=torch.view_as_complex(x.view(2, 3, 5, 4, 2)).conj().imag,
                                                                                              gate=x[..., :4].contiguous())]
    for kw in bad:
        with pytest.raises((ValueError, IndexError)):
            g.gated_scan_forward(**{**dict(x=x, gate=x), **kw})
    with pytest.raises(ValueError, match="saved"):
        long = torch.randn(2, 3, 40, 8, device="cuda")
        g.gated_scan_vjp(long, None, long, long, (None, None))
    with pytest.raises(ValueError):
        g.gated_step(x, x, x.half())
    with pytest.raises(ValueError):
        g.gated_step(x, x, None)
    d = g.make_scan_dims(0, 2, 3, 5, 8)
    y = torch.empty_like(x)
    for args in ((x, x, None, x, None, None), (x, x, s, y, s, None), (x, x, None, y, y, None), (y[:, 1:], x, None, y, None, None)):
        with pytest.raises(g.GleamError) as e:
            g.gleam_gated_scan_forward(*args, d)
        assert e.value.status == -6
    with pytest.raises(g.GleamError) as e:
        g.gleam_gated_scan_forward(x.cpu(), x, None, y, None, None, d)
    assert e.value.status == -4


@pytest.mark.parametrize("shape,dim", [((2, 3, 20, 4, 6), 2), ((2, 50, 8), 1), ((4, 33), 1)])
@pytest.mark.parametrize("reverse", [False, True])
def test_autograd(shape, dim, reverse):
    """Gradients of the node against the definition's, with cotangents in another order and unused outputs."""
    import paper_2207_08393_b200 as g
    leaves = [torch.randn(shape, device="cuda", requires_grad=True) for _ in range(2)]
    state = torch.randn(shape[:dim] + shape[dim + 1:], device="cuda", requires_grad=True)
    four = (shape[0], int(np.prod(shape[1:dim])), shape[dim], int(np.prod(shape[dim + 1:])))
    x, gate = host(leaves[0]).reshape(four), host(leaves[1]).reshape(four)
    st = host(state).reshape(four[0], four[1], four[3])
    before = so.forward(x, gate, st, None, reverse)[2]
    cot = torch.randn(shape[::-1], device="cuda").permute(*range(len(shape) - 1, -1, -1))
    dlast = torch.randn_like(state)
    for use_y, use_last in ((True, True), (True, False), (False, True)):
        y, last = g.gated_scan(*leaves, state, None, dim, reverse)
        loss = (y * cot).sum() * use_y + (last * dlast).sum() * use_last if use_y and use_last else (y * cot).sum() if use_y else (last * dlast).sum()
        got = torch.autograd.grad(loss, leaves + [state])
        ref = so.vjp(host(cot).reshape(four) * use_y, host(dlast).reshape(st.shape) * use_last, x, gate, before, None, reverse)
        for a, r in zip(got, ref):
            close(a, r.reshape(a.shape), torch.float32, 500.0, "gradient")
    wide = torch.randn(shape[:-1] + (2 * shape[-1],), device="cuda", requires_grad=True)      # slices that the calls refuse are copied
    y, _ = g.gated_scan(wide[..., ::2], wide[..., 1::2], None, None, dim, reverse)
    y.sum().backward()
    assert bool(torch.isfinite(wide.grad).all())


def test_gradients_by_differences():
    import paper_2207_08393_b200 as g
    torch.manual_seed(2)
    x, gate = torch.randn(1, 2, 9, 3, device="cuda", requires_grad=True), torch.randn(1, 2, 9, 3, device="cuda", requires_grad=True)
    loss = lambda: (g.gated_scan(x, gate, reverse=True)[0] ** 2).sum().double()
    grads = torch.autograd.grad(loss(), (x, gate))
    with torch.no_grad():
        for t, grad in zip((x, gate), grads):
            move = torch.randn_like(t)
            t += 1e-2 * move
            up = loss()
            t -= 2e-2 * move
            down = loss()
            t += 1e-2 * move
            # the quotient's own error: 1e-4 of the third derivative, and 32-bit sums
            assert abs(float((up - down) / 2e-2 - (grad * move).sum())) < 2e-2 * float(grad.norm() * move.norm())


@pytest.mark.parametrize("shape", [(1, 8, 20, 640), (1, 1, 4000, 64), (1, 3, 9000, 1), (2, 100, 21, 1)])
def test_repeats_other_streams_and_graphs(shape):
    """The same bits again, on another stream, and from two replayed graphs with workspaces of their own."""
    import paper_2207_08393_b200 as g
    x, gate, dy, state, dlast = inputs(shape, torch.bfloat16, 6)

    def both(x, gate, dy):
        y, last, saved = g.gated_scan_forward(x, gate, state)
        return (y, last) + g.gated_scan_vjp(dy, dlast, x, gate, saved)

    first = both(x, gate, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both(x, gate, dy)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        here = [t.clone() for t in (x, gate, dy)]
        with torch.cuda.graph(graph):
            out = both(*here)
        graphs.append((graph, here, out))
    graphs[1][1][0].neg_()
    for graph, _, _ in graphs + graphs:
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, graphs[0][2]))
    other = both(graphs[1][1][0], gate, dy)
    assert all(torch.equal(a, b) for a, b in zip(other, graphs[1][2]))


def test_outputs_stay_inside():
    """Canaries around the outputs of raw calls with strided outputs."""
    import paper_2207_08393_b200 as g
    for shape in ((2, 3, 21, 10), (2, 3, 21, 1), (1, 1, 3001, 1), (1, 1, 2000, 34)):
        b, c, t, n = shape
        x, gate, dy, state, dlast = inputs(shape, torch.float16, 7)
        wide = [torch.full((b, 2 * c, t, n), 77.0, dtype=torch.float16, device="cuda") for _ in range(3)]
        s = (2 * c * t * n, t * n, n)
        vec = [torch.full((b * c * n + 8,), 55.0, device="cuda") for _ in range(2)]
        mk = lambda strides: g.make_scan_dims(1, b, c, t, n, strides=strides, stream=torch.cuda.current_stream())
        d = mk([(0, 0, 0), (0, 0, 0), s])
        need = g.gleam_gated_scan_saved_size(d)
        saved = torch.full((need // 4 + 4,), 33.0, device="cuda")
        ws = torch.full((g.gleam_gated_scan_workspace_size(d) + 256,), 11, dtype=torch.uint8, device="cuda")
        d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel() - 256
        g.gleam_gated_scan_forward(x, gate, state, wide[0], vec[0], saved, d)
        d = mk([(0, 0, 0), (0, 0, 0), (0, 0, 0), s, s])
        d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel() - 256
        g.gleam_gated_scan_vjp(dy, dlast, x, gate, state, saved, wide[1], wide[2], vec[1], d)
        torch.cuda.synchronize()
        assert all(bool((w[:, c:] == 77.0).all()) for w in wide) and all(bool((v[-8:] == 55.0).all()) for v in vec)
        assert bool((saved[need // 4:] == 33.0).all()) and bool((ws[-256:] == 11).all())
        y, last, sv = g.gated_scan_forward(x, gate, state)
        dx, dg, ds = g.gated_scan_vjp(dy, dlast, x, gate, sv)
        for a, w in zip((y, dx, dg), wide):
            assert torch.equal(a, w[:, :c])
        assert torch.equal(last.reshape(-1), vec[0][:-8]) and torch.equal(ds.reshape(-1), vec[1][:-8])


def test_writes_in_place_are_seen_by_autograd():
    import paper_2207_08393_b200 as g
    x, gate = torch.randn(2, 6, 8, device="cuda", requires_grad=True), torch.randn(2, 6, 8, device="cuda")
    state = torch.zeros(2, 8, device="cuda")
    y, _ = g.gated_scan(x, gate, state, dim=1)
    with torch.no_grad():
        g.gated_step(x[:, 0], gate[:, 0], state)                       # the state that the backward pass needs
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with pytest.raises(ValueError, match="gated_scan"):
        g.gated_step(x[:, 0], gate[:, 0], state)
    with torch.inference_mode():
        s = torch.zeros(2, 8, device="cuda")
        assert torch.equal(g.gated_step(x[:, 0], gate[:, 0], s), s)
    with pytest.raises(ValueError, match="save=False"):
        y, last, saved = g.gated_scan_forward(x.detach(), gate, dim=1, save=False)
        g.gated_scan_vjp(y, None, x.detach(), gate, saved, dim=1)


@pytest.mark.parametrize("shape", [(1, 1, 4, 1200000001), (1, 1, 4, 1200000000), (1, 1200000000, 4, 1), (2, 3100000, 700, 1)])
def test_arrays_beyond_32_bits(shape):
    """Over 2^32 elements: places in the first, the last and a middle chain, which take patterns of their own."""
    import paper_2207_08393_b200 as g
    b, c, t, n = shape
    x = torch.zeros(shape, dtype=torch.float16, device="cuda")
    gate = torch.full(shape, -1.0, dtype=torch.float16, device="cuda")
    chains = [(0, 0, 0), (b - 1, c - 1, n - 1), (b - 1, c * 9 // 10, n * 9 // 10)]
    torch.manual_seed(8)
    for i, j, k in chains:
        x[i, j, :, k] = torch.randn(t, device="cuda").half()
        gate[i, j, :, k] = torch.randn(t, device="cuda").half()
    y, last, saved = g.gated_scan_forward(x, gate)
    dx, dg, _ = g.gated_scan_vjp(x, None, x, gate, saved, state_grad=False)
    for i, j, k in chains:
        cut = lambda v: host(v[i, j, :, k]).reshape(1, 1, t, 1)
        ry, rlast, before = so.forward(cut(x), cut(gate))
        rdx, rdg, _ = so.vjp(cut(x), None, cut(x), cut(gate), before)
        for got, ref in ((y, ry), (dx, rdx), (dg, rdg)):
            close(got[i, j, :, k].reshape(1, 1, t, 1), ref, torch.float16, 500.0, "chain %d %d %d" % (i, j, k))
        assert abs(float(last[i, j, k]) - float(rlast[0, 0, 0])) < 1e-4
    assert int(torch.count_nonzero(last)) <= 3


# The forms: private pieces, strips, narrow rows, short series, series that share tiles, single chains, parts of both
FORMS = [(1, 2, 3, 2048), (1, 3, 2, 1025), (1, 300, 2, 7), (1, 2000, 5, 1), (1, 200, 90, 1), (1, 30, 3000, 1), (1, 1, 4000, 264), (1, 1, 3000, 131)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape", FORMS)
def test_gates_far_from_zero(shape, reverse, dtype):
    """f and 1 - f one by one, as 32-bit numbers: the first step has the gate and x = 1, the others keep the state.  last is 1 - f from a state of
    zero, and what comes back from a cotangent of 1 is f.

    32-bit gates: the exponential is off by 2^-22 at most, the sum in front of the division by 2^-24, the division by 2^-23, a product by 2^-24: 2^-21.
    Gates of 16 bits: also |gate| 2^-23, for the rounded argument of the exponential (2^-24) and the constant in it (2^-26)."""
    import paper_2207_08393_b200 as g
    b, c, t, n = shape
    first = t - 1 if reverse else 0
    x, gate = torch.ones(shape, dtype=TYPES[dtype], device="cuda"), torch.full(shape, float("inf"), dtype=TYPES[dtype], device="cuda")
    gate[:, :, first] = torch.linspace(-86.0, 86.0, b * c * n, device="cuda").view(b, c, n).to(TYPES[dtype])
    y, last, saved = g.gated_scan_forward(x, gate, reverse=reverse)
    ds = g.gated_scan_vjp(torch.zeros_like(x), torch.ones(b, c, n, device="cuda"), x, gate, saved, reverse=reverse)[2]
    state = torch.ones(b, c, n, device="cuda")
    g.gated_step(torch.zeros(b, c, n, dtype=TYPES[dtype], device="cuda"), gate[:, :, first].contiguous(), state)
    at = gate[:, :, first].double()
    most = 2.0 ** -21 + (0.0 if dtype == "float32" else at.abs() * 2.0 ** -23)
    for got, want in ((last, 1 / (1 + torch.exp(at))), (ds, 1 / (1 + torch.exp(-at))), (state, 1 / (1 + torch.exp(-at)))):
        assert bool(((got.double() / want - 1).abs() <= most).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("shape", MAPS + SERIES)
def test_norms_of_the_errors(shape, reverse, dtype):
    """Against norms instead of the worst case.  A step is off by less than 2^-21 (2^-23 to 2^-22 as a rule), and a chain remembers 56 steps:
    errors of random signs give sqrt(56) 2^-22 = 1.8e-6 of the result, gates of 16 bits (up to 9, on average below 2) half as much again; the few elements
    of a small array may have no averages, 56 * 2^-21 = 2.7e-5.  What is stored in 16 bits differs from the rounded definition where that
    lies so near to the border of two numbers: 3e-6 of a typical value against steps of 2^-11 of it and less, 1 % of the elements, 3 with
    differences h - x that are small.  An h of 16 bits in the gate's gradient would change most of them (tests/test_scan_ops.py)."""
    import paper_2207_08393_b200 as g
    kind = TYPES[dtype]
    x, gate, dy, state, dlast = inputs(shape, kind, 9)
    y, last, saved = g.gated_scan_forward(x, gate, state, None, 2, reverse)
    dx, dg, ds = g.gated_scan_vjp(dy, dlast, x, gate, saved, None, 2, reverse)
    ry, rlast, before = so.forward(host(x), host(gate), host(state), None, reverse)
    rdx, rdg, rds = so.vjp(host(dy), host(dlast), host(x), host(gate), before, None, reverse)
    for what, got, ref in (("y", y, ry), ("last", last, rlast), ("grad_x", dx, rdx), ("grad_gate", dg, rdg), ("grad_state", ds, rds)):
        most = 3e-5 if ref.size < 1000 else 2e-6 if kind is torch.float32 else 3e-6
        if got.dtype is torch.float32:
            assert np.sqrt(((host(got) - ref) ** 2).sum()) <= most * np.sqrt((ref ** 2).sum()) + 1e-35, what
            continue
        want = torch.from_numpy(ref).to(kind).cuda()
        assert float((got.double() - want.double()).abs().max()) <= torch.finfo(kind).eps * np.abs(ref).max(), what
        if ref.size >= 1000:
            assert int((got != want).sum()) <= 0.03 * ref.size, what


@pytest.mark.parametrize("shape", [(3, 800000001), (5, 2, 300000000)])
def test_steps_beyond_2_to_31_elements(shape):
    import paper_2207_08393_b200 as g
    x, gate = torch.zeros(shape, dtype=torch.float16, device="cuda"), torch.full(shape, -1.0, dtype=torch.float16, device="cuda")
    state = torch.zeros(shape, device="cuda")
    flat = [t.view(-1) for t in (x, gate, state)]
    n = flat[0].numel()
    at = torch.tensor([0, 1, shape[-1] - 1, shape[-1], n // 2, n - shape[-1], n - 2, n - 1], device="cuda")
    torch.manual_seed(9)
    for t in flat:
        t[at] = torch.randn(len(at), device="cuda").to(t.dtype)
    want = so.forward(*[host(t[at]).reshape(1, 1, 1, -1) for t in flat[:2]], host(flat[2][at]).reshape(1, 1, -1))[1].reshape(-1)
    y = g.gated_step(x, gate, state)
    close(flat[2][at], want, torch.float32, 4.0, "state")
    assert torch.equal(y.view(-1)[at], flat[2][at].half()) and int(torch.count_nonzero(state)) == len(at)
