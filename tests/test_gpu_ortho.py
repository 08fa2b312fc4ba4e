"""Orthogonalised updates on the GPU against their definition in 64 bits (oracle.ortho_oracle states the tolerance)."""
import numpy as np
import pytest

from oracle import ortho_oracle as oo

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, its, dtype, what=""):
    """The last iterate; storing rounds by half a step of the type (float16: or of its smallest numbers)."""
    ref, got = its[-1], host(got)
    norm = np.sqrt((ref ** 2).sum())
    most = oo.tolerance(its)
    if dtype != torch.float32:
        most += torch.finfo(dtype).eps / 2 * norm + torch.finfo(dtype).smallest_normal * np.sqrt(ref.size)
    assert np.isfinite(got).all() and got.shape == ref.shape, what
    assert np.sqrt(((got - ref) ** 2).sum()) <= most + 2.0 ** -23 * norm, what


def matrices(count, rows, cols, dtype=torch.float32, seed=0, spread=1.0):
    """Singular values that fall off."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = min(rows, cols)
    u, v = torch.randn(count, rows, n, generator=gen, device="cuda"), torch.randn(count, n, cols, generator=gen, device="cuda")
    return (spread * (u / (1 + torch.arange(n, device="cuda"))) @ v).to(dtype)


SHAPES = [(1, 1, 1), (1, 1, 200), (1, 200, 1), (3, 7, 5), (2, 64, 64), (2, 100, 900), (2, 900, 100), (1, 127, 129), (1, 129, 127), (1, 128, 128), (1, 130, 1000),
          (1, 257, 300), (1, 300, 257), (1, 640, 651), (5, 2, 900), (2, 100, 18), (1, 60, 5000), (1, 384, 1024)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalise(shape, steps, dtype):
    import paper_2207_08393_b200 as g
    x = matrices(*shape, dtype=TYPES[dtype])
    before = x.clone()
    y = g.orthogonalise(x, steps)
    assert y.dtype == x.dtype and torch.equal(x, before)
    for k in range(shape[0]):
        close(y[k], oo.iterates(host(x[k]), steps), TYPES[dtype])


@pytest.mark.parametrize("spread", [1e-12, 1e-4, 1e6, 1e12])
def test_any_magnitude(spread):
    import paper_2207_08393_b200 as g
    x = matrices(1, 40, 70, spread=spread)
    close(g.orthogonalise(x)[0], oo.iterates(host(x[0]), 5), torch.float32)


def test_other_coefficients_and_many_turns():
    """1.875, -1.25, 0.375 converge: after enough turns the rows are orthonormal."""
    import paper_2207_08393_b200 as g
    x = torch.randn(2, 50, 120, device="cuda")
    y = g.orthogonalise(x, 20, (1.875, -1.25, 0.375))
    eye = torch.eye(50, dtype=torch.float64, device="cuda")
    assert float((y.double() @ y.double().mT - eye).abs().max()) < 1e-5
    close(g.orthogonalise(x, 2, (2.0, -1.5, 0.5))[0], oo.iterates(host(x[0]), 2, (2.0, -1.5, 0.5)), torch.float32)


def test_zeros_ones_and_matrices_that_are_not_numbers():
    import paper_2207_08393_b200 as g
    x = matrices(5, 130, 200)
    want = g.orthogonalise(x)
    x[1] = 0
    x[2, 5, 7] = float("nan")
    x[3, 129, 199] = float("inf")
    y = g.orthogonalise(x)
    assert int(torch.count_nonzero(y[1])) == 0
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())
    assert torch.equal(y[0], want[0]) and torch.equal(y[4], want[4])
    close(g.orthogonalise(torch.ones(1, 9, 33, device="cuda"))[0], oo.iterates(np.ones((9, 33)), 5), torch.float32)


def test_more_matrices_than_a_launch_takes():
    import paper_2207_08393_b200 as g
    x = matrices(150, 12, 40)
    y = g.orthogonalise(x.view(3, 50, 12, 40)).view(150, 12, 40)
    for k in (0, 63, 64, 127, 128, 149):
        assert torch.equal(y[k], g.orthogonalise(x[k].clone()))


@pytest.mark.parametrize("shape", [(40, 90, 130), (2, 300, 700), (1, 1030, 2100), (70, 20, 30)])
def test_the_bits_repeat_and_do_not_depend_on_the_neighbours(shape):
    import paper_2207_08393_b200 as g
    x = matrices(*shape)
    y = g.orthogonalise(x)
    assert torch.equal(y, g.orthogonalise(x))
    close(y[-1], oo.iterates(host(x[-1]), 5), torch.float32)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("shape", [(3, 60, 540), (2, 100, 18), (1, 2, 900), (2, 200, 150), (66, 5, 9)])
def test_muon_step(shape, nesterov, dtype):
    import paper_2207_08393_b200 as g
    count, rows, cols = shape
    t = TYPES[dtype]
    w = [v.clone() for v in torch.randn(shape, device="cuda").to(t)]
    grads = [v.clone() for v in matrices(*shape, dtype=t, seed=1)]
    mom = [v.clone() for v in matrices(*shape, seed=2)]
    keep = [[v.clone() for v in s] for s in (w, grads, mom)]
    lr, mu, wd, scale = 0.125, 0.75, 0.25, 2.0
    g.muon_step(w, grads, mom, lr, mu, nesterov, wd, scale, steps=2)
    for k in (0, count - 1):
        m = mu * host(keep[2][k]) + host(keep[1][k])
        assert np.abs(host(mom[k]) - m).max() <= 2.0 ** -23 * np.abs(m).max()
        its = oo.iterates(host(keep[1][k]) + mu * m if nesterov else m, 2)
        ref = (1 - lr * wd) * host(keep[0][k]) - lr * scale * its[-1]
        norm = np.sqrt((ref ** 2).sum())
        # the source is rounded once more than in orthogonalise: 2^-23 of it, at most 14 times as much of a turn's result
        most = lr * scale * (oo.tolerance(its) + 14 * 5 * 2.0 ** -23 * np.sqrt((its[1] ** 2).sum())) + (torch.finfo(t).eps / 2 + 2.0 ** -23) * norm
        assert np.sqrt(((host(w[k]) - ref) ** 2).sum()) <= most
    assert all(torch.equal(a, b) for a, b in zip(grads, keep[1]))


def test_canaries_and_overlaps():
    import paper_2207_08393_b200 as g
    st = torch.cuda.current_stream()
    for rows, cols in ((33, 70), (70, 33), (130, 257)):
        n = rows * cols
        d = g.make_matrix_dims(0, 2, rows, cols, stream=st)
        need = g.gleam_orthogonalise_workspace_size(d)
        ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
        d.workspace, d.workspace_bytes = ws.data_ptr(), need
        x = matrices(2, rows, cols)
        out = torch.full((2 * n + 16,), 9.0, device="cuda")
        parts = [out[4:4 + n], out[8 + n:8 + 2 * n]]
        g.gleam_orthogonalise([x[0], x[1]], parts, d)
        g.gleam_orthogonalise_check_status(d)
        assert bool((ws[need:] == 7).all()) and bool((out[:4] == 9).all()) and bool((out[4 + n:8 + n] == 9).all()) and bool((out[8 + 2 * n:] == 9).all())
        assert torch.equal(torch.stack(parts).view(2, rows, cols), g.orthogonalise(x))
        for xs, outs in (([x[0], x[1]], [x[0], parts[1]]), ([x[0], x[1]], [parts[0], parts[0]]), ([x[0], x[1]], [out[:n], out[n - 1:]]), ([ws, x[1]], parts)):
            with pytest.raises(g.GleamError) as e:
                g.gleam_orthogonalise(xs, outs, d)
            assert e.value.status == -6
        g.gleam_orthogonalise([x[0], x[0]], parts, d)                   # the same matrix twice is read twice
        assert torch.equal(parts[0], parts[1])


def test_refusals():
    import paper_2207_08393_b200 as g
    x = torch.randn(4, 6, device="cuda")
    for bad in (x[0], x.double(), x.t(), x[:, ::2]):
        with pytest.raises(ValueError):
            g.orthogonalise(bad)
    m = torch.zeros(4, 6, device="cuda")
    for w, gr, mo in ((x, x.half(), m), (x, x[:3], m), (x, x, m.half()), (x, x.t().contiguous().t(), m), (x.t().contiguous().t(), x, m), (x, x.cpu(), m), (x[0], x[0], m[0])):
        with pytest.raises(ValueError):
            g.muon_step([w], [gr], [mo], 0.1)
    with pytest.raises(g.GleamError):
        g.muon_step([x], [x.clone()], [m], 0.1, momentum=1.5)
    with pytest.raises(g.GleamError):
        g.muon_step([x, x], [x.clone(), x.clone()], [m, m.clone()], 0.1)
    assert g.orthogonalise(torch.empty(0, 4, 6, device="cuda")).shape == (0, 4, 6)
    assert g.orthogonalise(torch.empty(2, 0, 6, device="cuda")).shape == (2, 0, 6)
    g.muon_step([], [], [], 0.1)


def test_other_streams_and_graphs():
    import paper_2207_08393_b200 as g
    x = matrices(3, 150, 400)
    first = g.orthogonalise(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = g.orthogonalise(x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)
    graphs = []
    for _ in range(2):
        here, graph = x.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = g.orthogonalise(here)
        graphs.append((graph, here, out))
    graphs[1][1].copy_(matrices(3, 150, 400, seed=9))
    for graph, _, _ in graphs + graphs:
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, graphs[0][2]) and torch.equal(g.orthogonalise(graphs[1][1]), graphs[1][2])


def test_the_optimiser_is_the_step():
    """Weights of several shapes and orders, a missing gradient, and a resumed run."""
    import paper_2207_08393_b200 as g
    torch.manual_seed(4)
    shapes = [(16, 2, 3, 3), (16, 16, 3, 3), (16, 16, 3, 3), (2, 16, 3, 3), (12, 20), (5, 7)]

    def params():
        torch.manual_seed(5)
        ps = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in shapes]
        ps[1].data = ps[1].data.contiguous(memory_format=torch.channels_last)
        return ps

    torch.manual_seed(6)
    grads = [[torch.randn(s, device="cuda") for s in shapes] for _ in range(4)]
    kw = dict(lr=0.05, momentum=0.9, weight_decay=0.1)
    a = params()
    opt = g.Muon(a, **kw)
    w = [p.detach().contiguous().clone() for p in a]
    m = [torch.zeros_like(v) for v in w]
    for turn in grads[:2]:
        for p, v in zip(a[:-1], turn):
            p.grad = v.contiguous(memory_format=torch.channels_last) if v.dim() == 4 else v.clone()
        opt.step()
        for k, v in enumerate(turn[:-1]):
            g.muon_step([w[k]], [v], [m[k]], 0.05, 0.9, True, 0.1, 0.2 * max(w[k].shape[0], w[k][0].numel()) ** 0.5)
    for p, v in zip(a, w):
        assert torch.equal(p.detach().contiguous(), v)
    b = params()
    for p, q in zip(b, a):
        p.data.copy_(q.data)
    other = g.Muon(b, **kw)
    other.load_state_dict(opt.state_dict())
    for turn in grads[2:]:
        for ps, o in ((a, opt), (b, other)):
            for p, v in zip(ps[:-1], turn):
                p.grad = v.clone()
            o.step()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_half_precision_weights_keep_a_32_bit_momentum():
    import paper_2207_08393_b200 as g
    p = torch.nn.Parameter(torch.randn(8, 24, device="cuda", dtype=torch.bfloat16))
    opt = g.Muon([p])
    p.grad = torch.randn_like(p)
    opt.step()
    assert opt.state[p]["momentum"].dtype == torch.float32
    again = g.Muon([p])
    again.load_state_dict(opt.state_dict())
    assert again.state[p]["momentum"].dtype == torch.float32
    assert torch.equal(again.state[p]["momentum"], opt.state[p]["momentum"])


def test_writes_in_place_are_seen_by_autograd():
    import paper_2207_08393_b200 as g
    w = torch.randn(4, 6, device="cuda", requires_grad=True)
    y = (w * w).sum()
    before = w._version
    with torch.no_grad():
        g.muon_step([w], [torch.randn(4, 6, device="cuda")], [torch.zeros(4, 6, device="cuda")], 0.1)
    assert w._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("shape", [(1, 128, 1024), (1, 128, 1025), (1, 112, 2048), (1, 113, 1500), (9, 16, 7000), (1, 16, 30000), (40, 128, 900), (20, 48, 6000)])
def test_where_the_resident_kernel_ends(shape):
    """The most that a cluster holds, and a little more, which the general kernels take."""
    import paper_2207_08393_b200 as g
    x = matrices(*shape)
    y = g.orthogonalise(x, 3)
    for k in (0, shape[0] - 1):
        close(y[k], oo.iterates(host(x[k]), 3), torch.float32)
    t = g.orthogonalise(x.mT.contiguous(), 3)
    close(t[0], [i.T for i in oo.iterates(host(x[0]), 3)], torch.float32)


@pytest.mark.parametrize("rows, cols", [(24, 130), (150, 200)])
def test_status_of_several_launches(rows, cols):
    """More matrices than one launch takes, with a workspace that held something else."""
    import paper_2207_08393_b200 as g
    st = torch.cuda.current_stream()
    d = g.make_matrix_dims(0, 70, rows, cols, stream=st)
    need = g.gleam_orthogonalise_workspace_size(d)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = ws.data_ptr(), need
    x = matrices(70, rows, cols)
    out = torch.empty_like(x)
    g.gleam_orthogonalise(list(x), list(out), d)
    g.gleam_orthogonalise_check_status(d)
    assert torch.equal(out, g.orthogonalise(x))


@pytest.mark.parametrize("rows, cols", [(24, 130), (150, 200)])
def test_a_norm_beyond_32_bits_gives_zeros(rows, cols):
    import paper_2207_08393_b200 as g
    x = torch.full((2, rows, cols), 1e19, device="cuda")             # squares of 1e38, thousands of them
    x[1] = matrices(1, rows, cols)[0]
    y = g.orthogonalise(x)
    assert not bool(y[0].any())
    x[0] = 0
    assert torch.equal(y, g.orthogonalise(x))                        # the other matrix is untouched by it


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(4, 512, 4608), (1, 1024, 9216), (2, 300, 2500), (32, 100, 900), (16, 60, 1620), (9, 30, 700)])
def test_the_bits_of_many_calls(shape, dtype):
    """Products whose order is left open would lose an update of a sum once in a while: the same bits over many calls, with other work between
    them and a workspace that held something else."""
    import paper_2207_08393_b200 as g
    x = matrices(*shape, dtype=TYPES[dtype])
    first = g.orthogonalise(x)
    other = torch.randn(1024, 1024, device="cuda")
    differs = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(60):
        if k % 3 == 1:
            other = torch.tanh(other @ other)
        if k % 5 == 2:
            torch.empty(1 << 26, dtype=torch.uint8, device="cuda").fill_(k + 1)
        differs += torch.count_nonzero(g.orthogonalise(x) != first)
    assert int(differs) == 0


@pytest.mark.parametrize("rows, cols", [(24, 130), (150, 200)])
@pytest.mark.parametrize("eps", [1e-30, 1e-38, 1.5e-45])
def test_zeros_stay_zeros_whatever_eps(rows, cols, eps):
    import paper_2207_08393_b200 as g
    x = torch.zeros(2, rows, cols, device="cuda")
    x[1] = matrices(1, rows, cols)[0]
    y = g.orthogonalise(x, eps=eps)
    assert not bool(y[0].any()) and not bool(torch.isnan(y[0]).any())
    assert torch.equal(y[1], g.orthogonalise(x[1], eps=1e-30))
    w = [torch.ones(rows, cols, device="cuda")]
    g.muon_step(w, [x[0].clone()], [torch.zeros(rows, cols, device="cuda")], 0.5, weight_decay=0.5, eps=eps)
    assert bool((w[0] == 0.75).all())


# ---- beside the same turns in 32-bit products (oracle.ortho_oracle.near)

def turns(x, steps, coefficients=oo.COEFFICIENTS, eps=1e-7):
    """The definition in x's type, over the shorter side."""
    a, b, c = coefficients
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.mT if tall else x


def near_32_bits(x, y, steps, **kw):
    """Every matrix of y = orthogonalise(x) within ``near`` of 64 bits."""
    assert not torch.backends.cuda.matmul.allow_tf32
    for u, v in zip(x, y):
        ref = turns(u.double(), steps, **kw)
        norm = float(ref.norm())
        assert norm > 0.0 and np.isfinite(norm)
        err32 = float((turns(u, steps, **kw).double() - ref).norm()) / norm
        off = float((v.double() - ref).norm()) / norm
        most = oo.near(err32, max(u.shape))
        assert off <= most, "%g, 32-bit products %g, allowed %g" % (off, err32, most)


@pytest.mark.parametrize("steps", [1, 3, 5])
@pytest.mark.parametrize("shape", [(2, 100, 900), (1, 60, 5000), (2, 900, 2), (1, 130, 1000), (2, 257, 300), (2, 300, 257), (1, 640, 651), (1, 384, 1024),
                                   (1, 1030, 2100), (1, 2048, 2048), (1, 4100, 3000), (1, 512, 12000), (40, 90, 130), (16, 60, 1620)])
def test_as_near_as_pieces_allow(shape, steps):
    import paper_2207_08393_b200 as g
    x = matrices(*shape, seed=11)
    near_32_bits(x, g.orthogonalise(x, steps), steps)
    x = torch.randn(shape, device="cuda")                            # singular values of one size
    near_32_bits(x, g.orthogonalise(x, steps), steps)


@pytest.mark.parametrize("rows, cols", [(100, 900), (900, 60), (150, 200), (300, 700)])
@pytest.mark.parametrize("norm", [1e-6, 1e-7, 3e-8, 1e-9, 1e-10, 1e-11, 1e-12, 1e-13, 1e-16, 1e-18, 1e-20])
def test_norms_small_against_eps(rows, cols, norm):
    """X starts far below 1 and keeps its digits."""
    import paper_2207_08393_b200 as g
    x = matrices(2, rows, cols, seed=12)
    x = (x.double() * (norm / x.double().norm(dim=(-2, -1), keepdim=True))).float()
    for steps in (1, 2, 5, 9):
        near_32_bits(x, g.orthogonalise(x, steps), steps)
    near_32_bits(x, g.orthogonalise(x, 3, (0.25, -0.5, 0.25), 1e-9), 3, coefficients=(0.25, -0.5, 0.25), eps=1e-9)       # norms that shrink
    w, mom = [torch.zeros(rows, cols, device="cuda")], [torch.zeros(rows, cols, device="cuda")]
    g.muon_step(w, [x[0]], mom, 1.0, 0.0)
    near_32_bits(x[:1], [-w[0]], 5)


@pytest.mark.parametrize("shape", [(16384, 16400), (130, 1 << 20), (1 << 20, 40), (7000, 16384)])
def test_the_largest_sides(shape):
    import paper_2207_08393_b200 as g
    x = torch.randn((1,) + shape, device="cuda")
    near_32_bits(x, g.orthogonalise(x, 1), 1)


@pytest.mark.parametrize("rows, cols", [(100, 900), (150, 600), (60, 60)])
@pytest.mark.parametrize("share", [1e-2, 1e-4, 1e-6, 1e-9])
def test_rows_that_are_small_beside_the_others(rows, cols, share):
    """Stored values have an absolute step: X, A and P are off by 2^-35 each.  In a row that is small, five turns of the usual coefficients
    stretch X's 2^-35 sqrt(L) by 3.45^5 + ... + 3.45 = 682, and what P's row is off by, 2^-35 (1 + 4.78 + 2.04 * 1.56) sqrt(S) times |X| <= 1.25,
    by 3.45^4 + ... + 1 = 198.  The rest is relative to the row, as of a whole matrix."""
    import paper_2207_08393_b200 as g
    x = matrices(1, rows, cols, seed=13)
    x[0, 7] *= share
    y, ref, half = g.orthogonalise(x)[0, 7].double(), turns(x[0].double(), 5)[7], turns(x[0], 5)[7].double()
    norm = float(ref.norm())
    most = 2.0 ** -35 * (682 * cols ** 0.5 + 198 * 11.3 * rows ** 0.5) + norm * oo.near(float((half - ref).norm()) / norm, cols)
    assert float((y - ref).norm()) <= most


def test_gradients_are_not_dropped_in_silence():
    """Neither call is differentiable, and weights are written in place: as with torch's own operators, not under gradients."""
    import paper_2207_08393_b200 as g
    x = torch.randn(4, 6, device="cuda", requires_grad=True)
    others = [torch.randn(4, 6, device="cuda"), torch.zeros(4, 6, device="cuda")]
    with pytest.raises(ValueError, match="no_grad"):
        g.orthogonalise(x)
    with pytest.raises(ValueError, match="no_grad"):
        g.orthogonalise(x * 2)
    for lists in (([x], [others[0]], [others[1]]), ([x * 2], [others[0]], [others[1]]), ([others[0]], [x], [others[1]]), ([others[0]], [others[0].clone()], [x])):
        with pytest.raises(ValueError, match="no_grad"):
            g.muon_step(*lists, 0.1)
    assert not bool(others[1].any())
    with torch.no_grad():
        want = g.orthogonalise(x)
        g.muon_step([x], [others[0]], [others[1]], 0.1)
    assert torch.equal(g.orthogonalise(others[0]), g.orthogonalise(others[0].detach())) and want.shape == x.shape


def test_a_first_step_is_not_captured():
    """Its momenta would be emptied by every replay."""
    import paper_2207_08393_b200 as g
    p = torch.nn.Parameter(torch.randn(8, 24, device="cuda"))
    opt = g.Muon([p], lr=0.1)
    grad = torch.randn_like(p)
    p.grad = grad.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        try:
            with pytest.raises(RuntimeError, match="before a capture"):
                opt.step()
        finally:
            graph.capture_end()
    torch.cuda.synchronize()
    assert not opt.state[p]
    opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for _ in range(3):
        graph.replay()
    q = torch.nn.Parameter(p.detach().clone())
    m = torch.zeros_like(grad)
    for _ in range(4):
        m = 0.95 * m + grad
    torch.cuda.synchronize()
    assert float((opt.state[p]["momentum"] - m).norm()) <= 1e-6 * float(m.norm())


@pytest.mark.parametrize("shape", [(4096, 4096), (512, 60000), (130, 1 << 18), (60000, 300), (2500, 2200)])
def test_sums_of_many_terms(shape):
    """Terms of one sign, added up so often that cutting off alone would show: one float32 in the tensor core all along leaves 3e-5 to 1e-4."""
    import paper_2207_08393_b200 as g
    for x in (matrices(1, *shape, seed=14), torch.rand((1,) + shape, device="cuda")):
        for steps in (1, 5):
            near_32_bits(x, g.orthogonalise(x, steps), steps)


@pytest.mark.parametrize("rows, cols", [(100, 900), (150, 200)])
@pytest.mark.parametrize("eps", [0.5, 1.0, 3.0, 1e6, 1e20])
def test_eps_that_are_large_beside_the_norm(rows, cols, eps):
    import paper_2207_08393_b200 as g
    x = matrices(2, rows, cols, seed=15)
    x = x / x.norm(dim=(-2, -1), keepdim=True)
    for steps in (1, 5, 8):
        near_32_bits(x, g.orthogonalise(x, steps, eps=eps), steps, eps=eps)
