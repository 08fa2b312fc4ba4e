"""The recurrence and the orthogonalised update together, as the module loop uses them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def plain_convolutions():
    before = torch.backends.cudnn.allow_tf32, torch.backends.cudnn.deterministic
    torch.backends.cudnn.allow_tf32, torch.backends.cudnn.deterministic = False, True
    yield
    torch.backends.cudnn.allow_tf32, torch.backends.cudnn.deterministic = before


def reference(prior, x, lengths):
    """The prior in 64 bits on the CPU, frame after frame."""
    F = torch.nn.functional
    par = {k: v.detach().double().cpu().requires_grad_(True) for k, v in prior.named_parameters()}
    conv = lambda name, v, pad=1: F.conv2d(v, par[name + ".weight"], par[name + ".bias"], padding=pad)
    x = x.detach().double().cpu().requires_grad_(True)
    B, _, T, n0, n1, n2 = x.shape
    h = x.permute(0, 2, 3, 1, 4, 5).reshape(B * T * n0, 2, n1, n2)
    f = conv("head", h)
    u = conv("gates", f).view(B, T, n0, -1, n1, n2)
    N = f.shape[1]
    total = torch.zeros(B, T, n0, N, n1, n2, dtype=torch.float64)
    for way in range(u.shape[3] // (2 * N)):
        rows = []
        for b in range(B):
            state, ys = torch.zeros(n0, N, n1, n2, dtype=torch.float64), [None] * T
            for t in (range(T) if way == 0 else range(T - 1, -1, -1)):
                if t >= lengths[b]:
                    ys[t] = torch.zeros_like(state)
                    continue
                gate = torch.sigmoid(u[b, t, :, (2 * way + 1) * N:(2 * way + 2) * N])
                state = gate * state + (1 - gate) * u[b, t, :, 2 * way * N:(2 * way + 1) * N]
                ys[t] = state
            rows.append(torch.stack(ys))
        total = total + torch.stack(rows)
    f = f + conv("mix", total.reshape(f.shape), 0)
    for k in range(len(prior.blocks)):
        f = f + conv("blocks.%d.3" % k, F.relu(conv("blocks.%d.1" % k, F.relu(f))))
    h = h + conv("tail", f)
    return h.reshape(B, T, n0, 2, n1, n2).permute(0, 3, 1, 2, 4, 5), x, par


def close(got, ref, what):
    """Convolutions and gates in 32 bits leave relative errors of some 1e-6."""
    got, ref = got.detach().double().cpu(), ref.detach()
    assert float((got - ref).norm()) <= 1e-4 * float(ref.norm()) + 1e-12, what


@pytest.mark.parametrize("recurrent", ["causal", "both"])
@pytest.mark.parametrize("n0,lengths", [(1, None), (1, [5, 2]), (2, [0, 5])])
def test_gradients_of_the_prior(recurrent, n0, lengths):
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(3)
    prior = gl.ResidualPrior(6, 1, recurrent=recurrent).cuda()
    x = torch.randn(2, 2, 5, n0, 11, 12, device="cuda", requires_grad=True)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = prior(x, n)
    ref, x64, par = reference(prior, x, lengths or [5, 5])
    close(out, ref, "output")
    cot = torch.randn_like(out)
    out.backward(cot)
    ref.backward(cot.double().cpu())
    close(x.grad, x64.grad, "x")
    for k, v in prior.named_parameters():
        close(v.grad, par[k].grad, k)


@pytest.mark.parametrize("norm,last", [(False, False), (True, False), (False, True)])
def test_live_frames_are_the_cine(norm, last):
    """Convolutions of one frame and of a batch of frames may sum in another order; also with the features last in memory."""
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(1)
    prior = gl.ResidualPrior(8, 2, norm=norm, recurrent="causal").cuda().eval()
    if last:
        prior = prior.to(memory_format=torch.channels_last)
    x = torch.randn(2, 2, 6, 1, 12, 10, device="cuda")
    whole, state = prior(x), None
    for t in range(6):
        out, state = prior.live(x[:, :, t:t + 1], state)
        close(out[:, :, 0], whole[:, :, t].double().cpu(), "frame %d" % t)


def test_greedy_minibatches_with_recurrent_priors_and_muon(oracle):
    """Alg. 1 on padded cines: every parameter gets a gradient and moves, the same seeds give the same bits, the state resumes."""
    from oracle.oracle import Dims, MASK_READOUT_INVARIANT
    from paper_2207_08393_b200 import gleam_loop as gl, workloads as wl
    n, T = (1, 32, 48), 4
    w = wl.scaled(wl.WORKLOADS["cine"], batch=2, coils=4, frames=T, n=n)
    inp = wl.make_inputs(w)
    d = Dims(2, 4, T, 2, n, 0, MASK_READOUT_INVARIANT)
    y = oracle.apply_A(inp["x_true"], inp["sens"], inp["mask"], d).astype(np.complex64)
    x0 = oracle.apply_AH(y, inp["sens"], inp["mask"], d).astype(np.complex64)
    dev = torch.device("cuda:0")
    step = gl.DataConsistencyStep(torch.from_numpy(y).to(dev), torch.from_numpy(inp["sens"]).to(dev), torch.from_numpy(inp["mask"]).to(dev),
                                  w.eta, torch.from_numpy(inp["x_true"]).to(dev), lengths=torch.tensor([4, 3], dtype=torch.int32, device=dev))
    x0_ch = torch.from_numpy(oracle.complex_to_channels(x0)).to(dev)
    results = []
    for _ in range(2):
        torch.manual_seed(0)
        mods = [gl.GleamModule(2, 8, 1, recurrent="both").to(dev) for _ in range(2)]
        start = [[t.detach().clone() for t in m.parameters()] for m in mods]
        opts = [gl.module_optimizer(m, lr=1e-3) for m in mods]
        for turn in range(3):
            if turn == 2:                              # as a resumed run would
                states = [o.state_dict() for o in opts]
                opts = [gl.module_optimizer(m, lr=1e-3) for m in mods]
                for o, s in zip(opts, states):
                    o.load_state_dict(s)
            losses, x = gl.greedy_step(mods, opts, x0_ch, step)
        assert all(np.isfinite(losses)) and bool(torch.isfinite(x).all())
        for m, s in zip(mods, start):
            assert all(t.grad is not None and bool(torch.isfinite(t.grad).all()) for t in m.parameters())
            assert all(not torch.equal(t.detach(), u) for t, u in zip(m.parameters(), s))
        results.append((losses, x))
    assert results[0][0] == results[1][0] and torch.equal(results[0][1], results[1][1])


def test_a_captured_training_step():
    """Forward, gradients and update of a recurrent prior in one graph: replays go on training as eager steps do."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import gleam_loop as gl
    x = torch.randn(1, 2, 4, 1, 16, 24, device="cuda")
    kept = []
    for captured in (False, True):
        torch.manual_seed(2)
        prior = gl.ResidualPrior(8, 1, recurrent="both").cuda()
        params = [p for p in prior.parameters() if p.dim() >= 2]
        opt = g.Muon(params, lr=0.01)

        def once():
            for p, v in zip(params, torch.autograd.grad(prior(x).square().mean(), params)):
                p.grad = v
            opt.step()
            for p in params:
                p.grad = None

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            once()
            once()
        torch.cuda.current_stream().wait_stream(side)
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                once()
            for _ in range(3):
                graph.replay()
        else:
            for _ in range(3):
                once()
        torch.cuda.synchronize()
        kept.append([p.detach().clone() for p in params])
    for a, b in zip(*kept):
        assert float((a - b).norm()) <= 1e-5 * float(a.norm())


def test_a_prior_under_autocast():
    """Half precision convolutions around the recurrence: outputs and gradients near those in single precision."""
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(4)
    prior = gl.ResidualPrior(8, 1, recurrent="both").cuda()
    x = torch.randn(1, 2, 5, 1, 12, 16, device="cuda")
    want = prior(x)
    grads = torch.autograd.grad(want.square().mean(), list(prior.parameters()))
    with torch.autocast("cuda", dtype=torch.bfloat16):
        got = prior(x)
    half = torch.autograd.grad(got.float().square().mean(), list(prior.parameters()))
    # eleven roundings of 2^-9 on the way to an output, twice as many to a gradient; sums of such errors stay far below
    assert float((got.float() - want).norm()) <= 0.05 * float(want.norm())
    for a, b in zip(grads, half):
        assert bool(torch.isfinite(b).all()) and float((a - b).norm()) <= 0.1 * float(a.norm()) + 1e-4


def test_a_float16_prior_with_a_gradient_scaler():
    """module_optimizer under torch.amp: a step with finite gradients moves everything, one with infinite ones nothing."""
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(5)
    prior = gl.ResidualPrior(8, 1, recurrent="both").cuda()
    opt, scaler = gl.module_optimizer(prior, lr=1e-3), torch.amp.GradScaler("cuda", init_scale=128.0)
    x = torch.randn(1, 2, 5, 1, 12, 16, device="cuda")
    for factor, moves in ((1.0, True), (float("inf"), False), (1.0, True)):
        before = [p.detach().clone() for p in prior.parameters()]
        opt.zero_grad()
        with torch.autocast("cuda", dtype=torch.float16):
            loss = prior(x).float().square().mean() * factor
        scaler.scale(loss).backward()
        scaler.step(opt)
        scaler.update()
        assert all(torch.equal(p, q) != moves and bool(torch.isfinite(p).all()) for p, q in zip(prior.parameters(), before))


@pytest.mark.parametrize("recurrent", [None, "causal", "both"])
@pytest.mark.parametrize("shape", [(0, 2, 5, 1, 8, 9), (2, 2, 0, 1, 8, 9)])
def test_a_batch_without_frames(shape, recurrent):
    from paper_2207_08393_b200 import gleam_loop as gl
    prior = gl.ResidualPrior(4, 1, recurrent=recurrent).cuda()
    x = torch.randn(shape, device="cuda", requires_grad=True)
    out = prior(x)
    assert out.shape == x.shape
    out.sum().backward()
    assert x.grad.shape == x.shape and all(p.grad is not None and not bool(p.grad.any()) for p in prior.parameters())
