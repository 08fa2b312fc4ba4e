"""The prior with layer norms and dropout in the module loop: a run of the operators as a block uses them, against a CPU
restatement in 64 bits, and captured into a graph."""
import numpy as np
import pytest

from oracle import prior_oracle as po

torch = pytest.importorskip("torch")


def test_dropout_without_a_generator_is_refused():
    from paper_2207_08393_b200 import gleam_loop as gl
    with pytest.raises(ValueError, match="generator"):
        gl.ResidualPrior(8, 2, dropout=0.1)
    with pytest.raises(ValueError, match="probability"):
        gl.ResidualPrior(8, 2, dropout=1.5)
    assert set(gl.ResidualPrior(8, 2).state_dict()) == {k for k in gl.ResidualPrior(8, 2, norm=True).state_dict() if "norm" not in k}


def reference(prior, x, p, offsets, seed):
    """The prior in 64 bits on the CPU; masks from the oracle."""
    F = torch.nn.functional
    get = lambda t: t.detach().double().cpu().requires_grad_(True)
    par = {k: get(v) for k, v in prior.named_parameters()}
    conv = lambda name, v: F.conv2d(v, par[name + ".weight"], par[name + ".bias"], padding=1)

    def norm(v, k):
        mean = v.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + 1e-5)
        return (v - mean) * rstd * par["norm_weight.%d" % k].view(1, -1, 1, 1) + par["norm_bias.%d" % k].view(1, -1, 1, 1)

    B, _, T, n0, n1, n2 = x.shape
    x = get(x)
    h = x.permute(0, 2, 3, 1, 4, 5).reshape(B * T * n0, 2, n1, n2)
    f = conv("head", h)
    normed = "norm_weight.0" in par
    y = norm(f, 0) if normed else f
    for k in range(len(prior.blocks)):
        u = conv("blocks.%d.3" % k, F.relu(conv("blocks.%d.1" % k, F.relu(y))))
        if p > 0:
            u = u * torch.from_numpy(po.kept(tuple(u.shape), p, seed, offsets[k]) * po.scale(p))
        f = f + u
        y = norm(f, k + 1) if normed else f
    out = h + conv("tail", y)
    return out.reshape(B, T, n0, 2, n1, n2).permute(0, 3, 1, 2, 4, 5), x, par


def assert_close(got, ref, what):
    got, ref = got.detach().double().cpu(), ref.detach()
    assert float((got - ref).norm()) <= 1e-4 * float(ref.norm()) + 1e-12, what


@pytest.mark.gpu
@pytest.mark.parametrize("norm,p", [(True, 0.3), (True, 0.0), (False, 0.3)])
@pytest.mark.parametrize("features,n1,n2", [(8, 20, 24), (12, 15, 13)])
def test_gradients_of_the_prior(norm, p, features, n1, n2):
    """Convolutions without TF32 leave relative errors of some 1e-6; 1e-4 covers what the norms make of them."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(3)
    before = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        gen = g.DropoutGenerator(17)
        gen.take(1000)
        prior = gl.ResidualPrior(features, 3, norm=norm, dropout=p, generator=gen).cuda()
        for t in prior.parameters():
            t.data.add_(0.05 * torch.randn_like(t))
        x = torch.randn(2, 2, 3, 1, n1, n2, device="cuda", requires_grad=True)
        start = gen.offset
        out = prior(x)
        n = 6 * features * n1 * n2
        offsets = [start + k * ((n + 3) // 4) for k in range(3)]
        assert gen.offset == start + (3 * ((n + 3) // 4) if p > 0 or norm else 0)
        ref, x64, par = reference(prior, x, p, offsets, 17)
        assert_close(out, ref, "output")
        cot = torch.randn_like(out)
        out.backward(cot)
        ref.backward(cot.double().cpu())
        assert_close(x.grad, x64.grad, "x")
        for k, v in prior.named_parameters():
            assert_close(v.grad, par[k].grad, k)
        prior.eval()
        assert_close(prior(x), reference(prior, x, 0.0, offsets, 17)[0], "evaluation drops nothing")
    finally:
        torch.backends.cudnn.allow_tf32 = before


@pytest.mark.gpu
def test_a_greedy_minibatch_with_norms_and_dropout(oracle):
    """Alg. 1 runs with such modules, every parameter gets a gradient, and the same seeds give the same bits."""
    from oracle.oracle import Dims, MASK_READOUT_INVARIANT
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import gleam_loop as gl, workloads as wl
    n, T = (1, 32, 48), 2
    w = wl.scaled(wl.WORKLOADS["cine"], batch=1, coils=4, frames=T, n=n)
    inp = wl.make_inputs(w)
    d = Dims(1, 4, T, 2, n, 0, MASK_READOUT_INVARIANT)
    y = oracle.apply_A(inp["x_true"], inp["sens"], inp["mask"], d).astype(np.complex64)
    x0 = oracle.apply_AH(y, inp["sens"], inp["mask"], d).astype(np.complex64)
    dev = torch.device("cuda:0")
    step = gl.DataConsistencyStep(torch.from_numpy(y).to(dev), torch.from_numpy(inp["sens"]).to(dev), torch.from_numpy(inp["mask"]).to(dev),
                                  w.eta, torch.from_numpy(inp["x_true"]).to(dev))
    x0_ch = torch.from_numpy(oracle.complex_to_channels(x0)).to(dev)
    results = []
    deterministic = torch.backends.cudnn.deterministic
    torch.backends.cudnn.deterministic = True
    try:
        for _ in range(2):
            torch.manual_seed(0)
            gen = g.DropoutGenerator(5)
            mods = [gl.GleamModule(2, 8, 2, norm=True, dropout=0.1, generator=gen).to(dev) for _ in range(2)]
            start = [[t.detach().clone() for t in m.parameters()] for m in mods]
            opts = [torch.optim.SGD(m.parameters(), lr=1e-2) for m in mods]
            losses, x = gl.greedy_step(mods, opts, x0_ch, step)
            assert all(np.isfinite(losses)) and bool(torch.isfinite(x).all())
            for m, s in zip(mods, start):
                assert all(t.grad is not None and bool(torch.isfinite(t.grad).all()) for t in m.parameters())
                assert all(not torch.equal(t.detach(), u) for t, u in zip(m.parameters(), s))
            results.append((losses, x))
    finally:
        torch.backends.cudnn.deterministic = deterministic
    assert results[0][0] == results[1][0] and torch.equal(results[0][1], results[1][1])


@pytest.mark.gpu
def test_a_captured_training_step_of_the_prior():
    """Forward and gradients in one graph with the device counter: replays differ from one another and repeat with it."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(1)
    gen = g.DropoutGenerator(8, capturable=True)
    prior = gl.ResidualPrior(8, 2, norm=True, dropout=0.5, generator=gen).cuda()
    x = torch.randn(1, 2, 2, 1, 16, 24, device="cuda")
    params = list(prior.parameters())

    def once():
        grads = torch.autograd.grad(prior(x).square().sum(), params)
        gen.advance()
        return grads
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            once()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = once()
    seen = []
    for turn in (3, 4, 3):
        gen.step.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert int(gen.step) == turn + 1
        seen.append([t.clone() for t in grads])
    norms = [t.norm() for t in seen[0]]
    assert any(float((a - b).norm()) > 1e-3 * float(n) for a, b, n in zip(seen[0], seen[1], norms))
    # the convolutions' gradients may add in any order
    assert all(float((a - b).norm()) <= 1e-4 * float(n) + 1e-12 for a, b, n in zip(seen[0], seen[2], norms))


@pytest.mark.gpu
def test_a_prior_under_activation_checkpointing():
    """Recomputed blocks draw the masks of the forward pass: the same bits as without checkpointing."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200.gleam_loop import ResidualPrior
    from torch.utils.checkpoint import checkpoint
    x = torch.randn(2, 2, 3, 1, 12, 10, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    got = []
    for again in (False, True):
        torch.manual_seed(2)
        gen = g.DropoutGenerator(17)
        priors = [ResidualPrior(8, 2, norm=norm, dropout=0.3, generator=gen).cuda() for norm in (True, False)]
        leaf = x.clone().requires_grad_()
        h = leaf
        with torch.backends.cudnn.flags(enabled=True, benchmark=False, deterministic=True):
            for prior in priors:
                h = checkpoint(prior, h, use_reentrant=False, context_fn=gen.recompute) if again else prior(h)
            h.square().sum().backward()
        got.append([h.detach(), leaf.grad] + [p.grad for prior in priors for p in prior.parameters()])
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_checkpointing_with_a_device_counter():
    """Masks of the counter's value come back in the recomputation; a counter that moved before the backward pass raises."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200.gleam_loop import ResidualPrior
    from torch.utils.checkpoint import checkpoint
    x = torch.randn(1, 2, 2, 1, 12, 10, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    got = []
    for again, moved in ((False, False), (True, False), (True, True)):
        torch.manual_seed(2)
        gen = g.DropoutGenerator(17, capturable=True)
        gen.advance()
        prior = ResidualPrior(8, 2, norm=True, dropout=0.3, generator=gen).cuda()
        leaf = x.clone().requires_grad_()
        with torch.backends.cudnn.flags(enabled=True, benchmark=False, deterministic=True):
            h = checkpoint(prior, leaf, use_reentrant=False, context_fn=gen.recompute) if again else prior(leaf)
            if moved:
                gen.advance()
                with pytest.raises(RuntimeError, match="counter"):
                    h.square().sum().backward()
                continue
            h.square().sum().backward()
        got.append([h.detach(), leaf.grad] + [p.grad for p in prior.parameters()])
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [True, False])
def test_an_evaluation_leaves_the_masks_of_the_training_alone(norm):
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200.gleam_loop import ResidualPrior
    x = torch.randn(1, 2, 2, 1, 12, 10, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    gen = g.DropoutGenerator(17)
    torch.manual_seed(2)
    prior = ResidualPrior(8, 2, norm=norm, dropout=0.3, generator=gen).cuda()
    with torch.backends.cudnn.flags(enabled=True, benchmark=False, deterministic=True):
        want = prior(x)
        taken = gen.offset
        gen.offset = 0
        for _ in range(3):
            prior.eval()(x)
        assert gen.offset == 0 and taken > 0
        assert torch.equal(prior.train()(x), want) and gen.offset == taken


@pytest.mark.gpu
def test_without_dropout_the_counter_does_not_matter():
    """p = 0 reads no mask in the backward pass either, so the counter may move before it."""
    import paper_2207_08393_b200 as g
    gen = g.DropoutGenerator(1, capturable=True)
    t = torch.randn(3, 8, 20, device="cuda", requires_grad=True)
    y, total = g.dropout_add_layer_norm(t, t.detach(), None, None, 0.0, gen, dim=1)
    z = g.dropout(t, 0.0, gen)
    gen.advance()
    (total + z).sum().backward()
    assert gen.offset == 0 and torch.equal(t.grad, torch.full_like(t, 2.0))


def composite(prior, x, kept, scale):
    """The prior with the library's operators restated in torch: the same convolutions, sums and norms in 64 bits that are rounded
    where the operators round."""
    def norm(v, k):
        v64 = v.double()
        mean = v64.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt(((v64 - mean) ** 2).mean(1, keepdim=True) + 1e-5)
        w, b = prior.norm_weight[k].double().view(1, -1, 1, 1), prior.norm_bias[k].double().view(1, -1, 1, 1)
        return ((v64 - mean) * rstd * w + b).float().to(v.dtype)

    B, _, T, n0, n1, n2 = x.shape
    h = x.permute(0, 2, 3, 1, 4, 5).reshape(B * T * n0, 2, n1, n2)
    f = prior.head(h)
    y = norm(f, 0) if prior.norm_weight is not None else f
    for k, blk in enumerate(prior.blocks):
        u = blk(y)
        f = (f.double() + torch.where(kept[k], u.double() * scale, 0.0)).float().to(f.dtype)
        y = norm(f, k + 1) if prior.norm_weight is not None else f
    out = h + prior.tail(y)
    return out.reshape(B, T, n0, 2, n1, n2).permute(0, 3, 1, 2, 4, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
def test_a_prior_under_autocast_and_with_features_last(kind, last, norm):
    """Autocast hands the operators 16-bit maps with 32-bit weights, channels_last rows of features; the default 16 features.

    Against the restatement on the same convolutions.  In 16 bits (u half a step) a value that the operators' 32 bits leave on the other
    side of a border of the type is off by 2 u; fewer than one in a thousand are, so that a map is off by less than 0.1 u in L2, and
    four norms and the convolutions between them make less than 4 u of it.  The restatement's gradients have up to two
    roundings more in each of three blocks, threefold by the convolutions and norms: less than 20 u.  A wrong mask is
    off by more than 0.3."""
    import paper_2207_08393_b200 as g
    from paper_2207_08393_b200 import gleam_loop as gl
    p, seed, n1, n2 = 0.3, 23, 21, 26
    torch.manual_seed(4)
    gen = g.DropoutGenerator(seed)
    gen.take(40)
    prior = gl.ResidualPrior(16, 3, norm=norm, dropout=p, generator=gen).cuda()
    for t in prior.parameters():
        t.data.add_(0.05 * torch.randn_like(t))
    if last:
        prior = prior.to(memory_format=torch.channels_last)
    x = torch.randn(2, 2, 3, 1, n1, n2, device="cuda")
    shape, order = ((6, n1, n2, 16), (0, 3, 1, 2)) if last else ((6, 16, n1, n2), (0, 1, 2, 3))
    count = 6 * 16 * n1 * n2 // 4
    kept = [torch.from_numpy(po.kept(shape, p, seed, 10 + k * count)).cuda().permute(order) for k in range(3)]
    half = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[kind]
    seen, grads, outs = [], [], []
    prior.head.register_forward_hook(lambda m, i, o: seen.append(o))
    cot = torch.randn_like(x)
    allow = torch.backends.cudnn.allow_tf32
    torch.backends.cudnn.allow_tf32 = False
    try:
        with torch.backends.cudnn.flags(enabled=True, benchmark=False, deterministic=True, allow_tf32=False):
            for f in (prior, lambda v: composite(prior, v, kept, po.scale(p))):
                leaf = x.clone().requires_grad_()
                with torch.autocast("cuda", dtype=getattr(torch, kind), enabled=kind != "float32"):
                    out = f(leaf)
                outs.append(out.detach())
                grads.append(torch.autograd.grad(out, [leaf] + list(prior.parameters()), cot))
    finally:
        torch.backends.cudnn.allow_tf32 = allow
    assert seen[0].dtype == getattr(torch, kind)
    assert seen[0].is_contiguous(memory_format=torch.channels_last if last else torch.contiguous_format)
    off = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())
    # 32 bits: convolutions in another order for another input leave some 1e-6
    assert off(outs[0], outs[1]) <= (1e-5 if kind == "float32" else 4 * half)
    for a, b in zip(*grads):
        assert off(a, b) <= (1e-4 if kind == "float32" else 20 * half)
