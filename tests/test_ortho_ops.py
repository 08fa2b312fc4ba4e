"""Orthogonalised updates without a GPU: the definition two ways, and the host-side refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2207_08393_b200 as g
from oracle import ortho_oracle as oo
from paper_2207_08393_b200 import _build, binding


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return g.load_library()


@pytest.mark.parametrize("shape", [(1, 1), (5, 9), (9, 5), (7, 7)])
def test_products_act_on_the_singular_values(shape):
    x = np.random.default_rng(0).normal(size=shape)
    for steps in (1, 3, 5):
        assert np.allclose(oo.iterates(x, steps)[-1], oo.by_singular_values(x, steps), rtol=0, atol=1e-12)


def test_five_turns_bring_singular_values_near_one():
    x = np.random.default_rng(1).normal(size=(20, 50))
    s = np.linalg.svd(oo.iterates(x, 5)[-1], compute_uv=False)
    assert s.min() > 0.6 and s.max() < 1.25


def test_struct_layouts_match_the_header():
    d = binding.gleam_matrix_dims
    assert (d.count.offset, d.turns.offset, d.eps.offset, d.stream.offset, d.workspace_bytes.offset) == (8, 32, 48, 56, 72)
    assert ctypes.sizeof(d) == 80 and ctypes.sizeof(binding.gleam_muon_args) == 20


A = 1 << 30                                         # addresses that are never dereferenced
BAD, NULL = binding.GLEAM_ERR_BAD_DIMS, binding.GLEAM_ERR_NULL_POINTER


def dims(**kw):
    args = dict(dtype=0, count=2, rows=20, cols=30)
    args.update(kw)
    return g.make_matrix_dims(**args)


def status(call, *args):
    with pytest.raises(g.GleamError) as e:
        call(*args)
    return e.value.status


def muon(**kw):
    args = dict(lr=0.1, momentum=0.9, weight_decay=0.0, scale=1.0, nesterov=1)
    args.update(kw)
    return g.gleam_muon_args(**args)


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(count=-1), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 20) + 1), dict(rows=16385, cols=20000),
                                dict(rows=2000, cols=1 << 20), dict(turns=0), dict(turns=101), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                                dict(coefficients=(17.0, 0, 0)), dict(coefficients=(1.0, float("nan"), 0)), dict(coefficients=(1.0, 0, float("inf")))])
def test_bad_sizes(lib, kw):
    d = dims(workspace=8 * A, workspace_bytes=1 << 40, **kw)
    assert status(g.gleam_orthogonalise_workspace_size, d) == BAD
    assert status(g.gleam_orthogonalise, [A, 2 * A], [3 * A, 4 * A], d) == BAD
    assert status(g.gleam_orthogonalise_check_status, d) == BAD
    assert status(g.gleam_muon_step, [A, 2 * A], [3 * A, 4 * A], [5 * A, 6 * A], muon(), d) == BAD


@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(lr=float("nan")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-0.1), dict(weight_decay=float("inf")),
                                dict(scale=float("nan")), dict(nesterov=2)])
def test_bad_steps(lib, kw):
    assert status(g.gleam_muon_step, [A, 2 * A], [3 * A, 4 * A], [5 * A, 6 * A], muon(**kw), dims(workspace=8 * A, workspace_bytes=1 << 40)) == BAD


def test_pointers_workspace_and_versions(lib):
    need = g.gleam_orthogonalise_workspace_size(dims())
    assert need > 0
    assert status(g.gleam_orthogonalise, [A, 2 * A], [3 * A, 4 * A], dims()) == NULL
    assert status(g.gleam_orthogonalise, [A, 2 * A], [3 * A, 4 * A], dims(workspace=8 * A, workspace_bytes=need - 1)) == binding.GLEAM_ERR_WORKSPACE_TOO_SMALL
    assert status(g.gleam_orthogonalise_check_status, dims(workspace=8 * A, workspace_bytes=need - 1)) == binding.GLEAM_ERR_WORKSPACE_TOO_SMALL
    assert status(g.gleam_orthogonalise, [A, 2 * A], [3 * A, 4 * A], dims(workspace=8 * A + 128, workspace_bytes=need)) == BAD
    d = dims(workspace=8 * A, workspace_bytes=need)
    for at in range(2):
        for k in range(2):
            lists = [[A, 2 * A], [3 * A, 4 * A]]
            lists[at][k] = None
            assert status(g.gleam_orthogonalise, *lists, d) == NULL
            lists[at][k] = A + 2
            assert status(g.gleam_orthogonalise, *lists, d) == BAD
    for at in range(3):
        lists = [[A, 2 * A], [3 * A, 4 * A], [5 * A, 6 * A]]
        lists[at][1] = None
        assert status(g.gleam_muon_step, *lists, muon(), d) == NULL
    d.struct_version = 2
    assert status(g.gleam_orthogonalise, [A, 2 * A], [3 * A, 4 * A], d) == BAD
    assert lib.gleam_orthogonalise(None, None, None) == NULL
    assert lib.gleam_muon_step(None, None, None, None, None) == NULL


def test_nothing_to_do(lib):
    for kw in (dict(count=0), dict(rows=0), dict(cols=0)):
        d = dims(**kw)
        assert g.gleam_orthogonalise_workspace_size(d) == 0
        g.gleam_orthogonalise([], [], d)
        g.gleam_orthogonalise_check_status(d)
        g.gleam_muon_step([], [], [], muon(), d)


def test_the_torch_layer_refuses():
    x = torch.zeros(3, 4)
    with pytest.raises(ValueError, match="CUDA"):
        g.orthogonalise(x)
    with pytest.raises(ValueError, match="CUDA"):
        g.muon_step([x], [x], [x], 0.1)
    with pytest.raises(ValueError, match="1 weights"):
        g.muon_step([x], [], [x], 0.1)
    p = torch.nn.Parameter(x)
    for kw in (dict(lr=-1.0), dict(momentum=1.0), dict(weight_decay=-1.0), dict(scale="adam")):
        with pytest.raises(ValueError):
            g.Muon([p], **kw)
    with pytest.raises(ValueError, match="another optimiser"):
        g.Muon([torch.nn.Parameter(torch.zeros(5))])


def test_priors_along_frames_are_asked_for():
    from paper_2207_08393_b200 import gleam_loop as gl
    with pytest.raises(ValueError, match="recurrent"):
        gl.ResidualPrior(8, 2, recurrent="backward")
    with pytest.raises(RuntimeError, match="causal"):
        gl.ResidualPrior(8, 2, recurrent="both").live(torch.zeros(1, 2, 1, 1, 4, 4))
    with pytest.raises(ValueError, match="one frame"):
        gl.ResidualPrior(8, 2, recurrent="causal").live(torch.zeros(1, 2, 3, 1, 4, 4))
    plain = gl.ResidualPrior(8, 2)
    assert not any("gates" in k or "mix" in k for k in plain.state_dict())
    opt = gl.module_optimizer(gl.GleamModule(2, 8, 1, norm=True, recurrent="both"), lr=0.01)
    assert [type(o).__name__ for o in opt.optimizers] == ["Muon", "Adam"]
    with pytest.raises(ValueError):
        opt.load_state_dict([])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_a_loaded_momentum_keeps_its_32_bits(dtype):
    """Whatever the weights' type: a run that is taken up again goes on with the very same momenta."""
    torch.manual_seed(3)
    a = [torch.nn.Parameter(torch.randn(5, 7).to(dtype)) for _ in range(3)]
    opt = g.Muon([{"params": a[:1]}, {"params": a[1:], "lr": 0.5}])
    for p in a[:1] + a[2:]:                                        # one has not been updated yet
        opt.state[p]["momentum"] = torch.randn(5, 7)
    kept = opt.state_dict()
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    other = g.Muon([{"params": b[:1]}, {"params": b[1:]}])
    other.load_state_dict(kept)
    assert other.param_groups[1]["lr"] == 0.5 and "momentum" not in other.state[b[1]]
    for p, q in ((a[0], b[0]), (a[2], b[2])):
        m = other.state[q]["momentum"]
        assert m.dtype == torch.float32 and torch.equal(m, opt.state[p]["momentum"]) and m.data_ptr() != opt.state[p]["momentum"].data_ptr()


def test_a_loaded_momentum_has_its_weights_shape():
    a, b = torch.nn.Parameter(torch.zeros(4, 6)), torch.nn.Parameter(torch.zeros(6, 6))
    opt = g.Muon([a])
    opt.state[a]["momentum"] = torch.zeros(1, 6)
    with pytest.raises(ValueError):
        g.Muon([b]).load_state_dict(opt.state_dict())


def in_pieces(x, steps, pieces, coefficients=oo.COEFFICIENTS, eps=1e-7):
    """The turns with X, A and P stored as one or two float16 numbers of 2^10 times their values (X times a power of two where its norm is
    small), everything else in 64 bits."""
    a, b, c = coefficients

    def stored(v):
        v = v * 1024.0
        hi = v.astype(np.float16).astype(np.float64)
        lo = (v - hi).astype(np.float16).astype(np.float64) if pieces == 2 else 0.0 * v
        return hi / 1024.0, lo / 1024.0

    def product(u, v):
        return u[0] @ v[0] + u[0] @ v[1] + u[1] @ v[0]

    norm = np.sqrt((x.astype(np.float64) ** 2).sum())
    most = norm / (norm + eps)
    x = x.astype(np.float64) / (norm + eps)
    for _ in range(steps):
        e = np.ceil(np.log2(most)) if most <= 0.5 else 0.0
        s = stored(x * 2.0 ** -e)
        p = stored(b * product(s, [v.T for v in s]) + c * 2.0 ** (2 * e) * product(*[stored(product(s, [v.T for v in s]))] * 2))
        x = 2.0 ** e * (a * (s[0] + s[1]) + 2.0 ** (2 * e) * product(p, s))
        most = most * (abs(a) + most ** 2 * (abs(b) + most ** 2 * abs(c))) if most <= 0.5 else 1.0
    return x


@pytest.mark.parametrize("norm", [1.0, 1e-6, 1e-8, 1e-11, 1e-13, 1e-16])
@pytest.mark.parametrize("shape", [(60, 540), (130, 257), (100, 900)])
@pytest.mark.parametrize("steps", [1, 5])
def test_the_bound_takes_two_pieces_and_not_one(shape, steps, norm):
    rng = np.random.default_rng(3)
    n = shape[0]
    x = (rng.normal(size=(n, n)) / (1 + np.arange(n))) @ rng.normal(size=(n, shape[1]))
    x = (x * norm / np.sqrt((x ** 2).sum())).astype(np.float32)
    ref = oo.iterates(x, steps)[-1]
    off = lambda y: np.sqrt(((y - ref) ** 2).sum() / (ref ** 2).sum())
    most = oo.near(off(oo.in_32_bits(x, steps)), shape[1])
    # 32-bit products leave up to 2.7e-6 after five turns (100 x 900), of which four times, 900 * 2^-28 and 2^-21 are 1.5e-5
    assert off(in_pieces(x, steps, 2)) <= most < 2e-5
    assert off(in_pieces(x, steps, 1)) > 10 * most


def pair_of_optimizers():
    from paper_2207_08393_b200 import gleam_loop as gl
    torch.manual_seed(0)
    a, b = torch.nn.Parameter(torch.randn(3, 4)), torch.nn.Parameter(torch.randn(5))
    return gl.Optimizers([torch.optim.SGD([a], lr=0.5, momentum=0.9), torch.optim.Adam([b], lr=0.25)]), a, b


def test_optimizers_take_schedules_and_gradient_scalers():
    import copy
    import pickle
    opt, a, b = pair_of_optimizers()
    schedule = torch.optim.lr_scheduler.StepLR(opt, 1, gamma=0.5)
    scaler = torch.amp.GradScaler("cpu", init_scale=4.0, growth_interval=1)
    assert [g["params"] for g in opt.param_groups] == [[a], [b]]

    def turn(factor):
        opt.zero_grad()
        scaler.scale(factor * ((a ** 2).sum() + (b ** 2).sum())).backward()
        scaler.step(opt)
        scaler.update()
        schedule.step()

    before = [a.detach().clone(), b.detach().clone()]
    want = before[0] - 0.5 * 2 * before[0]
    turn(1.0)
    assert torch.allclose(a, want) and not torch.equal(b, before[1])
    assert [o.param_groups[0]["lr"] for o in opt.optimizers] == [0.25, 0.125] and scaler.get_scale() == 8.0
    before = [a.detach().clone(), b.detach().clone()]
    turn(float("inf"))                                   # gradients that are not finite: no step, of neither
    assert torch.equal(a, before[0]) and torch.equal(b, before[1]) and scaler.get_scale() == 4.0
    state = copy.deepcopy(opt.state_dict())
    other, c, d = pair_of_optimizers()
    other.load_state_dict(state)
    assert [g["lr"] for g in other.param_groups] == [g["lr"] for g in opt.param_groups] and set(other.state) == {c, d}
    with torch.no_grad():
        c.copy_(a)
        d.copy_(b)
    loss = other.step(lambda: sum((p ** 2).sum() for p in (c, d)).backward())
    opt.zero_grad()
    sum((p ** 2).sum() for p in (a, b)).backward()
    opt.step()
    assert loss is None and torch.equal(a, c) and torch.equal(b, d)
    for again in (copy.deepcopy(opt), pickle.loads(pickle.dumps(opt))):
        assert len(again.optimizers) == 2 and len(again.param_groups) == 2
        again.step()
    with pytest.raises(ValueError, match="belongs to one"):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.zeros(2))]})
    from paper_2207_08393_b200 import gleam_loop as gl
    gl.Optimizers([]).step()
    repr(opt)


def test_a_refused_group_is_not_kept():
    opt = g.Muon([torch.nn.Parameter(torch.zeros(3, 4))])
    with pytest.raises(ValueError, match="no matrix"):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.zeros(2, 2)), torch.nn.Parameter(torch.zeros(5))]})
    assert len(opt.param_groups) == 1
    opt.add_param_group({"params": torch.nn.Parameter(torch.zeros(2, 2))})
    assert len(opt.param_groups) == 2
