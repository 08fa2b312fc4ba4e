"""Operators of the learned prior without a GPU: the definition of the mask, host-side refusals of the C calls, and the views
that the torch layer makes of strided tensors."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2207_08393_b200 as g
from oracle import prior_oracle as po
from paper_2207_08393_b200 import _build, binding, prior_ops


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return g.load_library()


@pytest.mark.parametrize("counter,key,out", [       # published test vectors of Philox4x32-10
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, out):
    assert tuple(po.philox(counter, key)) == out


@pytest.mark.parametrize("offset,step", [(0, 0), (2 ** 32 - 2, 5), (2 ** 64 - 3, 2 ** 40 + 1)])
def test_vectorised_words_are_philox(offset, step):
    seed = 0x0123456789ABCDEF
    got = po.words(23, seed, offset, step)
    for i in range(23):
        block = (offset + i // 4) % 2 ** 64
        ref = po.philox((block & 0xFFFFFFFF, block >> 32, step & 0xFFFFFFFF, step >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        assert int(got[i]) == ref[i % 4]


def test_the_oracle_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(0)
    x, w, b, dy = rng.normal(size=(2, 5, 3)), rng.normal(size=5), rng.normal(size=5), rng.normal(size=(2, 5, 3))
    y, mean, rstd = po.layer_norm(x, w, b, 1e-3)
    gx, gw, gb = po.layer_norm_vjp(dy, x, w, mean, rstd)
    f = lambda x, w, b: float((po.layer_norm(x, w, b, 1e-3)[0] * dy).sum())
    for which, grad in ((0, gx), (1, gw), (2, gb)):
        args = [x, w, b]
        for at in np.ndindex(args[which].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[which][at] += 1e-6
            down[which][at] -= 1e-6
            assert abs((f(*up) - f(*down)) / 2e-6 - grad[at]) < 1e-6


def test_struct_layout_matches_the_header():
    d = binding.gleam_feature_dims
    assert (d.eps.offset, d.outer.offset, d.pitch.offset, d.stream.offset) == (12, 16, 40, 80)
    assert ctypes.sizeof(d) == 104 and ctypes.sizeof(binding.gleam_dropout_args) == 32


A = 1 << 30                                         # addresses that are never dereferenced
BAD, NULL = binding.GLEAM_ERR_BAD_DIMS, binding.GLEAM_ERR_NULL_POINTER


def feature_dims(**kw):
    args = dict(dtype=0, weight_dtype=0, outer=4, features=8, inner=1, eps=1e-5)
    args.update(kw)
    return g.make_feature_dims(**args)


def status(call, *args):
    with pytest.raises(g.GleamError) as e:
        call(*args)
    return e.value.status


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), BAD), (dict(dtype=-1), BAD), (dict(weight_dtype=1), BAD), (dict(dtype=1, weight_dtype=2), BAD),
    (dict(features=0), BAD), (dict(outer=-1), BAD), (dict(inner=-2), BAD), (dict(pitch=[7]), BAD), (dict(pitch=[0, -8]), BAD),
    (dict(features=(1 << 24) + 1), BAD), (dict(inner=1 << 50), BAD), (dict(outer=1 << 45), BAD), (dict(pitch=[1 << 47]), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD),
])
def test_bad_dims(lib, kw, code):
    d = feature_dims(**kw)
    assert status(g.gleam_layer_norm_forward, A, None, None, 2 * A, None, None, d) == code
    if "eps" not in kw:
        assert status(g.gleam_layer_norm_workspace_size, d) == code
        assert status(g.gleam_dropout_forward, A, None, 2 * A, g.make_dropout_args(0.5), d) == code
    d.struct_version = 7
    assert status(g.gleam_layer_norm_forward, A, None, None, 2 * A, None, None, d) == BAD


@pytest.mark.parametrize("p", [-0.1, 1.0000001, float("nan")])
def test_bad_probabilities(lib, p):
    assert status(g.gleam_dropout_forward, A, None, 2 * A, g.make_dropout_args(p), feature_dims()) == BAD
    assert status(g.gleam_dropout_add_layer_norm_forward, A, 2 * A, None, None, 3 * A, 4 * A, None, None,
                  g.make_dropout_args(p), feature_dims()) == BAD


def test_null_pointers(lib):
    d, m = feature_dims(), g.make_dropout_args(0.5)
    for at in (0, 3):
        args = [A, None, None, 2 * A, None, None, d]
        args[at] = None
        assert status(g.gleam_layer_norm_forward, *args) == NULL
    for at in (0, 1, 3, 4, 5):
        args = [A, 2 * A, None, 3 * A, 4 * A, 5 * A, None, None, d]
        args[at] = None
        assert status(g.gleam_layer_norm_vjp, *args) == NULL
    for at in (0, 2):
        args = [A, None, 2 * A, m, d]
        args[at] = None
        assert status(g.gleam_dropout_forward, *args) == NULL
    for at in (0, 1, 4, 5):
        args = [A, 2 * A, None, None, 3 * A, 4 * A, None, None, m, d]
        args[at] = None
        assert status(g.gleam_dropout_add_layer_norm_forward, *args) == NULL
    for at in (0, 2, 4, 5, 6, 7):
        args = [A, None, 2 * A, None, 3 * A, 4 * A, 5 * A, 6 * A, None, None, m, d]
        args[at] = None
        assert status(g.gleam_dropout_add_layer_norm_vjp, *args) == NULL
    lib = g.load_library()
    assert lib.gleam_dropout_vjp(A, 2 * A, None, ctypes.byref(d)) == NULL
    assert lib.gleam_dropout_vjp(A, 2 * A, ctypes.byref(m), None) == NULL
    assert lib.gleam_layer_norm_workspace_size(ctypes.byref(d), None) == NULL


def test_misaligned_pointers_and_workspace(lib):
    d = feature_dims()
    assert status(g.gleam_layer_norm_forward, A + 2, None, None, 2 * A, None, None, d) == BAD
    assert status(g.gleam_layer_norm_forward, A, 3 * A + 2, None, 2 * A, None, None, d) == BAD
    assert status(g.gleam_dropout_forward, A, None, 2 * A, g.make_dropout_args(0.5, step=3 * A + 4), d) == BAD
    args = (A, 2 * A, None, 3 * A, 4 * A, 5 * A, 6 * A, None)
    assert status(g.gleam_layer_norm_vjp, *args, d) == NULL                                   # a weight gradient needs scratch
    assert status(g.gleam_layer_norm_vjp, *args, feature_dims(workspace=7 * A, workspace_bytes=8)) == binding.GLEAM_ERR_WORKSPACE_TOO_SMALL
    assert status(g.gleam_layer_norm_vjp, *args, feature_dims(workspace=7 * A + 16, workspace_bytes=1 << 20)) == BAD


def test_calls_on_nothing_need_no_pointers(lib):
    for kw in (dict(outer=0), dict(inner=0)):
        d, m = feature_dims(**kw), g.make_dropout_args(0.5)
        assert g.gleam_layer_norm_workspace_size(d) == 0
        g.gleam_layer_norm_forward(None, None, None, None, None, None, d)
        g.gleam_dropout_forward(None, None, None, m, d)
        g.gleam_dropout_vjp(None, None, m, d)
        g.gleam_layer_norm_vjp(None, None, None, None, None, None, None, None, d)
        g.gleam_dropout_add_layer_norm_forward(None, None, None, None, None, None, None, None, m, d)


def test_cpu_tensors_are_refused():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="no CPU fallback"):
        g.layer_norm_forward(x)
    with pytest.raises(ValueError, match="no CPU fallback"):
        g.dropout_forward(x, 0.5, 0, 0)


def address(view, o, c, k):
    pitch = view.pitch or view.features * view.inner
    return o * pitch + (c * view.inner + k)


@pytest.mark.parametrize("make,dim", [
    (lambda: torch.empty(3, 4, 5), 1), (lambda: torch.empty(3, 4, 5), 0), (lambda: torch.empty(3, 4, 5), 2),
    (lambda: torch.empty(3, 9, 5)[:, 2:6], 1),                       # features of a wider array
    (lambda: torch.empty(6, 4, 5)[::2], 1),                          # every other slice
    (lambda: torch.empty(3, 7, 4, 5)[:, 1:2], 2),
    (lambda: torch.empty(2, 4, 3, 5).to(memory_format=torch.channels_last), 1),
    (lambda: torch.empty(7, 4).t(), 0),                              # features last in memory
    (lambda: torch.empty(7, 6)[:, :4], 1),
    (lambda: torch.empty(1, 4, 5).expand(1, 4, 5), 1),
    (lambda: torch.empty(5), 0),
])
def test_views_address_the_elements(make, dim):
    t = make()
    v = prior_ops._view(t, dim)
    index = torch.arange(t.numel()).view(t.shape)
    assert v.outer * v.features * v.inner == t.numel() and v.features == t.shape[dim]
    flat = [sum(i * s for i, s in zip(at, t.stride())) for at in np.ndindex(*t.shape)]
    order = (index.movedim(dim, -1) if v.last else index).reshape(v.outer, v.features, v.inner)
    for o in range(v.outer):
        for c in range(v.features):
            for k in range(v.inner):
                assert flat[int(order[o, c, k])] == address(v, o, c, k)
    like = prior_ops._like(t, dim, v)
    assert like.shape == t.shape and prior_ops._view(like, dim).pitch in (0, v.features * v.inner)
    assert (prior_ops._view(like, dim).outer, prior_ops._view(like, dim).inner) == (v.outer, v.inner)


@pytest.mark.parametrize("make,dim", [
    (lambda: torch.empty(4, 3, 5).transpose(0, 2), 1),
    (lambda: torch.empty(1, 4, 5).expand(3, 4, 5), 1),               # the same memory three times
    (lambda: torch.empty(3, 4, 10)[:, :, ::2], 1),
    (lambda: torch.empty(4, 6, 4, 5)[::2, ::3], 2),                  # uneven steps before the features
])
def test_other_orders_are_refused(make, dim):
    with pytest.raises(ValueError, match="contiguous"):
        prior_ops._view(make(), dim)


def test_generator_ranges_do_not_meet():
    gen = prior_ops.DropoutGenerator(3, device="cpu", capturable=True)
    assert [gen.take(n) for n in (1, 4, 5, 0, 8)] == [0, 1, 2, 4, 4] and gen.offset == 6
    gen.advance()
    assert int(gen.step) == 1
    with pytest.raises(RuntimeError):
        prior_ops.DropoutGenerator(3, device="cpu").advance()


def test_only_an_order_is_changed_for_a_call():
    x = torch.zeros(2, 3, 4)
    turned = torch.arange(24.).view(2, 4, 3).transpose(1, 2)
    got = prior_ops._match(x, turned, 1)
    assert got.is_contiguous() and torch.equal(got, turned)
    for other in (turned.double(), turned.to("meta"), turned[:1]):   # another type, device or shape is for the call to refuse
        assert prior_ops._match(x, other, 1) is other


def test_a_recomputed_pass_takes_its_ranges_again():
    from torch.utils.checkpoint import checkpoint
    gen, taken = prior_ops.DropoutGenerator(3, device="cpu"), []

    def block(x):
        for _ in range(2):
            taken.append(gen.take(x.numel()))
            x = x.sin()
        return x

    x = torch.ones(10, requires_grad=True)
    y = checkpoint(block, x, use_reentrant=False, context_fn=gen.recompute)
    z = checkpoint(block, y, use_reentrant=False, context_fn=gen.recompute)
    assert taken == [0, 3, 6, 9] and gen.offset == 12
    z.sum().backward(retain_graph=True)
    again = taken[4:]
    assert again == [6, 9, 0, 3] and gen.offset == 12
    z.sum().backward()                                               # a kept graph runs its blocks again
    assert set(taken[8:]) <= {0, 3, 6, 9} and gen.offset == 12


def test_a_recomputed_pass_after_the_counter_has_moved_is_refused():
    """Masks of a capturable generator depend on its counter: a recomputation behind advance() would draw others than the
    outputs were made with, so it raises; without advance() it runs."""
    from torch.utils.checkpoint import checkpoint
    for moved in (False, True):
        gen = prior_ops.DropoutGenerator(3, device="cpu", capturable=True)

        def block(x):
            gen.take(x.numel())
            return x.sin()

        x = torch.ones(10, requires_grad=True)
        y = checkpoint(block, x, use_reentrant=False, context_fn=gen.recompute)
        if not moved:
            y.sum().backward()
            assert torch.allclose(x.grad, torch.ones(10).cos()) and gen.offset == 3
            continue
        gen.advance()
        with pytest.raises(RuntimeError, match="counter"):
            y.sum().backward()
        assert gen.offset == 3 and gen.take(1) == 3              # the generator can be used on


def in_a_thread(f):
    import threading
    t = threading.Thread(target=f)
    t.start()
    t.join(60)
    assert not t.is_alive()


def test_threads_get_ranges_of_their_own():
    import sys
    import threading
    gen, taken = prior_ops.DropoutGenerator(3), []

    class Size:                                                      # a size whose evaluation lets another thread in
        def __int__(self):
            in_a_thread(lambda: taken.append(gen.take(8)))
            return 8

    taken.append(gen.take(Size()))
    assert sorted(taken) == [0, 2] and gen.offset == 4
    before = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        many = [threading.Thread(target=lambda: taken.extend([gen.take(1) for _ in range(3000)])) for _ in range(4)]
        for t in many:
            t.start()
        for t in many:
            t.join()
    finally:
        sys.setswitchinterval(before)
    assert sorted(taken) == [0, 2] + list(range(4, 12004)) and gen.offset == 12004


def test_a_recomputed_pass_and_other_threads():
    """What another thread takes during a forward pass or its recomputation belongs to neither."""
    from torch.utils.checkpoint import checkpoint
    gen, taken, other = prior_ops.DropoutGenerator(3, device="cpu"), [], []

    def block(x):
        for _ in range(2):
            taken.append(gen.take(x.numel()))
            in_a_thread(lambda: other.append(gen.take(4)))
            x = x.sin()
        return x

    x = torch.ones(8, requires_grad=True)
    checkpoint(block, x, use_reentrant=False, context_fn=gen.recompute).sum().backward()
    assert taken == [0, 3, 0, 3] and other == [2, 5, 6, 7] and gen.offset == 8


def test_nested_recomputations_take_their_ranges_again():
    from torch.utils.checkpoint import checkpoint
    gen, taken = prior_ops.DropoutGenerator(3, device="cpu"), []

    def inner(x):
        taken.append(gen.take(8))
        return x.sin().sin()

    def outer(x):
        taken.append(gen.take(4))
        x = checkpoint(inner, x.sin(), use_reentrant=False, context_fn=gen.recompute)
        taken.append(gen.take(12))
        return x.sin().sin()

    x = torch.ones(8, requires_grad=True)
    y = checkpoint(outer, x, use_reentrant=False, context_fn=gen.recompute)
    assert taken == [0, 1, 3] and gen.offset == 6
    y.sum().backward()
    assert taken[3:6] == [0, 1, 3] and set(taken[6:]) <= {1} and gen.offset == 6
    plain = torch.ones(8, requires_grad=True)
    plain.sin().sin().sin().sin().sin().sum().backward()
    assert torch.allclose(x.grad, plain.grad)


def test_a_recomputed_pass_that_takes_other_ranges_is_refused():
    gen = prior_ops.DropoutGenerator(3)
    first, again = gen.recompute()
    with first:
        gen.take(8)
        gen.take(4)
    for sizes in ((4,), (8, 8), (8, 4, 1)):
        with pytest.raises(RuntimeError, match="recomputed"):
            with again:
                for n in sizes:
                    gen.take(n)
        assert gen.offset == 3
    with again:
        assert (gen.take(8), gen.take(4)) == (0, 2)
    assert gen.take(1) == 3


def test_a_pass_that_fails_leaves_nothing_behind():
    """A forward pass or recomputation that raises ends its context; later ranges are not theirs."""
    gen = prior_ops.DropoutGenerator(3)
    first, again = gen.recompute()
    with pytest.raises(KeyError):
        with first:
            gen.take(8)
            raise KeyError
    gen.take(4)
    with pytest.raises(KeyError):
        with again:
            assert gen.take(8) == 0
            raise KeyError
    assert gen.take(4) == 3 and gen.offset == 4
    with again:
        assert gen.take(8) == 0
        with pytest.raises(RuntimeError):                            # only the one range is its own
            gen.take(4)


@pytest.mark.parametrize("how", ["deepcopy", "pickle"])
def test_copies_of_a_generator(how):
    """A copy, as of a module that holds the generator, stands where the first one stood and goes its own way."""
    import copy
    import pickle
    gen = prior_ops.DropoutGenerator(3, device="cpu", capturable=True)
    gen.take(8)
    gen.advance()
    other = copy.deepcopy(gen) if how == "deepcopy" else pickle.loads(pickle.dumps(gen))
    gen.advance()
    assert gen.take(4) == 2 and (other.seed, other.offset, int(other.step)) == (3, 2, 1)
    assert other.take(4) == 2 and gen.offset == other.offset == 3


def test_where_nothing_is_dropped_no_range_is_taken(monkeypatch):
    """p = 0 draws no mask: no range, no counter; also without a generator."""
    for name in ("_Dropout", "_Tail"):
        monkeypatch.setattr(prior_ops, name, type("Node", (), {"apply": staticmethod(lambda *a: a)}))
    gen = prior_ops.DropoutGenerator(3, device="cpu", capturable=True)
    x = torch.zeros(4, 8)
    for p, g_ in ((0.0, gen), (0.0, None), (0, gen)):
        assert prior_ops.dropout(x, p, g_) == (x, None, p, 0, 0, None)
        assert prior_ops.dropout_add_layer_norm(x, x, None, None, p, g_)[4:] == (p, 0, 0, 1e-5, -1, None)
        assert gen.offset == 0
    assert prior_ops.dropout(x, 0.5, gen)[2:] == (0.5, 3, 0, gen.step) and gen.offset == 8
    assert prior_ops.dropout_add_layer_norm(x, x, None, None, 0.5, gen)[4:] == (0.5, 3, 8, 1e-5, -1, gen.step) and gen.offset == 16
    for call in (lambda: prior_ops.dropout(x, 0.5, None), lambda: prior_ops.dropout_add_layer_norm(x, x, None, None, 0.5)):
        with pytest.raises(ValueError, match="generator"):
            call()


@pytest.mark.parametrize("make", [
    lambda: torch.empty(2, 6, 4, 5), lambda: torch.empty(2, 6, 4, 5).to(memory_format=torch.channels_last), lambda: torch.empty(9, 6)[:, :4],
    lambda: torch.empty(7, 4).t(), lambda: torch.empty(3, 1, 5), lambda: torch.empty(5, 1), lambda: torch.empty(0, 3)])
def test_a_residual_is_brought_into_the_order_of_x(make):
    """What the call takes as it is stays as it is; another order of the same shape is copied into x's."""
    x = make()
    shape = tuple(x.shape)
    values = torch.arange(float(x.numel())).view(shape)
    turned = torch.empty(shape[::-1]).permute(*range(len(shape) - 1, -1, -1)).copy_(values)
    spread = torch.empty(shape[:-1] + (2 * shape[-1],))[..., ::2].copy_(values)
    for t in (values, turned, spread, torch.zeros(1).expand(shape)):
        got = prior_ops._residual_beside(x, t)
        assert torch.equal(got, t)
        prior_ops._flat(x, got)                                      # refuses what the call cannot take
    wide = torch.empty_strided(shape, x.stride()).copy_(values)
    assert prior_ops._residual_beside(x, wide) is wide and prior_ops._residual_beside(x, None) is None
    for other in (values.double(), values.to("meta"), torch.zeros(shape + (2,))):
        assert prior_ops._residual_beside(x, other) is other         # for the call to refuse


@pytest.mark.parametrize("capturable", [False, True])
def test_a_resumed_run_goes_on_where_it_was(tmp_path, capturable):
    """Saved and loaded next to a model's and an optimiser's state; the counter stays the tensor that a graph may read."""
    gen = prior_ops.DropoutGenerator(2 ** 63 + 5, device="cpu", capturable=capturable)
    gen.take(8)
    if capturable:
        gen.advance()
    torch.save({"generator": gen.state_dict()}, tmp_path / "run.pt")
    gen.take(80)
    later = prior_ops.DropoutGenerator(1, device="cpu", capturable=capturable)
    step = later.step
    later.load_state_dict(torch.load(tmp_path / "run.pt", weights_only=True)["generator"])
    assert (later.seed, later.offset) == (2 ** 63 + 5, 2) and later.step is step
    assert not capturable or int(step) == 1
    assert later.take(4) == 2
    with pytest.raises(ValueError, match="capturable"):
        prior_ops.DropoutGenerator(1, device="cpu", capturable=not capturable).load_state_dict(gen.state_dict())
    for bad in ({}, {"seed": 1, "offset": 2}, {"seed": 1, "offset": "x", "step": 1 if capturable else None}):
        with pytest.raises((KeyError, ValueError)):
            later.load_state_dict(bad)
        assert later.offset == 3 and later.seed == 2 ** 63 + 5       # nothing is half loaded


def test_a_bad_counter_leaves_a_generator_as_it_was():
    gen = prior_ops.DropoutGenerator(3, device="cpu", capturable=True)
    with pytest.raises(ValueError):
        gen.load_state_dict({"seed": 4, "offset": 5, "step": "x"})
    assert (gen.seed, gen.offset, int(gen.step)) == (3, 0, 0)


def test_a_residual_or_cotangent_that_torch_negates_is_resolved():
    x = torch.zeros(4, 1)
    for lazy in (torch.randn(4, 1, dtype=torch.complex64).conj().imag, torch._neg_view(torch.randn(4, 1))):
        for got in (prior_ops._match(x, lazy, 1), prior_ops._residual_beside(x, lazy)):
            assert not got.is_neg() and torch.equal(got, lazy)


def test_kept_structures_go_by_the_value_of_eps(monkeypatch):
    """eps may be anything that is a number, a tensor too, whose value can change between calls."""
    monkeypatch.setattr(prior_ops, "_check_kind", lambda x: None)
    monkeypatch.setattr(prior_ops, "_stream", lambda x: 0)
    x, eps = torch.zeros(4, 8), torch.tensor(0.5)
    for value in (0.5, 0.25):
        eps.fill_(value)
        c = prior_ops._call(x, -1, torch.float32, eps)
        assert prior_ops._new_dims(c.template).eps == value
