"""The gated recurrence without a GPU: its definition against differences, and the host-side refusals of the C calls."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2207_08393_b200 as g
from oracle import scan_oracle as so
from paper_2207_08393_b200 import _build, binding, scan_ops


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return g.load_library()


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("lengths", [None, [3, 0], [4, 1]])
def test_the_oracle_gradient_is_the_difference_quotient(reverse, lengths):
    rng = np.random.default_rng(1)
    x, gate, dy = (rng.normal(size=(2, 2, 4, 3)) for _ in range(3))
    state, dlast = rng.normal(size=(2, 2, 3)), rng.normal(size=(2, 2, 3))
    before = so.forward(x, gate, state, lengths, reverse)[2]
    grads = so.vjp(dy, dlast, x, gate, before, lengths, reverse)

    def f(x, gate, state):
        y, last, _ = so.forward(x, gate, state, lengths, reverse)
        return float((y * dy).sum() + (last * dlast).sum())

    for which, grad in enumerate(grads):
        args = [x, gate, state]
        for at in np.ndindex(args[which].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[which][at] += 1e-6
            down[which][at] -= 1e-6
            assert abs((f(*up) - f(*down)) / 2e-6 - grad[at]) < 1e-7


def test_struct_layout_matches_the_header():
    d = binding.gleam_scan_dims
    assert (d.batch.offset, d.stride.offset, d.lengths.offset, d.workspace_bytes.offset) == (16, 48, 168, 192)
    assert ctypes.sizeof(d) == 200


A = 1 << 30                                         # addresses that are never dereferenced
BAD, NULL, ALIAS = binding.GLEAM_ERR_BAD_DIMS, binding.GLEAM_ERR_NULL_POINTER, binding.GLEAM_ERR_ALIAS


def scan_dims(**kw):
    args = dict(dtype=0, batch=2, channels=3, steps=5, inner=8)
    args.update(kw)
    return g.make_scan_dims(**args)


def status(call, *args):
    with pytest.raises(g.GleamError) as e:
        call(*args)
    return e.value.status


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(reverse=2), dict(batch=-1), dict(channels=-1), dict(steps=-1), dict(inner=-1),
                                dict(steps=(1 << 31) + 1), dict(batch=1 << 20, channels=1 << 20), dict(lengths=A + 2)])
def test_bad_sizes(lib, kw):
    d = scan_dims(**kw)
    assert status(g.gleam_gated_scan_workspace_size, d) == BAD
    assert status(g.gleam_gated_scan_saved_size, d) == BAD
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == BAD
    assert status(g.gleam_gated_scan_vjp, A, None, 2 * A, 3 * A, None, 4 * A, 5 * A, 6 * A, None, d) == BAD


@pytest.mark.parametrize("strides", [(-120, 40, 8), (120, 40, 7), (120, 39, 8), (119, 40, 8), (120, 0, 8), (0, 40, 8), (120, 40, 0), (8, 8, 8),
                                     (1 << 62, 40, 8)])
def test_elements_that_share_memory(lib, strides):
    """Arrays of 2 x 3 x 5 x 8."""
    d = scan_dims(strides=[strides])
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == BAD
    d = scan_dims(strides=[(0, 0, 0), (0, 0, 0), strides])
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == BAD


def test_null_pointers_and_versions(lib):
    d = scan_dims()
    for at in (0, 1, 3):
        args = [A, 2 * A, None, 3 * A, None, None, d]
        args[at] = None
        assert status(g.gleam_gated_scan_forward, *args) == NULL
    d = scan_dims(steps=40)                             # states are saved between chunks of steps
    assert g.gleam_gated_scan_saved_size(d) > 0
    for at in (0, 2, 3, 5, 6, 7):
        args = [A, None, 2 * A, 3 * A, None, 4 * A, 5 * A, 6 * A, None, d]
        args[at] = None
        assert status(g.gleam_gated_scan_vjp, *args) == NULL
    d = scan_dims(steps=1)
    for at in range(4):
        args = [A, 2 * A, 3 * A, 4 * A, d]
        args[at] = None
        assert status(g.gleam_gated_step, *args) == NULL
    assert status(g.gleam_gated_step, A, 2 * A, 3 * A, 4 * A, scan_dims(steps=2)) == BAD
    assert status(g.gleam_gated_step, A, 2 * A, 3 * A, 4 * A, scan_dims(steps=1, lengths=5 * A)) == BAD
    d.struct_version = 9
    assert status(g.gleam_gated_step, A, 2 * A, 3 * A, 4 * A, d) == BAD
    assert lib.gleam_gated_step(A, A, A, A, None) == NULL


def test_alignment(lib):
    d = scan_dims(steps=40)
    for at, off in ((0, 2), (1, 1), (2, 2), (3, 2), (4, 2), (5, 8)):
        args = [A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, d]
        args[at] += off
        assert status(g.gleam_gated_scan_forward, *args) == BAD


def test_long_chains_of_few_need_a_workspace(lib):
    kw = dict(dtype=2, batch=1, channels=1, steps=51200, inner=1024)
    d = scan_dims(**kw)
    need = g.gleam_gated_scan_workspace_size(d)
    assert need > 0
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == NULL
    d = scan_dims(workspace=8 * A, workspace_bytes=need - 1, **kw)
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == binding.GLEAM_ERR_WORKSPACE_TOO_SMALL
    d = scan_dims(workspace=8 * A + 128, workspace_bytes=need, **kw)
    assert status(g.gleam_gated_scan_forward, A, 2 * A, None, 3 * A, None, None, d) == BAD
    assert g.gleam_gated_scan_workspace_size(scan_dims(dtype=2, batch=1, channels=60, steps=20, inner=30720)) == 0


def test_calls_without_elements_touch_nothing(lib):
    for kw in (dict(batch=0), dict(channels=0), dict(inner=0)):
        d = scan_dims(**kw)
        g.gleam_gated_scan_forward(None, None, None, None, None, None, d)
        g.gleam_gated_scan_vjp(None, None, None, None, None, None, None, None, None, d)
        assert g.gleam_gated_scan_saved_size(d) == g.gleam_gated_scan_workspace_size(d) == 0
        g.gleam_gated_step(None, None, None, None, scan_dims(steps=1, **kw))


@pytest.mark.parametrize("make", [lambda: torch.zeros(2, 3, 4, 5), lambda: torch.zeros(2, 3)])
def test_the_torch_layer_has_no_cpu_fallback(make):
    x = make()
    for call in (lambda: g.gated_scan(x, x), lambda: g.gated_scan_forward(x, x), lambda: g.gated_step(x, x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def strides_of(t, dim):
    c = scan_ops._Chains.__new__(scan_ops._Chains)
    c.dim, shape = dim, t.shape
    numel = scan_ops._numel
    c.sizes = (shape[0] if dim else 1, numel(shape[1:dim]), shape[dim], numel(shape[dim + 1:]))
    return c._strides(t, "t")


def test_strides_of_slices():
    wide = torch.zeros(2, 6, 5, 4, 3)
    assert strides_of(wide, 2) == (0, 0, 0)
    assert strides_of(wide[:, :3], 2) == (360, 60, 12)
    assert strides_of(wide[:, :, :4], 2) == (360, 60, 12)
    assert strides_of(wide[:, :, :, :2], 2) == (360, 60, 12)
    assert strides_of(wide[:1, :, 1:2], 2) == (1, 60, 1)
    tokens = torch.zeros(2, 7, 10)
    assert strides_of(tokens[..., :5], 1) == (70, 1, 10)
    for t, dim in ((wide[..., :2], 2), (wide[:, :, :, ::2], 2), (wide.transpose(3, 4), 2), (wide[:, ::2, ::2].expand(2, 3, 3, 4, 3)[..., :1].expand(2, 3, 3, 4, 3), 2),
                   (torch.zeros(2, 1, 5, 4).expand(2, 6, 5, 4), 2), (torch.zeros(1, 6, 5, 4).expand(2, 6, 5, 4), 2),
                   (torch.zeros(2, 6, 1, 4).expand(2, 6, 5, 4), 2)):
        with pytest.raises(ValueError, match="contiguous"):
            strides_of(t, dim)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 2, 21, 129), (1, 16, 20, 1), (1, 2, 400, 33)])
def test_a_rounded_state_shows_in_the_gates_gradient(shape, dtype):
    """The measures of tests/test_gpu_scan.py::test_norms_of_the_errors for an h_(t-1) that went through the arrays' type (float32: bfloat16)."""
    rng = np.random.default_rng(2)
    rounded = lambda v, kind=dtype: torch.from_numpy(v).to(kind).double().numpy()
    x, dy = rounded(rng.normal(size=shape)), rounded(rng.normal(size=shape))
    gate = rounded(np.clip(1.5 * rng.normal(size=shape) + 1.0, -9, 4))
    before = so.forward(x, gate)[2]
    right = so.vjp(dy, None, x, gate, before)[1]
    wrong = so.vjp(dy, None, x, gate, rounded(before, torch.bfloat16 if dtype is torch.float32 else dtype))[1]
    if dtype is torch.float32:
        assert np.sqrt(((wrong - right) ** 2).sum()) > 1e-4 * np.sqrt((right ** 2).sum())
    else:
        # h is off by a quarter of its step on average and about half as large as h - x, whose step decides: an eighth of the elements
        assert (rounded(wrong) != rounded(right)).mean() > 0.1


def test_sizes_of_steps_on_contiguous_tensors(lib):
    """Any shape whose axes fit, however many elements it has; the call's own limits hold for what comes out."""
    big = 1 << 31
    for shape, want in (((), (1, 1)), ((7,), (1, 7)), ((20, 160), (1, 3200)), ((big,), (1, big)), ((3, big), (3, big)), ((3, 1200000000), (3, 1200000000)),
                        ((2, 3, 5, 1 << 29), (6, 5 << 29) if 5 << 29 <= big else (30, 1 << 29)), ((1, 1, big, 2), (big, 2))):
        batch, inner = scan_ops._step_sizes(shape)
        assert (batch, inner) == want and batch * inner == scan_ops._numel(shape)
        assert g.gleam_gated_scan_workspace_size(scan_dims(dtype=1, batch=batch, channels=1, steps=1, inner=inner)) == 0
    for shape in ((big + 1,), (big + 1, 1), (2, big + 1)):
        with pytest.raises(ValueError, match="2\\^31"):
            scan_ops._step_sizes(shape)
