"""Host-side checks of the expert feed-forward block and of 8-bit checkpoints: the
oracle's gradients against differences of its outputs, the format's error bound,
and the refusals of the C entry points and of the binding (every call below fails
validation, which happens before any HIP call)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import ffn as X
from paper_2608_00573_amd import abi, offline

NULL, SHAPE, DTYPE, WORKSPACE = -1, -2, -3, -6
RELU, SWIGLU = abi.ACT_RELU, abi.ACT_SWIGLU


@pytest.mark.parametrize("gated", [False, True])
def test_gradient_is_the_difference_quotient(gated):
    r = np.random.default_rng(3)
    E, d, F, n = 3, 4, 5, 7
    off = [1, 4, 4, 6]  # an expert without rows, rows of no expert at both ends
    wu, wd, x, dy = (r.normal(size=s) for s in ((E, F, d), (E, d, F), (n, d), (n, d)))
    wg = r.normal(size=(E, F, d)) if gated else None
    _, u, g = X.forward(wu, wg, wd, x, off)
    grads = X.backward(wu, wg, wd, x, dy, u, g, off)

    # central differences of a smooth function of size ~10: h^2 and 1e-16 * 10 / h
    # balance at h = 1e-5, leaving about 1e-9 (relu: no u within h of 0 in these inputs)
    assert gated or np.abs(u[1:6]).min() > 1e-3
    h, tol = 1e-5, 1e-8
    args = [x, wu, wg, wd]
    for which, (arr, grad) in enumerate(zip(args, grads)):
        if arr is None:
            assert grad is None
            continue
        for idx in np.ndindex(arr.shape):
            out = []
            for step in (h, -h):
                moved = list(args)
                moved[which] = arr.copy()
                moved[which][idx] += step
                out.append(float((dy * X.forward(moved[1], moved[2], moved[3], moved[0], off)[0]).sum()))
            assert abs((out[0] - out[1]) / (2 * h) - grad[idx]) < tol, (which, idx)
    assert not grads[0][[0, 6]].any() and not grads[1][1].any() and not grads[3][1].any()


def test_codes_are_within_their_bound():
    r = np.random.default_rng(4)
    x = r.normal(size=(50, 77)) * np.exp(4 * r.normal(size=(50, 1)))
    x[3] = 0.0
    x[4, :5] = [127.4, 127.5, 127.9, -127.9, 64.0]
    q, s = X.pack(x)
    back = X.unpack(q, s)
    top = np.repeat(np.abs(np.pad(x, ((0, 0), (0, 19))).reshape(50, 3, 32)).max(2), 32, 1)[:, :77]
    assert (np.abs(back - x) <= top / 127).all()
    q2, s2 = X.pack(back)  # what was a code stays one
    assert np.array_equal(X.unpack(q2, s2), back)
    assert not back[3].any()


def test_blocks_that_are_not_finite_come_back_as_nan():
    x = np.ones((2, 64))
    x[0, 3], x[1, 40] = np.nan, np.inf
    back = X.unpack(*X.pack(x))
    assert np.isnan(back[0, :32]).all() and (back[0, 32:] == 1).all()
    assert (back[1, :32] == 1).all() and np.isnan(back[1, 32:]).all()


# ------------------------------------------------------------- refusals --
P = 1 << 20  # an aligned address that is never read


def _size(name, *dims):
    out = C.c_size_t(0)
    rc = getattr(abi.lib(), name + "_workspace_size")(*dims, C.byref(out))
    return rc, out.value


def _forward(dtype=abi.BF16, act=SWIGLU, E=4, d=64, F=128, n=10, keep=1, ws_bytes=None, **over):
    a = dict(w_up=P, w_gate=P if act == SWIGLU else None, w_down=P, x=P, offsets=P, y=P, up=P,
             up_scale=P, gate=P, gate_scale=P, ws=P)
    a.update(over)
    if ws_bytes is None:
        ws_bytes = _size("trimmoe_expert_ffn", dtype, act, E, d, F, n, keep)[1]
    return abi.lib().trimmoe_expert_ffn(dtype, act, E, d, F, n, keep, *a.values(), ws_bytes, None)


def _backward(dtype=abi.BF16, act=SWIGLU, E=4, d=64, F=128, n=10, keep=1, x_packed=0, ws_bytes=None,
              **over):
    a = dict(w_up=P, w_gate=P if act == SWIGLU else None, w_down=P, x=P, x_scale=P, dy=P, offsets=P,
             up=P, up_scale=P, gate=P, gate_scale=P, dx=P, dw_up=P,
             dw_gate=P if act == SWIGLU else None, dw_down=P, ws=P)
    a.update(over)
    if ws_bytes is None:
        ws_bytes = _size("trimmoe_expert_ffn_backward", dtype, act, E, d, F, n, x_packed)[1]
    return abi.lib().trimmoe_expert_ffn_backward(dtype, act, E, d, F, n, keep, x_packed, *a.values(),
                                                 ws_bytes, None)


@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("status,over", [
    (DTYPE, dict(dtype=2)), (DTYPE, dict(act=2)), (DTYPE, dict(keep=3)), (DTYPE, dict(keep=-1)),
    (SHAPE, dict(E=0)), (SHAPE, dict(E=257)), (SHAPE, dict(d=65)), (SHAPE, dict(d=0)),
    (SHAPE, dict(F=96)), (SHAPE, dict(F=0)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=(1 << 21) + 1)),
    (SHAPE, dict(d=(1 << 20) + 64)), (SHAPE, dict(d=1 << 20, F=1 << 20, E=2)),
    (NULL, dict(w_up=None)), (NULL, dict(w_gate=None)), (NULL, dict(w_down=None)),
    (NULL, dict(x=None)), (NULL, dict(offsets=None)), (NULL, dict(ws=None)), (NULL, dict(up=None)),
    (NULL, dict(gate=None)), (NULL, dict(keep=2, up_scale=None)),
    (NULL, dict(keep=2, gate_scale=None)),
    (SHAPE, dict(act=RELU, w_gate=P)), (SHAPE, dict(w_up=P + 8)), (SHAPE, dict(w_gate=P + 2)),
    (SHAPE, dict(w_down=P + 4)), (SHAPE, dict(x=P + 8)), (SHAPE, dict(up=P + 8)),
    (SHAPE, dict(keep=2, gate=P + 8)), (SHAPE, dict(offsets=P + 2)),
    (WORKSPACE, dict(ws=P + 128)), (WORKSPACE, dict(ws_bytes=100)),
])
def test_refusals(call, status, over):
    assert call(**over) == status


def test_refusals_of_one_direction():
    assert _forward(y=None) == NULL
    assert _forward(y=P + 8) == SHAPE
    assert _forward(dtype=abi.F32, y=P + 2) == SHAPE
    assert _backward(keep=0) == DTYPE
    assert _backward(dy=None) == NULL
    assert _backward(x_packed=1, x_scale=None) == NULL
    assert _backward(act=RELU, dw_gate=P) == SHAPE
    for name in ("dy", "dx", "dw_up", "dw_gate", "dw_down"):
        assert _backward(**{name: P + 8}) == SHAPE
        assert _backward(dtype=abi.F32, **{name: P + 2}) == SHAPE
    one = _size("trimmoe_expert_ffn_backward", abi.BF16, SWIGLU, 4, 64, 128, 10, 0)[1]
    assert _backward(x_packed=1, ws_bytes=one) == WORKSPACE  # (the rows' values need room)
    assert abi.lib().trimmoe_expert_ffn_workspace_size(abi.BF16, SWIGLU, 1, 64, 64, 1, 0, None) == NULL


def test_workspaces_hold_the_activations():
    for dtype, size in ((abi.F32, 4), (abi.BF16, 2)):
        for n in (0, 1, 40, 300, 3000, 100000):
            act = n * 256 * size
            for keep in (0, 1, 2):
                got = _size("trimmoe_expert_ffn", dtype, SWIGLU, 8, 64, 256, n, keep)[1]
                assert act * (3 if dtype == abi.F32 and keep == 2 else 1) <= got < 4 * act + (1 << 28)
            for packed in (0, 1):
                got = _size("trimmoe_expert_ffn_backward", dtype, SWIGLU, 8, 64, 256, n, packed)[1]
                assert 3 * act + packed * n * 64 * size <= got < 6 * act + (1 << 28)


@pytest.mark.parametrize("name", ["pack", "unpack"])
def test_checkpoint_refusals(name):
    f = getattr(abi.lib(), "trimmoe_checkpoint_" + name)
    assert f(2, 1, 32, P, P, P, None) == DTYPE
    for n, c in ((-1, 32), (1, 0), ((1 << 21) + 1, 32), (1, (1 << 20) + 1)):
        assert f(abi.F32, n, c, P, P, P, None) == SHAPE
    for at in range(3):
        p = [P, P, P]
        p[at] = None
        assert f(abi.BF16, 1, 32, *p, None) == NULL
    x = 0 if name == "pack" else 2
    for dtype, off in ((abi.BF16, 1), (abi.F32, 2)):
        p = [P, P, P]
        p[x] += off
        assert f(dtype, 1, 32, *p, None) == SHAPE


def _t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("over", [
    dict(w_up=_t(2, 8)), dict(w_gate=_t(2, 8, 5)), dict(w_down=_t(2, 8, 4)), dict(x=_t(3, 5)),
    dict(x=_t(3, 4, dtype=torch.bfloat16)), dict(x=_t(4, 3).t()), dict(offsets=None),
    dict(offsets=_t(3)), dict(offsets=_t(2, dtype=torch.int32)), dict(keep="8bit"),
])
def test_binding_refuses(over):
    a = dict(w_up=_t(2, 8, 4), w_gate=_t(2, 8, 4), w_down=_t(2, 4, 8), x=_t(3, 4),
             offsets=_t(3, dtype=torch.int32))
    a.update(over)
    with pytest.raises((ValueError, TypeError)):
        abi.trimmoe_expert_ffn(**a)


@pytest.mark.parametrize("over", [
    dict(dy=_t(2, 4)), dict(kept=_t(3, 8)), dict(kept=(_t(3, 8), None)), dict(kept=(_t(3, 7), _t(3, 8))),
    dict(kept=((_t(3, 8), _t(3, 1)), (_t(3, 8), _t(3, 1)))),
    dict(kept=(_t(3, 8), (_t(3, 8, dtype=torch.int8), _t(3, 1, dtype=torch.uint8)))),
    dict(x=(_t(3, 4, dtype=torch.int8), _t(3, 2, dtype=torch.uint8))), dict(x=_t(3, 5)),
])
def test_binding_refuses_in_the_backward(over):
    a = dict(w_up=_t(2, 8, 4), w_gate=_t(2, 8, 4), w_down=_t(2, 4, 8), x=_t(3, 4), dy=_t(3, 4),
             kept=(_t(3, 8), _t(3, 8)), offsets=_t(3, dtype=torch.int32))
    a.update(over)
    with pytest.raises((ValueError, TypeError)):
        abi.trimmoe_expert_ffn_backward(**a)


def test_binding_refuses_cpu_tensors_and_other_types():
    with pytest.raises(ValueError):
        abi.trimmoe_checkpoint_pack(_t(2, 32))
    with pytest.raises(TypeError):
        abi.trimmoe_checkpoint_pack(_t(2, 32, dtype=torch.float16))
    with pytest.raises(ValueError):
        abi.trimmoe_checkpoint_pack(_t(64))
    with pytest.raises(ValueError):
        abi.trimmoe_checkpoint_unpack(_t(2, 32, dtype=torch.int8), _t(2, 2, dtype=torch.uint8))


def test_rows_by_expert():
    target = torch.tensor([[2, 0], [-1, 2], [0, 5], [3, 2]], dtype=torch.int16)
    row, offsets = offline.expert_rows(target, 4)
    assert offsets.tolist() == [0, 2, 2, 5, 6] and offsets.dtype == torch.int32
    assert row.tolist() == [0, 2, 0, 1, 3, 3, 1, 2]  # experts 0, 2, 3; then no expert
    row, offsets = offline.expert_rows(torch.full((3, 1), -1, dtype=torch.int16), 2)
    assert offsets.tolist() == [0, 0, 0] and sorted(row.tolist()) == [0, 1, 2]
