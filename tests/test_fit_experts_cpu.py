"""The descent of offline.fit_experts on the CPU, its block and gradient by the fp64
oracle: what it keeps, the rows it takes, and each step against the formula."""
import numpy as np
import pytest
import torch

from oracle import ffn as X
from paper_2608_00573_amd import abi, offline

U = 2.0 ** -24


def _np(t):
    return None if t is None else t.double().numpy()


@pytest.fixture
def kept_as(monkeypatch):
    """The forms in which the forward was asked to keep its activations."""
    asked = []

    def borders(offsets, n):
        return [0, n] if offsets is None else offsets.tolist()

    def forward(wu, wg, wd, x, offsets=None, keep=None, stream=None):
        asked.append(keep)
        y, u, g = X.forward(_np(wu), _np(wg), _np(wd), _np(x), borders(offsets, len(x)))
        return torch.from_numpy(y).to(x.dtype), (u, g)

    def backward(wu, wg, wd, x, dy, kept, offsets=None, want_dx=True, want_dw=True, stream=None):
        grads = X.backward(_np(wu), _np(wg), _np(wd), _np(x), _np(dy), *kept, borders(offsets, len(x)))
        return tuple(None if g is None else torch.from_numpy(g).to(x.dtype) for g in grads)

    monkeypatch.setattr(abi, "trimmoe_expert_ffn", forward)
    monkeypatch.setattr(abi, "trimmoe_expert_ffn_backward", backward)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    return asked


def _experts(dtype, gated, E=3, d=6, F=10, n=20, seed=1):
    r = np.random.default_rng(seed)
    t = lambda *s: torch.from_numpy(r.normal(size=s) * s[-1] ** -0.5).to(dtype)  # noqa: E731
    w = (t(E, F, d), t(E, F, d) if gated else None, t(E, d, F))
    return w, t(n, d) * 2, t(n, d)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("dtype,form", [(torch.bfloat16, "packed"), (torch.float32, "full")])
def test_activations_are_kept_in_8_bits_for_bf16_rows_only(kept_as, dtype, form, gated):
    w, x, y = _experts(dtype, gated)
    offsets = torch.tensor([0, 7, 7, 18], dtype=torch.int32)
    offline.fit_experts(*w, x, y, offsets, 2, 0.1)
    assert kept_as == [form] * 2
    for keep in ("full", "packed"):
        del kept_as[:]
        offline.fit_experts(*w, x, y, offsets, 1, 0.1, keep=keep)
        assert kept_as == [keep]


def _step(w, x, y, borders, lr):
    """(weights, loss) of a step in fp64."""
    wn = [_np(v) for v in w]
    out, u, g = X.forward(*wn, _np(x), borders)
    live = np.zeros((len(x), 1), bool)
    live[max(borders[0], 0):borders[-1]] = True
    off, n = np.where(live, out - _np(y), 0.0), max(int(live.sum()), 1)
    grads = X.backward(*wn, _np(x), off / n, u, g, borders)[1:]
    return [None if v is None else v - lr * dv for v, dv in zip(wn, grads)], 0.5 * (off ** 2).sum() / n


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("borders", [[0, 7, 7, 18], [2, 7, 20, 20], [0, 0, 0, 0]])
def test_a_step_goes_down_the_gradient(kept_as, borders, gated):
    w, x, y = _experts(torch.float32, gated)
    y[:borders[0]], y[borders[-1]:] = np.nan, np.inf  # (rows of no expert have no target)
    got, losses = offline.fit_experts(*w, x, y, torch.tensor(borders, dtype=torch.int32), 1, 0.25)
    want, loss = _step(w, x, y, borders, 0.25)
    # the oracle's gradient of an output rounded to fp32 (u of it), rounded itself: the
    # chain has fewer than 64 roundings of values below 4, and gradients below 8
    for v, a, b in zip(w, got, want):
        assert (a is None) == (b is None)
        if a is not None:
            assert np.abs(b - _np(v)).max() < 0.25 * 8
            np.testing.assert_allclose(_np(a), b, rtol=0, atol=64 * U * 8)
    assert abs(float(losses[0]) - loss) <= 64 * U * (loss + 1)


@pytest.mark.parametrize("gated", [True, False])
def test_without_borders_all_rows_are_one_expert_s(kept_as, gated):
    w, x, y = _experts(torch.float32, gated, E=1)
    got, losses = offline.fit_experts(*w, x, y, None, 3, 0.25)
    want, loss = offline.fit_experts(*w, x, y, torch.tensor([0, len(x)], dtype=torch.int32), 3, 0.25)
    assert torch.equal(losses, loss)
    for a, b in zip(got, want):
        assert a is b is None or torch.equal(a, b)
