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
