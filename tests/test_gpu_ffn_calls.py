"""Calls of the feed-forward block and of 8-bit activations that the GPU tests of their
results do not make."""
import numpy as np
import pytest
import torch

from oracle import ffn as X
from paper_2608_00573_amd import abi, offline
from test_gpu_ffn import BF16, DEV, F32, U, Block, _kept_np, _mat, _np

pytestmark = pytest.mark.gpu


def test_rows_past_32_bits_are_refused():
    """More rows than a call takes, with few in the lower 32 bits."""
    n = 2 ** 32 + 5
    x = torch.empty(n, 1, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="checkpoint_pack"):
        abi.trimmoe_checkpoint_pack(x)
    del x
    codes = torch.empty(n, 1, dtype=torch.int8, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="checkpoint_unpack"):
        abi.trimmoe_checkpoint_unpack(codes, codes.view(torch.uint8))
    del codes
    w = torch.ones(1, 1, 1, device=DEV)
    x = torch.empty(n, 1, device=DEV)
    offsets = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    with pytest.raises(abi.TrimmoeError, match="expert_ffn"):
        abi.trimmoe_expert_ffn(w, w, w, x, offsets)
    with pytest.raises(abi.TrimmoeError, match="expert_ffn_backward"):
        abi.trimmoe_expert_ffn_backward(w, None, w, x, x, (x, None), offsets, want_dx=False)


def _check_y(b, y):
    """y within Block.check_forward's bound, computed in fp64 on the GPU."""
    h = 2.0 ** -8
    for e, (i, j) in enumerate(X.groups(b.off, b.n)):
        if i == j:
            continue
        wu, wd, x = b.w[0][e].double(), b.w[2][e].double(), b.xd[i:j].double()
        u, eu = x @ wu.T, (b.d + 8) * U * (x.abs() @ wu.abs().T)
        if b.gated:
            wg = b.w[1][e].double()
            g, eg = x @ wg.T, (b.d + 8) * U * (x.abs() @ wg.abs().T)
            s = torch.sigmoid(g)
            a = s * g * u
            ea = (s * g).abs() * eu + 1.1 * u.abs() * eg + 1.1 * eu * eg + (8 + 2 * g.abs()) * U * a.abs() * 1.01
        else:
            a, ea = u.clamp_min(0.0), eu
        ra = ea + h * (a.abs() + ea)
        want = a @ wd.T
        ey = (ra @ wd.abs().T + (b.F + 8) * U * (a.abs() @ wd.abs().T)) * 1.01
        bad = ~((y[i:j].double() - want).abs() <= ey + h * (want.abs() + ey))
        assert not bad.any(), (e, int(bad.sum()), bad.nonzero()[:4].tolist())
    out = torch.ones(b.n, dtype=torch.bool, device=DEV)
    out[int(b.off[0]):int(b.off[-1])] = False
    assert not y[out].any()


@pytest.mark.parametrize("gated,d,F,sizes", [
    (True, 1024, 4096, [900, 0, 901]),       # y in large tiles, all of them in pieces of K,
    (False, 1024, 4160, [1799]),             # ... 65 slices of it,
    (True, 4096, 4096, [2300, 2, 2250]),     # ... and behind whole tiles
    (False, 4032, 4160, [4500, 300]),        # columns cut short too
])
def test_large_tiles_of_y_in_pieces(gated, d, F, sizes):
    b = Block(70, BF16, gated, d, F, sizes, 1, 2)
    y, _ = b.forward(None)
    _check_y(b, y)
    assert torch.equal(y, b.forward("packed")[0])


@pytest.mark.parametrize("case", [(F32, True, 41, 97, [130, 0, 3], 2, 3), (F32, False, 33, 1500, [3], 1, 2),
                                  (BF16, False, 64, 256, [5, 0, 9, 1], 0, 1),
                                  (BF16, True, 192, 128, [600, 1, 700], 1, 0)])
def test_rows_in_8_bits_of_other_sizes(case):
    b = Block(71, *case)
    _, kept = b.forward("full")
    x8 = abi.trimmoe_checkpoint_pack(b.xd)
    x = X.unpack(x8.codes.cpu().numpy(), x8.scale.cpu().numpy())
    got = b.backward(kept, x=x8)
    b.check_backward(got, _kept_np(kept), x=x)
    dx, *dw = b.backward(kept, x=x8, want_dw=False)
    assert torch.equal(dx, got[0]) and dw == [None] * 3


def test_codes_at_any_address():
    x = torch.randn(10, 40, device=DEV)
    p = abi.trimmoe_checkpoint_pack(x)
    codes = torch.empty(403, dtype=torch.int8, device=DEV)
    scale = torch.empty(23, dtype=torch.uint8, device=DEV)
    for dtype in (BF16, F32):
        want = abi.trimmoe_checkpoint_unpack(*p, dtype=dtype)
        for at in (1, 2, 3):
            q, s = codes[at:at + 400].view(10, 40), scale[at:at + 20].view(10, 2)
            q.copy_(p.codes)
            s.copy_(p.scale)
            assert torch.equal(abi.trimmoe_checkpoint_unpack(q, s, dtype=dtype), want)


@pytest.mark.parametrize("gated", [True, False])
def test_bf16_experts_fitted_with_activations_in_8_bits(gated):
    """A step as fit_experts makes it by default: the gradient that it takes is the
    oracle's of what was kept, and the weights move by it."""
    b = Block(72, BF16, gated, 128, 192, [40, 0, 25], 1, 2)
    y, yn = _mat(72, 9, (b.n, b.d), 1.0, BF16)
    y = y.to(DEV)
    y[0], y[-2:] = float("nan"), float("inf")
    lr, n = 2.0, 65
    out, kept = b.forward("packed")
    b.check_forward(out, kept, "packed")
    live = torch.zeros(b.n, 1, dtype=torch.bool, device=DEV)
    live[1:66] = True
    off = torch.where(live, out.float() - y.float(), 0.0)
    dy = (off / n).to(BF16)
    b.dyd, b.dy = dy, (dy, _np(dy))
    _, *dw = b.backward(kept, want_dx=False)
    b.check_backward((None, *dw), _kept_np(kept))
    got, losses = offline.fit_experts(*b.w, b.xd, y, b.offd, 1, lr)
    for w, g, t in zip(b.w, dw, got):
        if w is None:
            assert g is None and t is None
            continue
        w, g = _np(w), _np(g)
        want = w - lr * g
        # rounded to bf16 once, after two operations in fp32
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * (np.abs(w) + lr * np.abs(g))
        assert (np.abs(_np(t) - want) <= bound).all() and np.abs(lr * g).max() > 0.01
        assert not g[1].any()  # an expert without rows stays
    # a sum of 65 * 128 squares in fp32, in any order
    loss = 0.5 * (np.where(live.cpu().numpy(), _np(out) - yn, 0.0) ** 2).sum() / n
    assert abs(float(losses[0]) - loss) <= 10000 * U * loss
