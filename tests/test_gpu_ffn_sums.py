"""How exact fp32 sums of few rows are.

A sum of K products of random signs in one chain of fp32 additions rounds K partial
sums, the k-th of size sqrt(k) of a product's.  A rounding is off by u^2 / 6 of the value
squared on average (u = 2^-24: u^2 / 3 at the lower end of a binade, u^2 / 12 at its
upper), so the sums are off by u sqrt(K / 12) of their norm together.  Four chains of K / 4
are off by half of that (and their joining by some u): the bound lies in the middle, and
with some ten thousand sums the mean is sharp to some percent."""
import pytest
import torch

from paper_2608_00573_amd import abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
K = 2048


def _off(got, want):
    """Distance from the exact sums in units of one chain's."""
    return float((got.double() - want).norm() / want.norm()) / (U * (K / 12) ** 0.5)


def _randn(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV)


@pytest.mark.parametrize("n", [9, 40])
def test_pre_activations(n):
    x, wu, wg, wd = _randn(1, n, K), _randn(2, K, K), _randn(3, K, K), _randn(4, K, K)
    _, kept = abi.trimmoe_expert_ffn(wu, wg, wd, x, keep="full")
    for k, w in zip(kept, (wu, wg)):
        assert _off(k, x.double() @ w.double().T) < 0.75


@pytest.mark.parametrize("n", [9, 40])
def test_outputs_and_gradients(n):
    """relu blocks in which all but one product are exact."""
    x, w, dy = _randn(1, n, K).abs(), _randn(2, K, K), _randn(3, n, K)
    eye = torch.eye(K, device=DEV)
    y, kept = abi.trimmoe_expert_ffn(eye, None, w, x, keep="full")
    assert torch.equal(kept[0], x) and _off(y, x.double() @ w.double().T) < 0.75
    # du = da = dy w, dx = du
    dx, *_ = abi.trimmoe_expert_ffn_backward(eye, None, w, x, dy, kept, want_dw=False)
    assert _off(dx, dy.double() @ w.double()) < 0.75
    # du = dy, dx = dy w
    dx, *_ = abi.trimmoe_expert_ffn_backward(w, None, eye, x, dy, kept, want_dw=False)
    assert _off(dx, dy.double() @ w.double()) < 0.75
