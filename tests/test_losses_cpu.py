"""Host-side checks of the training losses: the oracle's gradients against
differences of its losses, and the refusals of the C entry points (every call
below fails validation, which happens before any HIP call)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import losses as X
from paper_2608_00573_amd import abi, offline

NULL, SHAPE, DTYPE, WORKSPACE = -1, -2, -3, -6


def _rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("with_bias", [False, True])
def test_head_gradient_is_the_difference_quotient(with_bias):
    r = _rng(1)
    V, d, Q = 11, 5, 7
    W, H, g = r.normal(size=(V, d)), r.normal(size=(Q, d)), r.normal(size=Q)
    b = r.normal(size=V) if with_bias else None
    y = np.array([0, 3, 10, -1, 11, 5, 3])
    dH, dW, db = X.head_loss_grad(W, H, y, g, b)

    def total(W_, H_, b_):
        return float(g @ X.head_loss(W_, H_, y, b_)[0])

    # central differences of a smooth function of size ~10: h^2 and 1e-16 * 10 / h
    # balance at h = 1e-5, leaving about 1e-9
    h, tol = 1e-5, 1e-8
    for arr, grad, which in ((W, dW, 0), (H, dH, 1)) + (((b, db, 2),) if with_bias else ()):
        for idx in np.ndindex(arr.shape):
            lo, hi = arr.copy(), arr.copy()
            lo[idx] -= h
            hi[idx] += h
            args = [W, H, b]
            args[which] = hi
            up = total(*args)
            args[which] = lo
            assert abs((up - total(*args)) / (2 * h) - grad[idx]) < tol, (which, idx)
    assert not dH[3].any() and not dH[4].any()


def test_balance_gradient_is_the_difference_quotient():
    r = _rng(2)
    E, d, Q = 6, 5, 9
    W, H, b = r.normal(size=(E, d)), r.normal(size=(Q, d)), r.normal(size=E)
    t = r.integers(-1, E, size=(Q, 2))
    t[4] = -1
    dH, dW, db, _ = X.balance_grad(W, H, t, 0.7, b)
    h, tol = 1e-5, 1e-9
    for arr, grad, which in ((W, dW, 0), (H, dH, 1), (b, db, 2)):
        for idx in np.ndindex(arr.shape):
            args_hi, args_lo = [W, H, b], [W, H, b]
            args_hi[which], args_lo[which] = arr.copy(), arr.copy()
            args_hi[which][idx] += h
            args_lo[which][idx] -= h
            up = X.balance_loss(args_hi[0], args_hi[1], t, args_hi[2])[0]
            dn = X.balance_loss(args_lo[0], args_lo[1], t, args_lo[2])[0]
            assert abs(0.7 * (up - dn) / (2 * h) - grad[idx]) < tol, (which, idx)
    assert not dH[4].any()


def test_balance_loss_of_an_even_load_is_one():
    E, Q = 4, 8
    W, H = np.zeros((E, 3)), np.ones((Q, 3))
    t = (np.arange(Q) % E).reshape(Q, 1)
    loss, counts, ps, p = X.balance_loss(W, H, t)
    assert loss == 1.0 and counts.tolist() == [2, 2, 2, 2, 8]
    assert X.balance_loss(W, H, np.full((Q, 2), -1))[0] == 0.0


def test_rows_without_any_logit_take_no_part():
    W, H = np.ones((3, 2)), np.ones((2, 2))
    b = np.full(3, -np.inf)
    loss, lse = X.head_loss(W, H, [0, 1], b)
    assert (loss == 0).all() and np.isneginf(lse).all()
    D, _, live = X.head_loss_d(W, H, [0, 1], [1, 1], b)
    assert not D.any() and not live.any()


# --------------------------------------------------------------- refusals --
A = 4096                 # a non-null, aligned address that no call below reaches
BIG = 1 << 62            # a workspace size that is always enough


def _p(x):
    return C.c_void_p(x)


def _loss(dtype=1, V=512, d=64, Q=8, w=A, b=0, h=A, y=A, loss=A, lse=A, ws=A, n=BIG):
    return abi.lib().trimmoe_head_cross_entropy(dtype, V, d, Q, _p(w), _p(b), _p(h), _p(y),
                                                _p(loss), _p(lse), _p(ws), n, None)


def _loss_b(dtype=1, V=512, d=64, Q=8, w=A, b=0, h=A, y=A, lse=A, g=A, dh=A, dw=A, db=0, ws=A,
            n=BIG):
    return abi.lib().trimmoe_head_cross_entropy_backward(
        dtype, V, d, Q, _p(w), _p(b), _p(h), _p(y), _p(lse), _p(g), _p(dh), _p(dw), _p(db), _p(ws),
        n, None)


def _bal(dtype=1, E=8, k=2, d=64, Q=8, w=A, b=0, h=A, t=A, loss=A, c=A, ps=A, p=A, ws=A, n=BIG):
    return abi.lib().trimmoe_balance_loss(dtype, E, k, d, Q, _p(w), _p(b), _p(h), _p(t), _p(loss),
                                          _p(c), _p(ps), _p(p), _p(ws), n, None)


def _bal_b(dtype=1, E=8, k=2, d=64, Q=8, w=A, h=A, t=A, p=A, c=A, g=A, dh=A, dw=A, db=A, ws=A,
           n=BIG):
    return abi.lib().trimmoe_balance_loss_backward(
        dtype, E, k, d, Q, _p(w), _p(h), _p(t), _p(p), _p(c), _p(g), _p(dh), _p(dw), _p(db), _p(ws),
        n, None)


BAD_DIMS = [(dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE), (dict(d=96), SHAPE),
            (dict(d=0), SHAPE), (dict(dtype=0, d=0), SHAPE), (dict(d=(1 << 20) + 64), SHAPE),
            (dict(Q=-1), SHAPE), (dict(Q=(1 << 21) + 1), SHAPE)]
BAD_BUFFERS = [(dict(w=0), NULL), (dict(ws=0), NULL), (dict(h=0), NULL), (dict(w=A + 8), SHAPE),
               (dict(h=A + 2), SHAPE), (dict(dtype=0, h=A + 2), SHAPE), (dict(ws=A + 128), WORKSPACE),
               (dict(n=64), WORKSPACE)]


@pytest.mark.parametrize("over,code", BAD_DIMS + BAD_BUFFERS + [
    (dict(V=0), SHAPE), (dict(V=(1 << 28) + 1), SHAPE), (dict(y=0), NULL), (dict(loss=0), NULL),
    (dict(lse=0), NULL)])
def test_head_loss_refuses(over, code):
    assert _loss(**over) == code


@pytest.mark.parametrize("over,code", BAD_DIMS + BAD_BUFFERS + [
    (dict(V=0), SHAPE), (dict(y=0), NULL), (dict(lse=0), NULL), (dict(g=0), NULL),
    (dict(dh=A + 4), SHAPE), (dict(dw=A + 8), SHAPE)])
def test_head_loss_backward_refuses(over, code):
    assert _loss_b(**over) == code


@pytest.mark.parametrize("over,code", BAD_DIMS + BAD_BUFFERS + [
    (dict(E=0), SHAPE), (dict(E=257), SHAPE), (dict(k=0), SHAPE), (dict(k=9, E=16), SHAPE),
    (dict(k=3, E=2), SHAPE), (dict(t=0), NULL), (dict(loss=0), NULL), (dict(c=0), NULL),
    (dict(ps=0), NULL), (dict(p=0), NULL)])
def test_balance_loss_refuses(over, code):
    assert _bal(**over) == code


@pytest.mark.parametrize("over,code", BAD_DIMS + BAD_BUFFERS + [
    (dict(E=257), SHAPE), (dict(k=9, E=16), SHAPE), (dict(t=0), NULL), (dict(p=0), NULL),
    (dict(c=0), NULL), (dict(g=0), NULL), (dict(dh=A + 8), SHAPE), (dict(dw=A + 2), SHAPE)])
def test_balance_loss_backward_refuses(over, code):
    assert _bal_b(**over) == code


def test_calls_without_rows_and_without_gradients_return_at_once():
    # no rows: the row arrays may be NULL, and the forward has nothing to launch
    assert _loss(Q=0, h=0, y=0, loss=0, lse=0) == 0
    # no gradient asked for
    assert _loss_b(dh=0, dw=0, db=0) == 0
    assert _bal_b(dh=0, dw=0, db=0) == 0


SIZES = [("trimmoe_head_cross_entropy", (512, 64)), ("trimmoe_head_cross_entropy", (151936, 2048)),
         ("trimmoe_head_cross_entropy_backward", (512, 64)),
         ("trimmoe_head_cross_entropy_backward", (32000, 4096)),
         ("trimmoe_balance_loss", (60, 4, 2048)), ("trimmoe_balance_loss_backward", (60, 4, 2048))]


@pytest.mark.parametrize("name,dims", SIZES)
@pytest.mark.parametrize("dtype", [0, 1])
def test_workspace_sizes(name, dims, dtype):
    f = getattr(abi.lib(), name + "_workspace_size")
    n = C.c_size_t(0)
    assert f(dtype, *dims, 8, None) == NULL
    assert f(2, *dims, 8, C.byref(n)) == DTYPE
    assert f(dtype, *dims, -1, C.byref(n)) == SHAPE
    for rows in (0, 1, 37, 64, 65, 1000, 8192, 100000, 1 << 21):
        assert f(dtype, *dims, rows, C.byref(n)) == 0 and n.value % 256 == 0
    # far less than the logits of a large batch
    if "cross_entropy" in name and dims[0] > 1000:
        assert f(dtype, *dims, 1 << 20, C.byref(n)) == 0
        assert n.value < (1 << 20) * dims[0] * 2


def test_wrappers_refuse_host_and_mismatched_tensors():
    w, h = torch.zeros(8, 64), torch.zeros(4, 64)
    y = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        abi.trimmoe_head_cross_entropy(w, h, y)                    # not on a GPU
    with pytest.raises(ValueError):
        abi.trimmoe_head_cross_entropy(w, h, y.long())             # not int32
    with pytest.raises(ValueError):
        abi.trimmoe_head_cross_entropy(w[:, :32], h, y)            # another d
    with pytest.raises(ValueError):
        abi.trimmoe_head_cross_entropy(w, h.t().contiguous().t(), y)  # not contiguous
    with pytest.raises(TypeError):
        abi.trimmoe_head_cross_entropy(w.half(), h.half(), y)
    with pytest.raises(ValueError):
        abi.trimmoe_balance_loss(w, h, y)                          # target not [Q, k] int16


# ---------------------------------------------------------- offline descent --
@pytest.fixture
def oracle_losses(monkeypatch):
    """offline.balance_routers on the CPU, its losses and gradients by the oracle."""
    def forward(w, h, t, b=None):
        l, c, s, p = X.balance_loss(w.numpy(), h.numpy(), t.numpy(), None if b is None else b.numpy())
        return (torch.tensor([l]).float(), torch.from_numpy(c).int(), torch.from_numpy(s).float(),
                torch.from_numpy(p).float())

    def backward(w, h, t, prob, counts, dloss, want_dh=True):
        # (dz from prob alone: the bias is in it)
        E, cn = w.shape[0], counts.numpy().astype(np.float64)
        p, c = prob.double().numpy(), cn[:E]
        live = ((t >= 0) & (t < E)).any(1).numpy()
        dz = float(dloss) * E / (c.sum() * cn[E]) * p * (c - (p @ c)[:, None]) * live[:, None]
        f = lambda x: torch.from_numpy(x).float()
        return None, f(dz.T @ h.double().numpy()), f(dz.sum(0))

    monkeypatch.setattr(abi, "trimmoe_balance_loss", forward)
    monkeypatch.setattr(abi, "trimmoe_balance_loss_backward", backward)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)


def _skewed_router(E=8, k=2, d=16, Q=512):
    r = _rng(7)
    w = torch.from_numpy(r.normal(size=(E, d)).astype(np.float32) * d ** -0.5)
    b = torch.from_numpy((-0.5 * np.log(1 + np.arange(E))).astype(np.float32))
    h = torch.from_numpy(r.normal(size=(Q, d)).astype(np.float32))
    t = np.argsort(-X.logits(w.numpy(), h.numpy(), b.numpy()), axis=1, kind="stable")[:, :k]
    t[r.random(Q) < 0.1] = -1                       # inactive rows
    t[3], t[4] = [-1, t[3, 0]], [t[4, 0], E]        # rows of fewer slots
    return w, b, h, torch.from_numpy(t.astype(np.int16))


def _load(w, b, h, t):
    """Slots per expert of the router (w, b) over the rows that t routes."""
    E = w.shape[0]
    order = np.argsort(-X.logits(w.numpy(), h.numpy(), b.numpy()), axis=1, kind="stable")
    live = ((t >= 0) & (t < E)).numpy().sum(1)
    return np.bincount(np.concatenate([o[:n] for o, n in zip(order, live)]), minlength=E)


def test_balanced_routers_balance_the_load_they_make(oracle_losses):
    # a step moves probability away from the experts that the router of that step loads
    # most: over many steps the load itself becomes even and stays so
    w, b, h, t = _skewed_router()
    start = _load(w, b, h, t)
    assert start.max() > 1.5 * start.mean()
    for epochs in (20, 100):
        (w1, b1, losses, counts), = offline.balance_routers([(w, b)], [h], [t], epochs, 0.5)
        load = _load(w1, b1, h, t)
        assert load.sum() == start.sum() and load.max() / load.mean() - 1 < (start.max() / start.mean() - 1) / 2, \
            (epochs, load)


def test_balanced_routers_report_the_loss_of_their_own_routing(oracle_losses):
    w, b, h, t = _skewed_router()
    live = ((t >= 0) & (t < 8)).any(1)
    whole = [offline.balance_routers([(w, b)], [h], [t], n, 0.5)[0] for n in range(5)]
    for n in range(1, 5):
        # step n starts from the router that n - 1 steps end with
        w0, b0 = whole[n - 1][:2]
        load = _load(w0, b0, h, t)
        losses, counts = whole[n][2], whole[n][3]
        assert counts.tolist() == [*load.tolist(), int(live.sum())]
        p = X.balance_loss(w0.numpy(), h.numpy(), t.numpy(), b0.numpy())[2]
        want = 8 * float(load @ p) / (float(load.sum()) * int(live.sum()))
        assert abs(float(losses[n - 1]) - want) <= 4 * 2.0 ** -24 * want  # rounded to fp32
        assert torch.equal(whole[4][2][:n], losses)


def test_balanced_routers_without_a_bias_start_from_zero(oracle_losses):
    w, b, h, t = _skewed_router()
    got = offline.balance_routers([(w, None)], [h], [t], 3, 0.5)[0]
    want = offline.balance_routers([(w, torch.zeros(8))], [h], [t], 3, 0.5)[0]
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and got[1].any()


def test_softmax_heads_step_down_the_gradient(monkeypatch):
    # a step of lr lowers the mean loss by lr |g|^2, up to the second order: the Hessian of a
    # row's loss in (w, b) is at most (|h|^2 + 1) / 2, and lr^2 / 2 times it times |g|^2 is
    # what a step may differ by
    def forward(w, h, y, b=None):
        loss, lse = X.head_loss(w.numpy(), h.numpy(), y.numpy(), b.numpy())
        return torch.from_numpy(loss).float(), torch.from_numpy(lse).float()

    def backward(w, h, y, lse, g, b=None, want_dh=True):
        _, dw, db = X.head_loss_grad(w.numpy(), h.numpy(), y.numpy(), g.numpy(), b.numpy())
        return None, torch.from_numpy(dw).float(), torch.from_numpy(db).float()

    monkeypatch.setattr(abi, "trimmoe_head_cross_entropy", forward)
    monkeypatch.setattr(abi, "trimmoe_head_cross_entropy_backward", backward)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    r = _rng(8)
    V, d, Q, lr = 13, 6, 40, 0.1
    w = torch.from_numpy(r.normal(size=(V, d)).astype(np.float32))
    h = torch.from_numpy(r.normal(size=(Q, d)).astype(np.float32))
    y = torch.from_numpy(r.integers(-1, V, size=Q).astype(np.int32))
    live = (y >= 0).numpy()
    (w1, b1, losses), = offline.train_softmax_heads([h], y, w, 1, lr)
    start, end = (float(X.head_loss(a.numpy(), h.numpy(), y.numpy(), b.numpy())[0].sum()) /
                  live.sum() for a, b in ((w, torch.zeros(V)), (w1, b1)))
    g2 = (float((w1 - w).double().square().sum()) + float(b1.double().square().sum())) / lr ** 2
    most = float((h.double().square().sum(1) + 1)[y >= 0].mean()) / 2
    u = 2.0 ** -24
    assert abs(float(losses[0]) - start) <= 100 * u * start   # a sum of 40 fp32 terms and weights
    assert abs(end - start + lr * g2) <= lr ** 2 / 2 * most * g2 * 1.01
    assert lr * most / 2 < 0.9 and g2 > 0.05                  # (so that the loss does fall)
