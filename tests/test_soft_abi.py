"""ps_soft without a GPU: symbols, refusals of the C ABI and of the binding, and the 64-bit reference of the
GPU tests against automatic differentiation."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import soft_ref
from paper_1410_8043_amd import ps_soft

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF = float("inf")


def test_header_and_binding_name_the_same_functions():
    with open(os.path.join(ROOT, "include", "ps_soft.h")) as f:
        text = f.read()
    names = set(re.findall(r"^(?:int|void|const char \*)\s*(ps_soft_\w+)\(", text, re.M))
    assert names == set(ps_soft.SYMBOLS)
    for name in names:
        assert getattr(ps_soft._lib, name)
    for py, c in (("EINVAL", "EINVAL"), ("ENOMEM", "ENOMEM"), ("EDEVICE", "EDEVICE"), ("ESTATE", "ESTATE"), ("F32", "F32"),
                  ("BF16", "BF16"), ("F16", "F16"), ("OPT_DEVICE", "OPT_DEVICE"), ("OPT_SPLITS", "OPT_SPLITS"),
                  ("OPT_SEARCH", "OPT_SEARCH")):
        m = re.search(r"#define PS_SOFT_%s \(?(-?\d+)\)?" % c, text)
        assert m and int(m.group(1)) == getattr(ps_soft, py)


@pytest.mark.parametrize("items,K,type", [(0, 8, 0), (-1, 8, 0), (2**31 - 64, 8, 0), (8, 0, 0), (8, 513, 0), (8, 8, -1), (8, 8, 3)])
def test_create_refuses(items, K, type):
    with pytest.raises(ps_soft.PsSoftError) as e:
        ps_soft.ps_soft_create(items, K, type)
    assert e.value.code == ps_soft.EINVAL
    h = ctypes.c_void_p(1)
    assert ps_soft._lib.ps_soft_create(items, K, type, ctypes.byref(h)) == ps_soft.EINVAL and not h.value
    assert ps_soft._lib.ps_soft_create(8, 8, 0, None) == ps_soft.EINVAL


def test_null_handles():
    lib = ps_soft._lib
    assert lib.ps_soft_set_option(None, 1, 0) == ps_soft.EINVAL
    assert lib.ps_soft_set_stream(None, None) == ps_soft.EINVAL
    assert lib.ps_soft_reserve(None, 1, 1, 1) == ps_soft.EINVAL
    assert lib.ps_soft_xent(None, *([0, None, 8, None, 8, None, None, None, 0] + [None] * 4 + [8, None, 8])) == ps_soft.EINVAL
    assert lib.ps_soft_last_error(None) == b""
    lib.ps_soft_destroy(None)


@pytest.fixture
def handle():
    h = ps_soft.ps_soft_create(10, 8, ps_soft.F32)
    yield h
    ps_soft._lib.ps_soft_destroy(h)


@pytest.mark.parametrize("key,value", [(0, 0), (99, 0), (ps_soft.OPT_DEVICE, -2), (ps_soft.OPT_DEVICE, 4096), (ps_soft.OPT_SPLITS, -1),
                                       (ps_soft.OPT_SPLITS, 1025), (ps_soft.OPT_SEARCH, -2), (ps_soft.OPT_SEARCH, 2)])
def test_options_refused(handle, key, value):
    assert ps_soft._lib.ps_soft_set_option(handle, key, value) == ps_soft.EINVAL
    assert ps_soft._lib.ps_soft_last_error(handle)


P = 4096  # a pointer that no refused call reads


def xent_args(**over):
    a = dict(n=4, X=P, ldx=8, W=P, ldw=8, row_ptr=None, item=P, value=None, entries=4, weight=None, loss=P, lse=P, dX=None, lddx=8,
             dW=None, lddw=8) | over
    return list(a.values())


@pytest.mark.parametrize("over", [dict(n=-1), dict(n=2**31), dict(X=None), dict(W=None), dict(ldx=7), dict(ldw=7), dict(dX=P, lddx=7),
                                  dict(dW=P, lddw=0), dict(entries=3), dict(entries=-1), dict(item=None), dict(row_ptr=P, entries=2**31),
                                  dict(row_ptr=P, item=None)])
def test_xent_refuses(handle, over):
    assert ps_soft._lib.ps_soft_xent(handle, *xent_args(**over)) == ps_soft.EINVAL
    assert ps_soft._lib.ps_soft_last_error(handle)


@pytest.mark.parametrize("over", [dict(n=-1), dict(k=0), dict(ldt=2), dict(tau=0.0), dict(tau=-1.0), dict(tau=INF), dict(tau=float("nan")),
                                  dict(item=None), dict(score=None), dict(X=None), dict(n=2**30, k=3, ldt=3), dict(dX=P, lddx=1)])
def test_distill_refuses(handle, over):
    a = dict(n=4, X=P, ldx=8, W=P, ldw=8, k=3, item=P, score=P, ldt=3, tau=1.0, tlse=None, weight=None, loss=P, lse=P, dX=None, lddx=8,
             dW=None, lddw=8) | over
    assert ps_soft._lib.ps_soft_distill(handle, *a.values()) == ps_soft.EINVAL
    assert ps_soft._lib.ps_soft_last_error(handle)


@pytest.mark.parametrize("over", [dict(n=-1), dict(k=0), dict(k=257, ldo=257), dict(ldo=2), dict(W=None), dict(entries=-1),
                                  dict(row_ptr=P, entries=5), dict(best=None), dict(score=None), dict(ldx=0)])
def test_top_refuses(handle, over):
    a = dict(n=4, X=P, ldx=8, W=P, ldw=8, k=3, row_ptr=None, item=None, entries=0, best=P, score=P, ldo=3) | over
    assert ps_soft._lib.ps_soft_top(handle, *a.values()) == ps_soft.EINVAL
    assert ps_soft._lib.ps_soft_last_error(handle)


@pytest.mark.parametrize("args", [(-1, 0, 0), (0, -1, 0), (0, 0, 257), (0, 0, -1), (2**31, 0, 0)])
def test_reserve_refuses(handle, args):
    assert ps_soft._lib.ps_soft_reserve(handle, *args) == ps_soft.EINVAL


def test_top_of_no_rows_needs_no_device(handle):
    assert ps_soft._lib.ps_soft_top(handle, 0, None, 8, P, 8, 3, None, None, 0, None, None, 3) == ps_soft.OK


def test_binding_refuses_cpu_tensors_and_wrong_shapes():
    with pytest.raises(ValueError):
        ps_soft.PsSoft(10, 8, torch.float64)
    with ps_soft.PsSoft(10, 8) as h:
        X, W, item = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int32)
        for call in (lambda: h.xent(X, W, item), lambda: h.top(X, W, 2), lambda: h.distill(X, W, item[:, None], X[:, :1])):
            with pytest.raises(ValueError, match="GPU"):
                call()
        with pytest.raises(ValueError, match="n x 8"):
            h.xent(torch.zeros(4, 7), W, item)
        with pytest.raises(ValueError, match="float32"):
            h.xent(X.half(), W, item)
    with pytest.raises(ValueError, match="closed"):
        h.xent(X, W, item)


def test_factorization_calls_refuse_without_factors():
    from paper_1410_8043_amd import ps_mf

    lib = ps_mf._lib
    assert lib.ps_mf_softmax_loss(None, ctypes.byref(ctypes.c_double())) == ps_mf.EINVAL
    assert lib.ps_mf_top_items(None, None, 0, 1, 0, None, None) == ps_mf.EINVAL
    assert lib.ps_mf_device_factors(None, None, None, None) == ps_mf.EINVAL
    with ps_mf.PsMf(4, 5, 3, 1, 0, 0.1, 0.0, host_only=True) as g:
        assert lib.ps_mf_softmax_loss(g.h, None) == ps_mf.EINVAL
        g.load_ratings(np.array([0, 3]), np.array([1, 2]), np.ones(2))
        for call in (g.softmax_loss, lambda: g.top_items(2), g.device_factors):
            with pytest.raises(ps_mf.PsMfError) as e:
                call()
            assert e.value.code == ps_mf.ESTATE


# ---- the reference against automatic differentiation, and that its bounds mean something
def torch_loss(x, w, y, extra, weight, tau):
    s = x @ w.T / tau
    return (weight * tau * tau * (extra + y.sum(1) * torch.logsumexp(s, 1) - (y * s).sum(1))).sum()


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_reference_gradients(tau):
    g = torch.Generator().manual_seed(5)
    n, M, K = 7, 13, 5
    x = torch.randn(n, K, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(M, K, generator=g, dtype=torch.float64, requires_grad=True)
    weight = torch.randn(n, generator=g, dtype=torch.float64)
    y = torch.rand(n, M, generator=g, dtype=torch.float64) * (torch.rand(n, M, generator=g) < 0.3)
    y[2] = 0
    extra = torch.rand(n, generator=g, dtype=torch.float64)
    live = (y != 0).any(1)
    weight[2] = 0
    torch_loss(x, w, y, extra, weight, tau).backward()
    (loss, lse, dX, dW), bounds = soft_ref.dense_loss(x.detach().numpy(), w.detach().numpy(), y.numpy(), extra.numpy(), live.numpy(),
                                                      weight.numpy(), tau)
    assert np.abs(dX - x.grad.numpy()).max() < 1e-12 and np.abs(dW - w.grad.numpy()).max() < 1e-12
    assert lse[2] == pytest.approx(np.log(M)) and loss[2] == 0
    for v, b in zip((loss, lse, dX, dW), bounds):
        assert b.shape == v.shape and (b >= 0).all() and b.max() < 1e-3 * max(1.0, np.abs(v).max())


def test_reference_distillation_is_a_divergence():
    g = torch.Generator().manual_seed(6)
    X, W = torch.randn(5, 4, generator=g), torch.randn(9, 4, generator=g)
    tau = 1.7
    s = X @ W.T
    item = torch.arange(9, dtype=torch.int32).repeat(5, 1)
    (loss, lse, dX, dW), _ = soft_ref.distill(X, W, item, s, tau)
    assert np.abs(loss).max() < 1e-5 and np.abs(dX).max() < 1e-5  # the teacher is the student
    (loss2, *_), _ = soft_ref.distill(X, W, item, s + torch.randn(5, 9, generator=g), tau)
    assert (loss2 > 0).all()
    t = torch.nn.functional
    want = t.kl_div(torch.log_softmax(s.double() / tau, 1), torch.log_softmax(2 * s.double() / tau, 1), log_target=True, reduction="none")
    (loss3, *_), _ = soft_ref.distill(X, W, item, 2 * s, tau)
    assert np.abs(loss3 - tau * tau * want.sum(1).numpy()).max() < 1e-5


def test_a_planted_mistake_is_outside_the_bounds():
    g = torch.Generator().manual_seed(7)
    X, W = torch.randn(20, 16, generator=g), torch.randn(50, 16, generator=g)
    item = torch.randint(0, 50, (20,), generator=g, dtype=torch.int32)
    vals, bounds = soft_ref.xent(X, W, item)
    for v, b in zip(vals, bounds):
        assert soft_ref.near(torch.from_numpy(v).float(), v, b) <= 1
        assert soft_ref.near(torch.from_numpy(v * (1 + 2e-3)), v, b) > 1
    other, _ = soft_ref.xent(X, W, (item + 1) % 50)
    assert soft_ref.near(torch.from_numpy(other[2]), vals[2], bounds[2]) > 1
