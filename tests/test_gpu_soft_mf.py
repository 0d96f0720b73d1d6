"""The operators over all items on a factorization's own handle: softmax loss, best items, device factors (MI355X)."""
import sys

import numpy as np
import pytest
import torch

import soft_ref
from paper_1410_8043_amd import synth

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1410_8043_amd import ps_mf

    return ps_mf


def softmax_loss(w, L, R):
    """In 64 bits, and its bound: each user's fp32 part is off by what soft_ref allows of one."""
    ptr = np.zeros(L.shape[0] + 1, np.int64)
    np.add.at(ptr, w.user + 1, 1)
    ptr = torch.from_numpy(ptr.cumsum())
    order = np.argsort(w.user, kind="stable")
    vals, bounds = soft_ref.xent(torch.from_numpy(L), torch.from_numpy(R), torch.from_numpy(w.item[order]), ptr,
                                 torch.from_numpy(w.val[order]))
    return vals[0].sum(), (bounds[0] + 2.0 ** -24 * np.abs(vals[0])).sum()


@pytest.mark.parametrize("K,s,B,step,policy", [(16, 2, 1, 0, 0), (33, 0, 3, 0, 2), (20, 1, 2, 2, 0), (128, 3, 1, 0, 3)])
def test_softmax_loss_and_top_items_of_a_run(gpu, K, s, B, step, policy):
    spec = synth.CONFIGS["tiny"]
    w = synth.generate(spec, K=K)
    w.L0 *= 6  # scores of some size
    w.R0 *= 6
    say(f"softmax loss K={K} s={s} B={B} step={step} policy={policy}")
    eta = 0.01 if step == 0 else 1e-3
    with gpu.PsMf(spec.N, spec.M, K, spec.P, s, eta, spec.lam, B=B, step=step, policy=policy) as g:
        with pytest.raises(gpu.PsMfError) as e:
            g.softmax_loss()
        assert e.value.code == gpu.ESTATE
        g.load_ratings(w.user, w.item, w.val)
        for call in (g.softmax_loss, lambda: g.top_items(3), lambda: g.device_factors()):
            with pytest.raises(gpu.PsMfError) as e:
                call()
            assert e.value.code == gpu.ESTATE
        g.set_factors(w.L0, w.R0)
        for clocks in (0, 4):
            g.clock(clocks)
            L, R = g.get_factors()
            squared = g.loss()
            want, bound = softmax_loss(w, L, R)
            got = g.softmax_loss()
            say(f"  {clocks} clocks: {got!r} against {want!r}, bound {bound:.3g}")
            assert abs(got - want) <= bound and g.softmax_loss() == got
            ptr = np.zeros(spec.N + 1, np.int64)
            np.add.at(ptr, w.user + 1, 1)
            ptr = torch.from_numpy(ptr.cumsum())
            lists = torch.from_numpy(w.item[np.argsort(w.user, kind="stable")])
            Lt, Rt = torch.from_numpy(L), torch.from_numpy(R)
            best, score = soft_ref.top(Lt, Rt, 12)
            items, scores = g.top_items(12, exclude_rated=False)
            assert np.array_equal(items, best) and np.allclose(scores, score, rtol=2.0 ** -23, atol=0)
            best, score = soft_ref.top(Lt, Rt, 12, ptr, lists)
            items, scores = g.top_items(12)
            assert np.array_equal(items, best)
            some = np.array([999, 3, 3, 0, 512, 7], np.int32)
            items, scores = g.top_items(12, users=some)
            assert np.array_equal(items, best[some]) and np.allclose(scores, score[some], rtol=2.0 ** -23, atol=0)
            assert g.top_items(5, users=np.zeros(0, np.int32))[0].shape == (0, 5)
            assert g.loss() == squared  # nothing of the run changed
            torch.cuda.synchronize()
            dL, dR = g.device_factors()
            assert np.array_equal(dL.cpu().numpy(), L) and np.array_equal(dR.cpu().numpy(), R)


def test_refusals(gpu):
    spec = synth.CONFIGS["tiny"]
    w = synth.generate(spec)
    with gpu.PsMf(spec.N, spec.M, spec.K, spec.P, 1, 0.01, 0.05) as g:
        g.load_ratings(w.user, w.item, w.val)
        g.set_factors(w.L0, w.R0)
        for args in (dict(k=0), dict(k=257), dict(k=3, users=[-1]), dict(k=3, users=[5, spec.N])):
            with pytest.raises(gpu.PsMfError) as e:
                g.top_items(**args)
            assert e.value.code == gpu.EINVAL, args
        with pytest.raises(gpu.PsMfError) as e:
            gpu.ps_mf_top_items(g.h, None, 5, 3)
        assert e.value.code == gpu.EINVAL
        assert np.isfinite(g.softmax_loss())


def test_users_without_ratings_and_on_another_stream(gpu):
    N, M, K = 30, 40, 8
    rng = np.random.default_rng(3)
    user, item = np.array([2, 2, 2, 9], np.int32), np.array([0, 7, 7, 39], np.int32)
    L, R = (rng.standard_normal((n, K)).astype(np.float32) for n in (N, M))
    got = []
    for stream in (None, torch.cuda.Stream()):
        with gpu.PsMf(N, M, K, 2, 1, 0.01, 0.0, stream=stream) as g:
            g.load_ratings(user, item, np.ones(4, np.float32))
            g.set_factors(L, R)
            items, _ = g.top_items(M)
            assert (items[2, -2:] == -1).all() and not {0, 7} & set(items[2]) and sorted(items[5]) == list(range(M))
            got.append(g.softmax_loss())
            gpu.ps_mf_set_stream(g.h, torch.cuda.Stream())
            assert g.softmax_loss() == got[-1]
    assert got[0] == got[1] > 0
    with gpu.PsMf(N, M, K, 2, 1, 0.01, 0.0, B=3) as g:  # no rating at all
        g.load_ratings(user[:0], item[:0], np.ones(0, np.float32))
        g.set_factors(L, R)
        assert g.softmax_loss() == 0.0 and (g.top_items(3)[0] >= 0).all()


def test_gradients_on_device_factors(gpu):
    # a batch of users' gradients from the handle's own table, without a copy of it
    from paper_1410_8043_amd import ps_soft

    spec = synth.CONFIGS["tiny"]
    w = synth.generate(spec, K=20)
    with gpu.PsMf(spec.N, spec.M, 20, spec.P, 2, 0.01, 0.05, stream=torch.cuda.current_stream()) as g, ps_soft.PsSoft(spec.M, 20) as h:
        g.load_ratings(w.user, w.item, w.val)
        g.set_factors(w.L0, w.R0)
        g.clock(3)
        torch.cuda.synchronize()
        L, R = g.device_factors()
        assert L.stride(0) == 32
        item = torch.from_numpy(w.item[:200].copy()).cuda()
        vals, bounds = soft_ref.xent(L[:200], R, item)
        got = h.xent(L[:200], R, item)
        for a, v, b in zip(got, vals, bounds):
            assert soft_ref.near(a, v, b) <= 1
