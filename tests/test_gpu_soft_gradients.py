"""ps_soft's item gradients on the device, number by number, and its teachers' scores, against 64 bits.

Bounds: those of soft_ref for fp32 tables, whatever the tables' type (scores, weights in two planes of 11 bits,
sums), and one rounding to the gradient's type: half of its step at the number's own size.
"""
import sys

import numpy as np
import pytest
import torch

import soft_ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# bits behind the first, and the smallest step's exponent
STEP = {F32: (23, -149), BF16: (7, -133), F16: (10, -24)}


@pytest.fixture(scope="module")
def soft():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1410_8043_amd import ps_soft

    return ps_soft


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def half_step(size, dtype):
    bits, least = STEP[dtype]
    _, e = np.frexp(size)  # size in [2^(e-1), 2^e)
    return np.exp2(np.maximum(e - 1 - bits, least) - 1.0)


def off(got, want, bound, dtype):
    """The largest |got - want| over its bound and one rounding to dtype."""
    got = soft_ref.f64(got)
    assert np.isfinite(got).all()
    return float((np.abs(got - want) / (bound + half_step(np.abs(want) + bound, dtype))).max())


def tables(n, M, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    X, W = torch.randn(n, K, generator=g) * 0.3, torch.randn(M, K, generator=g) * 0.3
    return X.to(dtype).cuda(), W.to(dtype).cuda(), g


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,M,K,splits", [(64, 100, 16, 0), (90, 130, 33, 2), (48, 70, 128, 0), (40, 65, 256, 0), (33, 40, 400, 0)])
def test_item_gradients_are_rounded_once(soft, n, M, K, splits, dtype):
    # weights rounded to fewer bits than two planes hold send numbers to the neighbour of the nearest
    X, W, g = tables(n, M, K, dtype, K)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    weight = (torch.rand(n, generator=g) + 0.5).cuda()
    want, bounds = soft_ref.xent(X.float(), W.float(), item, weight=weight)
    score = torch.randn(n, 5, generator=g).cuda()
    ids = torch.stack([torch.randperm(M, generator=g)[:5] for _ in range(n)]).int().cuda()
    want2, bounds2 = soft_ref.distill(X.float(), W.float(), ids, score, 2.0, weight=weight)
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        for name, got, v, b in (("xent", h.xent(X, W, item, weight=weight), want, bounds),
                                ("distill", h.distill(X, W, ids, score, tau=2.0, weight=weight), want2, bounds2)):
            for part, q in (("dX", 2), ("dW", 3)):
                most = off(got[q], v[q], b[q], dtype)
                say(f"{name} n={n} M={M} K={K} {dtype} {part}: {most:.3f} of its bound")
                assert most <= 1, (name, part, most)


def item_gradients(x, w, y, weight, tau=1.0):
    """dW in 64 bits, and what fp32 sums of weights in two planes may be off, item by item: scores, log-sum-exps and
    exponentials as in soft_ref, and each weight 2^-25 where the item's own largest one is at least 2^6."""
    n, K = x.shape
    M = w.shape[0]
    U = soft_ref.U
    s, a = x @ w.T / tau, np.abs(x) @ np.abs(w).T / tau
    top = s.max(1, keepdims=True)
    lse = np.log(np.exp(s - top).sum(1, keepdims=True)) + top
    g = (weight * tau)[:, None]
    soft = g * y.sum(1, keepdims=True) * np.exp(s - lse)
    want = (soft - g * y).T @ x
    es = (K + 16) * 2 * U * a
    ep = es + es.max(1, keepdims=True) + (M + 64) * U + 4 * U * np.abs(lse) + 2.0 ** -20 + (M + n + 64) * U
    ey = (n + M + 16) * U
    bound = (np.abs(soft) * ep + np.abs(g * y) * ey).T @ np.abs(x)
    largest = np.maximum(np.abs(soft), np.abs(g * y)).max(0)
    bound += 2.0 ** -31 * largest[:, None] * np.abs(x).sum(0) + 2.0 ** -37 * (np.abs(soft) + np.abs(g * y)).sum(0)[:, None] * np.abs(x).max()
    return want, bound


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("dtype,depth", [(F32, 10), (F32, 20), (F32, 28), (F32, 60), (BF16, 20), (BF16, 28), (BF16, 60), (F16, 10)])
def test_improbable_items_beside_targets(soft, dtype, depth, splits):
    # every other item has probabilities of e^-depth of its neighbours', which are targets: their gradients keep their digits
    n, M, K = 300, 64, 4
    X, W, g = tables(n, M, K, dtype, depth)
    X[:, 0] = 4
    W[:, 0] = -(torch.arange(M) % 2).to(dtype).cuda() * depth / 4
    item = (torch.randint(0, M // 2, (n,), generator=g, dtype=torch.int32) * 2).cuda()
    y = np.zeros((n, M))
    y[np.arange(n), item.cpu()] = 1
    want, bound = item_gradients(soft_ref.f64(X), soft_ref.f64(W), y, np.ones(n))
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        most = off(h.xent(X, W, item)[3], want, bound, dtype)
    say(f"improbable e^-{depth} {dtype} splits={splits}: {most:.3f} of its bound")
    assert most <= 1


@pytest.mark.parametrize("power", [10, 20, 40])
def test_one_heavy_row(soft, power):
    # a row of weight 2^power that only knows one item: the other items' gradients are the light rows'
    n, M, K = 200, 100, 8
    X, W, g = tables(n, M, K, F32, power)
    W[:, 0] = 0
    W[33, 0] = 32
    X[:, 0] = 0
    X[50] = 0
    X[50, 0] = 4
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32)
    item[50] = 33
    weight = torch.ones(n)
    weight[50] = 2.0 ** power
    y = np.zeros((n, M))
    y[np.arange(n), item] = 1
    want, bound = item_gradients(soft_ref.f64(X), soft_ref.f64(W), y, weight.numpy().astype(np.float64))
    with soft.PsSoft(M, K) as h:
        most = off(h.xent(X, W, item.cuda(), weight=weight.cuda())[3], want, bound, F32)
    say(f"heavy row 2^{power}: {most:.3f} of its bound")
    assert most <= 1


@pytest.mark.parametrize("splits", [0, 1, 4])
@pytest.mark.parametrize("spread", [0, 12, 60])
def test_shares_and_values_of_either_sign_and_far_sizes(soft, spread, splits):
    # rows whose values add up to something negative or to nothing, weights of either sign over 2^spread, a row after another
    # growing or shrinking, items twice in a list, values of 0
    n, M, K = 260, 97, 12
    X, W, g = tables(n, M, K, F32, spread + 1)
    value = torch.randn(n, 6, generator=g)
    value[:, 5] = -value[:, :5].sum(1) * (torch.arange(n) % 3 == 0)
    value[::7, 2] = 0
    item = torch.randint(0, M, (n, 6), generator=g, dtype=torch.int32)
    item[::5, 1] = item[::5, 0]
    e = torch.rand(n, generator=g) * spread
    e[:100] = e[:100].sort().values  # rows that grow, and rows that shrink
    e[100:200] = e[100:200].sort(descending=True).values
    weight = torch.exp2(e) * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)
    y = np.zeros((n, M))
    np.add.at(y, (np.arange(n)[:, None], item.numpy()), soft_ref.f64(value))
    wt = soft_ref.f64(weight)
    want, bound = item_gradients(soft_ref.f64(X), soft_ref.f64(W), y, wt)
    # a sum of six fp32 values is off by 6 u of the values', where they cancel
    sizes = soft_ref.f64(value.abs()).sum(1)
    p = np.exp(soft_ref.f64(X) @ soft_ref.f64(W).T)
    p /= p.sum(1, keepdims=True)
    ya = np.zeros((n, M))
    np.add.at(ya, (np.arange(n)[:, None], item.numpy()), soft_ref.f64(value.abs()))
    bound += 6 * soft_ref.U * (np.abs(wt)[:, None] * (sizes[:, None] * p + 2 * ya)).T @ np.abs(soft_ref.f64(X))
    ptr = torch.arange(0, 6 * n + 1, 6).cuda()
    with soft.PsSoft(M, K, splits=splits) as h:
        got = h.xent(X, W, item.flatten().cuda(), row_ptr=ptr, value=value.flatten().cuda(), weight=weight.cuda())[3]
        again = h.xent(X, W, item.flatten().cuda(), row_ptr=ptr, value=value.flatten().cuda(), weight=weight.cuda(), grad="W")[3]
    most = off(got, want, bound, F32)
    say(f"shares over 2^{spread} splits={splits}: {most:.3f} of its bound")
    assert most <= 1 and torch.equal(got, again)


def test_tiny_and_huge_weights(soft):
    # all rows' weights scaled by a power of two scale the gradients exactly; the smallest and the largest of them together
    n, M, K = 70, 80, 10
    X, W, g = tables(n, M, K, F32, 5)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    weight = torch.randn(n, generator=g).cuda()
    with soft.PsSoft(M, K) as h:
        base = h.xent(X, W, item, weight=weight)
        for e in (-90, -40, 30, 100):
            far = h.xent(X, W, item, weight=weight * 2.0 ** e)
            assert torch.equal(far[2] * 2.0 ** -e, base[2]) and torch.equal(far[3] * 2.0 ** -e, base[3]), e
        weight[::2] *= 2.0 ** -120
        weight[1] = 2.0 ** 100
        out = h.xent(X, W, item, weight=weight)
        assert all(torch.isfinite(t).all() for t in out)


@pytest.mark.parametrize("tau,full", [(1.0, False), (0.75, False), (3.3, False), (2.0, True), (0.5, True)])
@pytest.mark.parametrize("far", [300, -3000, 30_000])
def test_teachers_of_far_scores(soft, far, tau, full):
    # a number added to all of a teacher's scores changes nothing: the sums are exact here (multiples of 2^-8 below 2^15), so the
    # bounds are those of the scores without it
    n, M, K, k = 70, 300, 16, 20
    X, W, g = tables(n, M, K, F32, far % 97)
    score = (torch.randn(n, k, generator=g) * 512).round() / 256
    score[3, 5:] = -float("inf")
    ids = torch.stack([torch.randperm(M, generator=g)[:k] for _ in range(n)]).int()
    ids[4] = -1
    ids, score = ids.cuda(), score.cuda()
    tlse = (torch.logsumexp(score / tau, 1) * 256 + 100).round() / 256 if full else None
    weight = torch.rand(n, generator=g).cuda()
    want, bounds = soft_ref.distill(X, W, ids, score, tau, tlse, weight)
    with soft.PsSoft(M, K) as h:
        got = h.distill(X, W, ids, score + far, tau=tau, tlse=None if tlse is None else tlse + far / tau, weight=weight)
        only = h.distill(X, W, ids, score + far, tau=tau, tlse=None if tlse is None else tlse + far / tau, weight=weight, grad=False)
    for part, a, v, b in zip(("loss", "lse", "dX", "dW", "loss alone", "lse alone"), (*got, *only), (*want, *want[:2]), (*bounds, *bounds[:2])):
        most = soft_ref.near(a, v, b)
        say(f"teacher far={far} tau={tau} full={full} {part}: {most:.3f} of its bound")
        assert most <= 1, part


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("power", [-24, -80, -100])
def test_temperatures_whose_square_is_out_of_range(soft, power, few):
    # at a temperature near 0 both softmaxes are one item, and loss = tau (the student's best score - its score of the teacher's
    # item): about tau, where tau^2 in fp32 would be 0.  tau a power of two: scores / tau are exact
    n, M, K, k = 40, 200, 8, 5
    X, W, g = tables(n, M, K, F32, 3)
    ids = torch.stack([torch.randperm(M, generator=g)[:k] for _ in range(n)]).int().cuda()
    score = torch.randn(n, k, generator=g).cuda()
    tau = 2.0 ** power
    with soft.PsSoft(M, K, splits=0 if few else 2) as h:
        loss = soft_ref.f64(h.distill(X, W, ids, score, tau=tau, grad=not few)[0])
    s = soft_ref.f64(X) @ soft_ref.f64(W).T
    want = s.max(1) - s[np.arange(n), soft_ref.f64(ids.gather(1, score.argmax(1, keepdim=True)))[:, 0].astype(int)]
    # scores in fp32 as in soft_ref; ties of the best within tau add at most log M
    a = np.abs(soft_ref.f64(X)) @ np.abs(soft_ref.f64(W)).T
    bound = ((K + 16) * 4 + 8) * soft_ref.U * a.max(1) + tau * np.log(M) * 2
    most = float((np.abs(loss / tau - want) / bound).max())
    say(f"tau=2^{power} few={few}: {most:.3f} of its bound")
    assert most <= 1


@pytest.mark.parametrize("splits,grad", [(0, False), (0, True), (3, True)])
def test_scores_far_below_zero(soft, splits, grad):
    # every score of a row near -2^110: one item takes all, lse is its score, the loss what the target is below it
    n, M, K = 33, 90, 4
    X, W, g = tables(n, M, K, F32, 9)
    X, W = X.abs() + 1, -(W.abs() + 1)
    W[:, 0] -= torch.arange(M).cuda()
    X, W = X * 2.0 ** 55, W * 2.0 ** 55
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    s = soft_ref.f64(X) @ soft_ref.f64(W).T
    want = s.max(1) - s[np.arange(n), soft_ref.f64(item).astype(int)]
    bound = (K + 16) * 4 * soft_ref.U * np.abs(s).max(1)  # all products of one sign: |x||w| is |s|
    with soft.PsSoft(M, K, splits=splits) as h:
        out = h.xent(X, W, item, grad=grad)
    if grad:  # rows' weights agree with their own scores, whatever these are off by
        assert torch.isfinite(out[2]).all()
    for part, got, v in (("loss", out[0], want), ("lse", out[1], s.max(1))):
        most = float((np.abs(soft_ref.f64(got) - v) / bound).max())
        say(f"far below zero splits={splits} grad={grad} {part}: {most:.3f} of its bound")
        assert most <= 1


@pytest.mark.parametrize("M", [33_554_432 + 100, 40_000, 32_700])
def test_every_record_of_a_list_counts_once(soft, M):
    # tiles of items that take three sorting passes (from 2^20 tiles on), two, and one; items in every row's list, items of one row,
    # lists that no item of which is another row's.  A record lost, taken twice or moved is at least 1/200 of an item's sum
    n, K, per = 40, 1, 3000
    g = torch.Generator(device="cuda").manual_seed(M)
    X = (torch.randint(1, 4, (n, K), generator=g, device="cuda") / 4).float()
    W = torch.randint(-2, 3, (M, K), generator=g, device="cuda").float()
    item = torch.randint(0, M, (n, per), generator=g, device="cuda", dtype=torch.int32)
    item[:, 5] = M - 1
    item[:, 77] = M // 2
    item[:, 2000:2040] = torch.arange(40, device="cuda").int() * (M // 40)
    value = torch.randint(1, 6, (n, per), generator=g, device="cuda").float()
    ptr = torch.arange(0, per * n + 1, per, device="cuda")
    say(f"records M={M}")
    with soft.PsSoft(M, K) as h:
        dW = h.xent(X, W, item.flatten(), row_ptr=ptr, value=value.flatten(), grad="W")[3]
        again = h.xent(X, W, item.flatten(), row_ptr=ptr, value=value.flatten(), grad="W")[3]
    assert torch.equal(dW, again)
    del again
    x, w = X[:, 0].double(), W[:, 0].double()
    want, size = torch.zeros(M, dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda")
    for i in range(n):
        part = value[i].double().sum() * torch.softmax(x[i] * w, 0) * x[i]
        want += part
        size += part.abs()
        want.index_add_(0, item[i].long(), -value[i].double() * x[i])
        size.index_add_(0, item[i].long(), value[i].double() * x[i])
    # scores and values are exact; a weight is off by 2^-20 (exponential, log-sum-exp, planes), a sum of n weights and of a
    # list's records in it by n u
    assert float(((dW[:, 0].double() - want).abs() / size).max()) <= 2.0 ** -19 + n * soft_ref.U


@pytest.mark.parametrize("splits", [0, 2])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_row_that_lists_an_item_thousands_of_times(soft, dtype, splits):
    # and a popular item beside it, and neighbours of either that hardly any row wants
    n, M, K, times = 70, 64, 6, 3000
    X, W, g = tables(n, M, K, dtype, 11)
    X[:, 0] = 4
    W[:, 0] = 0
    W[20:30, 0] = -4
    lists = [[int(j)] for j in torch.randint(0, M, (n,), generator=g)]
    for i in range(n):
        lists[i].append(22)
    lists[40] = [7] * times
    y = np.zeros((n, M))
    for i, l in enumerate(lists):
        np.add.at(y[i], l, 1.0)
    ptr = torch.tensor(np.cumsum([0] + [len(l) for l in lists])).cuda()
    item = torch.tensor([j for l in lists for j in l], dtype=torch.int32).cuda()
    weight = torch.full((n,), 2.0 ** -8)
    want, bound = item_gradients(soft_ref.f64(X), soft_ref.f64(W), y, soft_ref.f64(weight))
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        got = h.xent(X, W, item, row_ptr=ptr, weight=weight.cuda())[3]
    most = off(got, want, bound, dtype)
    say(f"thousands of times {dtype} splits={splits}: {most:.3f} of its bound")
    assert most <= 1


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("size", [30.0, 1e3, 3e4, 1e6])
def test_confident_rows_of_large_scores(soft, size, dtype, splits):
    # a row's target takes its whole softmax: what is left of p - 1 may not depend on how large the scores are.  A score's error e
    # moves p to at most p / (p + (1 - p) exp(+-2 e)); the exponentials, log-sum-exps and planes are 2^-20, sums 2 u a term
    n, M, K = 200, 220, 32
    W, g = torch.randn(M, K, generator=torch.Generator().manual_seed(int(size))), torch.Generator().manual_seed(3)
    scale = (size / K) ** 0.5
    X = (W[:n] * (1 + 0.02 * torch.randn(n, K, generator=g)) * scale).to(dtype).cuda()
    W = (W * scale).to(dtype).cuda()
    item = torch.arange(n).int()
    item[::16] += 5
    x, w = soft_ref.f64(X), soft_ref.f64(W)
    s, a = x @ w.T, np.abs(x) @ np.abs(w).T
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    p, rest = e / e.sum(1, keepdims=True), np.empty_like(e)
    for j in range(M):  # 1 - p without cancellation
        rest[:, j] = np.delete(e, j, 1).sum(1) / e.sum(1)
    y = np.zeros((n, M))
    y[np.arange(n), item] = 1
    want = (p - y).T @ x
    es = np.minimum((K + 16) * 2 * soft_ref.U * a.max(1, keepdims=True), 300)
    with np.errstate(divide="ignore", invalid="ignore"):
        up = p / (p + rest * np.exp(-2 * es)) - p
        down = p - p / (p + rest * np.exp(2 * es))
    moved = np.where(p > 0, np.maximum(np.abs(np.nan_to_num(up)), np.abs(np.nan_to_num(down))), 0)
    bound = (moved + p * (2.0 ** -20 + 2 * (M + 16) * soft_ref.U) + y * (n + 16) * soft_ref.U + 2.0 ** -31).T @ np.abs(x)
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        got = h.xent(X, W, item.cuda())
    most = off(got[3], want, bound, dtype)
    say(f"confident size={size} {dtype} splits={splits}: {most:.3f} of its bound")
    assert most <= 1 and torch.isfinite(got[2]).all()
