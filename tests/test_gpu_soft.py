"""ps_soft on the device against the operators in 64 bits (soft_ref), with bounds derived there.

Sizes from one row and one item to several tiles and pieces, odd ones among them; element types; strided
and misaligned tables; lists that are empty, repeat, are padded or out of range; masked rows that hold NaN;
other streams, captured graphs, two handles; equal bits of equal calls.
"""
import contextlib
import gc
import sys

import numpy as np
import pytest
import torch

import soft_ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SHAPES = [(1, 1, 1), (1, 2, 3), (2, 33, 5), (33, 31, 16), (31, 65, 17), (64, 100, 32), (100, 333, 33), (5, 1000, 64), (130, 257, 100),
          (65, 515, 128), (40, 300, 200), (37, 129, 256), (33, 200, 300), (20, 140, 512), (3, 4097, 24), (700, 50, 20)]


@pytest.fixture(scope="module")
def soft():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1410_8043_amd import ps_soft

    return ps_soft


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@contextlib.contextmanager
def capture(graph):
    """torch.cuda.graph without the garbage collector: a graph left in a cycle (an exception's frames hold
    one) that it frees inside a capture waits for the device there, which ends the process."""
    gc.collect()
    gc.disable()
    try:
        with torch.cuda.graph(graph):
            yield
    finally:
        gc.enable()


def gen(*seed):
    g = torch.Generator()
    g.manual_seed(sum(int(v) * 7919 ** (k + 1) for k, v in enumerate(seed)) % (2**31))
    return g


def tables(n, M, K, dtype, g, scale=1.0):
    X = torch.randn(n, K, generator=g) * (scale * 2 / K) ** 0.5
    W = torch.randn(M, K, generator=g) * (scale * 2 / K) ** 0.5 * torch.exp(0.4 * torch.randn(M, 1, generator=g))
    return X.to(dtype).cuda(), W.to(dtype).cuda()


def lists(n, M, mean, g, bad=True):
    """Lists of 0 to 3 mean entries, some twice, some < 0."""
    length = (torch.rand(n, generator=g) * 2 * mean).round().long()
    if n > 2:
        length[1] = 0
        length[-1] = 3 * mean
    else:
        length += 1
    ptr = torch.zeros(n + 1, dtype=torch.int64)
    ptr[1:] = length.cumsum(0)
    item = (torch.rand(int(ptr[-1]), generator=g) ** 2 * M).int().clamp(max=M - 1)
    if bad and n > 4:
        item[torch.rand(item.shape, generator=g) < 0.1] = -1
    return ptr.cuda(), item.cuda()


def check(name, got, want, bounds, dtype):
    for part, a, v, b in zip(("loss", "lse", "dX", "dW"), got, want, bounds):
        off = soft_ref.near(a, v, b, dtype if part[0] == "d" else F32)
        say(f"  {name} {part}: {off:.3f} of its bound")
        assert off <= 1, (name, part, off)


def same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.numel() else x, y.view(torch.uint8) if y.numel() else y) for x, y in zip(a, b))


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K", SHAPES)
def test_xent_one_target(soft, n, M, K, dtype, splits):
    g = gen(1, n, M, K)
    X, W = tables(n, M, K, dtype, g)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32)
    weight = torch.randn(n, generator=g)
    if n > 4:
        item[3] = -1
        weight[4] = 0
        X[3:5] = float("nan")
    item, weight = item.cuda(), weight.cuda()
    Xr = torch.where(X.isnan(), torch.zeros_like(X), X)
    want, bounds = soft_ref.xent(Xr, W, item, weight=weight)
    say(f"xent one n={n} M={M} K={K} {dtype} splits={splits}")
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        got = h.xent(X, W, item, weight=weight)
        again = h.xent(X, W, item, weight=weight)
        only = h.xent(X, W, item, weight=weight, grad=False)
        dx = h.xent(X, W, item, weight=weight, grad="X")
        dw = h.xent(X, W, item, weight=weight, grad="W")
    check("xent", got, want, bounds, dtype)
    assert same(got, again) and dx[3] is None and dw[2] is None
    check("loss only", only, want, bounds, dtype)
    check("dX only", dx[:3], want, bounds, dtype)
    check("dW only", (dw[0], dw[1]), want, bounds, dtype)
    assert soft_ref.near(dw[3], want[3], bounds[3], dtype) <= 1
    if n > 4:
        assert float(got[0][3]) == 0 and float(got[0][4]) == 0 and not got[2][3:5].any()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K,mean,splits", [(1, 50, 8, 5, 0), (33, 31, 16, 40, 2), (31, 65, 17, 1, 0), (100, 333, 33, 20, 0),
                                               (5, 1000, 64, 300, 4), (130, 257, 100, 9, 0), (65, 515, 128, 70, 0), (37, 129, 256, 3, 0),
                                               (20, 140, 512, 11, 2), (1100, 60, 20, 12, 0), (50, 3000, 40, 200, 0)])
def test_xent_lists(soft, n, M, K, mean, splits, dtype):
    g = gen(2, n, M, K)
    X, W = tables(n, M, K, dtype, g)
    ptr, item = lists(n, M, mean, g)
    value = (torch.rand(item.shape, generator=g) * 5 - 1).cuda()
    value[item < 0] = float("nan")
    weight = torch.rand(n, generator=g).cuda()
    vr = torch.where(item < 0, torch.zeros_like(value), value)
    want, bounds = soft_ref.xent(X, W, item, ptr, vr, weight)
    say(f"xent lists n={n} M={M} K={K} entries={item.numel()} {dtype}")
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        got = h.xent(X, W, item, row_ptr=ptr, value=value, weight=weight)
        again = h.xent(X, W, item, row_ptr=ptr, value=value, weight=weight)
        ones = h.xent(X, W, item, row_ptr=ptr)
    check("xent", got, want, bounds, dtype)
    assert same(got, again)
    want, bounds = soft_ref.xent(X, W, item, ptr)
    check("no values", ones, want, bounds, dtype)


def test_xent_the_same_item_many_times(soft):
    # rows that list an item two to nine times, dense lists, values of either sign: added in the list's order
    n, M, K = 150, 45, 24
    g = gen(20)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n, 90), generator=g, dtype=torch.int32)
    item[:, 5:9] = item[:, 4:5]
    ptr = torch.arange(0, 90 * n + 1, 90).cuda()
    item = item.flatten().cuda()
    value = torch.randn(item.shape, generator=g).cuda()
    want, bounds = soft_ref.xent(X, W, item, ptr, value)
    say("xent many times")
    with soft.PsSoft(M, K) as h:
        got = h.xent(X, W, item, row_ptr=ptr, value=value)
        again = h.xent(X, W, item, row_ptr=ptr, value=value)
    check("many times", got, want, bounds, F32)
    assert same(got, again)


def test_xent_items_of_many_digits_and_popular_items(soft):
    # items beyond 2^18 take three sorting passes; one item in every row's list goes over many chunks
    n, M, K = 3000, 300_000, 8
    g = gen(3)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n, 4), generator=g, dtype=torch.int32)
    item[:, 1] = 299_999
    item[:, 2] = 262_144 + 7
    item[: n // 2, 3] = 5
    ptr = torch.arange(0, 4 * n + 1, 4)
    say("xent many digits")
    with soft.PsSoft(M, K) as h:
        dW = h.xent(X, W, item.flatten().cuda(), row_ptr=ptr.cuda(), grad="W")[3]
        again = h.xent(X, W, item.flatten().cuda(), row_ptr=ptr.cuda(), grad="W")[3]
    assert torch.equal(dW, again)
    x, w = X.double(), W.double()
    want = torch.zeros(M, K, dtype=torch.float64, device="cuda")
    room = torch.zeros(M, K, dtype=torch.float64, device="cuda")
    for a in range(0, n, 500):
        s = x[a:a + 500] @ w.T
        p = 4 * torch.softmax(s, 1)
        want += p.T @ x[a:a + 500]
        room += p.T @ x[a:a + 500].abs()
    for c in range(4):
        j = item[:, c].long().cuda()
        want.index_add_(0, j, -x)
        room.index_add_(0, j, x.abs())
    # scores within 2 u (K + 16) (|x||w| below 40), their weights twice that, 2^-20 of the exponential, sums of n and of M
    rel = 4 * (K + 16) * soft_ref.U * 40 + 2.0 ** -20 + (n + M + 64) * soft_ref.U
    assert float(((dW.double() - want).abs() / (room * rel + 1e-30)).max()) <= 1


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K,k,tau,full,splits", [(1, 10, 4, 3, 1.0, False, 0), (33, 31, 16, 31, 2.0, False, 0), (100, 333, 33, 10, 0.7, True, 0),
                                                     (70, 515, 128, 64, 2.0, True, 3), (40, 200, 256, 100, 4.0, False, 0),
                                                     (20, 140, 512, 1, 1.5, True, 0), (1500, 40, 20, 7, 1.0, False, 0)])
def test_distill(soft, n, M, K, k, tau, full, splits, dtype):
    g = gen(4, n, M, K)
    X, W = tables(n, M, K, dtype, g)
    t = X.cpu().float() @ W.cpu().float().T + torch.randn(n, M, generator=g)
    tlse = torch.logsumexp(t / tau, 1).cuda() if full else None
    score, item = torch.topk(t, k, 1)
    item = item.int()
    weight = torch.randn(n, generator=g)
    if n > 10:
        item[3] = -1  # a masked row
        score[3] = float("nan")
        item[5, k // 2:] = -1  # a shorter list, ended by ids and by scores
        score[5, k // 2:] = float("nan")
        score[6, k // 2:] = -float("inf")
        score[7] = -float("inf")
        weight[8] = 0
        if k > 2:
            item[9, 1] = item[9, 0]  # the same item twice
        if full:
            tlse[3] = float("nan")
    item, score, weight = item.cuda(), score.cuda(), weight.cuda()
    sr = torch.where(item < 0, torch.zeros_like(score), score)
    want, bounds = soft_ref.distill(X, W, item, sr, tau, tlse, weight)
    say(f"distill n={n} M={M} K={K} k={k} tau={tau} full={full} {dtype}")
    with soft.PsSoft(M, K, dtype, splits=splits) as h:
        got = h.distill(X, W, item, score, tau=tau, tlse=tlse, weight=weight)
        again = h.distill(X, W, item, score, tau=tau, tlse=tlse, weight=weight)
        only = h.distill(X, W, item, score, tau=tau, tlse=tlse, weight=weight, grad=False)
    check("distill", got, want, bounds, dtype)
    check("loss only", only, want, bounds, dtype)
    assert same(got, again)
    if n > 10:
        assert not got[0][[3, 7, 8]].any() and not got[2][[3, 7, 8]].any()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K,k,mean,splits", [(1, 1, 1, 1, 0, 0), (1, 50, 8, 60, 5, 0), (3, 300, 17, 256, 0, 0), (33, 700, 64, 10, 40, 3),
                                                 (200, 1111, 100, 64, 0, 0), (7, 20_000, 128, 100, 300, 0), (20, 900, 512, 5, 9, 0),
                                                 (600, 5000, 32, 20, 30, 0), (1, 100_000, 48, 256, 50, 0)])
def test_top(soft, n, M, K, k, mean, splits, dtype, search=None):
    g = gen(5, n, M, K)
    X, W = tables(n, M, K, dtype, g)
    ptr, item = lists(n, M, mean, g) if mean else (None, None)
    want, score = soft_ref.top(X, W, k, ptr, item)
    say(f"top n={n} M={M} K={K} k={k} {dtype}")
    with soft.PsSoft(M, K, dtype, splits=splits, search=search) as h:
        got = h.top(X, W, k, row_ptr=ptr, item=item)
    assert np.array_equal(got[0].cpu().numpy(), want)
    # the 64-bit sum in another order, rounded to fp32: at most a step of fp32 apart
    a, b = got[1].cpu().numpy(), score
    assert np.array_equal(np.isinf(a), np.isinf(b))
    fine = np.isfinite(b)
    assert np.all(np.abs(a[fine] - b[fine]) <= 2 * soft_ref.U * np.abs(b[fine]) + 1e-30)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K,k,mean,splits", [(33, 2049, 1, 3, 0, 0), (40, 2100, 15, 256, 30, 0), (65, 3000, 16, 10, 20, 3), (257, 2500, 31, 64, 0, 0),
                                                 (300, 4100, 100, 33, 500, 0), (130, 9000, 128, 100, 0, 5), (50, 2600, 200, 20, 10, 0),
                                                 (64, 2300, 256, 7, 0, 0), (34, 2400, 300, 40, 9, 0), (90, 2222, 512, 12, 0, 0),
                                                 (1000, 20_011, 40, 50, 100, 0)])
def test_top_of_many_rows(soft, n, M, K, k, mean, splits, dtype):
    # both searches
    test_top(soft, n, M, K, k, mean, splits, dtype, 0)
    test_top(soft, n, M, K, k, mean, splits, dtype, 1)


@pytest.mark.parametrize("n,M,K,k", [(1, 1, 1, 1), (3, 40, 7, 50), (70, 500, 33, 256), (9, 2000, 64, 100)])
def test_top_by_candidates_of_few_items(soft, n, M, K, k):
    # no threshold, more candidates than room: forms that the sizes would not choose
    test_top(soft, n, M, K, k, 5 if M > 20 else 0, 0, F32, 1)


def test_top_forms_agree(soft):
    # the largest case that both take in a moment, bit for bit
    g = gen(22)
    for n, M, K, k, dtype in ((3000, 17_770, 128, 64, F32), (700, 30_011, 100, 200, F16), (4100, 5000, 64, 10, BF16)):
        X, W = tables(n, M, K, dtype, g)
        ptr, item = lists(n, M, 50, g)
        say(f"top forms n={n} M={M} K={K} k={k} {dtype}")
        with soft.PsSoft(M, K, dtype, search=0) as a, soft.PsSoft(M, K, dtype, search=1) as b, soft.PsSoft(M, K, dtype) as c:
            x, y, z = (h.top(X, W, k, row_ptr=ptr, item=item) for h in (a, b, c))
        assert same(x, y) and same(x, z)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,M,K", [(1, 1, 1), (1, 17_770, 128), (2, 70, 33), (3, 999, 7), (9, 5000, 100), (17, 64, 512), (40, 2049, 50)])
def test_loss_alone_of_few_rows(soft, n, M, K, dtype):
    g = gen(24, n, M, K)
    X, W = tables(n, M, K, dtype, g, 3.0)
    ptr, item = lists(n, M, 5, g)
    weight = torch.ones(n)
    if n > 8:
        weight[5] = 0
        X[5] = float("nan")
        X[6] = X[6] * 100  # one item takes all
    Xr = torch.where(X.isnan(), torch.zeros_like(X), X)
    want, bounds = soft_ref.xent(Xr, W, item, ptr, weight=weight.cuda())
    say(f"few rows n={n} M={M} K={K} {dtype}")
    with soft.PsSoft(M, K, dtype) as h:
        got = h.xent(X, W, item, row_ptr=ptr, weight=weight.cuda(), grad=False)
        assert same(got, h.xent(X, W, item, row_ptr=ptr, weight=weight.cuda(), grad=False))
        Wn = W.clone()
        Wn[M // 2, K - 1] = float("nan")
        assert h.xent(Xr, Wn, item, row_ptr=ptr, grad=False)[1].isnan().all()
    check("few", got, want, bounds, dtype)


def test_equal_calls_give_equal_bits(soft):
    # several tiles and pieces, enough workgroups that their order differs from call to call
    g = gen(23)
    for n, M, K, dtype in ((4096, 9000, 128, F32), (1500, 20_000, 256, BF16), (5000, 3000, 512, F32), (700, 4000, 40, F16)):
        X, W = tables(n, M, K, dtype, g)
        ptr, item = lists(n, M, 30, g)
        for splits in (0, 16, 5):
            say(f"equal bits n={n} M={M} K={K} {dtype} splits={splits}")
            with soft.PsSoft(M, K, dtype, splits=splits) as h:
                first = h.xent(X, W, item, row_ptr=ptr)
                for _ in range(8):
                    assert same(h.xent(X, W, item, row_ptr=ptr), first)


def test_top_of_uneven_tables(soft):
    # rows and items of far lengths, a few items above all, near scores, rows of zeros or not finite, many equal items
    g = gen(21)
    n, M, K, k = 100, 5000, 48, 30
    X, W = tables(n, M, K, F32, g)
    W *= torch.exp(1.5 * torch.randn(M, 1, generator=g)).cuda()
    X *= torch.exp2(torch.randint(-40, 20, (n, 1), generator=g).float()).cuda()
    W[100:140] *= 300
    W[2000:2600] = W[1999]  # 601 equal items
    W[3000:4500] = W[1999] + 1e-6 * torch.randn(1500, K, generator=g).cuda()  # and 1500 near ones
    X[:50] = W[1999] * X[:50].norm(dim=1, keepdim=True)  # half of the rows like them best
    X[60] = 0
    ptr = torch.zeros(n + 1, dtype=torch.int64)
    ptr[3:] = 4990  # row 2 leaves ten
    ptr[11:] += 40  # row 10 excludes the longest
    item = torch.cat((torch.arange(4990), torch.arange(100, 140))).int().cuda()
    for name, w in (("finite", W), ("nan", W.clone()), ("inf", W.clone())):
        if name != "finite":
            w[777, 5] = float(name)
        want, score = soft_ref.top(X, w, k, ptr, item)
        say(f"top uneven {name}")
        with soft.PsSoft(M, K, search=0) as h, soft.PsSoft(M, K, search=1) as h1:
            best, val = h.top(X, w, k, row_ptr=ptr.cuda(), item=item)
            assert same((best, val), h1.top(X, w, k, row_ptr=ptr.cuda(), item=item))
        got = best.cpu().numpy()
        if name == "finite":
            # equal up to the order of scores whose 64-bit sums differ in their last bits
            s = soft_ref.f64(X) @ soft_ref.f64(w).T
            for i in range(n):
                if not np.array_equal(got[i], want[i]):
                    a, b = s[i, got[i]], s[i, want[i]]
                    assert (got[i] >= 0).all() and np.abs(a - b).max() <= 64 * 2.0 ** -53 * np.abs(s[i]).max(), i
                    assert len(set(got[i])) == k
            assert (got[2, 10:] == -1).all() and (got[60] == np.arange(k)).all()
        else:
            rows = [i for i in range(n) if i != 2]
            s = soft_ref.f64(X) @ soft_ref.f64(w).T
            for i in rows:
                if np.isnan(s[i, 777]) or s[i, 777] == np.inf:
                    assert got[i, 0] == 777, (name, i)
                else:
                    assert 777 not in got[i]


@pytest.mark.parametrize("search", [0, 1])
def test_top_ties_masks_and_nan(soft, search):
    # whole numbers: many equal scores, exact in any order; the lowest items win
    g = gen(6)
    n, M, K, k = 50, 4000, 8, 100
    X = torch.randint(-2, 3, (n, K), generator=g).float().cuda()
    W = torch.randint(-2, 3, (M, K), generator=g).float().cuda()
    X[7] = 0  # every score equal
    ptr = torch.zeros(n + 1, dtype=torch.int64)
    ptr[9:] = M  # row 8 excludes everything
    ptr[10:] += M - 3  # row 9 all but three
    item = torch.cat((torch.arange(M), torch.arange(3, M))).int().cuda()
    want, score = soft_ref.top(X, W, k, ptr, item)
    say("top ties")
    with soft.PsSoft(M, K, search=search) as h:
        best, val = h.top(X, W, k, row_ptr=ptr.cuda(), item=item)
        W2 = W.clone()
        W2[1234, 3] = float("nan")
        nan_best, nan_val = h.top(X, W2, 3)
        W2[1234, 3] = float("inf")
        X2 = X.abs() + 1
        inf_best, inf_val = h.top(X2, W2, 3)
    assert np.array_equal(best.cpu().numpy(), want) and np.array_equal(val.cpu().numpy(), score)
    assert (best[8] == -1).all() and (best[9, :3] == torch.tensor([0, 1, 2], device="cuda")).sum() >= 1 and (best[9, 3:] == -1).all()
    assert (best[7].cpu() == torch.arange(k)).all()
    assert (nan_best[:, 0] == 1234).all() and nan_val[:, 0].isnan().all() and not nan_val[:, 1:].isnan().any()
    assert (inf_best[:, 0] == 1234).all() and torch.isinf(inf_val[:, 0]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K,pad,shift", [(20, 3, 1), (64, 4, 0), (33, 31, 5)])
def test_strided_and_misaligned_tables(soft, K, pad, shift, dtype):
    n, M = 70, 200
    g = gen(7, K)
    Xd, Wd = tables(n, M, K, dtype, g)
    xs = torch.full((n * (K + pad) + shift,), float("nan"), dtype=dtype, device="cuda")[shift:].view(n, K + pad)
    ws = torch.full((M * (K + pad) + shift,), float("nan"), dtype=dtype, device="cuda")[shift:].view(M, K + pad)
    xs[:, :K], ws[:, :K] = Xd, Wd
    ptr, item = lists(n, M, 6, g)
    say(f"strided K={K} pad={pad} shift={shift} {dtype}")
    with soft.PsSoft(M, K, dtype) as h:
        a = h.xent(Xd, Wd, item, row_ptr=ptr)
        b = h.xent(xs[:, :K], ws[:, :K], item, row_ptr=ptr)
        c, d = h.top(Xd, Wd, 9), h.top(xs[:, :K], ws[:, :K], 9)
        with pytest.raises(ValueError, match="contiguous"):
            h.xent(Xd.t().contiguous().t(), Wd, item, row_ptr=ptr)
        # gradients into strided rows of the caller: what lies between them stays
        out = torch.full((M, K + pad), 7.0, dtype=dtype, device="cuda")
        rc = soft._lib.ps_soft_xent(h.h, n, Xd.data_ptr(), K, Wd.data_ptr(), K, ptr.data_ptr(), item.data_ptr(), None, item.numel(), None,
                                    None, None, None, 0, out.data_ptr(), K + pad)
        assert rc == soft.OK
    assert same(a, b) and same(c, d)
    assert torch.equal(out[:, :K], a[3]) and (out[:, K:] == 7).all()


def test_numbers_of_far_magnitudes(soft):
    # tables scaled by powers of two give the same scores; rows far below the largest; large scores
    n, M, K = 40, 300, 32
    g = gen(8)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    with soft.PsSoft(M, K) as h:
        say("magnitudes: powers of two")
        base = h.xent(X, W, item)
        for e in (-100, -60, 40, 90, 100):
            far = h.xent(X * 2.0 ** e, W * 2.0 ** -e, item)
            assert torch.equal(far[0], base[0]) and torch.equal(far[1], base[1])
            assert torch.equal(far[2] * 2.0 ** e, base[2]) and torch.equal(far[3] * 2.0 ** -e, base[3])
        for name, x, w in (("rows", X * torch.exp2(-torch.arange(n).cuda() / 2.0)[:, None], W),
                           ("items", X, W * torch.exp2(-torch.arange(M).cuda() / 20.0)[:, None]), ("large", X * 12, W * 4)):
            say(f"magnitudes: {name}")
            want, bounds = soft_ref.xent(x, w, item)
            check(name, h.xent(x, w, item), want, bounds, F32)
        say("magnitudes: zeros")
        z = h.xent(X * 0, W * 0, item)
        want, bounds = soft_ref.xent(X * 0, W * 0, item)
        assert soft_ref.near(z[1], want[1], bounds[1]) <= 1 and not z[2].any() and not z[3].any()


def test_weights_far_apart(soft):
    n, M, K = 64, 90, 16
    g = gen(9)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    weight = (torch.exp2(-torch.arange(n) / 4.0) * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)).cuda()
    want, bounds = soft_ref.xent(X, W, item, weight=weight)
    with soft.PsSoft(M, K) as h:
        check("weights", h.xent(X, W, item, weight=weight), want, bounds, F32)


def test_fitted_rows_keep_small_gradients(soft):
    # the target's weight is almost all of the softmax: p - 1 is small and must not drown in roundings of p
    n, M, K = 96, 96, 64
    g = gen(10)
    W = torch.randn(M, K, generator=g)
    X = W * (9.0 / K)
    item = torch.arange(n).int().cuda()
    for dtype in (F32, BF16, F16):
        x, w = X.to(dtype).cuda(), W.to(dtype).cuda()
        want, bounds = soft_ref.xent(x, w, item)
        say(f"fitted {dtype}")
        with soft.PsSoft(M, K, dtype) as h:
            got = h.xent(x, w, item)
        check("fitted", got, want, bounds, dtype)
        for a, b in zip(got[2:], want[2:]):
            rel = np.linalg.norm(soft_ref.f64(a) - b) / np.linalg.norm(b)
            # p is off by 2^-20, and what is left of 1 - p here is above 2^-9: 2^-11 of it, and the type's rounding
            assert rel <= 2.0 ** -11 + 2 * soft_ref.HALF[dtype], rel


def test_gradients_against_differences(soft):
    n, M, K = 50, 200, 24
    g = gen(11)
    X, W = tables(n, M, K, F32, g)
    ptr, item = lists(n, M, 5, g)
    dx, dw = torch.randn(n, K, generator=g).cuda(), torch.randn(M, K, generator=g).cuda()
    step = 2.0 ** -7
    with soft.PsSoft(M, K) as h:
        _, _, dX, dW = h.xent(X, W, item, row_ptr=ptr)
        along = {}
        for name, a, b in (("X", dx, 0 * dw), ("W", 0 * dx, dw)):
            up = h.xent(X + step * a, W + step * b, item, row_ptr=ptr, grad=False)[0].double().sum()
            down = h.xent(X - step * a, W - step * b, item, row_ptr=ptr, grad=False)[0].double().sum()
            along[name] = float((up - down) / (2 * step))
    for name, got in (("X", float((dX.double() * dx).sum())), ("W", float((dW.double() * dw).sum()))):
        say(f"differences {name}: {along[name]} against {got}")
        # the third derivative along a direction of length |d| |w| (about 8) is below 8^3 per unit of mass; step^2 / 6 of it,
        # and losses near 3000 in fp32 over 2 step
        assert abs(along[name] - got) <= step**2 / 6 * 512 * item.numel() + 3000 * 2.0 ** -22 / step


def test_bad_ids_and_pointers_touch_nothing(soft):
    n, M, K = 12, 40, 8
    g = gen(12)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32)
    item[4], item[6] = M, 2**31 - 1
    item = item.cuda()
    good = torch.ones(n, dtype=torch.bool)
    good[[4, 6]] = False
    clean = torch.where(good.cuda(), item, -1)
    say("bad ids")
    with soft.PsSoft(M, K) as h:
        got, want = h.xent(X, W, item), h.xent(X, W, clean)
        assert got[0][~good].isnan().all() and torch.equal(got[0][good], want[0][good]) and torch.equal(got[3], want[3])
        ptr = torch.arange(n + 1)
        ptr[5] = 100  # rows 4 and 5 have no list
        lst = torch.arange(n).int().cuda()
        say("bad pointers")
        loss = h.xent(X, W, lst, row_ptr=ptr.cuda())[0].cpu()
        assert loss[4:6].isnan().all() and not loss[:4].isnan().any() and not loss[6:].isnan().any()
        best, _ = h.top(X, W, 3, row_ptr=ptr.cuda(), item=torch.full((n,), M, dtype=torch.int32).cuda())
        assert torch.equal(best, h.top(X, W, 3)[0])
        score = torch.randn(n, 4, generator=g).cuda()
        ids = torch.randint(0, M, (n, 4), generator=g, dtype=torch.int32)
        ids[2, 1] = M + 5
        say("bad teacher ids")
        assert h.distill(X, W, ids.cuda(), score)[0].isnan().nonzero().flatten().tolist() == [2]


def test_no_rows_and_masked_batches(soft):
    M, K = 70, 12
    W = torch.randn(M, K, device="cuda")
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    with soft.PsSoft(M, K) as h:
        say("no rows")
        loss, lse, dX, dW = h.xent(W[:0], W, empty)
        assert loss.shape == (0,) and dX.shape == (0, K) and dW.shape == (M, K) and not dW.any()
        loss, lse, dX, dW = h.xent(W[:0], W, empty, row_ptr=torch.zeros(1, dtype=torch.int64, device="cuda"))
        assert not dW.any()
        assert h.top(W[:0], W, 3)[0].shape == (0, 3)
        say("all masked")
        X = torch.full((45, K), float("nan"), device="cuda")
        out = h.xent(X, W, torch.full((45,), -1, dtype=torch.int32, device="cuda"))
        assert not out[0].any() and not out[2].any() and not out[3].any()
        assert torch.allclose(out[1], torch.full_like(out[1], np.log(M)), atol=1e-5)
        out = h.xent(X, W, empty, row_ptr=torch.zeros(46, dtype=torch.int64, device="cuda"))
        assert not out[0].any() and not out[2].any() and not out[3].any()
    with soft.PsSoft(M, K) as h:  # a fresh workspace
        assert not h.xent(W[:0], W, empty)[3].any()


def test_nan_in_a_live_row_stays_in_its_row(soft):
    n, M, K = 40, 100, 16
    g = gen(13)
    X, W = tables(n, M, K, F32, g)
    item = torch.randint(0, M, (n,), generator=g, dtype=torch.int32).cuda()
    bad = X.clone()
    bad[11, 3] = float("nan")
    bad[12, 0] = float("inf")
    with soft.PsSoft(M, K) as h:
        a, b = h.xent(bad, W, item), h.xent(X, W, item)
    ok = torch.ones(n, dtype=torch.bool, device="cuda")
    ok[11:13] = False
    assert torch.equal(a[0][ok], b[0][ok]) and torch.equal(a[2][ok], b[2][ok])
    assert a[0][~ok].isnan().all() and a[3].isnan().all()


def run_all(h, d):
    return (*h.xent(d["X"], d["W"], d["item"], row_ptr=d["ptr"], weight=d["weight"]),
            *h.distill(d["X"], d["W"], d["ids"], d["score"], tau=2.0, weight=d["weight"]),
            *h.top(d["X"], d["W"], 7, row_ptr=d["ptr"], item=d["item"]))


def some(n, M, K, seed):
    g = gen(seed)
    X, W = tables(n, M, K, F32, g)
    ptr, item = lists(n, M, 6, g)
    return {"X": X, "W": W, "ptr": ptr, "item": item, "weight": torch.rand(n, generator=g).cuda(),
            "ids": torch.randint(0, M, (n, 5), generator=g, dtype=torch.int32).cuda(), "score": torch.randn(n, 5, generator=g).cuda()}


def test_streams_handles_and_a_growing_workspace(soft):
    small, large = some(40, 120, 20, 14), some(900, 120, 20, 15)
    with soft.PsSoft(120, 20) as h, soft.PsSoft(120, 20) as other:
        want = {id(d): run_all(h, d) for d in (small, large)}  # grows
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = []
        for k in range(6):  # streams in turn on one handle: each call waits for the one before
            d = (small, large)[k % 2]
            with torch.cuda.stream(side if k % 3 else torch.cuda.current_stream()):
                got.append((d, run_all(h, d)))
        with torch.cuda.stream(side):  # two handles at once
            a = run_all(other, large)
        b = run_all(h, small)
        torch.cuda.synchronize()
    for d, out in got + [(large, a), (small, b)]:
        assert same(out, want[id(d)])


def test_captured_and_replayed(soft):
    d = some(200, 300, 36, 16)
    e = some(200, 300, 36, 17)
    with soft.PsSoft(300, 36) as fresh:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(soft.PsSoftError) as err:
            with capture(graph):
                fresh.xent(d["X"], d["W"], d["item"], row_ptr=d["ptr"])
        assert err.value.code == soft.ESTATE
        del graph, err
        torch.cuda.synchronize()
    with soft.PsSoft(300, 36) as h, soft.PsSoft(300, 36) as eager:
        n_entries = max(x["item"].numel() for x in (d, e))
        h.reserve(200, max(n_entries, 200 * 5), 7)
        static = {k: v.clone() for k, v in d.items()}
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with capture(graph):
            out = run_all(h, static)
        for k in range(4):
            src = (d, e)[k % 2]
            if src["item"].numel() == static["item"].numel() or k % 2 == 0:
                for name, v in src.items():
                    static[name].copy_(v)
            else:  # the graph's lists have a fixed room: only the tables change
                for name in ("X", "W", "weight", "ids", "score"):
                    static[name].copy_(src[name])
            graph.replay()
            torch.cuda.synchronize()
            say(f"replay {k}")
            assert same(out, run_all(eager, static)), k
            big = some(700, 300, 36, 18)
            run_all(h, big)  # the handle grows; the graph's workspace stays
            torch.cuda.synchronize()


@pytest.mark.parametrize("M,K,dtype", [(300, 36, F32), (20_000, 64, F32), (5000, 256, BF16)])
def test_reserved_room_holds_every_smaller_call(soft, M, K, dtype):
    # captured calls cannot grow the workspace: each of these fits what was reserved for the largest
    with soft.PsSoft(M, K, dtype) as h:
        h.reserve(3000, 30_000, 50)
        for n in (1, 2, 5, 17, 40, 100, 130, 257, 513, 800, 1025, 1500, 2049, 3000):
            g = gen(25, n)
            X, W = tables(n, M, K, dtype, g)
            ptr, item = lists(n, M, 30_000 // (4 * n + 8), g, bad=False)
            ids = torch.randint(0, M, (n, 10), generator=g, dtype=torch.int32).cuda()
            score = torch.randn(n, 10, generator=g).cuda()
            say(f"reserved M={M} K={K} n={n} entries={item.numel()}")
            assert item.numel() <= 30_000
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with capture(graph):
                outs = [h.xent(X, W, item, row_ptr=ptr, grad=grad) for grad in (False, "X", "W", True)]
                outs.append(h.distill(X, W, ids, score))
                outs.append(h.top(X, W, min(50, M), row_ptr=ptr, item=item))
                outs.append(h.top(X, W, 3))
            graph.replay()
            torch.cuda.synchronize()
            with soft.PsSoft(M, K, dtype) as eager:
                assert same(outs[3], eager.xent(X, W, item, row_ptr=ptr))
                assert same(outs[0], eager.xent(X, W, item, row_ptr=ptr, grad=False))
                assert same(outs[5], eager.top(X, W, min(50, M), row_ptr=ptr, item=item))
            del graph


def test_many_rows_of_few_items(soft):
    # more rows than a launch has in its second dimension, one item
    n, K = 70_001, 3
    X, W = torch.randn(n, K, device="cuda"), torch.randn(1, K, device="cuda")
    item = torch.zeros(n, dtype=torch.int32, device="cuda")
    with soft.PsSoft(1, K) as h:
        loss, lse = h.xent(X, W, item, grad=False)
        assert torch.allclose(lse, X @ W[0], atol=1e-5) and float(loss.abs().max()) < 1e-5
        best, score = h.top(X, W, 2)
        assert (best == torch.tensor([0, -1], device="cuda", dtype=torch.int32)).all()
        loss, lse, dX, dW = h.xent(X, W, item)
        assert float(dX.abs().max()) < 1e-5 and float(dW.abs().max()) < 1e-2


def test_from_teacher_to_student(soft):
    # a trained factorization answers with its best items, and a smaller table learns from them
    from paper_1410_8043_amd import ps_mf, synth

    spec = synth.CONFIGS["tiny"]
    w = synth.generate(spec)
    with ps_mf.PsMf(spec.N, spec.M, spec.K, spec.P, 2, spec.eta, spec.lam, stream=torch.cuda.current_stream()) as mf:
        mf.load_ratings(w.user, w.item, w.val)
        mf.set_factors(w.L0, w.R0)
        mf.clock(5)
        L, R = (torch.from_numpy(a).cuda() for a in mf.get_factors())
    K = 6
    g = gen(19)
    X, W = tables(spec.N, spec.M, K, F32, g)
    with soft.PsSoft(spec.M, spec.K) as teacher, soft.PsSoft(spec.M, K) as student:
        item, score = teacher.top(L, R, 12)
        want, _ = soft_ref.top(L, R, 12)
        assert np.array_equal(item.cpu().numpy(), want)
        for step in range(3):
            vals, bounds = soft_ref.distill(X, W, item, score, 2.0)
            got = student.distill(X, W, item, score, tau=2.0)
            check(f"step {step}", got, vals, bounds, F32)
            X, W = X - 0.05 * got[2], W - 0.05 * got[3]


@pytest.mark.parametrize("n,M,K", [(2**24 + 5, 2, 1), (3, 2**24 + 5, 129)])
def test_more_workgroups_than_a_launch_dimension_takes(soft, n, M, K):
    # 2^22 workgroups of 4 rows, or of 4 items, and a few more rows; three kinds of rows, five of items
    xs, ws = torch.arange(n, device="cuda") % 3, torch.arange(M, device="cuda") % 5
    X = torch.zeros(n, K, dtype=BF16, device="cuda")
    W = torch.zeros(M, K, dtype=BF16, device="cuda")
    X[:, 0], W[:, 0] = (xs - 1) / 8, ws - 2
    item = (torch.arange(n, device="cuda") * 7919 % M).int()
    item[-1] = M - 1
    at = item.long()
    weight = float(2**24) if M > n else 1.0  # gradients of about 1
    with soft.PsSoft(M, K, BF16) as h:
        loss, lse, dX, dW = h.xent(X, W, item, weight=torch.full((n,), weight, device="cuda"))
    # by kinds, in 64 bits: M/5 items each, n/3 rows each
    nw, nx = torch.bincount(ws, minlength=5).double(), torch.bincount(xs, minlength=3).double()
    w, x = torch.arange(-2.0, 3, device="cuda").double(), torch.arange(-1.0, 2, device="cuda").double() / 8
    e = (x[:, None] * w).exp()
    total = (e * nw).sum(1)
    # values up to 2^5 rounded to half of 2^-19, and weights to 2^-21 (the exponent's and their own rounding)
    near = 2**-20 + 2**-20
    want = total.log()[xs]
    assert float((lse - want).abs().max()) <= near
    assert float((loss - (want - x[xs] * w[ws[at]])).abs().max()) <= near
    # dX: bf16's half step; sums of numbers up to 2 in pieces of 2 x 2048 instructions, half a step of fp32 each
    gx = weight * (((e * nw * w).sum(1) / total)[xs] - w[ws[at]])
    assert float(((dX[:, 0] - gx).abs() - 2**-8 * gx.abs()).max()) <= weight * 2**-11
    # dW: the same, weights of one plane of fp16, and, in a tile of 32 items with targets, to 2^-25 of 2 weight
    p = weight * e / total[:, None] * nx[:, None]
    gw = (p * x[:, None]).sum(0)[ws].index_add_(0, at, -weight * x[xs])
    size = (p * x.abs()[:, None]).sum(0)[ws].index_add_(0, at, weight * x[xs].abs())
    tile = torch.zeros(M // 32 + 1, dtype=torch.float64, device="cuda").index_fill_(0, at // 32, weight * n * 2**-24)
    slack = 2**-8 * gw.abs() + 2**-10 * size + tile[torch.arange(M, device="cuda") // 32]
    assert float(((dW[:, 0] - gw).abs() - slack).max()) <= 0
    if K > 1:
        assert not dX[:, 1:].any() and not dW[:, 1:].any()
