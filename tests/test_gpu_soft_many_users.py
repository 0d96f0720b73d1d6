"""The factorization's softmax loss with more users than one launch has threads for a wavefront each (2^26), their ratings in two
blocks."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_lists_of_two_blocks_of_many_users():
    from paper_1410_8043_amd import ps_mf

    N, M, K = 2**26 + 5, 7, 1
    user = np.array([0, 0, 3, 2**26 - 1, 2**26, 2**26 + 3, 2**26 + 4, 2**26 + 4], np.int32)
    item = np.array([1, 2, 0, 6, 3, 5, 4, 4], np.int32)
    val = np.array([1, 2, 3, 1, 2, 5, 4, 1], np.float32)
    L = np.zeros((N, K), np.float32)
    L[user, 0] = user % 5 - 1.5
    R = np.linspace(-1, 1, M, dtype=np.float32)[:, None]
    with ps_mf.PsMf(N, M, K, 1, 0, 0.01, 0.0, B=2) as g:
        print("loading", flush=True)
        g.load_ratings(user, item, val)
        print("factors", flush=True)
        g.set_factors(L, R)
        print("loss", flush=True)
        got = g.softmax_loss()
        best, _ = g.top_items(2, users=user)
    s = L[user, 0].astype(np.float64)[:, None] * R[:, 0].astype(np.float64)
    lse = np.log(np.exp(s).sum(1))
    want = float((val * (lse - s[np.arange(len(user)), item])).sum())
    # a user's part in fp32, sums of at most two terms: 2^-20 of the terms' sizes (scores below 4, log-sum-exps below 5)
    assert abs(got - want) <= 2.0**-20 * float((val * 9).sum())
    rated = [set(item[user == u]) for u in user]
    order = np.argsort(-s, axis=1, kind="stable")
    for r in range(len(user)):
        assert list(best[r]) == [j for j in order[r] if j not in rated[r]][:2]
