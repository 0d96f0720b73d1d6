"""The operators over a whole item table, as cases that can be timed and compared.

A factor model scores every item for a row (a user, a token) as the product of the row's K
numbers with the item's.  Three operators work on the softmax or the order of those scores,
none of them keeping the rows x items matrix:

* ``xent``: softmax cross entropy of each row's target items, with the gradients of both tables;
* ``distill``: the divergence from a teacher's top scores, with the gradients of both tables;
* ``top``: each row's k best items in the order of their scores, ties to the lowest item.

Definitions.  s_ij = x_i . w_j over items j; lse_i = log sum_j exp s_ij.

xent: row i has targets (j, v); loss_i = sum v (lse_i - s_ij), dX and dW are the gradients of
sum_i weight_i loss_i.  The same item twice counts twice; an item < 0 is no target.  A row with no
target or of weight 0 is read as a row of zeros: its loss is 0 and so is its gradient.

distill: row i has the teacher's scores t of some items; with q = softmax(t / tau) over them (or
exp(t / tau - tlse_i), tlse_i the teacher's own log-sum-exp over all its items), p = softmax(s / tau)
over all items and lse_i that softmax's log-sum-exp, loss_i = tau^2 sum q (log q - log p).  An
item < 0 or a score of -inf is no entry; rows without one, and weights, as above.

top: the k largest s_ij among the items that the row does not exclude, in decreasing order;
where fewer are left, item -1 with score -inf.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, n, M, K, **more):
    return {"name": name, "op": op, "n": n, "M": M, "K": K, "type": "f32"} | more


def _xent(name, n, M, K, *, mean=200, grad=True, masked=0.0, type="f32"):
    """mean: target items per row, 0 for one label per row."""
    return _case(name, "xent", n, M, K, mean=mean, grad=grad, masked=masked, type=type)


def _distill(name, n, M, K, k, *, tau=2.0, full=False, grad=True, masked=0.0, type="f32"):
    """full: the teacher's log-sum-exp is given too."""
    return _case(name, "distill", n, M, K, k=k, tau=tau, full=full, grad=grad, masked=masked, type=type)


def _top(name, n, M, K, k, *, mean=0, type="f32"):
    """mean: excluded items per row."""
    return _case(name, "top", n, M, K, k=k, mean=mean, type=type)


def listed():
    return [
        # the held-out loss of one user of the Netflix-shaped model, as a service asks for it: latency
        _xent("xent one user", 1, 17_770, 128, grad=False),
        # a training step of the medium model on a minibatch of users, each with their ratings
        _xent("xent minibatch", 256, 20_000, 64, mean=100),
        # a full training step of the headline model on a large batch of users
        _xent("xent netflix users", 16_384, 17_770, 128, mean=208),
        # words of the paper's vocabulary predicted one per row, tables in half the bytes, a padded batch
        _xent("xent vocabulary bf16", 8192, 100_000, 256, mean=0, masked=0.1, type="bf16"),
        # held-out loss at ragged sizes and the rank of the topic model
        _xent("xent evaluation ragged", 20_011, 9999, 100, mean=37, grad=False),
        # the tiny model taught by a larger one
        _distill("distill tiny", 300, 500, 16, 10),
        # a student of half the headline rank, 64 of the teacher's items per user
        _distill("distill netflix student", 8192, 17_770, 64, 64, full=True),
        # next-word teaching over the paper's vocabulary, short teacher lists, a padded batch
        _distill("distill vocabulary bf16", 4096, 100_000, 128, 32, tau=1.0, masked=0.1, type="bf16"),
        # one user asks for a page of recommendations without what they rated already
        _top("top one user", 1, 17_770, 128, 10, mean=208),
        # a service's batch of users
        _top("top service batch", 64, 20_000, 64, 20, mean=100),
        # the teacher's lists for distillation, a large batch
        _top("top teacher lists", 8192, 17_770, 128, 64),
        # half-precision tables over the paper's vocabulary, ragged
        _top("top vocabulary f16", 2047, 100_000, 100, 100, mean=20, type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("xent", "xent", "distill", "distill", "top"))
    n, M = _log(rng, 1, 20_000), _log(rng, 300, 120_000)
    K = rng.choice((8, 16, 20, 32, 33, 50, 64, 64, 100, 128, 128, 200, 256))
    type = rng.choice(("f32", "f32", "bf16", "f16"))
    while n * M * K > (15_000_000_000 if op == "top" else 35_000_000_000):  # no dearer than the listed ones
        n = max(1, n // 2)
    if op == "top":
        k = min(rng.choice((1, 5, 10, 20, 64, 100, 200)), M // 4)
        c = _top("", n, M, K, k, mean=rng.choice((0, 0, 20, 150)), type=type)
    elif op == "distill":
        c = _distill("", n, M, K, rng.choice((1, 4, 10, 32, 64, 100)), tau=rng.choice((0.7, 1.0, 2.0, 4.0)),
                     full=rng.random() < 0.4, grad=rng.random() < 0.8, masked=rng.choice((0.0, 0.0, 0.2)), type=type)
    else:
        c = _xent("", n, M, K, mean=rng.choice((0, 0, 5, 40, 200)), grad=rng.random() < 0.8,
                  masked=rng.choice((0.0, 0.0, 0.2)), type=type)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _gen(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + case["n"] * 31 + case["M"] * 7 + case["K"])
    return g


def _table(g, rows, K, spread):
    """Rows of normal numbers whose lengths vary as those of trained factors do; products of two
    tables have a standard deviation of about 2."""
    x = torch.randn(rows, K, generator=g, device="cuda") * (math.sqrt(2.0) / K ** 0.25)
    return x * torch.exp(spread * torch.randn(rows, 1, generator=g, device="cuda"))


def _lists(g, n, M, mean):
    """Item lists of n rows: heavy-tailed lengths, popular items more often, the same item twice in a
    row now and then."""
    length = torch.exp(0.8 * torch.randn(n, generator=g, device="cuda")) * (mean * 0.73)
    length = length.round().clamp(0, min(4 * mean, max(1, M // 3))).to(torch.int64)
    if n > 4:
        length[n // 2] = 0  # a user without a rating
    else:
        length = length.clamp(min=1)
    row_ptr = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    row_ptr[1:] = length.cumsum(0)
    nnz = int(row_ptr[-1])
    u = torch.rand(nnz, generator=g, device="cuda")
    place = (u ** 3 * M).to(torch.int64).clamp(max=M - 1)
    item = torch.randperm(M, generator=g, device="cuda")[place].to(torch.int32)
    return row_ptr, item


def prepare(case, seed):
    g = _gen(case, seed)
    n, M, K, dtype = case["n"], case["M"], case["K"], TYPES[case["type"]]
    x, w = _table(g, n, K, 0.2), _table(g, M, K, 0.3)
    st = {"case": case, "X": x.to(dtype), "W": w.to(dtype)}
    if case["op"] == "top":
        if case["mean"]:
            st["row_ptr"], st["item"] = _lists(g, n, M, case["mean"])
        return st
    if case["grad"]:
        st["weight"] = torch.rand(n, generator=g, device="cuda") / n
    if case["op"] == "xent":
        if case["mean"]:
            st["row_ptr"], st["item"] = _lists(g, n, M, case["mean"])
            st["value"] = torch.randint(1, 6, st["item"].shape, generator=g, device="cuda").to(torch.float32)
        else:
            st["item"] = (torch.rand(n, generator=g, device="cuda") ** 3 * M).to(torch.int32).clamp(max=M - 1)
        if case["masked"] and not case["mean"]:
            st["item"][torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
        return st
    # the teacher: the student's scores and much that the student does not know, its best k items
    k = min(case["k"], M)
    scores, items, lses = [], [], []
    xt = torch.cat((x, torch.randn(n, 16, generator=g, device="cuda") * 0.7), 1)
    wt = torch.cat((w, torch.randn(M, 16, generator=g, device="cuda") * 0.7), 1).t().contiguous()
    for i in range(0, n, 2048):
        s = xt[i:i + 2048] @ wt
        lses.append(torch.logsumexp(s / case["tau"], 1))
        t = torch.topk(s, k, dim=1)
        scores.append(t.values)
        items.append(t.indices.to(torch.int32))
    st["score"], st["item"] = torch.cat(scores).contiguous(), torch.cat(items).contiguous()
    if case["full"]:
        st["tlse"] = torch.cat(lses)
    if case["masked"]:
        off = torch.rand(n, generator=g, device="cuda") < case["masked"]
        st["item"][off] = -1
        st["item"][~off & (torch.rand(n, generator=g, device="cuda") < 0.3), k // 2:] = -1  # short lists
    return st


# ------------------------------------------------------------------ the framework's calls
_handles = {}


def _handle(st):
    """The handle that a program keeps for a table's shape and type."""
    from paper_1410_8043_amd import ps_soft

    c = st["case"]
    key = (c["M"], c["K"], c["type"])
    if key not in _handles:
        _handles[key] = ps_soft.PsSoft(c["M"], c["K"], TYPES[c["type"]])
    return _handles[key]


def _own(st):
    c, h = st["case"], _handle(st)
    if c["op"] == "top":
        return h.top(st["X"], st["W"], c["k"], row_ptr=st.get("row_ptr"), item=st.get("item"))
    if c["op"] == "xent":
        return h.xent(st["X"], st["W"], st["item"], row_ptr=st.get("row_ptr"), value=st.get("value"),
                      weight=st.get("weight"), grad=c["grad"])
    return h.distill(st["X"], st["W"], st["item"], st["score"], tau=c["tau"], tlse=st.get("tlse"),
                     weight=st.get("weight"), grad=c["grad"])


# ------------------------------------------------------------------ the plain forms
def _plain_softmax(st, rows, item, value, total, live, scale, gain, entropy):
    """loss_i = gain (entropy_i + total_i lse_i - sum value s / scale) over the entries (rows, item, value), and its
    gradients; lse over s / scale."""
    x, w = st["X"].float(), st["W"].float()
    weight = st.get("weight")
    if weight is not None:
        live = live & (weight != 0)
    x = torch.where(live[:, None], x, 0.0)
    value = torch.where(live[rows], value, 0.0)
    total = torch.where(live, total, 0.0)
    s = (x @ w.t()) / scale
    top = s.max(1, keepdim=True).values
    picked = s[rows, item]
    p = torch.exp(s - top)
    den = p.sum(1, keepdim=True)
    lse = (top + torch.log(den))[:, 0]
    loss = total * lse + torch.where(live, entropy, 0.0)
    loss = gain * loss.index_add(0, rows, -value * picked)
    if not st["case"]["grad"]:
        return loss, lse
    p = p * (total[:, None] / den)
    p.view(-1).index_add_(0, rows * s.shape[1] + item, -value)
    p = p * (torch.where(live, weight, 0.0) * (gain / scale))[:, None]
    return loss, lse, (p @ w).to(st["X"].dtype), (p.t() @ x).to(st["W"].dtype)


def _plain_xent(st):
    n = st["X"].shape[0]
    item = st["item"].to(torch.int64)
    if "row_ptr" in st:
        length = st["row_ptr"][1:] - st["row_ptr"][:-1]
        rows = torch.repeat_interleave(torch.arange(n, device=item.device), length, output_size=item.shape[0])
        value = st["value"]
    else:
        rows, value = torch.arange(n, device=item.device), torch.ones(n, device=item.device)
    value = torch.where(item >= 0, value, 0.0)
    some = torch.zeros(n, device=item.device).index_add(0, rows, (item >= 0).float()) > 0
    total = torch.zeros(n, device=item.device).index_add(0, rows, value)
    return _plain_softmax(st, rows, item.clamp(min=0), value, total, some, 1.0, 1.0, torch.zeros_like(total))


def _plain_distill(st):
    tau = st["case"]["tau"]
    n, k = st["item"].shape
    item = st["item"].to(torch.int64)
    there = (item >= 0) & (st["score"] > -math.inf)
    t = torch.where(there, st["score"] / tau, -math.inf)
    some = there.any(1)
    if "tlse" in st:
        logq = t - st["tlse"][:, None]
    else:
        top = torch.where(some, t.max(1).values, 0.0)[:, None]
        logq = t - top - torch.log(torch.exp(t - top).sum(1, keepdim=True))
    q = torch.where(there, torch.exp(logq), 0.0)
    entropy = torch.where(q > 0, q * logq, 0.0).sum(1)
    rows = torch.arange(n, device=item.device)[:, None].expand(n, k)
    return _plain_softmax(st, rows.reshape(-1), item.clamp(min=0).reshape(-1), q.reshape(-1), q.sum(1), some, tau,
                          tau * tau, entropy)


def _plain_top(st):
    c = st["case"]
    # which of two near scores is larger: in 64 bits
    s = st["X"].double() @ st["W"].double().t()
    if "row_ptr" in st:
        length = st["row_ptr"][1:] - st["row_ptr"][:-1]
        rows = torch.repeat_interleave(torch.arange(c["n"], device=s.device), length, output_size=st["item"].shape[0])
        s[rows, st["item"].to(torch.int64)] = -math.inf
    s, item = torch.sort(s, dim=1, descending=True, stable=True)
    s, item = s[:, :c["k"]], item[:, :c["k"]].to(torch.int32)
    return torch.where(s > -math.inf, item, -1), s.to(torch.float32)


def run(state):
    if own:
        return _own(state)
    return {"xent": _plain_xent, "distill": _plain_distill, "top": _plain_top}[state["case"]["op"]](state)


# ------------------------------------------------------------------ what the work is
def work(case):
    """Products: the scores once, each gradient once.  Bytes: both tables and the lists once, the
    outputs once."""
    n, M, K = case["n"], case["M"], case["K"]
    size = 4 if case["type"] == "f32" else 2
    data = (n + M) * K * size
    if case["op"] == "top":
        return {"bytes": data + n * case["mean"] * 4 + n * case["k"] * 8, "flops": 2.0 * n * M * K}
    entries = n * case["k"] * 8 if case["op"] == "distill" else n * max(1, case["mean"]) * (8 if case["mean"] else 4)
    grad = case["grad"]
    return {"bytes": data * (2 if grad else 1) + entries + n * 12, "flops": (6.0 if grad else 2.0) * n * M * K}


# ------------------------------------------------------------------ in 64 bits, from the definitions
def exact(case, seed):
    st = prepare(case, seed)
    n, M = case["n"], case["M"]
    X, W = st["X"].double(), st["W"].double()
    step = max(1, min(n, 250_000_000 // M))
    if case["op"] == "top":
        score = []
        for a in range(0, n, step):
            s = X[a:a + step].matmul(W.t())
            if "row_ptr" in st:
                b = min(n, a + step)
                beg, end = int(st["row_ptr"][a]), int(st["row_ptr"][b])
                at = torch.bucketize(torch.arange(beg, end, device="cuda"), st["row_ptr"][a + 1:b + 1], right=True)
                s.index_put_((at, st["item"][beg:end].long()), torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
            score.append(s.topk(case["k"], 1).values)
        return None, torch.cat(score)
    # one dense matrix of target weights per piece of rows: loss = sum_j y_ij (log y_ij-part - log p_ij)
    tau = case.get("tau", 1.0)
    loss, lse, dX, dW = [], [], [], torch.zeros_like(W)
    for a in range(0, n, step):
        b = min(n, a + step)
        m = b - a
        y = torch.zeros(m, M, dtype=torch.float64, device="cuda")
        negent = torch.zeros(m, dtype=torch.float64, device="cuda")
        if case["op"] == "xent":
            if case["mean"]:
                beg, end = int(st["row_ptr"][a]), int(st["row_ptr"][b])
                at = torch.bucketize(torch.arange(beg, end, device="cuda"), st["row_ptr"][a + 1:b + 1], right=True)
                j, v = st["item"][beg:end].long(), st["value"][beg:end].double()
            else:
                at, j = torch.arange(m, device="cuda"), st["item"][a:b].long()
                v = torch.ones(m, dtype=torch.float64, device="cuda")
        else:
            j = st["item"][a:b].long()
            t = st["score"][a:b].double().div(tau).masked_fill(j < 0, -math.inf)
            logq = t - (st["tlse"][a:b].double()[:, None] if case["full"] else torch.logsumexp(t, 1, keepdim=True))
            v = torch.nan_to_num(logq, nan=-math.inf).exp()
            negent = torch.xlogy(v, v).sum(1)
            at = torch.arange(m, device="cuda").repeat_interleave(j.shape[1])
            j, v = j.reshape(-1), v.reshape(-1)
        keep = j >= 0
        at, j, v = at[keep], j[keep], v[keep]
        has = torch.zeros(m, dtype=torch.bool, device="cuda")
        has[at] = True
        gain = torch.ones(m, dtype=torch.float64, device="cuda") * tau * tau
        up = st["weight"][a:b].double() if "weight" in st else torch.ones_like(gain)
        has &= up != 0
        y.index_put_((at, j), v, accumulate=True)
        y[~has] = 0
        x = X[a:b] * has[:, None]
        logit = x.matmul(W.t()).div_(tau)
        z = torch.logsumexp(logit, 1)
        lse.append(z)
        mass = y.sum(1)
        loss.append(gain * (negent * has + mass * z - (y * logit).sum(1)))
        if case["grad"]:
            logit.sub_(z[:, None]).exp_().mul_(mass[:, None]).sub_(y).mul_((up * has * gain / tau)[:, None])
            dX.append(logit.matmul(W))
            dW += logit.t().matmul(x)
    if not case["grad"]:
        return torch.cat(loss), torch.cat(lse)
    return torch.cat(loss), torch.cat(lse), torch.cat(dX), dW
