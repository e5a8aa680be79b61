"""The training side of the router and the pool, as cases that can be timed and compared.

The prefill router picks a pool entry for every history position (`ckv_route`); the pool rows it picks are what
attention reads.  Fitting the two takes, for each side (keys, values) and step, the five operators below.

  sort         positions ordered by the pool entry they picked, and where each entry's run begins
  loss         log-sum-exp of the router's scores, score of the picked entry, mean selection probability per entry, the
               load-balance loss sum_j p_j log(p_j m) and the peak loss -mean_i log sigmoid(score_i) of every group
  loss_grad    the gradients of both losses, and of whatever else depends on the picked scores, by x, W and bias
  gather       rows  user part | sigmoid(score) * pool row
  gather_grad  the gradients by the pool, the user parts and the scores

A position whose index lies outside [0, m) is padding: it takes no part, and its pool row is zero.

Shapes are those of the benchmark workloads (`synth.WORKLOADS`) and of the prefill cases, or lie between them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
BALANCE_WEIGHT, PEAK_WEIGHT = 1.0, 0.01   # what the paper trains with


def listed():
    return [
        # One user's history on its own: what an online learner handles at low load.  Launches and latency count.
        dict(name="sort_user", kind="sort", n=200, groups=2, pool=1024, zipf=0.0, pad=0.0),
        # The histories of a training batch, skewed towards few entries (workload cfg2's positions).
        dict(name="sort_batch", kind="sort", n=1048576, groups=8, pool=4096, zipf=1.1, pad=0.1),
        dict(name="loss_user", kind="loss", n=200, groups=2, pool=1024, d_in=64, spread=1.0, bias=True, pad=0.0),
        # A padded batch of odd size, a router without bias that has become decided.
        dict(name="loss_padded", kind="loss", n=10007, groups=3, pool=4099, d_in=32, spread=3.0, bias=False, pad=0.3),
        # 64 users of 512 positions against a large pool (workload cfg4's).
        dict(name="loss_batch", kind="loss", n=32768, groups=4, pool=16384, d_in=64, spread=1.0, bias=True, pad=0.0),
        dict(name="grad_user", kind="loss_grad", n=200, groups=2, pool=1024, d_in=64, spread=1.0, bias=True, pad=0.0,
             gated=True),
        dict(name="grad_padded", kind="loss_grad", n=10007, groups=3, pool=4099, d_in=128, spread=3.0, bias=False,
             pad=0.3, gated=True),
        # The balance and peak losses alone: the router is fitted behind a frozen model.
        dict(name="grad_batch", kind="loss_grad", n=32768, groups=4, pool=16384, d_in=64, spread=1.0, bias=True,
             pad=0.0, gated=False),
        # A small model in fp32, one user (workload cfg1).
        dict(name="gather_user", kind="gather", dtype="f32", n=200, groups=2, head_dim=32, d_user=4, pool=1024,
             zipf=0.0, pad=0.0, gated=True),
        # A batch's keys rebuilt (workload cfg2).
        dict(name="gather_batch", kind="gather", dtype="bf16", n=1048576, groups=8, head_dim=32, d_user=2, pool=4096,
             zipf=1.1, pad=0.0, gated=True),
        # A padded batch of odd size whose head of the pool takes most of the gradient.
        dict(name="gather_grad_padded", kind="gather_grad", dtype="bf16", n=20011, groups=4, head_dim=64, d_user=1,
             pool=10000, zipf=1.2, pad=0.3, gated=False),
        # A batch's key gradients (workload cfg4's pool).
        dict(name="gather_grad_batch", kind="gather_grad", dtype="bf16", n=1048576, groups=4, head_dim=64, d_user=4,
             pool=16384, zipf=1.05, pad=0.0, gated=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sort", "loss", "loss", "loss_grad", "loss_grad", "gather", "gather_grad", "gather_grad"])
    groups = rng.choice([1, 2, 3, 4, 8])
    pad = rng.choice([0.0, 0.0, 0.1, 0.5])
    case = dict(kind=kind, groups=groups, pad=pad)
    if kind in ("loss", "loss_grad"):
        pool = _log(rng, 64, 16384)
        n = min(_log(rng, 1, 131072), (1 << 31) // (pool * groups))
        case.update(n=n, pool=pool, d_in=rng.choice([32, 64, 64, 128]), spread=rng.choice([0.5, 1.0, 3.0]),
                    bias=rng.random() < 0.7)
        if case["d_in"] == 128:
            case["n"] = max(1, n // 2)
    else:
        case.update(n=_log(rng, 1, 1048576), pool=_log(rng, 64, 70000), zipf=rng.choice([0.0, 1.05, 1.1, 1.2]))
        if kind != "sort":
            dtype, head_dim = rng.choice([("bf16", 32), ("bf16", 64), ("bf16", 128), ("f32", 16), ("f32", 32)])
            case.update(dtype=dtype, head_dim=head_dim, d_user=rng.choice([0, 1, 2, 4, 5, 8]))
            case["n"] = max(1, min(case["n"], (1 << 28) // (groups * head_dim)))
    if kind not in ("sort", "loss"):
        case["gated"] = rng.random() < 0.6
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------

def _indices(g, n, groups, m, zipf):
    """[n][groups] int32; Zipf: P(rank r) ~ r^-s, ranks mapped to entries by a permutation per group."""
    if zipf == 0.0:
        return torch.randint(0, m, (n, groups), generator=g, device="cuda", dtype=torch.int32)
    w = torch.arange(1, m + 1, device="cuda", dtype=torch.float64).pow_(-zipf)
    cdf = torch.cumsum(w, 0).div_(w.sum()).float()
    rank = torch.searchsorted(cdf, torch.rand((n, groups), generator=g, device="cuda")).clamp_(max=m - 1)
    perm = torch.stack([torch.randperm(m, generator=g, device="cuda", dtype=torch.int32) for _ in range(groups)])
    return perm.gather(1, rank.t()).t().contiguous()


def _padding(g, idx, pad):
    """Whole positions without an entry, as a padded batch has them."""
    if pad > 0.0:
        idx[torch.rand(idx.shape[0], generator=g, device="cuda") < pad] = -1
    return idx


def _ordered(idx, m):
    """order [G][n], offset [G][m + 1], both int32: positions by entry, padding last."""
    key = torch.where((idx >= 0) & (idx < m), idx, m).t().contiguous()
    order = torch.sort(key, dim=1, stable=True)[1].int()
    count = torch.zeros((key.shape[0], m + 1), dtype=torch.int64, device=key.device)
    count.scatter_add_(1, key.long(), torch.ones_like(key, dtype=torch.int64))
    offset = torch.zeros((key.shape[0], m + 1), dtype=torch.int32, device=key.device)
    offset[:, 1:] = torch.cumsum(count[:, :m], 1)
    return order, offset


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, n, G, m = case["kind"], case["n"], case["groups"], case["pool"]
    st = dict(kind=kind, m=m, case=case)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)

    if kind in ("loss", "loss_grad"):
        d = case["d_in"]
        x, W = normal(n, d, std=d ** -0.5, dtype=torch.bfloat16), normal(G, m, d, std=case["spread"], dtype=torch.bfloat16)
        bias = normal(G, m, std=0.1) if case["bias"] else None
        picked = []
        for k in range(G):  # the router's choice
            s = x @ W[k].t()
            picked.append((s if bias is None else s.add_(bias[k])).argmax(1).int())
            del s
        idx = _padding(g, torch.stack(picked, 1), case["pad"])
        st.update(x=x, W=W, bias=bias, idx=idx)
        if kind == "loss_grad":
            loss, lse, score, mean = _plain_loss(st)
            st.update(lse=lse, score=score, mean=mean, sorted=_ordered(idx, m),
                      d_score=normal(n, G, std=0.01 / n) if case["gated"] else None)
        return st
    st["idx"] = _padding(g, _indices(g, n, G, m, case["zipf"]), case["pad"])
    if kind == "sort":
        return st
    dtype, D, du = DTYPES[case["dtype"]], case["head_dim"], case["d_user"]
    st.update(du=du, pool=normal(G, m, D - du, std=D ** -0.5, dtype=dtype),
              score=normal(n, G).add_(3.0) if case["gated"] else None)  # a winner's score lies well above the others'
    if kind == "gather":
        st["user"] = normal(n, G, du, std=D ** -0.5, dtype=dtype) if du else None
    else:
        st.update(d_out=normal(n, G, D, std=1.0 / n, dtype=dtype), sorted=_ordered(st["idx"], m))
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------

def _valid(st):
    return (st["idx"] >= 0) & (st["idx"] < st["m"])


def _scores(st):
    """[G][n][m]"""
    M = torch.matmul(st["x"].float(), st["W"].float().transpose(1, 2))
    return M if st["bias"] is None else M.add_(st["bias"][:, None, :])


def _plain_loss(st):
    valid, m = _valid(st), st["m"]
    M = _scores(st)
    rows = valid.sum(0)
    at = st["idx"].clamp(0, m - 1).long().t()[:, :, None]
    score = torch.where(valid, M.gather(2, at)[:, :, 0].t(), 0.0)
    top = M.amax(2, keepdim=True)
    e = M.sub_(top).exp_()
    total = e.sum(2, keepdim=True)
    lse = torch.where(valid, (total.log() + top)[:, :, 0].t(), 0.0)
    weight = torch.where(valid, 1.0, 0.0).t()[:, :, None] / total
    mean = e.mul_(weight).sum(1) / rows.clamp(min=1)[:, None]
    # sum_j p_j log(p_j m) in 64 bits: near balance the terms cancel (sum_j p_j = 1 is taken off term by term)
    y = mean.double() * m
    balance = torch.where(rows > 0, (torch.xlogy(y, y) - y + 1).mean(1), 0.0)
    soft = torch.clamp(-score, min=0) + torch.log1p(torch.exp(-score.abs()))     # -log sigmoid(score)
    peak = torch.where(valid, soft.double(), 0.0).sum(0) / rows.clamp(min=1)
    return torch.stack([balance, peak], 1).float(), lse.contiguous(), score.contiguous(), mean


def _plain_loss_grad(st):
    valid, m = _valid(st), st["m"]
    rows = valid.sum(0).clamp(min=1)
    p = _scores(st).sub_(st["lse"].t()[:, :, None]).exp_().mul_(valid.t()[:, :, None])
    h = torch.where(st["mean"] > 0, torch.log(st["mean"] * m), 0.0)
    r = (p * h[:, None, :]).sum(2, keepdim=True)
    dM = (h[:, None, :] - r).mul_(p).mul_((BALANCE_WEIGHT / rows)[:, None, None])
    del p
    d_score = -PEAK_WEIGHT / rows * torch.sigmoid(-st["score"])
    if st["d_score"] is not None:
        d_score = d_score + st["d_score"]
    d_score = torch.where(valid, d_score, 0.0).t()[:, :, None]
    dM.scatter_add_(2, st["idx"].clamp(0, m - 1).long().t()[:, :, None], d_score)
    dx = torch.matmul(dM, st["W"].float()).sum(0)
    dW = torch.matmul(dM.transpose(1, 2), st["x"].float())
    return dict(dx=dx.bfloat16(), dW=dW.bfloat16(), dbias=dM.sum(1))


def _gate(st):
    """[n][G]: 0 for padding."""
    one = torch.ones_like(st["idx"], dtype=torch.float32) if st["score"] is None else torch.sigmoid(st["score"])
    return torch.where(_valid(st), one, 0.0)


def _rows(st):
    """Flat pool row of every (position, group); padding points to row 0 of its group."""
    G, m = st["pool"].shape[:2]
    return torch.where(_valid(st), st["idx"], 0).long() + torch.arange(G, device="cuda") * m


def _plain_gather(st):
    pool = st["pool"].float().flatten(0, 1)
    out = pool[_rows(st)] * _gate(st)[:, :, None]
    return (out if st["user"] is None else torch.cat([st["user"].float(), out], 2)).to(st["pool"].dtype)


def _plain_gather_grad(st):
    G, m, ds = st["pool"].shape
    row, gate = _rows(st), _gate(st)
    d_row = st["d_out"][:, :, st["du"]:].float()
    d_pool = torch.zeros((G * m, ds), device="cuda")
    d_pool.index_add_(0, row.flatten(), (d_row * gate[:, :, None]).flatten(0, 1))
    out = dict(d_pool=d_pool.view(G, m, ds))
    if st["du"]:
        out["d_user"] = st["d_out"][:, :, :st["du"]].contiguous()
    if st["score"] is not None:
        out["d_score"] = (st["pool"].float().flatten(0, 1)[row] * d_row).sum(2) * gate * torch.sigmoid(-st["score"])
    return out


# ---- one pass -------------------------------------------------------------------------------------------------

def run(st):
    kind = st["kind"]
    if own:
        import paper_2601_19178_b200 as ckv
        if kind == "sort":
            order, offset = ckv.sort_indices(st["idx"], st["m"])
            return dict(order=order, offset=offset)
        if kind == "loss":
            loss, lse, score, mean = ckv.route_loss(st["x"], st["W"], st["bias"], st["idx"])
            return dict(loss=loss, lse=lse, score=score, mean=mean)
        if kind == "loss_grad":
            dx, dW, dbias = ckv.route_loss_grad(st["x"], st["W"], st["bias"], st["idx"], st["sorted"], st["lse"],
                                                st["score"], st["mean"], BALANCE_WEIGHT, PEAK_WEIGHT, st["d_score"])
            return dict(dx=dx, dW=dW, dbias=dbias)
        if kind == "gather":
            return ckv.gather(st["pool"], st["idx"], st["user"], st["score"])
        d_pool, d_user, d_score = ckv.gather_grad(st["pool"], st["sorted"], st["score"], st["d_out"])
        return {k: v for k, v in dict(d_pool=d_pool, d_user=d_user, d_score=d_score).items() if v is not None}
    if kind == "sort":
        order, offset = _ordered(st["idx"], st["m"])
        return dict(order=order, offset=offset)
    if kind == "loss":
        return dict(zip(("loss", "lse", "score", "mean"), _plain_loss(st)))
    if kind == "loss_grad":
        return _plain_loss_grad(st)
    return _plain_gather(st) if kind == "gather" else _plain_gather_grad(st)


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    """Inputs read once and outputs written once.  loss: one product per (position, entry); loss_grad: that one again
    and two more."""
    kind, n, G, m = case["kind"], case["n"], case["groups"], case["pool"]
    if kind == "sort":
        return {"bytes": 8.0 * n * G + 4.0 * G * (m + 1), "flops": 0}
    if kind in ("loss", "loss_grad"):
        d, pairs = case["d_in"], float(n) * m * G
        inputs = 2.0 * n * d + 2.0 * G * m * d + 4.0 * n * G + (4.0 * G * m if case["bias"] else 0)
        if kind == "loss":
            return {"bytes": inputs + 8.0 * n * G + 4.0 * G * m + 8.0 * G, "flops": 2.0 * d * pairs}
        more = 8.0 * n * G + 4.0 * G * m + (4.0 * n * G if case["gated"] else 0) + 4.0 * n * G
        return {"bytes": inputs + more + 2.0 * n * d + G * m * (2.0 * d + 4.0), "flops": 6.0 * d * pairs}
    e, D, du = BYTES[case["dtype"]], case["head_dim"], case["d_user"]
    bytes_ = 4.0 * n * G + (4.0 * n * G if case["gated"] else 0) + float(n) * G * (D + du) * e
    rows = min(float(n), float(m)) * G * (D - du)   # pool rows that can be touched
    if kind == "gather":
        return {"bytes": bytes_ + rows * e, "flops": float(n) * G * (D - du)}
    bytes_ += 4.0 * G * m * (D - du) + ((4.0 * n * G + rows * e) if case["gated"] else 0)
    return {"bytes": bytes_, "flops": (4.0 if case["gated"] else 1.0) * n * G * (D - du)}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

def _exact_loss(st):
    """Group by group and block of positions by block, from the sums as they are written."""
    n, G, m = st["x"].shape[0], st["W"].shape[0], st["m"]
    lse = torch.zeros((n, G), dtype=torch.float64, device="cuda")
    score, mean, loss = torch.zeros_like(lse), torch.zeros((G, m), dtype=torch.float64, device="cuda"), []
    for k in range(G):
        balance = peak = torch.zeros((), dtype=torch.float64, device="cuda")
        members = torch.nonzero((st["idx"][:, k] >= 0) & (st["idx"][:, k] < m))[:, 0]
        for part in members.split(4096):
            s = st["x"][part].double() @ st["W"][k].double().t()
            if st["bias"] is not None:
                s += st["bias"][k].double()
            lse[part, k] = torch.logsumexp(s, 1)
            score[part, k] = s[torch.arange(len(part), device="cuda"), st["idx"][part, k].long()]
            mean[k] += torch.softmax(s, 1).sum(0) / len(members)
        if len(members):
            balance = torch.xlogy(mean[k], mean[k] * m).sum()
            peak = -torch.nn.functional.logsigmoid(score[members, k]).mean()
        loss.append(torch.stack([balance, peak]))
    return dict(loss=torch.stack(loss), lse=lse, score=score, mean=mean)


def _exact_loss_grad(st):
    n, d = st["x"].shape
    G, m = st["W"].shape[0], st["m"]
    dx = torch.zeros((n, d), dtype=torch.float64, device="cuda")
    dW, dbias = torch.zeros((G, m, d), dtype=torch.float64, device="cuda"), torch.zeros((G, m), dtype=torch.float64, device="cuda")
    for k in range(G):
        members = torch.nonzero((st["idx"][:, k] >= 0) & (st["idx"][:, k] < m))[:, 0]
        u = st["mean"][k].double() * m
        h = torch.where(u > 0, torch.log(u), 0.0)
        for part in members.split(4096):
            x, W = st["x"][part].double(), st["W"][k].double()
            s = x @ W.t()
            if st["bias"] is not None:
                s += st["bias"][k].double()
            p = torch.exp(s - st["lse"][part, k].double()[:, None])
            t = p * (h - (p @ h)[:, None]) * (BALANCE_WEIGHT / len(members))
            picked = -PEAK_WEIGHT / len(members) / (1 + torch.exp(st["score"][part, k].double()))
            if st["d_score"] is not None:
                picked = picked + st["d_score"][part, k].double()
            t[torch.arange(len(part), device="cuda"), st["idx"][part, k].long()] += picked
            dx[part] += t @ W
            dW[k] += t.t() @ x
            dbias[k] += t.sum(0)
    return dict(dx=dx, dW=dW, dbias=dbias)


def _exact_gather(st):
    n, G = st["idx"].shape
    parts = []
    for k in range(G):
        i = st["idx"][:, k].long()
        real = (i >= 0) & (i < st["m"])
        row = st["pool"][k].double()[i.clamp(0, st["m"] - 1)]
        if st["score"] is not None:
            row = row / (1 + torch.exp(-st["score"][:, k].double()))[:, None]
        row[~real] = 0
        parts.append(row if st["user"] is None else torch.cat([st["user"][:, k].double(), row], 1))
    return torch.stack(parts, 1)


def _exact_gather_grad(st):
    n, G = st["idx"].shape
    m, du = st["m"], st["du"]
    d_pool, d_score = [], []
    for k in range(G):
        members = torch.nonzero((st["idx"][:, k] >= 0) & (st["idx"][:, k] < m))[:, 0]
        i = st["idx"][members, k].long()
        d_row = st["d_out"][members, k, du:].double()
        gate = torch.ones(len(members), dtype=torch.float64, device="cuda")
        if st["score"] is not None:
            gate = 1 / (1 + torch.exp(-st["score"][members, k].double()))
            ds = torch.zeros(n, dtype=torch.float64, device="cuda")
            ds[members] = gate * (1 - gate) * (st["pool"][k].double()[i] * d_row).sum(1)
            d_score.append(ds)
        d_pool.append(torch.zeros((m, d_row.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, i, gate[:, None] * d_row))
    out = dict(d_pool=torch.stack(d_pool))
    if du:
        out["d_user"] = st["d_out"][:, :, :du].double()
    if d_score:
        out["d_score"] = torch.stack(d_score, 1)
    return out


def exact(case, seed):
    if case["kind"] == "sort":
        return None
    st = prepare(case, seed)
    return {"loss": _exact_loss, "loss_grad": _exact_loss_grad, "gather": _exact_gather,
            "gather_grad": _exact_gather_grad}[case["kind"]](st)
