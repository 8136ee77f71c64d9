"""Operators on rows of factor tables and on the probabilities that factors give over all items, as cases
that can be timed and compared.

H (T x k) holds factor rows of users (or any queries), F (n x k) those of all items; z = scale H F^T + bias
are the scores of every item for every row, and p their softmax over the items.

* ``lookup``: rows of a table by id, scaled; ``lookup_grad``: its gradient, a sum over equal ids.
* ``score``: log sum of exponentials, log probabilities of given items, entropy, the best items.
* ``score_grad``: a training step on log probabilities and entropy: ``score``, then its gradient in H and F.
* ``distill``: a training step against a teacher's best items and their logits: the loss of each row
  (Kullback-Leibler divergence at a temperature) and its gradient in H and F.

Where ``own`` is false the operators are computed in elementary torch operations.  Inputs are synthetic,
from the seed alone: Gaussian factors whose scores spread over a few units, ids with Zipf popularity, a
popularity bias that excludes some items.  ``exact`` follows the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
MARGIN = 32  # candidates beyond the wanted best items that are ranked in 64 bits
_tsid = None


def listed():
    return [
        # serving: the factors of one user
        dict(name="lookup one", op="lookup", T=1, n=480_189, k=64, prec="bf16", pad=0.0),
        # the users of a training pass, by popularity, some of them padding
        dict(name="lookup pass", op="lookup", T=1_000_003, n=1_000_000, k=128, prec="fp32", pad=0.02),
        # a small mini-batch's gradient into a small table
        dict(name="lookup grad batch", op="lookup_grad", T=500, n=8192, k=32, prec="fp32", pad=0.0),
        # gradients of a long history of items into the largest table: a few ids hold much of it
        dict(name="lookup grad history", op="lookup_grad", T=2_000_003, n=1_000_000, k=128, prec="bf16", pad=0.02),
        # serving: ten items for one user out of a million
        dict(name="score one", op="score", T=1, n=1_000_000, k=128, prec="bf16", ids=1, top=10, bias=False),
        # evaluation on a catalogue of ratings: held-out items' probabilities and the best twenty, with a popularity bias
        dict(name="score catalogue", op="score", T=257, n=17_770, k=64, prec="fp32", ids=4, top=20, bias=True),
        # many users against the largest table
        dict(name="score million", op="score", T=2048, n=1_000_000, k=128, prec="bf16", ids=1, top=20, bias=False),
        # a policy step on a small table: log probability of the chosen item and an entropy bonus
        dict(name="score grad small", op="score_grad", T=1000, n=2048, k=32, prec="fp32", ids=1, bias=True),
        # the softmax loss over a whole large table
        dict(name="score grad large", op="score_grad", T=4096, n=100_000, k=128, prec="bf16", ids=1, bias=False),
        # a student of small rank on a template's columns
        dict(name="distill tiny", op="distill", T=200, n=160, k=8, prec="fp32", ids=8, tau=1.0, bias=False),
        # fp32 factors against the most observed items
        dict(name="distill mid", op="distill", T=4096, n=8192, k=64, prec="fp32", ids=20, tau=2.0, bias=True),
        # a large batch against a large table, the teacher's best fifty
        dict(name="distill large", op="distill", T=16_384, n=100_000, k=128, prec="bf16", ids=50, tau=2.0, bias=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: the operators as often as they are listed."""
    op = rng.choice(["lookup"] * 2 + ["lookup_grad"] * 2 + ["score"] * 3 + ["score_grad"] * 2 + ["distill"] * 3)
    k, prec = rng.choice([8, 16, 32, 64, 128]), rng.choice(["fp32", "bf16"])
    if op in ("lookup", "lookup_grad"):
        return dict(op=op, T=_log_uniform(rng, 1, 2_000_000), n=_log_uniform(rng, 100, 1_000_000), k=k, prec=prec,
                    pad=rng.choice([0.0, 0.02, 0.3]))
    n = _log_uniform(rng, 100, 1_000_000)
    most = 16_384 if op == "distill" else 4096
    T = _log_uniform(rng, 1, max(1, min(most, int((4e8 if prec == "fp32" else 1.2e9) / n))))
    case = dict(op=op, T=T, n=n, k=k, prec=prec, bias=rng.random() < 0.5)
    if op == "distill":
        return dict(case, ids=rng.randint(1, min(50, n)), tau=rng.choice([1.0, 2.0, 4.0]))
    if op == "score_grad":
        return dict(case, ids=rng.randint(1, 8))
    return dict(case, ids=rng.randint(1, 8), top=rng.randint(1, 50))


def _dtype(case):
    return torch.bfloat16 if case["prec"] == "bf16" else torch.float32


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 17)
    return g


def _normal(g, shape):
    return torch.randn(shape, generator=g, device=DEV)


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device=DEV)


def _zipf(g, shape, n):
    """Ids with density 1 / (1 + id), popular ones first."""
    r = torch.exp(torch.rand(shape, generator=g, device=DEV, dtype=torch.float64) * math.log(n + 1.0)).to(torch.int64) - 1
    return r.clamp_(0, n - 1)


def prepare(case, seed):
    g, T, n, k = _generator(seed), case["T"], case["n"], case["k"]
    s = dict(case)
    if case["op"] in ("lookup", "lookup_grad"):
        ids = _zipf(g, (T,), n)
        order = torch.randperm(n, generator=g, device=DEV)  # popular ids lie anywhere in the table
        ids = torch.where(_uniform(g, (T,)) < case["pad"], torch.full_like(ids, -1), order[ids])
        s["id"], s["scale"] = ids.to(torch.int32), math.sqrt(k)
        s["rows"] = (0.3 * _normal(g, (n if case["op"] == "lookup" else T, k))).to(_dtype(case))
        return s
    s["H"], s["F"] = _normal(g, (T, k)).to(_dtype(case)), _normal(g, (n, k)).to(_dtype(case))
    s["scale"] = 2.5 / math.sqrt(k)
    s["b"] = None
    if case["bias"]:
        b = -0.7 * torch.log1p(torch.randperm(n, generator=g, device=DEV).float())
        s["b"] = torch.where(_uniform(g, (n,)) < 0.02, torch.full_like(b, -math.inf), b)
    m = case["ids"]
    # a row's listed items differ from one another; popular ones are listed in many rows
    gaps = torch.randint(1, max(2, n // m), (T, m), generator=g, device=DEV)
    at = (_zipf(g, (T, 1), n) + torch.cumsum(gaps, 1) - gaps[:, :1]) % n
    s["id"] = torch.randperm(n, generator=g, device=DEV)[at].to(torch.int32)
    s["id"] = torch.where(_uniform(g, (T, m)) < 0.01, torch.full_like(s["id"], -1), s["id"])
    if case["op"] == "distill":
        s["teacher"] = 6.0 + torch.sort(2.0 * _normal(g, (T, m)), 1, descending=True).values
        s["dloss"] = (0.5 + _uniform(g, (T,))) / T
    if case["op"] == "score_grad":
        s["dlogp"] = -_normal(g, (T, m)) / T
        s["dentropy"] = -0.01 * (0.5 + _uniform(g, (T,))) / T
    return s


# ------------------------------------------------------------------------------------------ plain forms

def _plain_scores(s, tau):
    z = s["H"].float() @ s["F"].float().t()
    z *= s["scale"] / tau
    if s["b"] is not None:
        z += s["b"] / tau
    lse = torch.logsumexp(z, 1)
    return z, lse


def _plain_listed(s, z, lse):
    """The listed items' log probabilities (0 for none), and whether an entry is an item that may be had."""
    at = s["id"].to(torch.int64)
    there = at >= 0
    logp = z.gather(1, at.clamp(min=0)) - lse[:, None]
    return torch.where(there, logp, torch.zeros_like(logp)), there & (logp > -math.inf)


def _plain_best(s, z, lse):
    top = min(s["top"], s["n"])
    near = torch.topk(z, min(s["n"], top + MARGIN), 1).indices.sort(1).values
    exact = (s["H"].double()[:, None, :] * s["F"][near].double()).sum(2) * s["scale"]
    if s["b"] is not None:
        exact = exact + s["b"].double()[near]
    order = torch.sort(exact, dim=1, descending=True, stable=True)
    best = near.gather(1, order.indices[:, :top])
    return best.to(torch.int32), (order.values[:, :top] - lse[:, None]).float()


def _plain_entropy(logp):
    p = torch.exp(logp)
    return -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)


def _plain_products(s, dz, tau):
    dz *= s["scale"] / tau
    return (dz @ s["F"].float()).to(s["H"].dtype), (dz.t() @ s["H"].float()).to(s["F"].dtype)


def _plain(s):
    op = s["op"]
    if op == "lookup":
        at = s["id"].to(torch.int64)
        out = s["rows"][at.clamp(min=0)].float() * s["scale"]
        return torch.where((at >= 0)[:, None], out, torch.zeros_like(out)).to(s["rows"].dtype)
    if op == "lookup_grad":
        at, order = torch.sort(s["id"])
        ends = torch.searchsorted(at, torch.arange(s["n"] + 1, dtype=torch.int32, device=DEV))
        # an id's rows: a difference of running sums, along the contiguous axis
        sums = torch.cumsum(s["rows"][order].t().contiguous().double(), 1) * s["scale"]
        sums = torch.cat([sums.new_zeros((s["k"], 1)), sums], 1)
        return (sums[:, ends[1:]] - sums[:, ends[:-1]]).t().contiguous().to(s["rows"].dtype)
    if op == "score":
        z, lse = _plain_scores(s, 1.0)
        logp, _ = _plain_listed(s, z, lse)
        best, best_logp = _plain_best(s, z, lse)
        z -= lse[:, None]
        return dict(lse=lse, logp=logp, entropy=_plain_entropy(z), top_ids=best, top_logp=best_logp)
    if op == "score_grad":
        z, lse = _plain_scores(s, 1.0)
        logp, there = _plain_listed(s, z, lse)
        z -= lse[:, None]
        entropy = _plain_entropy(z)
        a = torch.where(there, s["dlogp"], torch.zeros_like(s["dlogp"]))
        p = torch.exp(z)
        dz = torch.where(p > 0, z + entropy[:, None], torch.zeros_like(z)).mul_(s["dentropy"][:, None]).add_(a.sum(1)[:, None])
        dz.mul_(p).neg_().scatter_add_(1, s["id"].to(torch.int64).clamp(min=0), a)
        dH, dF = _plain_products(s, dz, 1.0)
        return dict(logp=logp, entropy=entropy, dH=dH, dF=dF)
    tau = s["tau"]
    z, lse = _plain_scores(s, tau)
    logp, there = _plain_listed(s, z, lse)
    t = torch.where(there, s["teacher"] / tau, torch.full_like(logp, -math.inf))
    some = there.any(1)
    logw = t - torch.where(some, torch.logsumexp(t, 1), torch.zeros_like(lse))[:, None]
    w = torch.exp(logw)
    loss = tau * tau * torch.where(there, w * (logw - logp), torch.zeros_like(w)).sum(1)
    u = torch.where(some, s["dloss"], torch.zeros_like(s["dloss"])) * tau * tau
    z -= lse[:, None]
    dz = torch.exp_(z).mul_(u[:, None]).scatter_add_(1, s["id"].to(torch.int64).clamp(min=0), -w * u[:, None])
    dH, dF = _plain_products(s, dz, tau)
    return dict(loss=loss, lse=lse, dH=dH, dF=dF)


# ----------------------------------------------------------------------------------- the framework's calls

def _handle():
    global _tsid
    if _tsid is None:
        import paper_2608_00977_amd as tsid
        _tsid = tsid.Tsid(0)
    return _tsid


def _own(s):
    X, op = _handle(), s["op"]
    if op == "lookup":
        return X.lookup(s["rows"], s["id"], scale=s["scale"])
    if op == "lookup_grad":
        return X.lookup_grad(s["rows"], s["id"], s["n"], scale=s["scale"])
    if op == "score":
        r = X.score(s["H"], s["F"], ids=s["id"], scale=s["scale"], bias=s["b"], top=min(s["top"], s["n"]), entropy=True)
        return dict(lse=r.lse, logp=r.logp, entropy=r.entropy, top_ids=r.top_ids, top_logp=r.top_logp)
    if op == "score_grad":
        r = X.score(s["H"], s["F"], ids=s["id"], scale=s["scale"], bias=s["b"], entropy=True)
        dH, dF = X.score_grad(s["H"], s["F"], r.lse, ids=s["id"], dlogp=s["dlogp"], entropy=r.entropy,
                              dentropy=s["dentropy"], scale=s["scale"], bias=s["b"])
        return dict(logp=r.logp, entropy=r.entropy, dH=dH, dF=dF)
    loss, lse = X.distill(s["H"], s["F"], s["id"], s["teacher"], scale=s["scale"], temperature=s["tau"], bias=s["b"])
    dH, dF = X.distill_grad(s["H"], s["F"], s["id"], s["teacher"], lse, s["dloss"], scale=s["scale"],
                            temperature=s["tau"], bias=s["b"])
    return dict(loss=loss, lse=lse, dH=dH, dF=dF)


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work

def work(case):
    op, T, n, k = case["op"], case["T"], case["n"], case["k"]
    size = 2 if case["prec"] == "bf16" else 4
    if op == "lookup":
        return dict(bytes=4 * T + size * k * (T + min(T, n)), flops=T * k)
    if op == "lookup_grad":
        return dict(bytes=4 * T + size * k * (T + n), flops=T * k)
    m = case["ids"]
    ends = size * k * (T + n) + (4 * n if case["bias"] else 0)
    if op == "score":
        return dict(bytes=ends + 4 * T * (2 + 2 * m + 2 * case["top"]), flops=2 * T * n * k)
    return dict(bytes=ends + size * k * (T + n) + 4 * T * (2 + 3 * m), flops=6 * T * n * k)


# ---------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    ids = s["id"].to(torch.int64)
    if op == "lookup":
        table = torch.cat([s["rows"].double(), torch.zeros((1, s["k"]), dtype=torch.float64, device=DEV)])
        return s["scale"] * table[ids]  # the id -1 takes the last row
    if op == "lookup_grad":
        out = torch.zeros((s["n"] + 1, s["k"]), dtype=torch.float64, device=DEV)
        out.index_add_(0, ids % (s["n"] + 1), s["rows"].double())  # the id -1 adds to the last row
        return s["scale"] * out[:-1]
    tau = case.get("tau", 1.0)
    z = (s["H"].double() * (s["scale"] / tau)) @ s["F"].double().t()
    if s["b"] is not None:
        z += s["b"].double() / tau
    top = z.max(1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    logp = torch.where(ids < 0, 0.0, z.gather(1, ids.clamp(min=0)) - lse[:, None])
    have = (ids >= 0) & torch.isfinite(logp)
    if op == "distill":
        t = torch.exp((s["teacher"].double() - s["teacher"].double().max(1, keepdim=True).values) / tau) * have
        total = t.sum(1, keepdim=True)
        w = torch.where(total > 0, t / total.clamp(min=1e-300), 0.0)
        loss = tau ** 2 * torch.where(have, torch.special.xlogy(w, w) - w * logp, 0.0).sum(1)
        g = torch.exp(z - lse[:, None]) * (w.sum(1) * s["dloss"].double())[:, None]
        g.scatter_add_(1, ids.clamp(min=0), -w * s["dloss"].double()[:, None])
        g *= tau * s["scale"]
        return dict(loss=loss, lse=lse, dH=g @ s["F"].double(), dF=g.t() @ s["H"].double())
    q = z - lse[:, None]
    p = torch.exp(q)
    entropy = -(p * q.clamp(min=-1e6)).sum(1)
    if op == "score":
        best = torch.sort(z, dim=1, descending=True, stable=True) if s["n"] * s["T"] < 3e7 else None
        top = min(s["top"], s["n"])
        values = best.values[:, :top] if best else torch.topk(z, top, 1).values
        return dict(lse=lse, logp=logp, entropy=entropy, top_ids=best.indices[:, :top].to(torch.int32) if best else None,
                    top_logp=values - lse[:, None])
    a = torch.where(have, s["dlogp"].double(), 0.0)
    g = -p * (a.sum(1)[:, None] + s["dentropy"].double()[:, None] * (q.clamp(min=-1e6) + entropy[:, None]))
    g.scatter_add_(1, ids.clamp(min=0), a)
    g *= s["scale"]
    return dict(logp=logp, entropy=entropy, dH=g @ s["F"].double(), dF=g.t() @ s["H"].double())
