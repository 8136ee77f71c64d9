"""The row operators' definitions in 64 bits (numpy), and how far fp32 arithmetic may be from them.

Every bound counts roundings of half a step u = 2^-24 (fp32) or v = 2^-8 (bf16), first order, of
sums of absolute values; nothing in it comes from a run."""
import numpy as np

U, V = 2.0 ** -24, 2.0 ** -8
EXCLUDED = -1e7


def softmax_over(H, F, scale, bias, tau):
    """z / tau with -inf at excluded items, its log sums (-inf for an empty row), and the exclusions."""
    H, F = np.asarray(H, np.float64), np.array(F, np.float64)
    out = np.zeros(F.shape[0], bool) if bias is None else np.asarray(bias) < EXCLUDED
    F[out] = 0.0
    z = scale * (H @ F.T)
    if bias is not None:
        z = z + np.where(out, 0.0, bias)
    z = np.where(out[None, :], -np.inf, z / tau)
    if z.shape[1] == 0:
        return z, np.full(H.shape[0], -np.inf), out, F
    m = z.max(1)
    safe = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        lse = safe + np.log(np.exp(z - safe[:, None]).sum(1))
    return z, lse, out, F


def probabilities(z, lse):
    p = np.exp(z - np.where(np.isfinite(lse), lse, 0.0)[:, None])
    logp = np.where(p > 0, z - np.where(np.isfinite(lse), lse, 0.0)[:, None], 0.0)
    return p, logp


def score(H, F, ids, scale, bias, top):
    z, lse, out, _ = softmax_over(H, F, scale, bias, 1.0)
    p, lp = probabilities(z, lse)
    entropy = -(p * lp).sum(1)
    T, n = z.shape
    logp = np.zeros(ids.shape)
    for t in range(T):
        for j, i in enumerate(ids[t]):
            if 0 <= i < n:
                logp[t, j] = -np.inf if out[i] else z[t, i] - lse[t]
    best = np.full((T, top), -1, np.int64)
    best_logp = np.full((T, top), -np.inf)
    for t in range(T):
        order = [i for i in np.argsort(-z[t], kind="stable") if not out[i]][:top]
        best[t, :len(order)] = order
        best_logp[t, :len(order)] = z[t, order] - lse[t]
    return dict(lse=lse, logp=logp, entropy=entropy, top_ids=best, top_logp=best_logp)


def listed(ids, out, n):
    return (ids >= 0) & (ids < n) & ~out[np.clip(ids, 0, max(n - 1, 0))] if n else np.zeros(ids.shape, bool)


def scatter(ids, w, have, n):
    m = np.zeros((ids.shape[0], n))
    np.add.at(m, (np.arange(ids.shape[0])[:, None].repeat(ids.shape[1], 1)[have], ids[have]), w[have])
    return m


def teacher_weights(ids, teacher, out, n, tau, row_ok):
    have = listed(ids, out, n) & row_ok[:, None]
    t = np.where(have, np.asarray(teacher, np.float64) / tau, -np.inf)
    m = t.max(1, initial=-np.inf)
    some = np.isfinite(m)
    w = np.where(have, np.exp(t - np.where(some, m, 0.0)[:, None]), 0.0)
    s = w.sum(1)
    w = w / np.where(s > 0, s, 1.0)[:, None]
    logw = np.where(have, t - (np.where(some, m, 0.0) + np.log(np.where(s > 0, s, 1.0)))[:, None], 0.0)
    return w, logw, have, some


def distill(H, F, ids, teacher, scale, bias, tau):
    z, lse, out, _ = softmax_over(H, F, scale, bias, tau)
    w, logw, have, _ = teacher_weights(ids, teacher, out, z.shape[1], tau, np.isfinite(lse))
    logp = np.zeros(ids.shape)
    for t in range(ids.shape[0]):
        for j in range(ids.shape[1]):
            if have[t, j]:
                logp[t, j] = z[t, ids[t, j]] - lse[t]
    return tau * tau * np.where(w > 0, w * (np.where(w > 0, logw, 0.0) - logp), 0.0).sum(1), lse  # w log w -> 0


def dz_distill(H, F, ids, teacher, dloss, scale, bias, tau):
    """The gradient in the scores z / tau, and its size part by part."""
    z, lse, out, _ = softmax_over(H, F, scale, bias, tau)
    p, _ = probabilities(z, lse)
    w, _, have, some = teacher_weights(ids, teacher, out, z.shape[1], tau, np.isfinite(lse))
    u = np.where(some, np.asarray(dloss, np.float64), 0.0) * tau * tau
    s = scatter(ids, w, have, z.shape[1])
    return u[:, None] * (p - s), np.abs(u)[:, None] * (p + s)


def dz_score(H, F, ids, dlogp, dentropy, scale, bias):
    z, lse, out, _ = softmax_over(H, F, scale, bias, 1.0)
    p, lp = probabilities(z, lse)
    ok = np.isfinite(lse)
    have = listed(ids, out, z.shape[1]) & ok[:, None]
    a = np.where(have, np.asarray(dlogp, np.float64), 0.0)
    e = np.zeros(z.shape[0]) if dentropy is None else np.where(ok, np.asarray(dentropy, np.float64), 0.0)
    ent = -(p * lp).sum(1)
    s = scatter(ids, a, have, z.shape[1])
    size = p * np.abs(a).sum(1)[:, None] + np.abs(e)[:, None] * p * (np.abs(lp) + ent[:, None]) + scatter(
        ids, np.abs(a), have, z.shape[1])
    return s - p * a.sum(1)[:, None] - e[:, None] * p * (lp + ent[:, None]), size


def grads(dz, H, F, out, scale):
    F = np.where(out[:, None], 0.0, np.asarray(F, np.float64))
    return scale * dz @ F, scale * dz.T @ np.asarray(H, np.float64)


# ---------------------------------------------------------------- bounds

def z_bound(H, F, out, scale, tau, bias):
    """|error| of a score in fp32: k products and additions (each addition at most a whole step, 2 u), three
    dropped products of the parts of fp32 factors, the scale's rounding and the exponent's."""
    k = H.shape[1]
    F = np.where(out[:, None], 0.0, np.asarray(F, np.float64))
    size = abs(scale) / tau * (np.abs(np.asarray(H, np.float64)) @ np.abs(F).T)
    if bias is not None:
        size = size + np.where(out, 0.0, np.abs(bias))[None, :] / tau
    top = size.max(1, initial=0.0)
    return (2 * k + 16) * U * top


def lse_bound(zb, lse, n):
    """The largest score's error, n / 16 + 64 additions, the exponentials (2 u each) and the result's rounding."""
    return zb + (n / 16 + 72) * U + 2 * U * np.where(np.isfinite(lse), np.abs(lse), 0.0)


def entropy_bound(zb, entropy, n):
    """|d entropy| <= sum p |log p + entropy| |dz| <= 2 entropy |dz|, and the sums' roundings."""
    return 2 * (entropy + 1) * zb + (n / 16 + 72) * U * (2 * entropy + 2)


def grad_bounds(size, H, F, out, scale, zb, lse, n, T, bf16):
    """dH and dF: a probability is off by twice the scores' error and the log sum's; a term's rounding to bf16
    for bf16 factors; n (T) additions of at most a step; and the result's own rounding (added by the caller)."""
    rel = 2 * zb + lse_bound(zb, lse, n) + 8 * U + (V if bf16 else 0.0)
    Hs, Fs = np.abs(np.asarray(H, np.float64)), np.where(out[:, None], 0.0, np.abs(np.asarray(F, np.float64)))
    return (abs(scale) * ((size * (rel + 2 * (n + size.shape[1]) * U)[:, None]) @ Fs),
            abs(scale) * ((size * (rel + 2 * (T + size.shape[0]) * U)[:, None]).T @ Hs))
