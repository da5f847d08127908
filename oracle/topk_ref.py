"""Plain 64-bit reference of the operators on the record of a row's top
logits, row by row in numpy from their definitions (test infrastructure only;
it shares no code with the library)."""
import numpy as np

from .ref import bf16_to_f64

NAN, INF = float("nan"), float("inf")


def values(a):
    """Logits (float32, or uint16 bf16 patterns) as float64."""
    return bf16_to_f64(a) if a.dtype == np.uint16 else a.astype(np.float64)


def usable(x):
    """A row that has a softmax: a finite logit, no NaN and no +inf."""
    return not np.isnan(x).any() and not (x == INF).any() and (x > -INF).any()


def softmax(x):
    e = np.exp(x - x.max())
    return e / e.sum()


def inverse_cdf(mass, u):
    """Smallest index whose running sum exceeds u * total; the last one with
    mass where rounding leaves none.  Also the point's distance to the nearer
    edge of the interval taken."""
    c = np.cumsum(mass)
    point = float(u) * c[-1]
    over = np.nonzero(c > point)[0]
    j = int(over[0]) if len(over) else int(np.nonzero(mass > 0)[0][-1])
    before = c[j - 1] if j else 0.0
    return j, min(abs(c[j] - point), abs(point - before) if point > 0 else INF)


def topk(x, k, T, u=None):
    """Records of rows x [N, V]: ids, top (float64), rest, tokens, and the
    draws' margins."""
    z = values(x)
    N, V = z.shape
    ids, top = np.full((N, k), -1, np.int32), np.full((N, k), -INF)
    rest, tokens, margin = np.full(N, -INF), np.full(N, -1, np.int32), np.full(N, INF)
    for n in range(N):
        r = z[n]
        if not usable(r):
            continue
        order = np.lexsort((np.arange(V), -(r + 0.0)))[:k]
        order = order[r[order] > -INF]
        ids[n, :len(order)], top[n, :len(order)] = order, r[order]
        if T == 0:
            tokens[n] = order[0]
            continue
        out = np.delete(r, order)
        if (out > -INF).any():  # (relative to their largest: exp has no range for far ones)
            rest[n] = (out.max() - r[order[0]]) / T + np.log(np.exp((out - out.max()) / T).sum())
        if u is not None:
            s, margin[n] = inverse_cdf(np.exp((r[order] - r[order[0]]) / T), u[n])
            tokens[n] = order[s]
    return dict(ids=ids, top=top, rest=rest, tokens=tokens, margin=margin)


def record_ok(ids, top, V):
    """Whether one record is one: ids in range (-1: an empty slot), none twice,
    logits that are numbers, the first slot taken with mass."""
    held = ids[ids != -1]
    if ((held < 0) | (held >= V)).any() or len(set(held.tolist())) != len(held):
        return False
    t = top[ids != -1]
    return not np.isnan(t).any() and not (t == INF).any() and bool((t > -INF).any())


def xlogy(p, l):
    """p * l with 0 * anything = 0."""
    return np.where(p > 0, p * np.where(p > 0, l, 0.0), 0.0)


def distill(ids, top, rest, student, kind, beta, tau, mask=None):
    """Loss {mean, sum}, row losses and gradients of student [N, V] against
    records ids, top [N, k], rest [N] or None."""
    s, t = values(student), values(top)
    N, V = s.shape
    rows, grad = np.zeros(N), np.zeros((N, V))
    on = np.ones(N, bool) if mask is None else mask.reshape(-1) != 0
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        for n in np.nonzero(on)[0]:
            ok = usable(s[n]) and record_ok(ids[n], t[n], V) and ids[n, 0] != -1 and t[n, 0] > -INF
            if rest is not None:
                ok = ok and not np.isnan(rest[n]) and rest[n] != INF
            if not ok:
                rows[n], grad[n] = NAN, NAN
                continue
            held = ids[n] != -1
            at = ids[n][held]
            lt = (t[n][held] - t[n, 0]) / tau
            lt = np.append(lt, -INF if rest is None else float(rest[n]))
            lp = lt - lt.max() - np.log(np.exp(lt - lt.max()).sum())
            x = (s[n] - s[n].max()) / tau
            lse = np.log(np.exp(x).sum())
            lq = x - lse
            others = np.delete(lq, at)
            big = others.max() if len(others) else -INF
            Q = big + np.log(np.exp(others - big).sum()) if big > -INF else -INF
            lb = np.append(lq[at], Q)
            p, q = np.exp(lp), np.exp(lb)
            if kind == "fkl":
                D = xlogy(p, lp - lb).sum()
                f = np.where(q > 0, 1.0 - p / q, 0.0)
            elif kind == "rkl":
                D = xlogy(q, lb - lp).sum()
                f = lb - lp - D
            else:
                lm = lb if beta == 0 else lp if beta == 1 else np.log(beta * p + (1 - beta) * q)
                kq = xlogy(q, lb - lm).sum() if beta < 1 else 0.0
                D = (beta * xlogy(p, lp - lm).sum() if beta > 0 else 0.0) + (1 - beta) * kq
                f = (1 - beta) * (lb - lm - kq) if beta < 1 else np.zeros_like(lb)
            rows[n] = D
            qj = np.exp(lq)
            g = np.where(qj > 0, qj * f[-1], 0.0)
            g[at] = np.where(q[:-1] > 0, q[:-1] * f[:-1], 0.0)
            if kind == "fkl":  # q - p in the record; outside q_j - P q_j / Q, where q_j and Q may have no value
                share = np.exp(lq - big) if big > -INF else np.zeros(V)
                share[at] = 0.0
                g = qj - p[-1] * share / max(share.sum(), 1.0)
                g[at] = q[:-1] - p[:-1]
            grad[n] = g / tau
    total = float(rows[on].sum()) if on.any() else 0.0
    return np.array([total / on.sum() if on.any() else 0.0, total]), rows, grad


def verify(target, ids, top, tokens, u_accept, u_resample, T, draft_len=None):
    """accepted_len, out_tokens, reject_mask, and the smallest margin of each
    sequence's decisions (relative to the ratio for a test, in mass for a
    draw)."""
    t, d = values(target), values(top)
    B, K1, V = t.shape
    K = K1 - 1
    acc, out = np.full(B, -1, np.int32), np.full((B, K1), -1, np.int32)
    rmask, margin = np.zeros((B, K), np.uint8), np.full(B, INF)
    for b in range(B):
        kb = K if draft_len is None else int(draft_len[b])
        if kb < 1 or kb > K or ((tokens[b, :kb] < 0) | (tokens[b, :kb] >= V)).any():
            continue
        a, extra = kb, None
        for i in range(kb + 1):
            if not usable(t[b, i]):
                break
            p = softmax(t[b, i] / T)
            if i == kb:
                extra, m = inverse_cdf(p, u_resample[b])
                margin[b] = min(margin[b], m)
                break
            if not record_ok(ids[b, i], d[b, i], V):
                break
            q = np.zeros(V)
            held = ids[b, i] != -1
            q[ids[b, i][held]] = softmax(d[b, i][held] / T)
            y = tokens[b, i]
            uq = float(u_accept[b, i]) * q[y]
            margin[b] = min(margin[b], abs(uq - p[y]))
            if not uq < p[y]:
                a = i
                r = np.maximum(p - q, 0.0)
                extra, m = inverse_cdf(r if r.sum() > 0 else p, u_resample[b])
                margin[b] = min(margin[b], m)
                break
        if extra is None:
            continue
        acc[b] = a
        out[b, :a], out[b, a] = tokens[b, :a], extra
        if a < kb:
            rmask[b, a] = 1
    return acc, out, rmask, margin
