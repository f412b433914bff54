"""CPU checker (fp64, numpy) of the batch operators: token log probabilities, distillation from a teacher's top log
probabilities, batch routing and its gradient.  Written from the definitions, row by row; shares no code with the
library.  Masked places are -inf; what the definitions leave open (rows without any mass, NaN in the order of the
alternatives) follows the statements in ``include/draftexpert.h``."""
import numpy as np


def log_softmax(x):
    """log softmax of one row; a row of nothing but -inf stays -inf."""
    m = x.max() if not np.isnan(x).any() else np.nan
    if m == -np.inf:
        return np.full_like(x, -np.inf)
    with np.errstate(invalid="ignore"):
        u = x - m
        return u - np.log(np.exp(u).sum())


def order(z):
    """ids in descending order of z, ties to the lower id, NaN last."""
    return np.array(sorted(range(len(z)), key=lambda v: (np.isnan(z[v]), 0.0 if np.isnan(z[v]) else -z[v], v)))


def token_logprobs(z, tokens, n_top, temperature):
    N, V = z.shape
    out = {"logprob": np.zeros(N), "entropy": np.zeros(N), "top_ids": np.zeros((N, n_top), np.int64),
           "top_logprobs": np.zeros((N, n_top))}
    for t in range(N):
        lp = log_softmax(z[t] / temperature)
        p = np.exp(lp)
        if tokens[t] == -1:
            out["logprob"][t] = 0.0
        elif 0 <= tokens[t] < V:
            out["logprob"][t] = lp[tokens[t]]
        else:
            out["logprob"][t] = np.nan
        out["entropy"][t] = np.nan if np.isnan(lp).any() else -sum(p[p > 0] * lp[p > 0])
        if n_top:
            # (numpy's stable sort of the negated row puts equal values in the order of their ids and NaN last)
            ids = np.argsort(-z[t], kind="stable")[:n_top]
            out["top_ids"][t] = ids
            out["top_logprobs"][t] = lp[ids]
    return out


def distill_topk(z, ids, lp, tail, temperature, weight=None):
    """loss [N], dlogits [N, V], and the magnitudes the gradient is a difference of [N, V] (for error bounds)."""
    N, V = z.shape
    loss, grad, size = np.zeros(N), np.zeros((N, V)), np.zeros((N, V))
    for t in range(N):
        w = 1.0 if weight is None else float(weight[t])
        seen = {}
        for e, l in zip(ids[t], lp[t]):
            if 0 <= e < V and int(e) not in seen:
                seen[int(e)] = float(l)
        # (a list that is renormalised: relative to its largest entry, whose exponential may be out of range)
        top = max((l for l in seen.values() if l > -np.inf), default=0.0) if not tail else 0.0
        seen = {e: float(np.exp(np.float64(l) - top)) for e, l in seen.items()}
        if w == 0.0 or not seen:
            continue
        mass = sum(seen.values())
        if not tail and mass > 0:
            seen = {e: p / mass for e, p in seen.items()}
            mass = 1.0
        rest = max(0.0, 1.0 - mass) if tail else 0.0
        if not (z[t] > -np.inf).any():
            loss[t] = np.inf if mass + rest > 0 else 0.0
            continue
        logq = log_softmax(z[t] / temperature)
        q = np.exp(logq)
        beta = mass + rest
        d = beta * q
        s = beta * q
        total = 0.0
        for e, p in seen.items():
            if p > 0:
                total += p * (np.log(p) - logq[e])
            d[e] -= p
            s[e] += p
        if tail:
            other = np.ones(V, bool)
            other[list(seen)] = False
            x = z[t][other] / temperature
            if rest > 0:
                top = x.max() if len(x) else -np.inf
                if top == -np.inf:
                    total = np.inf
                else:
                    e = np.exp(x - top)
                    full = np.concatenate([x, z[t][~other] / temperature])
                    # (differences first: the maxima may be as large as a mask of the type's lowest value)
                    log_r = (top - full.max()) + np.log(e.sum()) - np.log(np.exp(full - full.max()).sum())
                    total += rest * (np.log(rest) - log_r)
                    d[other] -= rest * e / e.sum()
                    s[other] += rest * e / e.sum()
        loss[t] = total
        grad[t] = d * w / temperature
        size[t] = s * abs(w) / temperature
    return loss, grad, size


def scores(z, sigmoid):
    """Scores of one row; a masked (-inf) expert scores 0."""
    if sigmoid:
        with np.errstate(over="ignore"):
            return np.where(z == -np.inf, 0.0, 1.0 / (1.0 + np.exp(-z)))
    return np.exp(log_softmax(z)) if (z > -np.inf).any() else np.zeros_like(z)


def route(z, k, sigmoid, norm, scale, bias=None, groups=1, keep=1, top2=False):
    N, E = z.shape
    per = E // groups
    ids, w = np.zeros((N, k), np.int64), np.zeros((N, k))
    for t in range(N):
        masked = ~(z[t] > -np.inf)
        r = scores(z[t], sigmoid)
        v = z[t].astype(np.float64) if bias is None else r + bias
        g = np.where(masked, -np.inf, r if bias is None else v)
        v = np.where(masked, -np.inf, v)
        allowed = np.ones(E, bool)
        if groups > 1:
            best = []
            for i in range(groups):
                x = np.sort(g[i * per:(i + 1) * per])[::-1]
                x = x[x > -np.inf][:2 if top2 else 1]
                best.append(x.sum() if len(x) else -np.inf)
            kept = sorted(range(groups), key=lambda i: (-best[i], i))[:keep]
            allowed[:] = False
            for i in kept:
                allowed[i * per:(i + 1) * per] = True
        pick = sorted((e for e in range(E) if allowed[e]), key=lambda e: (-v[e], e))[:k]
        ids[t] = pick
        x = z[t][pick]
        if norm:
            live = x > -np.inf
            if live.any():
                # (ratios of the scores; the logarithms keep them where the scores themselves underflow)
                ls = -np.logaddexp(0.0, -x[live]) if sigmoid else x[live]
                e = np.exp(ls - ls.max())
                w[t][live] = scale * e / e.sum()
        else:
            w[t] = scale * r[pick]
    flat = ids.reshape(-1)
    perm = np.argsort(flat, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))])
    return ids, w, offsets, perm


def route_grad(z, ids, dw, sigmoid, norm, scale):
    """d_logits [N, E] and the magnitudes it is a difference of."""
    N, E = z.shape
    d, size = np.zeros((N, E)), np.zeros((N, E))
    for t in range(N):
        pairs = [(j, int(e)) for j, e in enumerate(ids[t]) if 0 <= e < E]
        r = scores(z[t], sigmoid)
        total = sum(r[e] for _, e in pairs)
        g = {j: scale * dw[t, j] for j, _ in pairs}
        c, a = np.zeros(E), np.zeros(E)
        if norm:
            if total == 0:
                continue
            mean = sum(g[j] * r[e] for j, e in pairs) / total
            mag = sum(abs(g[j]) * r[e] for j, e in pairs) / total
            for j, e in pairs:
                c[e] += (g[j] - mean) / total
                a[e] += (abs(g[j]) + mag) / total
        else:
            for j, e in pairs:
                c[e] += g[j]
                a[e] += abs(g[j])
        if sigmoid:
            d[t] = c * r * (1 - r)
            size[t] = a * r * (1 - r)
        else:
            d[t] = r * (c - (c * r).sum())
            size[t] = r * (a + (a * r).sum())
    return d, size
