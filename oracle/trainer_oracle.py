"""Float64 oracle of a trainer's calls on distilled rollouts: a row's top logits, distillation from them, cross entropy from
hidden states.  One row at a time, from the definitions."""
from __future__ import annotations

import numpy as np

ST_MASKED, ST_NONFINITE, ST_BAD_ID, ST_NOT_COMPUTED = 4, 8, 16, 64
UNUSABLE = 8 | 16 | 32 | 64
LEAST_REST = 2.0 ** -20


def _lse(z):
    m = z.max()
    return m if np.isinf(m) else m + np.log(np.exp(z - m).sum())


def supervised(V, target, advantage=None, corrected=None, teacher_top1=None, mask=None, rollout_status=None):
    """(token, coefficient, status) of every row; token -1: the row contributes nothing."""
    rows = []
    for i in range(len(target)):
        if mask is not None and mask[i] == 0:
            rows.append((-1, 0.0, ST_MASKED))
            continue
        if rollout_status is not None and int(rollout_status[i]) & UNUSABLE:
            rows.append((-1, 0.0, ST_NOT_COMPUTED))
            continue
        hit = corrected is not None and corrected[i] != 0
        tok = int(teacher_top1[i] if hit else target[i])
        coef = 1.0 if hit or advantage is None else float(advantage[i])
        if not np.isfinite(coef):
            rows.append((-1, 0.0, ST_NONFINITE))
        elif not 0 <= tok < V:
            rows.append((-1, 0.0, ST_BAD_ID))
        else:
            rows.append((tok, coef, 0))
    return rows


def linear_ce(hidden, weight, rows, tau=1.0, grad_scale=1.0, share=None):
    """hidden [N, d], weight [V, d] float64, rows of `supervised` -> dict of loss, logp_tok, lse, status, dhidden, dweight, and the sums of the magnitudes of
    the gradients' terms (dhidden_abs, dweight_abs) and of what share[i] of the probabilities has in them, before 1 is taken from the supervised one (dhidden_p, dweight_p)."""
    N = hidden.shape[0]
    out = {k: np.zeros(N) for k in ("loss", "logp_tok", "lse")}
    out["status"] = np.array([s for _, _, s in rows], dtype=np.uint32)
    out["dhidden"], out["dweight"] = np.zeros_like(hidden), np.zeros_like(weight)
    for kind in ("_abs", "_p"):
        out["dhidden" + kind], out["dweight" + kind] = np.zeros_like(hidden), np.zeros_like(weight)
    for i, (tok, coef, _) in enumerate(rows):
        if tok < 0:
            continue
        with np.errstate(all="ignore"):
            z = weight @ hidden[i] / tau
            lse = _lse(z)
        if not np.isfinite(lse) or not np.isfinite(z[tok]):
            out["status"][i], out["lse"][i] = ST_NONFINITE, np.nan
            continue
        logp = z - lse
        out["loss"][i], out["logp_tok"][i], out["lse"][i] = -coef * logp[tok], logp[tok], lse
        g = np.exp(logp)
        p = np.abs(g * (grad_scale * coef / tau)) * (0.0 if share is None else share[i])
        out["dhidden_p"][i] = p @ np.abs(weight)
        out["dweight_p"] += np.outer(p, np.abs(hidden[i]))
        g[tok] -= 1.0
        g *= grad_scale * coef / tau
        out["dhidden"][i] = g @ weight
        out["dweight"] += np.outer(g, hidden[i])
        out["dhidden_abs"][i] = np.abs(g) @ np.abs(weight)
        out["dweight_abs"] += np.abs(np.outer(g, hidden[i]))
    return out


def top_logits(x, k, tau=1.0):
    """x [N, V] float64 -> token [N, k], logit [N, k], lse [N], status [N]."""
    N, V = x.shape
    token, logit = np.full((N, k), -1, dtype=np.int32), np.full((N, k), -np.inf)
    lse, status = np.zeros(N), np.zeros(N, dtype=np.uint32)
    for i in range(N):
        if np.isnan(x[i]).any() or np.isposinf(x[i]).any():
            status[i], logit[i] = ST_NONFINITE, 0.0
            continue
        lse[i] = _lse(x[i] / tau)
        order = [v for v in np.argsort(-x[i], kind="stable")[:k] if x[i, v] > -np.inf]
        token[i, :len(order)], logit[i, :len(order)] = order, x[i, order]
    return token, logit, lse, status


def distill_top(s, token, logit, teacher_lse=None, reverse=False, tau=1.0, mask=None, grad_scale=1.0):
    """s [N, V], token [N, k], logit [N, k], teacher_lse [N] or None, float64 -> dict of loss, lse, grad, status."""
    N, V = s.shape
    loss, lse, grad, status = np.zeros(N), np.zeros(N), np.zeros((N, V)), np.zeros(N, dtype=np.uint32)
    for i in range(N):
        if mask is not None and mask[i] == 0:
            status[i] = ST_MASKED
            continue
        there = (token[i] != -1) & ~np.isneginf(logit[i])
        ids = token[i][there]
        if ((token[i] < -1) | (token[i] >= V)).any() or len(set(ids.tolist())) != len(ids):
            status[i] = ST_BAD_ID
            continue
        t = logit[i][there] / tau
        if (np.isnan(s[i]).any() or np.isposinf(s[i]).any() or np.isneginf(s[i]).all() or np.isneginf(s[i][ids]).any() or not np.isfinite(t).all()
                or (teacher_lse is not None and not np.isfinite(teacher_lse[i]))):
            status[i] = ST_NONFINITE
            continue
        z = s[i] / tau
        lse[i] = _lse(z)
        lp = z - lse[i]
        p = np.exp(lp)
        if teacher_lse is None and not len(ids):
            continue                       # nothing to learn from
        lw = t - (teacher_lse[i] if teacher_lse is not None else _lse(t))
        w = np.exp(lw)
        outside = np.ones(V, dtype=bool)
        outside[ids] = False
        W = w.sum()
        R, T, lT = 0.0, 0.0, 0.0
        if teacher_lse is not None and outside.any() and _lse(z[outside]) - lse[i] > -1000 * np.log(2):
            R, lT = max(1.0 - W, LEAST_REST), _lse(z[outside]) - lse[i]
            T = np.exp(lT)
        if reverse:
            rest = lT - np.log(R) if R else 0.0
            loss[i] = (p[ids] * (lp[ids] - lw)).sum() + T * rest
            g = np.where(p > 0, p * (rest - loss[i]), 0.0)
            g[ids] = p[ids] * (lp[ids] - lw - loss[i])
        else:
            loss[i] = (w * (lw - lp[ids])).sum() + (R * (np.log(R) - lT) if R else 0.0)
            g = p * (W + R) - (np.exp(lp - lT) * R if R else 0.0)
            g[ids] = p[ids] * (W + R) - w
        grad[i] = g * grad_scale / tau
    return {"loss": loss, "lse": lse, "grad": grad, "status": status}
