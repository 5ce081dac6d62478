"""Distillation of many rows against 64 bits on the GPU, for tests of rows that follow one another in a block."""
import torch

import paper_2609_36601_b200 as P

LEAST_REST = 2.0 ** -20


def check(s, token, logit, teacher_lse, reverse, rows=2048, repeats=1):
    """Loss, log-sum-exp and all of the gradient of finite rows (tokens apart, -1: no entry), with the terms' magnitudes and tolerances of test_gpu_distill_top.py: the loss to 2e-5 of its terms, the
    gradient to 2e-5 of its terms and half a step of its type.  Further calls give the same bits."""
    out, grad = P.distill_top(s, token, logit, teacher_lse, reverse=reverse)
    assert P.last_kernel() == 4
    for _ in range(repeats - 1):
        o, g = P.distill_top(s, token, logit, teacher_lse, reverse=reverse)
        assert all(torch.equal(o[k], out[k]) for k in out) and torch.equal(g, grad)
    assert not out["row_status"].any()
    half = 2.0 ** -8 if s.dtype == torch.bfloat16 else 2.0 ** -23
    for i in range(0, s.shape[0], rows):
        r = slice(i, i + rows)
        z = s[r].double()
        lse = torch.logsumexp(z, 1, keepdim=True)
        assert bool(((out["lse"][r].double() - lse[:, 0]).abs() <= 1e-5 + 2.0 ** -24 * lse[:, 0].abs()).all())
        lp = z - lse
        p = lp.exp()
        row, col = (token[r] >= 0).nonzero(as_tuple=True)
        v = token[r][row, col].long()
        lw = torch.full_like(lp, -float("inf"))
        lw[row, v] = logit[r].double()[row, col]
        lw = lw - (torch.logsumexp(lw, 1, keepdim=True) if teacher_lse is None else teacher_lse[r].double()[:, None])
        listed = lw > -float("inf")
        lw = torch.where(listed, lw, 0.0)
        w = torch.where(listed, lw.exp(), 0.0)
        W = w.sum(1, keepdim=True)
        S = torch.where(listed, 0.0, p).sum(1, keepdim=True)
        R = torch.zeros_like(W) if teacher_lse is None else (1 - W).clamp(min=LEAST_REST)
        lS = torch.logsumexp(torch.where(listed, -float("inf"), lp), 1, keepdim=True)
        lR = R.log() if teacher_lse is not None else torch.zeros_like(R)
        if teacher_lse is None:
            lS, S1 = torch.zeros_like(lS), torch.ones_like(S)
        else:
            S1 = S
        if reverse:
            loss = torch.where(listed, p * (lp - lw), 0.0).sum(1, keepdim=True) + S * (lS - lR)
            loss_mag = 1 + torch.where(listed, p * (1 + lp.abs() + lw.abs()), 0.0).sum(1, keepdim=True) + S * (lS.abs() + lR.abs())
            want = p * (torch.where(listed, lp - lw, lS - lR) - loss)
            mag = p * (1 + torch.where(listed, lp.abs() + lw.abs(), lS.abs() + lR.abs()) + loss_mag)
        else:
            loss = torch.where(listed, w * (lw - lp), 0.0).sum(1, keepdim=True) + R * (lR - lS)
            loss_mag = 1 + torch.where(listed, w * (1 + lw.abs() + lp.abs()), 0.0).sum(1, keepdim=True) + R * (1 + lR.abs() + lS.abs())
            want = torch.where(listed, p * (W + R) - w, p * (W + R - R / S1))
            mag = torch.where(listed, p * (W + R) + w, p * (W + R + R / S1))
        assert bool(((out["loss"][r].double() - loss[:, 0]).abs() <= 2e-5 * loss_mag[:, 0]).all())
        err = (grad[r].double() - want).abs()
        bound = 2e-5 * mag + half * want.abs() + 1e-37
        assert bool((err <= bound).all()), (i, float((err / bound).max()), (err > bound).nonzero()[:4].tolist())
    return out, grad
