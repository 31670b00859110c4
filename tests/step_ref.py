"""Plain 64-bit implementations of a training step's operators on the CPU, from
their formulas, with bounds of the rounding errors that the kernels may add."""
import math

import numpy as np
import torch


# -- batch tables -------------------------------------------------------------------
def tables(ids, tokens, free, block, width, cap):
    """Read by read, token by token. ids None: tokens holds the reads' lengths."""
    lead = np.asarray(tokens if ids is None else ids)
    tokens, free = np.asarray(tokens), np.asarray(free)
    G, n = lead.shape
    out = dict(start=np.zeros((G, n + 1), np.int32), table=np.full((G, n, width), -1, np.int32),
               slot=np.full((G, cap), -1, np.int64), row=np.full((G, cap), -1, np.int32),
               pos=np.full((G, cap), -1, np.int32), used=np.zeros((G, 3), np.int32))
    for g in range(G):
        done, t, taken, reads = False, 0, 0, 0
        for r in range(n):
            if ids is None:
                length = int(tokens[g, r])
            else:
                length = int(tokens[lead[g, r]]) if 0 <= lead[g, r] < tokens.size else 0
            length = max(length, 0)
            nb = (length + block - 1) // block
            done = done or nb > width or t + length > cap or taken + nb > free.shape[1]
            if not done:
                for j in range(nb):
                    out["table"][g, r, j] = free[g, taken + j]
                for p in range(length):
                    out["slot"][g, t + p] = int(free[g, taken + p // block]) * block + p % block
                    out["row"][g, t + p], out["pos"][g, t + p] = r, p
                t, taken, reads = t + length, taken + nb, reads + 1
            out["start"][g, r + 1] = t
        out["used"][g] = reads, t, taken
    return out


# -- attention ----------------------------------------------------------------------
UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}  # half a subnormal


def attention(q, k, v, start, scale, do=None):
    """o, lse (and dq, dk, dv) in 64 bits, and for each a bound of the kernels'
    error. With u the unit roundoff of the inputs' type and all sums in 32 bits:

    S is off by at most eS = (width + 4) 2^-24 scale sum |q||k| and the
    exponent's rounding, so P by a factor 1 +- e, e = 4 (eS + 2^-22 (max|S| +
    4) + L 2^-24); as a matrix operand P and dS are rounded by u more, outputs
    by u. o: (u + e) sum P|v| + u|o|. The gradient uses the rounded o, so its
    delta is off by eD_i = sum_d |do| (error of o) + width 2^-24 sum |do||o|;
    dS by (u + e)|dS| + P (eD_i + (width + 4) 2^-24 sum |do||v|); sums over
    those times the other operand, plus u of the output."""
    u, tiny, dt = UNIT[q.dtype], TINY[q.dtype], torch.float64
    T, H, D = q.shape
    Hk = k.shape[1]
    Q, K, V = (x.detach().cpu().to(dt) for x in (q, k, v))
    G = None if do is None else do.detach().cpu().to(dt)
    z = lambda *s: torch.zeros(s, dtype=dt)  # noqa: E731
    names = ["o"] + ([] if do is None else ["dq", "dk", "dv"])
    val = {x: z(T, Hk if x in ("dk", "dv") else H, D) for x in names}
    err = {x: z(*val[x].shape) for x in names}
    val["lse"], err["lse"] = torch.full((H, T), -math.inf, dtype=dt), z(H, T)
    for s in range(len(start) - 1):
        a, b = int(start[s]), int(start[s + 1])
        L = b - a
        if L == 0:
            continue
        low = torch.ones((L, L), dtype=torch.bool).tril()
        for h in range(H):
            g = h // (H // Hk)
            qh, kh, vh = Q[a:b, h], K[a:b, g], V[a:b, g]
            S = torch.where(low, scale * (qh @ kh.T), -math.inf)
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            o = P @ vh
            eS = (D + 4) * 2.0**-24 * scale * (qh.abs() @ kh.abs().T)
            big = torch.where(low, S.abs(), 0.0)
            e = 4 * (torch.where(low, eS, 0.0).amax(1) + 2.0**-22 * (big.amax(1) + 4) + L * 2.0**-24)
            eo = (u + e)[:, None] * (P @ vh.abs()) + u * o.abs() + L * (tiny * vh.abs().amax(0))
            val["o"][a:b, h], err["o"][a:b, h] = o, eo + tiny
            val["lse"][h, a:b], err["lse"][h, a:b] = lse, e + 2.0**-22 * (lse.abs() + 1)
            if do is None:
                continue
            gh = G[a:b, h]
            dP = gh @ vh.T
            dS = P * (dP - (gh * o).sum(1, keepdim=True))
            eD = (gh.abs() * eo).sum(1) + D * 2.0**-24 * (gh.abs() * o.abs()).sum(1)
            edS = (u + 2 * e)[:, None] * dS.abs() + P * (
                eD[:, None] + (D + 4) * 2.0**-23 * (gh.abs() @ vh.abs().T)) + tiny
            edS = torch.where(low, edS, 0.0)
            eP = torch.where(low, (u + 2 * e)[:, None] * P + tiny, 0.0)
            val["dq"][a:b, h] = scale * (dS @ kh)
            err["dq"][a:b, h] = scale * (edS @ kh.abs())
            val["dk"][a:b, g] += scale * (dS.T @ qh)
            err["dk"][a:b, g] += scale * (edS.T @ qh.abs())
            val["dv"][a:b, g] += P.T @ gh
            err["dv"][a:b, g] += eP.T @ gh.abs()
    for x in names[1:]:  # 32-bit sums, and the output's rounding
        err[x] = 1.01 * err[x] + u * val[x].abs() + tiny + 1e-30
    return val, err


# -- distillation -------------------------------------------------------------------
def distill(logits, index, teacher, tau, weight):
    """loss, gradient in 64 bits and bounds of the kernels' errors. Exponents x
    are off by 2^-22 (|x| + 2), so a row's q and p by that factor (x the largest
    that matters: below -100 nothing is left), the loss by that of its terms;
    the gradient by the sum of both and its own rounding."""
    u = UNIT[logits.dtype]
    s, y = logits.detach().cpu().double(), teacher.detach().cpu().double()
    x = index.cpu().long()
    T, V = s.shape
    w = torch.ones(T, dtype=torch.float64) if weight is None else weight.cpu().double()
    loss, grad = torch.zeros(T, dtype=torch.float64), torch.zeros((T, V), dtype=torch.float64)
    eloss, egrad = loss.clone(), grad.clone()
    for t in range(T):
        ok = (x[t] >= 0) & (x[t] < V) & (y[t] != -math.inf)
        if w[t] == 0 or not ok.any():
            continue
        at = x[t][ok]
        logp = torch.log_softmax(y[t][ok] / tau, 0)
        logq = torch.log_softmax(s[t] / tau, 0)
        p, q = logp.exp(), logq.exp()
        top = torch.where(logq > -100, logq.abs(), 0).max()
        e = 2.0**-21 * (float(torch.where(logp > -100, logp.abs(), 0).max() + top) + 4)
        e += (V / 64 + 32) * 2.0**-24  # a thread's sum of exponentials, then the threads'
        terms = torch.where(p > 0, p * (logp - logq[at]), 0.0)
        loss[t] = w[t] * tau * tau * terms.sum()
        eloss[t] = w[t].abs() * tau * tau * (
            4 * e * (p * (logp.abs() + logq[at].abs())).nan_to_num(0, 0, 0).sum() + 4 * e)
        d = q.clone()
        d.index_add_(0, at, -p)
        both = q.clone()
        both.index_add_(0, at, p)
        grad[t] = w[t] * tau * d
        egrad[t] = w[t].abs() * tau * (2 * e * both) + u * grad[t].abs() + TINY[logits.dtype] + 1e-38
    return loss, grad, eloss, egrad
