"""Plain 64-bit implementations of a token model's layers on the CPU, from their
formulas, with bounds of the rounding errors that the kernels may add. E = 2^-24,
half a step of 32 bits; u: of the output's type, `tiny` half of its smallest number."""
import math

import torch

E, LEAST = 2.0**-24, 2.0**-126
UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25, torch.float32: 2.0**-150}
F64 = torch.float64


def close(name, got, val, err):
    got = got.detach().cpu().to(F64)
    assert got.shape == val.shape, (name, got.shape, val.shape)
    bad = ~((got - val).abs() <= err)
    assert not bad.any(), (name, int(bad.sum()), float((got - val).abs()[bad].max()),
                           float((err / 1)[bad].min()))


def _wide(x):
    return x.detach().cpu().to(F64)


# -- embedding ----------------------------------------------------------------------
def names(ids, slot, V):
    """Every token's row of the embedding, -1 for padding; one after the other."""
    ids = ids.tolist()
    at = range(len(ids)) if slot is None else slot.tolist()
    out = []
    for s in at:
        v = ids[s] if 0 <= s < len(ids) else -1
        out.append(v if 0 <= v < V else -1)
    return out


def embed(weight, ids, slot, scale, dtype):
    """One product in 32 bits, rounded to the output's type: (u + E) of it."""
    w = _wide(weight)
    rows = names(ids, slot, w.shape[0])
    out = torch.zeros((len(rows), w.shape[1]), dtype=F64)
    for t, v in enumerate(rows):
        if v >= 0:
            out[t] = w[v] * scale
    return out, (UNIT[dtype] + 2 * E) * out.abs() + TINY[dtype] + TINY[torch.float32]


def embed_grad(dout, ids, slot, V, scale, dtype):
    """A row's m terms are added in 32 bits in some order: each sum is off by at most
    (m - 1) E of the terms' sum of absolute values; times scale; rounded."""
    d = _wide(dout)
    rows = names(ids, slot, V)
    val, mag = torch.zeros((V, d.shape[1]), dtype=F64), torch.zeros((V, d.shape[1]), dtype=F64)
    many = torch.zeros((V, 1), dtype=F64)
    for t, v in enumerate(rows):
        if v >= 0:
            val[v] += d[t]
            mag[v] += d[t].abs()
            many[v] += 1
    scale = abs(float(torch.tensor(scale, dtype=torch.float32))) * (1 if scale >= 0 else -1)
    val, mag = val * scale, mag * abs(scale)
    return val, 1.01 * (many + 1) * E * mag + UNIT[dtype] * val.abs() + TINY[dtype] + TINY[torch.float32]


# -- norms and rotations ---------------------------------------------------------------
def _pairs(R, interleaved):
    i = torch.arange(R // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)


def _turn(y, angle, R, interleaved):
    """y [..., width] with pair i turned by angle[..., i]; and the same of magnitudes."""
    a, b = _pairs(R, interleaved)
    out, c, s = y.clone(), angle.cos(), angle.sin()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def _both(m, R, interleaved):
    """What an element's error can come from: both of its pair."""
    a, b = _pairs(R, interleaved)
    out = m.clone()
    out[..., a] = out[..., b] = m[..., a] + m[..., b]
    return out


def rotate(x, pos, freq, weight, eps, interleaved, dout=None):
    """out (and dx, dweight) and bounds. With W the width: the sum of W squares is off
    by W E, r by half of it and a few roundings: er = (W / 2 + 8) E, z and y by one
    more each. An angle of t turns (|t| <= 1/2) is rounded to 32 bits (2 pi E / 2) and,
    in 64 bits, off by 2^-52 of all its turns; sine and cosine by 2 E: ea. An output
    by the error of y and ea times both elements of its pair, and its products' and
    sum's roundings, 3 E; rounded by u. Likewise the turned gradient g: eg = ea + 3 E
    of both. dot = mean of g w z: er + 2 E and eg of each term, (W + 2) E of the sum."""
    X, dt = _wide(x), x.dtype
    T, H, W = X.shape
    p = pos.cpu()
    there = (p >= 0)[:, None, None]
    X = torch.where(there, X, 0.0)
    w = torch.ones(W, dtype=F64) if weight is None else _wide(weight)
    R = 0 if freq is None else 2 * freq.numel()
    turns = torch.zeros((T, 1, R // 2), dtype=F64)
    if R:
        turns = p.to(F64)[:, None, None] * _wide(freq)
    # far angles are only as good as 64 bits make them
    far = (2.0**-52 * turns.abs()).amax(2, keepdim=True) if R else torch.zeros((T, 1, 1), dtype=F64)
    ea = 2 * far + (math.pi + 2) * E
    er = (W / 2 + 8) * E
    r = (X.square().mean(2, keepdim=True) + eps).rsqrt()
    z = X * r
    y = z * w
    val = {"out": _turn(y, turns, R, interleaved)}
    both = _both(y.abs(), R, interleaved)
    u, tiny = UNIT[dt], TINY[dt] + TINY[torch.float32]
    err = {"out": (ea + er + 6 * E) * both + u * val["out"].abs() + tiny}
    for d in (val, err):
        d["out"] = torch.where(there, d["out"], 0.0)
    if dout is None:
        return val, err
    G = torch.where(there, _wide(dout), 0.0)
    g = _turn(G, -turns, R, interleaved)
    eg = (ea + 3 * E) * _both(G.abs(), R, interleaved)
    gw = g * w
    dot = (gw * z).mean(2, keepdim=True)
    terms = (gw * z).abs()
    edot = ((er + 4 * E) * terms + eg * (w * z).abs() + (W + 2) * E * terms).mean(2, keepdim=True)
    dx = r * (gw - z * dot)
    edx = r * (eg * w.abs() + 2 * E * gw.abs() + z.abs() * edot + (2 * er + 6 * E) * (z * dot).abs()
               + (er + 4 * E) * gw.abs())
    val["dx"] = torch.where(there, dx, 0.0)
    err["dx"] = torch.where(there, edx + u * dx.abs() + tiny, 0.0)
    if weight is not None:
        gz = (g * z).abs()
        val["dw"] = (g * z).sum((0, 1))
        N = T * H
        err["dw"] = (1.01 * ((N + 2) * E * gz + (er + 2 * E) * gz + eg * z.abs()).sum((0, 1))
                     + UNIT[weight.dtype] * val["dw"].abs() + TINY[weight.dtype] + TINY[torch.float32])
    return val, err


# -- recurrence ---------------------------------------------------------------------------
def scan(x, gate, start, h0=None, dh=None, dlast=None):
    """h, last (and dx, dgate, dh0) token by token, and bounds.

    With s the smaller of a and k: s is off by 6 E (exponential 2, sum and reciprocal
    3, product 1), of gates in 16 bits by 1.3 |gate| E more (the exponent |gate| log2 e
    is rounded, and so is log2 e), and 0 below 2^-126; the larger, 1 - s, by E. A step's rounding is E of its result, E s
    of the difference in it, and 6 E s of that difference for s. A stretch's map adds
    3 E of A h and 2 E of B for each of its steps. All of it is at most 16 E of what
    the step's magnitudes come to, M_t = a M_(t-1) + k |x_t| and s (|x_t| + M_(t-1)),
    and decays with a. Likewise G, of magnitude N_t = |dh_t| + a N_(t+1)."""
    dt = x.dtype
    X, Gt = _wide(x), _wide(gate)
    T, C = X.shape
    n = len(start) - 1
    z = lambda *s: torch.zeros(s, dtype=F64)  # noqa: E731
    a, k = torch.sigmoid(Gt), torch.sigmoid(-Gt)
    s = torch.minimum(a, k)
    es = s * (0.0 if dt is torch.float32 else 1.3 * E * Gt.abs())
    val = dict(h=z(T, C), last=z(n, C) if h0 is None else _wide(h0))
    err = dict(h=z(T, C), last=z(n, C))
    before, ebefore, mag = z(T, C), z(T, C), z(T, C)
    u, tiny = UNIT[dt], TINY[dt] + TINY[torch.float32]
    for i in range(n):
        h, e = val["last"][i].clone(), z(C)
        M = h.abs()
        for t in range(int(start[i]), int(start[i + 1])):
            before[t], ebefore[t], mag[t] = h, e, M
            h = a[t] * h + k[t] * X[t]
            grow = s[t] * (X[t].abs() + M)
            M = a[t] * M + k[t] * X[t].abs()
            e = a[t] * e + 16 * E * (M + grow) + (es[t] + LEAST) * (X[t].abs() + mag[t]) + TINY[torch.float32]
            val["h"][t], err["h"][t] = h, e + u * h.abs() + tiny
        val["last"][i], err["last"][i] = h, e
    if dh is None:
        return val, err
    D = _wide(dh)
    val.update(dx=z(T, C), dgate=z(T, C), dh0=z(n, C) if dlast is None else _wide(dlast))
    err.update(dx=z(T, C), dgate=z(T, C), dh0=z(n, C))
    for i in range(n):
        R, e = val["dh0"][i].clone(), z(C)
        N = R.abs()
        for t in range(int(start[i + 1]) - 1, int(start[i]) - 1, -1):
            G, eG, NG = D[t] + R, e + E * (D[t].abs() + N), D[t].abs() + N
            diff, p = before[t] - X[t], a[t] * k[t]
            val["dx"][t] = k[t] * G
            err["dx"][t] = k[t] * (eG + 9 * E * NG) + (es[t] + LEAST) * NG + u * (k[t] * G).abs() + tiny
            val["dgate"][t] = p * diff * G
            err["dgate"][t] = (p * (diff.abs() * eG + (ebefore[t] + E * (X[t].abs() + mag[t])) * NG
                                    + 18 * E * diff.abs() * NG)
                               + (2 * es[t] + LEAST) * diff.abs() * NG
                               + u * (p * diff * G).abs() + tiny)
            R, N = a[t] * G, a[t] * NG
            e = a[t] * eG + 16 * E * N + 8 * E * s[t] * NG + (es[t] + LEAST) * NG + TINY[torch.float32]
        val["dh0"][i], err["dh0"][i] = R, e
    return val, err
