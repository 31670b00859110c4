"""The layers of a token model over a worker's packed samples, as timed cases.

``nopfs.batch_tables`` says where the tokens of the next reads lie. Between it
and ``nopfs.packed_attention`` a step on them needs

  embed   nopfs.token_embed: the rows of an embedding that the tokens name,
          scaled, and its gradient by sorted tokens
  rotate  nopfs.norm_rotate: the norms of queries and keys per head with the
          rotation by position, and its gradient
  scan    nopfs.gated_scan: a gated linear recurrence over each sample, which
          stands where attention may stand, and its gradient

``run`` computes them in plain torch operations in 32 bits, or, where ``own``
is true, with the library's kernels.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


# -- cases ------------------------------------------------------------------------
def _embed(name, weight, dtype, T, tail, V, D, skew, slots, train):
    return dict(name=name, kind="embed", weight=weight, dtype=dtype, T=T, tail=tail, V=V, D=D,
                skew=skew, slots=slots, train=train)


def _rotate(name, dtype, weight, Hq, Hkv, D, R, n, T, tail, sigma, mix, far, interleaved, train):
    return dict(name=name, kind="rotate", dtype=dtype, weight=weight, Hq=Hq, Hkv=Hkv, D=D, R=R, n=n,
                T=T, tail=tail, sigma=sigma, mix=mix, far=far, interleaved=interleaved, train=train)


def _scan(name, dtype, C, n, T, tail, sigma, mix, state, train):
    return dict(name=name, kind="scan", dtype=dtype, C=C, n=n, T=T, tail=tail, sigma=sigma, mix=mix,
                state=state, train=train)


def listed():
    return [
        # the next token of 32 sequences, as a generation's step has them: all latency
        _embed("embed-token", "bf16", "bf16", 32, 0, 32_768, 2_048, 1.0, False, False),
        # a small batch through a worker's token buffer, padding behind it, rows of an
        # odd width, weights in 32 bits under 16-bit activations
        _embed("embed-odd-train", "fp32", "fp16", 5_003, 170, 21_841, 250, 0.7, True, True),
        # a training step's batch of 32 documents, tokens as frequent as words are
        _embed("embed-batch-train", "bf16", "bf16", 16_384, 0, 32_768, 2_048, 1.0, True, True),
        # a large vocabulary, weights in 32 bits: the gradient is mostly rows no token names
        _embed("embed-large-train", "fp32", "bf16", 65_536, 0, 131_072, 1_024, 1.0, False, True),
        # the next token of 32 long sequences, far positions: all latency
        _rotate("rotate-token", "bf16", "bf16", 16, 4, 128, 128, 32, 32, 0, 0.0, 1, 100_000, False, False),
        # a batch of 32 documents in a training step, grouped heads
        _rotate("rotate-batch-train", "bf16", "bf16", 16, 4, 128, 128, 32, 16_384, 0, 0.7, 2, 0, False,
                True),
        # odd lengths, a width that is no power of two, half of it rotated, neighbours
        # as pairs, padding behind the last sample, weights in 32 bits
        _rotate("rotate-odd-train", "fp16", "fp32", 6, 2, 80, 40, 41, 5_003, 170, 1.2, 3, 0, True, True),
        # the evaluation of long documents, more heads
        _rotate("rotate-long", "bf16", "fp32", 32, 8, 128, 128, 3, 65_536, 0, 2.5, 4, 0, False, False),
        # the next token of 32 sequences from their states: all latency
        _scan("scan-token", "bf16", 2_048, 32, 32, 0, 0.0, 1, True, False),
        # odd lengths, samples of one token and of none, an odd number of channels,
        # states handed in and out, padding, all in 32 bits
        _scan("scan-odd-train", "fp32", 333, 41, 5_003, 170, 1.2, 3, True, True),
        # a batch of 32 documents in a training step
        _scan("scan-batch-train", "bf16", 2_048, 32, 16_384, 0, 0.7, 2, False, True),
        # one long document in a training step
        _scan("scan-long-train", "fp16", 1_024, 1, 65_536, 0, 0.0, 5, False, True),
    ]


_GRADIENT = 1.6e8      # of an embedding: elements of weight or activations
_ELEMENTS = 3.2e8      # of norms and rotations: elements of q and k, twice for training
_STATES = 6.5e7        # of a recurrence: elements


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["embed", "rotate", "scan"])
    tail = rng.choice([0, 0, rng.randint(1, 200)])
    if kind == "embed":
        while True:
            T, V, D = log_int(1, 100_000), log_int(2, 200_000), log_int(8, 8_192)
            D = rng.choice([D, D // 8 * 8])
            if max(T, V) * D <= _GRADIENT:
                break
        weight, dtype = rng.choice([("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp16"),
                                    ("fp32", "fp32")])
        c = _embed("", weight, dtype, T, tail, V, D, rng.choice([0.0, 0.7, 1.0, 1.0]),
                   rng.random() < 0.5, rng.random() < 0.7)
    elif kind == "rotate":
        while True:
            Hkv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
            D = rng.choice([64, 128, 64, 128, 32, 48, 80, 96, 112, 256])
            R = rng.choice([D, D, D // 16 * 8])
            n, T = log_int(1, 128), log_int(1, 100_000)
            train = rng.random() < 0.6
            if T * (Hkv * group + Hkv) * D * (2 if train else 1) <= _ELEMENTS:
                break
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        c = _rotate("", dtype, rng.choice([dtype, "fp32"]), Hkv * group, Hkv, D, R, n, T, tail,
                    rng.uniform(0.0, 2.0), rng.randint(10, 1_000_000),
                    rng.choice([0, 0, log_int(1_000, 1_000_000)]), rng.random() < 0.3, train)
    else:
        while True:
            C, n, T = log_int(1, 8_192), log_int(1, 256), log_int(1, 100_000)
            C = rng.choice([C, max(8, C // 8 * 8)])
            if T * C <= _STATES:
                break
        c = _scan("", rng.choice(["bf16", "bf16", "fp16", "fp32"]), C, n, T, tail,
                  rng.uniform(0.0, 2.0), rng.randint(10, 1_000_000), rng.random() < 0.5,
                  rng.random() < 0.6)
    del c["name"]
    return c


def _lengths(c):
    """Lengths of a case's samples (the same for every seed): their sum is T."""
    r = random.Random(c["mix"])
    w = [math.exp(c["sigma"] * r.gauss(0.0, 1.0)) for _ in range(c["n"])]
    if c["n"] > 8 and c["T"] > c["n"]:
        w[r.randrange(c["n"])] = 0.0  # a sample of no tokens, as a filtered one is
    total = sum(w)
    out = [int(c["T"] * x / total) for x in w]
    out[max(range(c["n"]), key=lambda i: w[i])] += c["T"] - sum(out)
    return out


# -- inputs -------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(2_000_003 + seed)
    kind, rows = case["kind"], case["T"] + case["tail"]

    def normal(*shape, dtype=case["dtype"], scale=1.0, mean=0.0):
        x = torch.randn(shape, generator=g, device="cuda")
        return x.mul_(scale).add_(mean).to(DTYPES[dtype])

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)

    if kind == "embed":
        V, D, T = case["V"], case["D"], case["T"]
        # frequencies go as 1 / id^skew: by the inverse of their integral
        u, e = uniform(T), 1.0 - case["skew"]
        x = torch.exp(u * math.log(V + 1)) if e == 0 else (u * ((V + 1) ** e - 1) + 1) ** (1 / e)
        ids = (x.long() - 1).clamp(0, V - 1)
        st = dict(weight=normal(V, D, dtype=case["weight"], scale=D ** -0.5), scale=math.sqrt(D))
        if case["slots"]:  # the tokens lie in blocks of a buffer
            block = 64
            blocks = -(-T // block) + 7
            order = torch.argsort(uniform(blocks)).repeat_interleave(block) * block
            slot = order + torch.arange(block, device="cuda").repeat(blocks)
            st["slot"] = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
            st["slot"][:T] = slot[:T]
            st["ids"] = torch.zeros(blocks * block, dtype=torch.int64, device="cuda")
            st["ids"][slot[:T]] = ids
        else:
            st["ids"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
            st["ids"][:T] = ids.int()
            st["slot"] = None
        if case["train"]:
            st["dout"] = normal(rows, D, scale=0.1)
    else:
        st = dict()
        start = [0]
        for x in _lengths(case):
            start.append(start[-1] + x)
        st["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    if kind == "rotate":
        Hq, Hkv, D, R = case["Hq"], case["Hkv"], case["D"], case["R"]
        qkv = normal(rows, Hq + 2 * Hkv, D, scale=1.5)  # one projection's output
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv])
        lengths = (st["start"][1:] - st["start"][:-1]).long()
        sample = torch.repeat_interleave(torch.arange(case["n"], device="cuda"), lengths)
        first = (uniform(case["n"]) * (case["far"] + 1)).long()  # tokens that stand before
        pos = torch.arange(case["T"], device="cuda") - st["start"][sample].long() + first[sample]
        st["pos"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        st["pos"][:case["T"]] = pos.int()
        i = torch.arange(0, R, 2, dtype=torch.float64, device="cuda")
        st["freq"] = 10_000.0 ** (-i / R)
        for name in ("q_weight", "k_weight"):
            st[name] = normal(D, dtype=case["weight"], scale=0.2, mean=1.0)
        st["eps"] = 1e-6
        if case["train"]:
            st.update(dq=normal(rows, Hq, D), dk=normal(rows, Hkv, D))
    elif kind == "scan":
        C, n = case["C"], case["n"]
        both = normal(rows, 2 * C)  # one projection's output
        both[:, C:].mul_(1.5).add_(2.5)  # gates that remember some ten to a hundred tokens
        st.update(x=both[:, :C], gate=both[:, C:], h0=None, dlast=None)
        if case["state"]:
            st["h0"] = normal(n, C, dtype="fp32")
        if case["train"]:
            st["dh"] = normal(rows, C)
            if case["state"]:
                st["dlast"] = normal(n, C, dtype="fp32")
    st["case"] = case
    return st


# -- the plain forms ------------------------------------------------------------------
def _token_ids(st):
    """Every row's token, and whether it has one."""
    ids, slot, V = st["ids"].long(), st["slot"], st["case"]["V"]
    if slot is not None:
        ids = torch.where(slot >= 0, ids[slot.clamp(min=0)], -1)
    there = (ids >= 0) & (ids < V)
    return torch.where(there, ids, 0), there


def _plain_embed(st):
    c = st["case"]
    ids, there = _token_ids(st)
    out = st["weight"][ids].float() * st["scale"]
    out.masked_fill_(~there[:, None], 0.0)
    out = out.to(DTYPES[c["dtype"]])
    if not c["train"]:
        return dict(out=out)
    d = st["dout"].float() * st["scale"]
    d.masked_fill_(~there[:, None], 0.0)
    dw = torch.zeros((c["V"], c["D"]), dtype=torch.float32, device="cuda")
    dw.index_add_(0, ids, d)
    return dict(out=out, dweight=dw.to(st["weight"].dtype))


def _pairs(x, R, interleaved):
    if interleaved:
        return x[..., 0:R:2], x[..., 1:R:2]
    return x[..., :R // 2], x[..., R // 2:R]


def _turn(x, cos, sin, R, interleaved):
    """x with its first R elements rotated pair by pair."""
    a, b = _pairs(x, R, interleaved)
    out = x.clone()
    u, v = _pairs(out, R, interleaved)
    u.copy_(a * cos - b * sin)
    v.copy_(b * cos + a * sin)
    return out


def _plain_rotate(st):
    c = st["case"]
    R, D = c["R"], c["D"]
    there = (st["pos"] >= 0)[:, None, None]
    angle = st["pos"].double()[:, None, None] * st["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {}
    for name in ("q", "k"):
        x, w = st[name], st[name + "_weight"]
        xf = torch.where(there, x.float(), 0.0)
        r = torch.rsqrt((xf * xf).sum(2, keepdim=True) / D + st["eps"])
        xh = xf * r
        y = _turn(xh * w.float(), cos, sin, R, c["interleaved"])
        out[name + "_out"] = torch.where(there, y, 0.0).to(x.dtype)
        if not c["train"]:
            continue
        g = torch.where(there, st["d" + name].float(), 0.0)
        g = _turn(g, cos, -sin, R, c["interleaved"])
        out[f"d{name}_weight"] = (g * xh).sum((0, 1)).to(w.dtype)
        g = g * w.float()
        dx = r * (g - xh * ((g * xh).sum(2, keepdim=True) / D))
        out["d" + name] = torch.where(there, dx, 0.0).to(x.dtype)
    return out


def _plain_linear_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first dimension, by doubling."""
    step = 1
    while step < a.shape[0]:
        b_next, a_next = b.clone(), a.clone()
        b_next[step:] += a[step:] * b[:-step]
        a_next[step:] *= a[:-step]
        a, b, step = a_next, b_next, 2 * step
    return b


def _plain_scan(st):
    c = st["case"]
    T, n, start, x16 = c["T"], c["n"], st["start"].long(), st["x"]
    x, gate = x16[:T].float(), st["gate"][:T].float()
    a, keep = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    full = start[1:] > start[:-1]
    first, final = start[:-1][full], start[1:][full] - 1  # of the samples that have tokens
    h0 = torch.zeros((n, c["C"]), device="cuda") if st["h0"] is None else st["h0"]
    carried = a.clone()
    carried[first] = 0.0
    b = keep * x
    b[first] += a[first] * h0[full]
    h = _plain_linear_scan(carried, b)
    last = h0.clone()
    last[full] = h[final]

    def rows(y):
        out = torch.zeros((T + c["tail"], c["C"]), dtype=x16.dtype, device="cuda")
        out[:T] = y
        return out

    out = dict(h=rows(h), last=last)
    if not c["train"]:
        return out
    before = torch.zeros_like(h)
    before[1:] = h[:-1]
    before[first] = h0[full]
    d = st["dh"][:T].float()
    if st["dlast"] is not None:
        d = d.clone()
        d[final] += st["dlast"][full]
    # G_t = d_t + a_{t+1} G_{t+1} within a sample
    behind = torch.zeros_like(carried)
    behind[:-1] = carried[1:]
    G = _plain_linear_scan(behind.flip(0), d.flip(0)).flip(0)
    out["dx"] = rows(keep * G)
    out["dgate"] = rows(a * keep * (before - x) * G)
    if st["h0"] is not None:
        dh0 = torch.zeros_like(h0) if st["dlast"] is None else st["dlast"].clone()
        dh0[full] = a[first] * G[first]
        out["dh0"] = dh0
    return out


# -- one pass ---------------------------------------------------------------------------
def _run_own(st):
    from paper_2101_08734_amd import nopfs

    c = st["case"]
    if c["kind"] == "embed":
        out = nopfs.token_embed(st["weight"], st["ids"], st["scale"], slot=st["slot"],
                                dtype=DTYPES[c["dtype"]])
        if not c["train"]:
            return dict(out=out)
        dw = nopfs.token_embed_grad(st["dout"], st["ids"], c["V"], st["scale"], slot=st["slot"],
                                    dtype=st["weight"].dtype)
        return dict(out=out, dweight=dw)
    if c["kind"] == "rotate":
        args = (st["q"], st["k"], st["pos"], st["freq"], st["q_weight"], st["k_weight"])
        how = dict(eps=st["eps"], interleaved=c["interleaved"])
        q, k = nopfs.norm_rotate(*args, **how)
        if not c["train"]:
            return dict(q_out=q, k_out=k)
        dq, dk, dqw, dkw = nopfs.norm_rotate_grad(st["dq"], st["dk"], *args, **how)
        return dict(q_out=q, dq_weight=dqw, dq=dq, k_out=k, dk_weight=dkw, dk=dk)
    h, last, carry = nopfs.gated_scan(st["x"], st["gate"], st["start"], st["h0"])
    if not c["train"]:
        return dict(h=h, last=last)
    dx, dgate, dh0 = nopfs.gated_scan_grad(st["dh"], st["x"], st["gate"], st["start"], carry,
                                           h0=st["h0"], dlast=st["dlast"])
    out = dict(h=h, last=last, dx=dx, dgate=dgate)
    if st["h0"] is not None:
        out["dh0"] = dh0
    return out


def run(state):
    if own:
        return _run_own(state)
    return dict(embed=_plain_embed, rotate=_plain_rotate, scan=_plain_scan)[state["case"]["kind"]](state)


def work(case):
    kind, T, rows, size = case["kind"], case["T"], case["T"] + case["tail"], SIZE[case["dtype"]]
    train = case["train"]
    if kind == "embed":
        V, D, wide = case["V"], case["D"], SIZE[case["weight"]]
        e, v = 1.0 - case["skew"], np.arange(1, V + 2, dtype=np.float64)
        upto = np.log(v) if e == 0 else (v ** e - 1) / e
        p = np.diff(upto) / upto[-1]
        distinct = float(-np.expm1(T * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())
        ids = rows * (16 if case["slots"] else 4)
        bytes_ = ids + distinct * D * wide + rows * D * size
        if train:
            bytes_ += ids + T * D * size + V * D * wide
        return {"bytes": int(bytes_), "flops": (2 if train else 1) * T * D}
    if kind == "rotate":
        D, heads = case["D"], case["Hq"] + case["Hkv"]
        x = size * heads * D
        small = rows * 4 + 4 * case["R"] + 2 * SIZE[case["weight"]] * D
        bytes_ = x * (T + rows) + small
        if train:
            bytes_ += x * (2 * T + rows) + small + 2 * SIZE[case["weight"]] * D
        return {"bytes": bytes_, "flops": (30 if train else 9) * T * heads * D}
    C, n = case["C"], case["n"]
    states = 4 * n * C
    bytes_ = size * C * (2 * T + rows) + 4 * (n + 1) + states * (2 if case["state"] else 1)
    if train:
        bytes_ += size * C * (3 * T + 2 * rows) + 4 * (n + 1) + (3 * states if case["state"] else 0)
    return {"bytes": bytes_, "flops": (30 if train else 8) * T * C}


# -- from the definitions, in 64 bits -------------------------------------------------------
def _exact_embed(st):
    c = st["case"]
    ids = st["ids"].cpu().numpy()
    slot = None if st["slot"] is None else st["slot"].cpu().numpy()
    names = ids if slot is None else np.array([ids[s] if s >= 0 else -1 for s in slot])
    rows = np.flatnonzero((names >= 0) & (names < c["V"]))
    at, names = torch.from_numpy(rows).cuda(), torch.from_numpy(names[rows].astype(np.int64)).cuda()
    out = torch.zeros((c["T"] + c["tail"], c["D"]), dtype=torch.float64, device="cuda")
    out[at] = st["scale"] * st["weight"][names].double()
    if not c["train"]:
        return dict(out=out)
    # a token's rows one after the other: differences of running sums at its ends
    order = torch.argsort(names, stable=True)
    token, many = torch.unique_consecutive(names[order], return_counts=True)
    ends = many.cumsum(0)
    dw = torch.zeros((c["V"], c["D"]), dtype=torch.float64, device="cuda")
    for a in range(0, c["D"], 256):
        run = st["dout"][at[order], a:a + 256].double().cumsum(0)[ends - 1]
        run[1:] = run[1:] - run[:-1].clone()
        dw[token, a:a + 256] = st["scale"] * run
    return dict(out=out, dweight=dw)


def _exact_rotate(st):
    """As complex numbers on the unit circle; gradients by autograd."""
    c = st["case"]
    R, D, T, rows = c["R"], c["D"], c["T"], c["T"] + c["tail"]
    angle = st["pos"][:T].double()[:, None, None] * st["freq"]
    circle = torch.polar(torch.ones_like(angle), angle)
    out = {}
    for name in ("q", "k"):
        x = st[name][:T].double().detach().requires_grad_(c["train"])
        w = st[name + "_weight"].double().detach().requires_grad_(c["train"])
        y = w * (x / (x.square().mean(2, keepdim=True) + st["eps"]).sqrt())
        z = y[..., :R]
        if c["interleaved"]:
            z = torch.view_as_complex(z.reshape(T, -1, R // 2, 2))
            z = torch.view_as_real(z * circle).reshape(T, -1, R)
        else:
            z = torch.complex(*z.reshape(T, -1, 2, R // 2).unbind(2)) * circle
            z = torch.cat([z.real, z.imag], 2)
        y = torch.cat([z, y[..., R:]], 2)

        def padded(a):
            p = torch.zeros((rows, *a.shape[1:]), dtype=torch.float64, device="cuda")
            p[:T] = a
            return p

        out[name + "_out"] = padded(y.detach())
        if c["train"]:
            dx, dw = torch.autograd.grad(y, (x, w), st["d" + name][:T].double())
            out[f"d{name}_weight"], out["d" + name] = dw, padded(dx)
    return out


def _exact_scan(st):
    """Token by token, forwards and backwards."""
    c = st["case"]
    T, n, C = c["T"], c["n"], c["C"]
    start = st["start"].tolist()
    f64 = dict(dtype=torch.float64, device="cuda")
    x, gate = st["x"].double(), st["gate"].double()
    a, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    b = keep * x
    h, before = torch.zeros((T + c["tail"], C), **f64), torch.zeros((T + c["tail"], C), **f64)
    last = torch.zeros((n, C), **f64) if st["h0"] is None else st["h0"].double()
    for s in range(n):
        for t in range(start[s], start[s + 1]):
            state = last[s] if t == start[s] else h[t - 1]
            torch.addcmul(b[t], a[t], state, out=h[t])
        if start[s + 1] > start[s]:
            i, e = start[s], start[s + 1]
            before[i] = last[s]
            before[i + 1:e] = h[i:e - 1]
            last[s] = h[e - 1]
    out = dict(h=h, last=last)
    if not c["train"]:
        return out
    dh = st["dh"].double()
    G = torch.zeros_like(h)
    dh0 = torch.zeros((n, C), **f64) if st["dlast"] is None else st["dlast"].double()
    for s in range(n):
        for t in range(start[s + 1] - 1, start[s] - 1, -1):
            if t == start[s + 1] - 1:
                torch.add(dh[t], dh0[s], out=G[t])
            else:
                torch.addcmul(dh[t], a[t + 1], G[t + 1], out=G[t])
        if start[s + 1] > start[s]:
            dh0[s] = a[start[s]] * G[start[s]]
    out["dx"] = keep * G
    out["dgate"] = a * keep * (before - x) * G
    out["dx"][T:] = 0.0
    out["dgate"][T:] = 0.0
    if st["h0"] is not None:
        out["dh0"] = dh0
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return dict(embed=_exact_embed, rotate=_exact_rotate, scan=_exact_scan)[case["kind"]](st)
