"""Operators of language-model training whose speed matters to a user of the library's single-kernel entry points:

* the gradient of the embedding lookup, summed over the tokens in sorted order,
* the gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(z), forward and backward,
* the orthogonalisation of an update by Newton-Schulz products, with its momentum.

With `own` false `run` computes them in elementary torch operations in fp32, with `own` true through the library.
"""
import ctypes

import numpy as np
import torch

own = False

STRIDE = 64                                   # the recurrence keeps the state that enters every 64th step
COEF = (3.4445, -4.7750, 2.0315)              # of the Newton-Schulz step a X + (b A + c A^2) X, A = X X^T
STEPS, EPS = 5, 1e-7
_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _embed(name=None, *, n, vocab, d, dtype, accumulate=False, pad=0.0, zipf=1.1):
    c = dict(op="embed_bwd", n=n, vocab=vocab, d=d, dtype=dtype, accumulate=accumulate, pad=pad, zipf=zipf)
    return dict(c, name=name) if name else c


def _scan_case(name=None, *, op, b, t, d, dtype, ragged=False, keep=True):
    c = dict(op=op, b=b, t=t, d=d, dtype=dtype, ragged=ragged, keep=keep)
    return dict(c, name=name) if name else c


def _ortho(name=None, *, batch, rows, cols, dtype, momentum=False):
    c = dict(op="orthogonalize", batch=batch, rows=rows, cols=cols, dtype=dtype, momentum=momentum)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The step of the smallest configuration anyone trains: 4 x 32 tokens, 256 symbols; a call is its latency.
        _embed("embed-grad-tiny", n=128, vocab=256, d=64, dtype="fp32"),
        # 32 streams of 150 tokens in a model 410 wide: rows off every alignment, bf16 gradients, the whole matrix written.
        _embed("embed-grad-410", n=4800, vocab=32768, d=410, dtype="bf16"),
        # The ordinary 512-wide decoder's step, 16 x 512 tokens, the gradient overwritten.
        _embed("embed-grad-512", n=8192, vocab=32768, d=512, dtype="fp32"),
        # A tied matrix of 50257 rows that already holds the output projection's gradient; a quarter of the batch is padding.
        _embed("embed-grad-tied-padded", n=8192, vocab=50257, d=1024, dtype="fp32", accumulate=True, pad=0.25),
        # Generation: one token for each of 64 streams.
        _scan_case("scan-token", op="scan_fwd", b=64, t=1, d=1024, dtype="bf16", keep=False),
        # A training segment of the 1024-wide model, forward ...
        _scan_case("scan-fwd-1024", op="scan_fwd", b=8, t=1024, d=1024, dtype="bf16"),
        # ... and backward.
        _scan_case("scan-bwd-1024", op="scan_bwd", b=8, t=1024, d=1024, dtype="bf16"),
        # One long document in fp32: few channels, many steps.
        _scan_case("scan-fwd-long", op="scan_fwd", b=1, t=65536, d=512, dtype="fp32"),
        # A padded batch of uneven lengths (an empty one among them), width off every alignment.
        _scan_case("scan-bwd-ragged", op="scan_bwd", b=7, t=777, d=410, dtype="fp32", ragged=True),
        # One feed-forward matrix of the smallest configuration.
        _ortho("ortho-tiny", batch=1, rows=64, cols=256, dtype="fp32"),
        # The second feed-forward matrices of four layers 410 wide (taller than wide, no whole tiles), with momentum.
        _ortho("ortho-tall-momentum", batch=4, rows=2100, cols=410, dtype="fp32", momentum=True),
        # The first feed-forward matrices of a 1024-wide model of 24 layers, bf16 gradients and updates.
        _ortho("ortho-1024", batch=24, rows=1024, cols=4096, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, lo, hi):
    """A whole number of tiles as often as not."""
    w = _log_int(rng, lo, hi)
    return max(lo, w // 64 * 64) if w >= 64 and rng.random() < 0.5 else w


def draw(rng):
    """One more call over the ranges between the smallest and the largest listed ones."""
    while True:
        dtype = rng.choice(("fp32", "bf16"))
        kind = rng.choice(("embed", "scan_fwd", "scan_bwd", "orthogonalize"))
        if kind == "embed":
            c = _embed(n=_log_int(rng, 1, 32768), vocab=_log_int(rng, 64, 65536), d=_width(rng, 16, 2048), dtype=dtype,
                       accumulate=rng.random() < 0.5, pad=rng.choice((0.0, 0.0, 0.25, 0.6)), zipf=rng.choice((1.0, 1.1, 1.3)))
        elif kind == "orthogonalize":
            c = _ortho(batch=_log_int(rng, 1, 24), rows=_width(rng, 16, 4096), cols=_width(rng, 16, 4096), dtype=dtype, momentum=rng.random() < 0.5)
        else:
            c = _scan_case(op=kind, b=_log_int(rng, 1, 64), t=rng.choice((1, _log_int(rng, 2, 65536), _log_int(rng, 2, 4096))), d=_width(rng, 16, 2048),
                           dtype=dtype, ragged=rng.random() < 0.3, keep=rng.random() < 0.7)
            if c["op"] == "scan_bwd":
                c["keep"] = True
            if c["b"] * c["t"] * c["d"] > 3.3e7:
                continue
        w = work(c)
        if w["bytes"] <= 4.5e8 and w["flops"] <= 1.6e12:
            return c


# ------------------------------------------------------------------------------ inputs
def _zipf(c):
    p = np.arange(1, c["vocab"] + 1, dtype=np.float64) ** -c["zipf"]
    return p / p.sum()


def _lens(c, gen):
    """Lengths from an empty stream to a full one; a seed deals the same ones to other streams."""
    if not c["ragged"]:
        return None
    b, t = c["b"], c["t"]
    every = torch.tensor([t * i // max(1, b - 1) if b > 1 else t // 2 for i in range(b)], dtype=torch.int32)
    return every[torch.randperm(b, generator=gen)].cuda()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    t_ = _DTYPE[c["dtype"]]
    s = {"case": c}

    def normal(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen).to(dtype)

    if c["op"] == "embed_bwd":
        cdf = torch.from_numpy(np.cumsum(_zipf(c))).cuda()
        u = torch.rand(c["n"], generator=gen, device="cuda", dtype=torch.float64)
        tok = torch.searchsorted(cdf, u).clamp_(max=c["vocab"] - 1).to(torch.int32)
        dh = normal(c["n"], c["d"]) * 1e-3
        if c["pad"]:                                   # the ends of the streams: token 0, no gradient
            pad = torch.arange(c["n"], device="cuda") % 128 >= 128 * (1 - c["pad"])
            tok[pad] = 0
            dh[pad] = 0
        s.update(tok=tok, dh=dh.to(t_), scale=c["d"] ** 0.5)
        s["dV"] = normal(c["vocab"], c["d"]) * 1e-3 if c["accumulate"] else torch.empty(c["vocab"], c["d"], device="cuda")
    elif c["op"] == "orthogonalize":
        # a gradient: a few strong directions over noise
        b, m, n = c["batch"], c["rows"], c["cols"]
        r = min(16, m, n)
        low = torch.matmul(normal(b, m, r) * torch.arange(1, r + 1, device="cuda") ** -0.5, normal(b, r, n))
        s["g"] = ((low + normal(b, m, n)) * 1e-4).to(t_)
        s["m"] = normal(b, m, n) * 1e-4 if c["momentum"] else None
        s["o"] = torch.empty(b, m, n, dtype=t_, device="cuda")
        s["scale"] = max(1.0, m / n) ** 0.5
    else:
        b, t, d = c["b"], c["t"], c["d"]
        s["z"] = (normal(b, t, d) * 1.5 + 1.5).to(t_)  # gates that mostly keep
        s["x"] = normal(b, t, d, dtype=t_)
        s["h0"], s["lens"] = normal(b, d), _lens(c, host)
        if c["op"] == "scan_fwd":
            s["h"] = torch.empty(b, t, d, dtype=t_, device="cuda")
            s["hT"] = torch.empty(b, d, device="cuda")
            s["states"] = torch.empty(b, -(-t // STRIDE), d, device="cuda") if c["keep"] else None
        else:
            # the forward pass of the same step left the states behind
            s["dh"], s["dhT"] = normal(b, t, d, dtype=t_), normal(b, d)
            s["states"] = _forward(s)["states"]
            s["dz"], s["dx"] = torch.empty_like(s["z"]), torch.empty_like(s["x"])
            s["dh0"] = torch.empty(b, d, device="cuda")
    return s


# -------------------------------------------------------------------------- plain forms
def _plain_scan(a, u):
    """h_t = a_t h_{t-1} + u_t from zero along axis 1, in log2 T doublings."""
    a, h, k = a.clone(), u.clone(), 1
    while k < h.shape[1]:
        h[:, k:] = h[:, k:] + a[:, k:] * h[:, :-k]
        a[:, k:] = a[:, k:] * a[:, :-k]
        k *= 2
    return h


def _gates(s):
    """f, (1 - f) and x in fp32, and which steps are taken; a step that is not taken keeps the state."""
    z, x = s["z"].float(), s["x"].float()
    live = None
    f, e = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    if s["lens"] is not None:
        live = (torch.arange(z.shape[1], device=z.device)[None, :] < s["lens"][:, None])[:, :, None]
        f, e, x = torch.where(live, f, 1.0), torch.where(live, e, 0.0), torch.where(live, x, 0.0)
    return f, e, x, live


def _forward(s):
    f, e, x, live = _gates(s)
    u = e * x
    u[:, 0] += f[:, 0] * s["h0"]
    h = _plain_scan(f, u)
    out = {"hT": h[:, -1].clone()}
    if s["case"]["keep"]:
        out["states"] = torch.cat([s["h0"][:, None], h[:, STRIDE - 1:-1:STRIDE]], 1)
    out["h"] = (h if live is None else torch.where(live, h, 0.0)).to(s["z"].dtype)
    return out


def _backward(s):
    f, e, x, live = _gates(s)
    u = e * x
    u[:, 0] += f[:, 0] * s["h0"]
    before = torch.cat([s["h0"][:, None], _plain_scan(f, u)[:, :-1]], 1)
    g = s["dh"].float() if live is None else torch.where(live, s["dh"].float(), 0.0)
    g = torch.cat([g[:, :-1], g[:, -1:] + s["dhT"][:, None]], 1)
    g = _plain_scan(torch.cat([f[:, 1:], f[:, :1]], 1).flip(1), g.flip(1)).flip(1)    # the first factor meets nothing
    t_ = s["z"].dtype
    return {"dz": (g * (before - x) * (f * e)).to(t_), "dx": (g * e).to(t_), "dh0": f[:, 0] * g[:, 0]}


def _embed_bwd(s):
    c = s["case"]
    out = s["dV"] if c["accumulate"] else torch.zeros(c["vocab"], c["d"], device="cuda")
    return {"dV": out.index_add_(0, s["tok"], s["dh"].float() * s["scale"])}


def _orthogonalize(s):
    x = s["g"].float()
    out = {}
    if s["m"] is not None:
        s["m"].mul_(0.95).add_(x)
        x = x + 0.95 * s["m"]
        out["m"] = s["m"]
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    out["o"] = ((x.transpose(1, 2) if tall else x) * s["scale"]).to(s["g"].dtype).contiguous()
    return out


# ----------------------------------------------------------------------------- own calls
def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _own(s):
    from paper_1909_06695_amd import binding as P

    L, c = P.lib(), s["case"]
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    dtype = 1 if c["dtype"] == "bf16" else 0

    def scratch(size, *of):
        if "scratch" not in s:                         # a program keeps it from call to call
            floats = size(*of)
            s["scratch"] = torch.empty(floats, device="cuda") if floats else None
        return _ptr(s["scratch"])

    if c["op"] == "embed_bwd":
        d = c["d"]
        P.check(L.ouro_op_embed_bwd_sorted(stream, dtype, _ptr(s["tok"]), _ptr(s["dh"]), d, _ptr(s["dV"]), d, c["n"], d, c["vocab"],
                                           s["scale"], int(c["accumulate"])))
        return {"dV": s["dV"]}
    if c["op"] == "orthogonalize":
        b, m, n = c["batch"], c["rows"], c["cols"]
        work = scratch(L.ouro_op_orthogonalize_scratch, b, m, n)
        P.check(L.ouro_op_orthogonalize(stream, dtype, b, m, n, _ptr(s["g"]), n, m * n, _ptr(s["m"]), 0.95, 1, _ptr(s["o"]), n, m * n,
                                        s["scale"], EPS, STEPS, work))
        return {"o": s["o"]} if s["m"] is None else {"m": s["m"], "o": s["o"]}
    b, t, d = c["b"], c["t"], c["d"]
    work = scratch(L.ouro_op_recurrence_scratch, b, t, d)
    if c["op"] == "scan_fwd":
        P.check(L.ouro_op_recurrence_fwd(stream, dtype, b, t, d, _ptr(s["z"]), d, _ptr(s["x"]), d, _ptr(s["h0"]), _ptr(s["lens"]),
                                         _ptr(s["h"]), d, _ptr(s["hT"]), _ptr(s["states"]), work))
        out = {"h": s["h"], "hT": s["hT"]}
        return dict(out, states=s["states"]) if c["keep"] else out
    P.check(L.ouro_op_recurrence_bwd(stream, dtype, b, t, d, _ptr(s["z"]), d, _ptr(s["x"]), d, _ptr(s["states"]), _ptr(s["lens"]),
                                     _ptr(s["dh"]), d, _ptr(s["dhT"]), _ptr(s["dz"]), d, _ptr(s["dx"]), d, _ptr(s["dh0"]), work))
    return {"dz": s["dz"], "dx": s["dx"], "dh0": s["dh0"]}


def run(state):
    if own:
        return _own(state)
    return {"embed_bwd": _embed_bwd, "scan_fwd": _forward, "scan_bwd": _backward, "orthogonalize": _orthogonalize}[state["case"]["op"]](state)


# ----------------------------------------------------------------------- work, and 64 bits
def work(case):
    """Bytes: every input read once and every output written once (of an accumulated matrix the rows of tokens that occur, as
    many as the distribution lets expect).  Flops: 1 multiply-add an embedded element; 8 a step of the recurrence forward, 16
    backward; for the Newton-Schulz step X X^T and its square by their symmetry once per pair, and the product onto X."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "embed_bwd":
        n, v, d = c["n"], c["vocab"], c["d"]
        rows = float((1 - (1 - _zipf(c)) ** (n * (1 - c["pad"]))).sum())
        return {"bytes": n * (4 + d * e) + d * 4 * (2 * rows if c["accumulate"] else v), "flops": 2 * n * d}
    if c["op"] == "orthogonalize":
        b, m, n = c["batch"], min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        return {"bytes": b * m * n * (2 * e + (8 if c["momentum"] else 0)), "flops": b * STEPS * (m * m * n + m ** 3 + 2 * m * m * n)}
    b, t, d = c["b"], c["t"], c["d"]
    live = b * t // 2 if c["ragged"] else b * t
    states = b * -(-t // STRIDE) * d * 4 if c["keep"] else 0
    if c["op"] == "scan_fwd":
        return {"bytes": (2 * live + b * t) * d * e + states + 8 * b * d, "flops": 8 * live * d}
    return {"bytes": (3 * live + 2 * b * t) * d * e + states + 8 * b * d, "flops": 16 * live * d}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "embed_bwd":
        # runs of equal tokens as differences of running sums
        key, order = torch.sort(s["tok"].long(), stable=True)
        total = torch.cat([torch.zeros(1, c["d"], dtype=torch.float64, device="cuda"), torch.cumsum(s["dh"].double()[order], 0)])
        first = torch.searchsorted(key, torch.arange(c["vocab"] + 1, device="cuda"))
        out = (total[first[1:]] - total[first[:-1]]) * s["scale"]
        return {"dV": out + s["dV"].double() if c["accumulate"] else out}
    if c["op"] == "orthogonalize":
        # the polynomial of the Gram matrix, applied once
        x, out = s["g"].double(), {}
        if s["m"] is not None:
            out["m"] = 0.95 * s["m"].double() + x
            x = x + 0.95 * out["m"]
        tall = c["rows"] > c["cols"]
        x = (x.transpose(1, 2) if tall else x).contiguous()
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        eye = torch.eye(gram.shape[1], dtype=torch.float64, device="cuda")
        q = eye.expand_as(gram).contiguous()
        for _ in range(STEPS):
            p = COEF[0] * eye + COEF[1] * gram + COEF[2] * torch.bmm(gram, gram)
            q, gram = torch.bmm(p, q), torch.bmm(p, torch.bmm(gram, p))
        o = torch.bmm(q, x) * s["scale"]
        out["o"] = (o.transpose(1, 2) if tall else o).contiguous()
        return out
    # the recurrence step by step
    b, t, d = c["b"], c["t"], c["d"]
    lens = torch.full((b, 1), t, device="cuda") if s["lens"] is None else s["lens"].long()[:, None]
    h = s["h0"].double()
    every = torch.empty(t + 1, b, d, dtype=torch.float64, device="cuda")
    every[0] = h
    f = torch.sigmoid(s["z"].double())
    x = s["x"].double()
    for i in range(t):
        h = torch.where(i < lens, torch.lerp(x[:, i], h, f[:, i]), h)
        every[i + 1] = h
    if c["op"] == "scan_fwd":
        taken = torch.arange(t, device="cuda")[None, :] < lens
        out = {"h": torch.where(taken[:, :, None], every[1:].transpose(0, 1), 0.0), "hT": h}
        if c["keep"]:
            out["states"] = every[0:t:STRIDE].transpose(0, 1).contiguous()
        return out
    g, dh = s["dhT"].double(), s["dh"].double()
    dz, dx = torch.empty_like(dh), torch.empty_like(dh)
    for i in range(t - 1, -1, -1):
        here = torch.where(i < lens, g + dh[:, i], 0.0)
        k = 1 - f[:, i]
        dx[:, i] = here * k
        dz[:, i] = here * (every[i] - x[:, i]) * f[:, i] * k
        g = torch.where(i < lens, here * f[:, i], g)
    return {"dz": dz, "dx": dx, "dh0": g}
