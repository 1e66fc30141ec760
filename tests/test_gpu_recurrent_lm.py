"""A training step of a recurrent language model put together from the single entry points, against 64 bits: tied embedding, a gated
linear recurrence over two segments whose state is carried on, cross-entropy, the gradients of all of it, and the
orthogonalised update of the two projections, after which single tokens continue.

Tolerance, by running error analysis: every number of the oracle carries a bound on what the device's may be off by.  A product and a sum
round once (2^-24 relative); a contraction of K terms adds (K + 2) 2^-23 of the sum of magnitudes (twice a rounding a term, for
sums that cut off); the gate's error is as in the tests of the recurrence, on top of what the error of z makes of it (a gate
changes by at most the factor exp(error of z)), and so are the 32 roundings of its scan; a softmax changes by at most the factor
exp(2 x largest error of its logits), and its own exponentials and sum by (|l| + |lse| + vocab + 16) 2^-24; what is stored as T rounds
once more, by half a step of T.  Over the whole step in bf16 such bounds grow beyond the gradients themselves, because they add up
what is independent; there the norm of an error is bounded too: ten numbers are stored on the longest way to a gradient (e, z, x, h,
logits, G, dh, dz, dx, de), each off by at most 2^-8 of itself, and contractions keep the ratio of independent errors to values, 10 x
2^-8 < 1/16."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {0: 0.0, 1: 2.0 ** -8}
VOCAB, LD, D, B, T = 61, 64, 40, 3, 70
SCALE = 1.5
LENS = [[70, 70, 70], [70, 33, 0]]                         # of the streams in the two segments


class Num:
    """A value and a bound on the error of what stands for it."""

    def __init__(self, v, e=None):
        self.v = np.asarray(v, dtype=np.float64)
        self.e = np.zeros_like(self.v) if e is None else e

    def _rounded(self, v, e, u=U):
        return Num(v, e + u * (np.abs(v) + e))

    def __add__(self, o):
        return self._rounded(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        return self._rounded(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        return self._rounded(self.v * o.v, np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e)

    def __matmul__(self, o):
        a, b = np.abs(self.v) + self.e, np.abs(o.v) + o.e
        e = a @ o.e + self.e @ np.abs(o.v)
        return Num(self.v @ o.v, e + (self.v.shape[-1] + 2) * 2 * U * (a @ b))

    def at(self, *i):
        return Num(self.v[i], self.e[i])

    @property
    def T(self):
        return Num(self.v.T, self.e.T)

    def stored(self, dtype):
        return self._rounded(self.v, self.e, HALF[dtype])

    def slack(self, u):
        return self._rounded(self.v, self.e, u)


def gates(z, live):
    """f, 1 - f of a step; (1, 0) for streams that have ended."""
    own = (np.abs(z.v) + z.e + 8) * U
    f, k = 1 / (1 + np.exp(-z.v)), 1 / (1 + np.exp(z.v))
    rel = np.expm1(z.e + 2 * own)
    return (Num(np.where(live, f, 1.0), np.where(live, f * rel, 0.0)), Num(np.where(live, k, 0.0), np.where(live, k * rel, 0.0)))


def slack(mag, q, u=32 * U):
    return Num(q.v, q.e + u * mag)


def recurrence(z, x, h0, lens):
    """h [B, T, D], the state before every step, the last state; mag: sums of magnitudes, which the scan's roundings are counted on."""
    h, mag = h0, np.abs(h0.v) + h0.e
    before, out = [], []
    for t in range(T):
        live = t < np.array(lens)[:, None]
        f, k = gates(z.at(slice(None), t), live)
        before.append(slack(mag, h))
        h = f * h + k * x.at(slice(None), t)
        mag = f.v * mag + k.v * (np.abs(x.v[:, t]) + x.e[:, t])
        out.append(Num(np.where(live, h.v, 0.0), np.where(live, h.e + 32 * U * mag, 0.0)))
    return out, before, slack(mag, h)


def recurrence_back(z, x, before, lens, dh, dhT):
    P, mag = dhT, np.abs(dhT.v) + dhT.e
    dz, dx = [None] * T, [None] * T
    for t in range(T - 1, -1, -1):
        live = t < np.array(lens)[:, None]
        f, k = gates(z.at(slice(None), t), live)
        d = Num(np.where(live, dh.v[:, t], 0.0), np.where(live, dh.e[:, t], 0.0))
        mag = mag + np.abs(d.v) + d.e
        G = slack(mag, P + d)
        dx[t] = k * G
        dz[t] = f * k * G * (before[t] - x.at(slice(None), t))
        P = f * (P + d)
        mag = f.v * mag
    return dz, dx, slack(mag, P)


def rows(steps, dtype):
    return Num(np.stack([q.v for q in steps], 1), np.stack([q.e for q in steps], 1)).stored(dtype)


def flat(q):
    return Num(q.v.reshape(B * T, -1), q.e.reshape(B * T, -1))


def split(q):
    return Num(q.v.reshape(B, T, -1), q.e.reshape(B, T, -1))


def oracle(V, W, h0, tok, tgt, dtype):
    """V [vocab, D], W [2, D, D] (the gate's and the input's projection), h0 [B, D]; tok, tgt [2, B*T] of the two segments.  Losses of the
    segments and the gradients of their sum."""
    V, W, state = Num(V), [Num(w) for w in W], Num(h0)
    kept, out = [], {"loss": []}
    n = B * T
    for s in range(2):
        e = Num(SCALE * V.v[tok[s]], U * np.abs(SCALE * V.v[tok[s]])).stored(dtype)
        z, x = (split((e @ w).stored(dtype)) for w in W)
        h, before, last = recurrence(z, x, state, LENS[s])
        h = flat(rows(h, dtype))
        logits = (h @ V.T).stored(dtype)
        top = logits.v.max(1, keepdims=True)
        lse = top + np.log(np.exp(logits.v - top).sum(1, keepdims=True))
        worst = logits.e.max(1, keepdims=True)
        own = (np.abs(logits.v) + np.abs(lse) + VOCAB + 16) * U
        prob = np.exp(logits.v - lse)
        prob = Num(prob, prob * np.expm1(2 * worst + 2 * own))
        hot = np.zeros((n, VOCAB))
        hot[np.arange(n), tgt[s]] = 1
        G = (prob - Num(hot)).slack(2 * U)
        G = Num(G.v / n, G.e / n).stored(dtype)
        loss = (lse - np.take_along_axis(logits.v, tgt[s][:, None], 1)).mean()
        out["loss"].append(Num(loss, (2 * worst + 2 * own.max(1, keepdims=True) * np.abs(lse)).mean() + (n + 4) * U * (np.abs(lse) + np.abs(logits.v)).mean(0).max()))
        out["h%d" % s], out["hT%d" % s] = h, last
        kept.append((e, z, x, before, h, G))
        state = last
    dV, dW, dstate = Num(np.zeros_like(V.v)), [Num(np.zeros_like(W[0].v)) for _ in W], Num(np.zeros((B, D)))
    for s in (1, 0):
        e, z, x, before, h, G = kept[s]
        dh = split((G @ V).stored(dtype))
        dz, dx, dstate = recurrence_back(z, x, before, LENS[s], dh, dstate)
        dz, dx = flat(rows(dz, dtype)), flat(rows(dx, dtype))
        dW = [dw + e.T @ q for dw, q in zip(dW, (dz, dx))]
        de = ((dz @ W[0].T).stored(dtype) + dx @ W[1].T).stored(dtype)
        pick = np.zeros((VOCAB, n))
        pick[tok[s], np.arange(n)] = SCALE
        dV = dV + G.T @ h + Num(pick) @ de
    out["dV"], out["dW0"], out["dW1"], out["dh0"] = dV, dW[0], dW[1], dstate
    return out


def problem(dtype):
    rng = np.random.default_rng(11)
    V, W, h0 = 0.3 * rng.standard_normal((VOCAB, D)), rng.standard_normal((2, D, D)) / np.sqrt(D), rng.standard_normal((B, D))
    as_stored = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16 if dtype else torch.float32).double().numpy()
    tok, tgt = rng.integers(0, VOCAB, (2, B * T)), rng.integers(0, VOCAB, (2, B * T))
    tok[rng.random(tok.shape) < 0.4] = 7                   # a frequent token
    return as_stored(V), as_stored(W), h0.astype(np.float32).astype(np.float64), tok, tgt


def test_the_oracle_against_differences():
    """Central differences in 64 bits with a step of 2^-14: their own error is a third derivative's times 2^-28 / 6, and 2^-52 of the loss
    over the step, below 1e-6 for derivatives of this size."""
    V, W, h0, tok, tgt = problem(0)
    ref = oracle(V, W, h0, tok, tgt, 0)
    rng = np.random.default_rng(12)
    for name in ("dV", "dW0", "dW1", "dh0"):
        to = rng.standard_normal(ref[name].v.shape)
        at = []
        for sign in (1, -1):
            v, w, h = V.copy(), W.copy(), h0.copy()
            target = {"dV": v, "dW0": w[0], "dW1": w[1], "dh0": h}[name]
            target += sign * 2.0 ** -14 * to
            at.append(sum(q.v for q in oracle(v, w, h, tok, tgt, 0)["loss"]))
        assert abs((at[0] - at[1]) * 2.0 ** 13 - (ref[name].v * to).sum()) < 1e-6, name


def L():
    import paper_1909_06695_amd as P
    return P.lib()


def stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def ok(rc):
    assert rc == 0, L().ouro_last_error()


def host(t):
    return t.double().cpu().numpy()


class Step:
    """The buffers of the step, and its calls."""

    def __init__(self, dtype):
        self.dtype = dtype
        V, W, h0, tok, tgt = problem(dtype)
        ty, f32 = dict(dtype=torch.bfloat16 if dtype else torch.float32, device="cuda"), dict(device="cuda")
        self.V, self.W, self.h0 = torch.tensor(V, **ty), torch.tensor(W, **ty), torch.tensor(h0, dtype=torch.float32, **f32)
        self.tok, self.tgt = (torch.tensor(a, dtype=torch.int32, **f32) for a in (tok, tgt))
        self.lens = torch.tensor(LENS, dtype=torch.int32, **f32)
        n = B * T
        new = lambda *shape, **kw: torch.full(shape, float("nan"), **kw)
        self.e, self.z, self.x, self.h, self.dh, self.dz, self.dx, self.de = (new(2, n, D, **ty) for _ in range(8))
        self.G = new(2, n, LD, **ty)
        self.kept = new(2, B, -(-T // 64), D, **f32)
        self.state, self.dstate = new(2, B, D, **f32), new(B, D, **f32)
        self.lse, self.rowloss, self.loss = new(2, n, **f32), new(2, n, **f32), new(2, **f32)
        self.dV, self.dW, self.momentum, self.update = new(VOCAB, D, **f32), new(2, D, D, **f32), new(2, D, D, **f32), new(2, D, D, **f32)
        self.w32 = self.W.float()
        self.flag = torch.zeros(1, dtype=torch.int32, **f32)
        self.rec = new(max(1, L().ouro_op_recurrence_scratch(B, T, D)), **f32)
        self.work = new(L().ouro_op_orthogonalize_scratch(2, D, D), **f32)

    def gemm(self, tA, tB, M, N, K, a, lda, b, ldb, c, ldc, f32=0, add=0, residual=None):
        ok(L().ouro_op_gemm(stream(), self.dtype, tA, tB, M, N, K, 1.0, p(a), lda, p(b), ldb, p(c), ldc, f32, add, None, p(residual), D if residual is not None else 0,
                            0, None, 0, 0))

    def gradients(self):
        n, ty = B * T, self.dtype
        self.G.zero_()
        for s in range(2):
            ok(L().ouro_op_embed_fwd(stream(), ty, p(self.tok[s]), p(self.V), None, p(self.e[s]), n, T, D, VOCAB, SCALE, p(self.flag)))
            self.gemm(0, 0, n, D, D, self.e[s], D, self.W[0], D, self.z[s], D)
            self.gemm(0, 0, n, D, D, self.e[s], D, self.W[1], D, self.x[s], D)
            ok(L().ouro_op_recurrence_fwd(stream(), ty, B, T, D, p(self.z[s]), D, p(self.x[s]), D, p(self.state[0] if s else self.h0), p(self.lens[s]), p(self.h[s]), D,
                                          p(self.state[s]), p(self.kept[s]), p(self.rec)))
            self.gemm(0, 1, n, VOCAB, D, self.h[s], D, self.V, D, self.G[s], LD)
            ok(L().ouro_op_softmax_ce(stream(), ty, p(self.G[s]), LD, p(self.tgt[s]), p(self.G[s]), LD, p(self.lse[s]), p(self.rowloss[s]), p(self.loss[s:]), n, VOCAB,
                                      p(self.flag)))
        self.dV.zero_(); self.dW.zero_(); self.dstate.zero_()
        for s in (1, 0):
            self.gemm(0, 0, n, D, VOCAB, self.G[s], LD, self.V, D, self.dh[s], D)
            ok(L().ouro_op_recurrence_bwd(stream(), ty, B, T, D, p(self.z[s]), D, p(self.x[s]), D, p(self.kept[s]), p(self.lens[s]), p(self.dh[s]), D, p(self.dstate),
                                          p(self.dz[s]), D, p(self.dx[s]), D, p(self.dstate), p(self.rec)))
            self.gemm(1, 0, D, D, n, self.e[s], D, self.dz[s], D, self.dW[0], D, 1, 1)
            self.gemm(1, 0, D, D, n, self.e[s], D, self.dx[s], D, self.dW[1], D, 1, 1)
            self.gemm(0, 1, n, D, D, self.dz[s], D, self.W[0], D, self.de[s], D)
            self.gemm(0, 1, n, D, D, self.dx[s], D, self.W[1], D, self.de[s], D, residual=self.de[s])
            self.gemm(1, 0, VOCAB, D, n, self.G[s], LD, self.h[s], D, self.dV, D, 1, 1)
            ok(L().ouro_op_embed_bwd_sorted(stream(), ty, p(self.tok[s]), p(self.de[s]), D, p(self.dV), D, n, D, VOCAB, SCALE, 1))
        self.momentum.fill_(0.25)
        ok(L().ouro_op_orthogonalize(stream(), 0, 2, D, D, p(self.dW), D, D * D, p(self.momentum), 0.9, 1, p(self.update), D, D * D, 0.2, 1e-7, 5, p(self.work)))

    def apply(self):
        ok(L().ouro_op_update(stream(), p(self.w32), None, None, p(self.W) if self.dtype else None, p(self.update), 1.0, None, 0.0, self.w32.numel(), 0, 0.02, 0.9,
                              0.999, 1e-8, 0))
        if not self.dtype:
            self.W.copy_(self.w32)

    def check(self, ref):
        for name, q in ref.items():
            if name == "loss":
                got = host(self.loss)
                assert all(abs(got[s] - q[s].v) <= q[s].e for s in range(2)), (got, [i.v for i in q], [i.e for i in q])
                continue
            i = int(name[-1]) if name[-1] in "01" else 0
            got = host({"h0": self.h[0], "h1": self.h[1], "hT0": self.state[0], "hT1": self.state[1], "dV": self.dV, "dW0": self.dW[0], "dW1": self.dW[1],
                        "dh0": self.dstate}[name])
            off = np.abs(got - q.v) - q.e
            assert np.all(off <= 0), (name, i, np.nanmax(off), np.abs(q.v).max(), q.e.max())
            if self.dtype:
                assert np.linalg.norm(got - q.v) <= np.linalg.norm(q.v) / 16, (name, np.linalg.norm(got - q.v), np.linalg.norm(q.v))
        assert self.flag.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
def test_gradients_of_the_step(dtype):
    s = Step(dtype)
    s.gradients()
    s.check(oracle(*problem(dtype), dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
def test_update_and_single_tokens(dtype):
    """The update is that of the gradients the device has (tolerance as in the tests of orthogonalised updates), and with the new weights the
    states of one segment come out the same token by token."""
    from tests import test_gpu_orthogonalize as ortho
    s = Step(dtype)
    s.gradients()
    before = host(s.w32)
    m = 0.9 * 0.25 + host(s.dW)
    u = host(s.dW) + 0.9 * m
    # u as the device rounds it is off by 3 roundings of magnitudes below |dW| + 0.9 |m|; they pass through five steps, each of slope 3.9
    for i in range(2):
        ref, tol = ortho.oracle(u[i], 0.2, 1e-7, 5)
        lost = 0.2 * 2 * 3.9 ** 5 * 3 * U * np.linalg.norm(np.abs(host(s.dW)[i]) + 0.9 * (0.9 * 0.25 + np.abs(host(s.dW)[i]))) / np.linalg.norm(u[i])
        assert np.linalg.norm(host(s.update)[i] - ref) <= tol + lost + U * np.linalg.norm(ref)
    s.apply()
    after = before - 0.02 * host(s.update)
    assert np.all(np.abs(host(s.w32) - after) <= 2 * U * (np.abs(before) + np.abs(after)))
    assert torch.equal(s.W, s.w32.to(s.W.dtype))
    s.gradients()                                          # (the state behind segment 0 with the new weights)
    n = B * T
    state, h = s.h0.clone(), torch.empty(B, D, dtype=s.W.dtype, device="cuda")
    z, x = s.z[0].view(B, T, D), s.x[0].view(B, T, D)
    for t in range(T):
        ok(L().ouro_op_recurrence_fwd(stream(), dtype, B, 1, D, p(z[:, t]), T * D, p(x[:, t]), T * D, p(state), None, p(h), D, p(state), None, None))
    ref = recurrence(Num(host(z)), Num(host(x)), Num(host(s.h0)), LENS[0])[2]
    for got in (state, s.state[0]):
        assert np.all(np.abs(host(got) - ref.v) <= ref.e)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
def test_the_step_as_a_graph(dtype):
    """Captured once and replayed with eager steps of another instance between the replays; tokens change between them."""
    s, other = Step(dtype), Step(dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.gradients()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.gradients()
    V, W, h0, tok, tgt = problem(dtype)
    for turn in range(3):
        now = np.roll(tok, turn, 1)
        s.tok.copy_(torch.from_numpy(now.astype(np.int32)))
        for t in (s.h, s.dV, s.dW, s.update, s.dstate):
            t.fill_(float("nan"))
        graph.replay()
        other.tok.copy_(s.tok)
        other.gradients()
        torch.cuda.synchronize()
        ref = oracle(V, W, h0, now, tgt, dtype)
        s.check(ref)
        other.check(ref)
