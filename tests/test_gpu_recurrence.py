"""The gated linear recurrence against a step-by-step loop in 64 bits, forward and backward.

Tolerance, by running error analysis: with a = sum of |terms| of a state (the same recursion on magnitudes) a step multiplies the
error by f and adds at most eps a: the gate's relative error, (|z| + 6) 2^-24 from the rounded exponent, the exponential, one addition,
the reciprocal and one product, and two roundings of the step; joining the parts of the scan adds a few roundings of what
passes through it, 32 in all.  What is stored as T rounds once more, by half a step of T."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {0: 0.0, 1: 2.0 ** -8}
STRIDE = 64


def L():
    import paper_1909_06695_amd as P
    return P.lib()


def stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def ok(rc):
    assert rc == 0, L().ouro_last_error()


def dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.bfloat16() if dtype else t


def host(t):
    return t.double().cpu().numpy()


def rows(a, dtype, gap, off):
    """[B, T, D] as rows `gap` elements apart with NaN between them, `off` elements behind an aligned address."""
    B, T, D = a.shape
    flat = torch.full((off + B * T * (D + gap),), float("nan"), dtype=torch.bfloat16 if dtype else torch.float32, device="cuda")
    v = flat[off:].view(B, T, D + gap)[:, :, :D]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)))
    return v


def make(B, T, D, dtype, seed, lens=None, gap=0, off=0, gate=1.0):
    rng = np.random.default_rng(seed)
    s = {"B": B, "T": T, "D": D, "dtype": dtype}
    for name, shift in (("z", gate), ("x", 0.0), ("dh", 0.0)):
        s[name] = rows(rng.standard_normal((B, T, D)) * (2.0 if name == "z" else 1.0) + shift, dtype, gap, off)
    s["h0"], s["dhT"] = dev(rng.standard_normal((B, D)), 0), dev(rng.standard_normal((B, D)), 0)
    s["lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["out"] = {k: rows(np.full((B, T, D), 5.0), dtype, gap, off) for k in ("h", "dz", "dx")}
    s["hT"], s["dh0"] = torch.full((B, D), 5.0, device="cuda"), torch.full((B, D), 5.0, device="cuda")
    s["states"] = torch.full((B, -(-T // STRIDE), D), 5.0, device="cuda")
    n = L().ouro_op_recurrence_scratch(B, T, D)
    s["scratch"] = torch.full((n,), float("nan"), device="cuda") if n else None
    return s


def forward(s, h0=True):
    ld = s["z"].stride(1)
    ok(L().ouro_op_recurrence_fwd(stream(), s["dtype"], s["B"], s["T"], s["D"], p(s["z"]), ld, p(s["x"]), ld, p(s["h0"]) if h0 else None, p(s["lens"]),
                                  p(s["out"]["h"]), ld, p(s["hT"]), p(s["states"]), p(s["scratch"])))


def backward(s, dhT=True):
    ld = s["z"].stride(1)
    ok(L().ouro_op_recurrence_bwd(stream(), s["dtype"], s["B"], s["T"], s["D"], p(s["z"]), ld, p(s["x"]), ld, p(s["states"]), p(s["lens"]),
                                  p(s["dh"]), ld, p(s["dhT"]) if dhT else None, p(s["out"]["dz"]), ld, p(s["out"]["dx"]), ld, p(s["dh0"]), p(s["scratch"])))


def oracle(s, h0=True, dhT=True):
    """Values and error bounds of every output."""
    B, T, D = s["B"], s["T"], s["D"]
    z, x, dh = host(s["z"]), host(s["x"]), host(s["dh"])
    lens = np.full(B, T) if s["lens"] is None else np.clip(s["lens"].cpu().numpy(), 0, T)
    live = (np.arange(T)[None] < lens[:, None])[:, :, None]
    z, x, dh = np.where(live, z, 0.0), np.where(live, x, 0.0), np.where(live, dh, 0.0)
    with np.errstate(over="ignore"):
        f, k = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
    f, k = np.where(live, f, 1.0), np.where(live, k, 0.0)
    finite = np.abs(z[np.isfinite(z)])
    eps = ((finite.max() if finite.size else 0.0) + 8) * U
    out, tol = {}, {}
    h = host(s["h0"]) if h0 else np.zeros((B, D))
    a, e = np.abs(h), np.zeros((B, D))
    H, A, E = np.empty((B, T + 1, D)), np.empty((B, T + 1, D)), np.empty((B, T + 1, D))
    for t in range(T + 1):
        H[:, t], A[:, t], E[:, t] = h, a, e + 32 * U * a
        if t < T:
            h = f[:, t] * h + k[:, t] * x[:, t]
            a = f[:, t] * a + k[:, t] * np.abs(x[:, t])
            e = f[:, t] * e + np.where(live[:, t], eps * a, 0.0)
    out["h"], tol["h"] = np.where(live, H[:, 1:], 0.0), np.where(live, E[:, 1:], 0.0)
    out["hT"], tol["hT"] = H[:, T], E[:, T]
    out["states"], tol["states"] = H[:, 0:T:STRIDE], E[:, 0:T:STRIDE]
    P = host(s["dhT"]) if dhT else np.zeros((B, D))
    a, e = np.abs(P), np.zeros((B, D))
    for n in ("dz", "dx"):
        out[n], tol[n] = np.zeros((B, T, D)), np.zeros((B, T, D))
    for t in range(T - 1, -1, -1):
        G, ga = P + dh[:, t], a + np.abs(dh[:, t])
        ge = np.where(live[:, t], e + (eps + 32 * U) * ga, e)
        v = H[:, t] - x[:, t]
        ve = E[:, t] + U * (np.abs(H[:, t]) + np.abs(x[:, t]))
        out["dx"][:, t], tol["dx"][:, t] = k[:, t] * G, k[:, t] * (ge + (eps + U) * np.abs(G))
        out["dz"][:, t] = G * v * f[:, t] * k[:, t]
        tol["dz"][:, t] = f[:, t] * k[:, t] * (ge * np.abs(v) + np.abs(G) * ve + (2 * eps + 4 * U) * np.abs(G * v))
        P, a, e = f[:, t] * G, f[:, t] * ga, f[:, t] * np.where(live[:, t], e + eps * ga, e)
    out["dh0"], tol["dh0"] = P, e + 32 * U * a
    for n in ("h", "dz", "dx"):
        tol[n] = tol[n] + HALF[s["dtype"]] * (np.abs(out[n]) + tol[n])
    return out, tol


def compare(s, names, out, tol):
    for n in names:
        got = host(s["out"][n] if n in s["out"] else s[n])
        off = np.abs(got - out[n]) - tol[n]
        assert np.all(off <= 0), (n, np.unravel_index(np.nanargmax(off), off.shape), np.nanmax(off))


SHAPES = [(1, 1, 1, 0, 0), (3, 1, 130, 0, 0), (70, 1, 64, 0, 0), (2, 2, 7, 3, 1), (2, 31, 64, 0, 0), (1, 32, 64, 0, 0), (1, 33, 65, 1, 1), (3, 64, 48, 8, 0),
          (2, 65, 129, 0, 3), (1, 513, 24, 0, 0), (2, 1030, 72, 0, 0), (1, 5000, 40, 2, 0), (600, 70, 8, 0, 0)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,D,gap,off", SHAPES)
def test_forward_and_backward(B, T, D, gap, off, dtype):
    """One step to several segments; rows apart and off every alignment; widths off the 16-byte pieces."""
    s = make(B, T, D, dtype, B + T + D, gap=gap, off=off)
    forward(s)
    out, tol = oracle(s)
    compare(s, ("h", "hT", "states"), out, tol)
    backward(s)
    compare(s, ("dz", "dx", "dh0"), out, tol)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,lens", [(1, [0, 1, 5, -3, 1]), (70, [0, 1, 70, 64, 69]), (1500, [0, 1500, 1, 700, 2000])])
def test_lengths(T, lens, dtype):
    """Streams of no step, one, all and more than all; behind a stream's end z, x and dh are NaN and the outputs zero."""
    s = make(5, T, 40, dtype, T, lens=lens)
    for b, n in enumerate(lens):
        for k in ("z", "x", "dh"):
            s[k][b, max(n, 0):] = float("nan")
    forward(s)
    out, tol = oracle(s)
    compare(s, ("h", "hT", "states"), out, tol)
    assert torch.equal(s["hT"][0], s["h0"][0])                   # no step: the state stays, bit for bit
    backward(s)
    compare(s, ("dz", "dx", "dh0"), out, tol)
    assert torch.equal(s["dh0"][0], s["dhT"][0])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,D,ragged", [(520, 600, 20, False), (130, 1100, 130, True), (180, 1100, 130, True), (1030, 300, 3, True)])
def test_streams_that_fill_the_chip(B, T, D, ragged, dtype):
    """Streams and strips of channels (64 in bf16, 32 in fp32) enough, 512 or more, for a workgroup to go through the segments of a stream one after the
    other, without a workspace; the second in fp32 only."""
    assert (L().ouro_op_recurrence_scratch(B, T, D) == 0) == (B * -(-D // 64) >= 512)
    lens = [(37 * b) % (T + 2) for b in range(B)] if ragged else None
    s = make(B, T, D, dtype, B, lens=lens)
    if ragged:
        late = torch.arange(T, device="cuda")[None] >= s["lens"][:, None]
        for k in ("z", "x", "dh"):
            s[k][late] = float("nan")
    forward(s)
    out, tol = oracle(s)
    compare(s, ("h", "hT", "states"), out, tol)
    backward(s)
    compare(s, ("dz", "dx", "dh0"), out, tol)


def test_offsets_beyond_32_bits():
    """Rows 2^25 elements apart, operands and results side by side in them: 70 rows end behind 2^31 elements."""
    B, T, D, ld = 1, 70, 8, 1 << 25
    s = make(B, T, D, 0, 21)
    wide = torch.empty(T * ld, device="cuda")
    assert wide.numel() > 2**31
    views = {k: wide.view(1, T, ld)[:, :, 100 * i:100 * i + D] for i, k in enumerate(("z", "x", "dh", "h", "dz", "dx"))}
    for k in ("z", "x", "dh"):
        views[k].copy_(s[k])
        s[k] = views[k]
    s["out"] = {k: views[k] for k in ("h", "dz", "dx")}
    forward(s)
    out, tol = oracle(s)
    compare(s, ("h", "hT", "states"), out, tol)
    backward(s)
    compare(s, ("dz", "dx", "dh0"), out, tol)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [3, 300])
def test_states_that_are_absent(T, dtype):
    """h0 and dhT NULL are zero; hT, states and dh0 need not be asked for."""
    s = make(2, T, 24, dtype, T)
    ld = s["z"].stride(1)
    out, tol = oracle(s, h0=False, dhT=False)
    forward(s, h0=False)
    compare(s, ("h", "hT", "states"), out, tol)
    backward(s, dhT=False)
    compare(s, ("dz", "dx", "dh0"), out, tol)
    want = {k: v.clone() for k, v in s["out"].items()}
    for v in s["out"].values():
        v.fill_(5.0)
    args = (stream(), dtype, 2, T, 24, p(s["z"]), ld, p(s["x"]), ld)
    ok(L().ouro_op_recurrence_fwd(*args, None, None, p(s["out"]["h"]), ld, None, None, p(s["scratch"])))
    ok(L().ouro_op_recurrence_bwd(*args, p(s["states"]), None, p(s["dh"]), ld, None, p(s["out"]["dz"]), ld, p(s["out"]["dx"]), ld, None, p(s["scratch"])))
    assert all(torch.equal(want[k], s["out"][k]) for k in want)


@pytest.mark.parametrize("dtype", [0, 1])
def test_infinite_gates(dtype):
    """z = +infinity keeps the state, -infinity replaces it, and their gradients are finite; the type's lowest value does what
    -infinity does.  A replaced state is x bit for bit (0 h + x); a kept one is the same number only up to the bound, because
    threads form it as (A h' + H) with the steps before grouped differently, each grouping rounding by itself."""
    s = make(1, 200, 16, dtype, 3)
    low = torch.finfo(s["z"].dtype).min
    s["z"][0, 50:120] = float("inf")
    s["z"][0, 130], s["z"][0, 140], s["z"][0, 150] = float("-inf"), low, -low
    forward(s)
    out, tol = oracle(s)
    compare(s, ("h", "hT", "states"), out, tol)
    h = s["out"]["h"][0]
    assert np.array_equal(out["h"][0, 50:120], np.broadcast_to(out["h"][0, 49], (70, 16)))
    assert torch.equal(h[130], s["x"][0, 130]) and torch.equal(h[140], s["x"][0, 140]) and torch.equal(h[150], h[149])
    backward(s)
    compare(s, ("dz", "dx", "dh0"), out, tol)


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_nan_reaches_later_steps_of_its_channel_only(dtype):
    s = make(2, 900, 24, dtype, 9)
    forward(s)
    clean = s["out"]["h"].clone()
    s["x"][1, 400, 5] = float("nan")
    forward(s)
    got = s["out"]["h"]
    assert torch.all(torch.isnan(got[1, 400:, 5]))
    got[1, 400:, 5] = clean[1, 400:, 5]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", [0, 1])
def test_token_by_token_equals_the_whole(dtype):
    """Single steps with the state carried in place give what one call over all steps gives, within both bounds."""
    s = make(3, 90, 50, dtype, 11)
    forward(s)
    out, tol = oracle(s)
    state, h = s["h0"].clone(), torch.empty_like(s["out"]["h"])
    for t in range(90):
        z, x, o = (v[:, t].contiguous() for v in (s["z"], s["x"], h))
        ok(L().ouro_op_recurrence_fwd(stream(), dtype, 3, 1, 50, p(z), 50, p(x), 50, p(state), None, p(o), 50, p(state), None, None))
        h[:, t] = o
    assert np.all(np.abs(host(h) - out["h"]) <= tol["h"])
    assert np.all(np.abs(host(state) - out["hT"]) <= tol["hT"])


@pytest.mark.parametrize("dtype", [0, 1])
def test_state_in_place_over_segments(dtype):
    """h0 and hT, and dhT and dh0, as one buffer in calls that are cut into segments."""
    s = make(1, 9000, 24, dtype, 13)
    assert s["scratch"] is not None
    forward(s)
    backward(s)
    h, hT, dh0 = s["out"]["h"].clone(), s["hT"].clone(), s["dh0"].clone()
    s["hT"] = s["h0"]
    s["dh0"] = s["dhT"]
    forward(s)
    backward(s)
    assert torch.equal(s["out"]["h"], h) and torch.equal(s["h0"], hT) and torch.equal(s["dhT"], dh0)


def test_gradients_against_differences():
    """Central differences of a weighted sum of h and hT, in fp32 arithmetic with steps of 2^-5: the third-derivative term is below
    step^2 |weights| T and the rounding below 64 2^-24 / step |weights| T."""
    s = make(1, 12, 4, 0, 17, gate=0.0)
    wT = host(s["dhT"])
    forward(s)
    backward(s)

    def value():
        forward(s)
        return float((host(s["out"]["h"]) * host(s["dh"])).sum() + (host(s["hT"]) * wT).sum())

    step, scale = 2.0 ** -5, 12 * (np.abs(host(s["dh"])).sum() + np.abs(wT).sum()) * (1 + np.abs(host(s["x"])).max())
    tol = (step ** 2 + 64 * U / step) * scale / 48
    for name, grad in (("z", s["out"]["dz"]), ("x", s["out"]["dx"]), ("h0", s["dh0"])):
        want = host(grad).copy()
        flat = s[name].reshape(-1) if name == "h0" else s[name].view(-1)
        for i in range(flat.numel()):
            old = flat[i].item()
            flat[i] = old + step
            up = value()
            flat[i] = old - step
            down = value()
            flat[i] = old
            assert abs((up - down) / (2 * step) - want.reshape(-1)[i]) <= tol, (name, i)


@pytest.mark.parametrize("dtype", [0, 1])
def test_streams_and_graphs(dtype):
    """On another stream, and captured with the segments' workspace: every replay equals the eager call bit for bit."""
    s = make(2, 3000, 40, dtype, 19, lens=[3000, 1234])
    assert s["scratch"] is not None
    forward(s)
    backward(s)
    eager = [t.clone() for t in (*s["out"].values(), s["hT"], s["dh0"], s["states"])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward(s)
        backward(s)
    torch.cuda.synchronize()
    now = lambda: (*s["out"].values(), s["hT"], s["dh0"], s["states"])
    assert all(torch.equal(a, b) for a, b in zip(eager, now()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward(s)
        backward(s)
    for i in range(3):
        s["x"].mul_(-0.5)
        for t in now():
            t.fill_(float("nan"))
        graph.replay()
        got = [t.clone() for t in now()]
        forward(s)
        backward(s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, now()))


def test_the_longest_stream():
    """2^30 steps of one channel in bf16, whose 2^23 tiles backward are two launches: windows at the start (the launches meet at step
    128), in the middle and at the end.  A window's oracle begins 400 steps before it and ends 400 behind it from zeros; what they leave out passes through 400 gates, a factor below 2^-200."""
    T, wide, far = 1 << 30, 600, 400
    gen = torch.Generator(device="cuda").manual_seed(23)
    s = {"B": 1, "T": T, "D": 1, "dtype": 1, "lens": None}
    for k in ("z", "x", "dh"):
        s[k] = torch.empty(1, T, 1, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    s["out"] = {k: torch.full_like(s["z"], float("nan")) for k in ("h", "dz", "dx")}
    s["h0"], s["dhT"] = dev([[2.0]], 0), dev([[-3.0]], 0)
    s["hT"], s["dh0"] = dev([[5.0]], 0), dev([[5.0]], 0)
    s["states"] = torch.full((1, T // STRIDE, 1), float("nan"), device="cuda")
    s["scratch"] = torch.full((L().ouro_op_recurrence_scratch(1, T, 1),), float("nan"), device="cuda")
    forward(s)
    backward(s)
    assert not any(torch.isnan(t).any() for t in (*s["out"].values(), s["states"]))
    for at in (0, T // 2 + 1, T - wide):
        lo, hi = max(0, at - far), min(T, at + wide + far)
        part = {"B": 1, "T": hi - lo, "D": 1, "dtype": 1, "lens": None, "h0": s["h0"] if lo == 0 else torch.zeros(1, 1, device="cuda"),
                "dhT": s["dhT"] if hi == T else torch.zeros(1, 1, device="cuda")}
        for k in ("z", "x", "dh"):
            part[k] = s[k][:, lo:hi]
        f = 1 / (1 + np.exp(-host(part["z"])[0, :, 0]))
        assert (lo == 0 or f[:far].prod() < 2.0**-200) and (hi == T or f[-far:].prod() < 2.0**-200)
        out, tol = oracle(part)
        for k in ("h", "dz", "dx"):
            got = host(s["out"][k][:, at:at + wide])
            assert np.all(np.abs(got - out[k][:, at - lo:at - lo + wide]) <= tol[k][:, at - lo:at - lo + wide]), (k, at)
        if hi == T:
            assert abs(s["hT"].item() - out["hT"].item()) <= tol["hT"].item()
        if lo == 0:
            assert abs(s["dh0"].item() - out["dh0"].item()) <= tol["dh0"].item()


@pytest.mark.parametrize("dtype", [0, 1])
def test_more_streams_than_a_launch(dtype):
    """2^26 + 5 streams of one token and one channel are two launches; some have no step.  h, dx and dz against the formulas in 64 bits."""
    B = (1 << 26) + 5
    gen = torch.Generator(device="cuda").manual_seed(29)
    ty = torch.bfloat16 if dtype else torch.float32
    z, x, dh = (torch.empty(B, dtype=ty, device="cuda").normal_(generator=gen) for _ in range(3))
    h0, dhT = (torch.empty(B, device="cuda").normal_(generator=gen) for _ in range(2))
    lens = torch.randint(0, 3, (B,), dtype=torch.int32, generator=gen, device="cuda")
    h, dz, dx = (torch.full_like(z, float("nan")) for _ in range(3))
    hT, dh0, states = (torch.full_like(h0, float("nan")) for _ in range(3))
    ok(L().ouro_op_recurrence_fwd(stream(), dtype, B, 1, 1, p(z), 1, p(x), 1, p(h0), p(lens), p(h), 1, p(hT), p(states), None))
    ok(L().ouro_op_recurrence_bwd(stream(), dtype, B, 1, 1, p(z), 1, p(x), 1, p(states), p(lens), p(dh), 1, p(dhT), p(dz), 1, p(dx), 1, p(dh0), None))
    assert torch.equal(states, h0)
    for lo, hi in ((0, 1 << 20), ((1 << 26) - (1 << 20), B)):
        at = slice(lo, hi)
        live = host(lens[at]) > 0
        part = {"B": hi - lo, "T": 1, "D": 1, "dtype": dtype, "lens": lens[at], "h0": h0[at, None], "dhT": dhT[at, None]}
        part.update(z=z[at, None, None], x=x[at, None, None], dh=dh[at, None, None])
        out, tol = oracle(part)
        for got, k in ((h, "h"), (hT, "hT"), (dz, "dz"), (dx, "dx"), (dh0, "dh0")):
            assert np.all(np.abs(host(got[at]) - out[k].reshape(-1)) <= tol[k].reshape(-1)), k
        assert not host(h[at])[~live].any()
    assert not any(torch.isnan(t).any() for t in (h, dz, dx, hT, dh0))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,D", [(1, 200, 16), (2, 1500, 40), (520, 600, 8)])
def test_a_kept_state_on_the_device(B, T, D, dtype):
    """Steps with z = +infinity in one tile, over several chained ones and over those that one workgroup goes through: their dz and dx are exactly 0, and h is what it
    was before them.  Threads and tiles form it from the steps before grouped differently, 32 roundings of at most the largest |h0| and |x| among those for
    either of the two that are compared, and as T each is off by half a step."""
    s = make(B, T, D, dtype, T + D)
    lo, hi = T // 4, T // 4 * 3
    s["z"][:, lo:hi] = float("inf")
    forward(s)
    backward(s)
    h = host(s["out"]["h"])
    most = np.maximum(np.abs(host(s["h0"])), np.abs(host(s["x"])[:, :lo]).max(1))
    tol = 2 * 32 * U * most + HALF[dtype] * (2 * np.abs(h[:, lo - 1]) + 64 * U * most) * (1 + 2 * HALF[dtype])
    assert np.all(np.abs(h[:, lo:hi] - h[:, lo - 1:lo]) <= tol[:, None])
    for k in ("dz", "dx"):
        assert not s["out"][k][:, lo:hi].any(), k
        assert s["out"][k][:, :lo].any() and s["out"][k][:, hi:].any(), k


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,D", [(2, 900, 24), (520, 600, 8)])
def test_an_infinity_stays_in_its_channel(B, T, D, dtype):
    """In x, h0, dh or dhT: not finite behind it (its gradients: before it), everything else as without it, bit for bit."""
    s = make(B, T, D, dtype, T)
    forward(s)
    backward(s)
    clean = {k: v.clone() for k, v in (*s["out"].items(), ("hT", s["hT"]), ("dh0", s["dh0"]))}
    at = T // 2

    def same_but(name, got, bad):
        assert not torch.isfinite(got[bad]).any(), name
        got = got.clone()
        got[bad] = clean[name][bad]
        assert torch.equal(got, clean[name]), name

    for value in (float("inf"), float("-inf")):
        kept = s["x"][1, at, 5].clone(), s["h0"][0, 3].clone()
        s["x"][1, at, 5] = s["h0"][0, 3] = value
        forward(s)
        bad = torch.zeros(B, T, D, dtype=torch.bool, device="cuda")
        bad[1, at:, 5] = bad[0, :, 3] = True
        same_but("h", s["out"]["h"], bad)
        same_but("hT", s["hT"], bad[:, -1])
        s["x"][1, at, 5], s["h0"][0, 3] = kept
        forward(s)
        kept = s["dh"][1, at, 5].clone(), s["dhT"][0, 3].clone()
        s["dh"][1, at, 5] = s["dhT"][0, 3] = value
        backward(s)
        bad = torch.zeros(B, T, D, dtype=torch.bool, device="cuda")
        bad[1, :at + 1, 5] = bad[0, :, 3] = True
        for k in ("dz", "dx"):
            same_but(k, s["out"][k], bad)
        same_but("dh0", s["dh0"], bad[:, 0])
        s["dh"][1, at, 5], s["dhT"][0, 3] = kept
