"""The precision of the orthogonalised update: its products of split operands against the same steps in fp32, each measured against 64 bits.

Tolerance: both forms add up in fp32.  What they add up differs: fp32 rounds a stored number by at most 2^-24 of itself, two fp16 halves by 2^-22, and a
product takes two of those and leaves out low x low, below 2^-22 of it again: three times 2^-22, 12 times what fp32 loses in a number.  The steps
carry both errors to the result alike, so the result may be off by 12 times what the fp32 form is (and half a step of fp32 for storing it).

The worst case over all matrices, which the other tests of the update allow, is some thousand times that.  This bound notices if a product of a high and
a low half is left out anywhere: on such matrices that costs 100 times the fp32 error and more (the tests on the CPU below)."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

COEF = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
TIMES = 12


def gradient(rng, b, r, c):
    """Four directions over noise of their size."""
    k = min(4, r, c)
    return (rng.standard_normal((b, r, k)) @ rng.standard_normal((b, k, c)) + rng.standard_normal((b, r, c))).astype(np.float32)


def plain(u, ty):
    tall = u.shape[0] > u.shape[1]
    x = (u.T if tall else u).astype(np.float64)
    x = (x / (np.linalg.norm(x) + EPS)).astype(ty)
    for _ in range(STEPS):
        a = x @ x.T
        x = ty(COEF[0]) * x + (ty(COEF[1]) * a + ty(COEF[2]) * (a @ a)) @ x
    return x.T if tall else x


def errors(u, *results):
    """Of the fp32 form and of each of `results`, relative to the norm of the result in 64 bits."""
    ref = plain(u, np.float64)
    return [np.linalg.norm(x - ref) / np.linalg.norm(ref) for x in (plain(u, np.float32), *results)]


# ------------------------------------------------------------ the arithmetic of the kernels, on the CPU
def split(x):
    v = x * np.float32(4096)
    hi = v.astype(np.float16)
    return hi.astype(np.float32), (v - hi.astype(np.float32)).astype(np.float16).astype(np.float32)


def product(l, r, without=""):
    """l r^T"""
    s = l[0] @ r[0].T
    if without != "high x low":
        s = s + l[0] @ r[1].T
    if without != "low x high":
        s = s + l[1] @ r[0].T
    return s * np.float32(2.0 ** -24)


def by_halves(u, pairs, without=("", "")):
    """Steps from split operands; `pairs`: two steps with X once.  without: which product leaves out what."""
    a, b, c = (np.float32(v) for v in COEF)
    tall = u.shape[0] > u.shape[1]
    x = (u.T if tall else u).astype(np.float64)
    x = split((x / (np.linalg.norm(x) + EPS)).astype(np.float32))
    times = lambda name, l, r: product(l, r, without[1] if without[0] == name else "")
    eye = np.eye(len(x[0]), dtype=np.float32)
    poly = lambda name, m: split(c * times(name, m, m) + (b * (m[0] + m[1]) * np.float32(2.0 ** -12) + a * eye))
    i = 0
    while i < STEPS:
        two = pairs and i + 1 < STEPS
        gram = split(times("A", x, x))
        by = first = poly("C", gram)
        if two:
            gram = split(times("C A C", split(times("C A", first, gram)), first))
            by = split(times("C' C", poly("C'", gram), first))
        x = split(times("X", by, tuple(v.T for v in x)))
        i += 1 + two
    x = (x[0] + x[1]) * np.float32(2.0 ** -12)
    return x.T if tall else x


PRODUCTS = {False: ("A", "C", "X"), True: ("A", "C", "C A", "C A C", "C'", "C' C", "X")}
ON_THE_CPU = [(64, 256, True), (200, 30, True), (64, 1000, True), (200, 700, True), (200, 260, False), (520, 530, False)]


@pytest.mark.parametrize("r,c,pairs", ON_THE_CPU)
def test_the_bound_holds_for_split_operands(r, c, pairs):
    u = gradient(np.random.default_rng(r + c), 1, r, c)[0]
    fp32, halves = errors(u, by_halves(u, pairs))
    assert halves <= TIMES * fp32 / 4                             # (in fact within 1.5; the bound keeps room for the worst case of every rounding)


@pytest.mark.parametrize("what", ["high x low", "low x high"])
@pytest.mark.parametrize("r,c,pairs", ON_THE_CPU)
def test_the_bound_notices_a_missing_product(r, c, pairs, what):
    u = gradient(np.random.default_rng(r + c), 1, r, c)[0]
    for name in PRODUCTS[pairs]:
        fp32, worse = errors(u, by_halves(u, pairs, (name, what)))
        assert worse > 4 * TIMES * fp32, (name, what, fp32, worse)


# ---------------------------------------------------------------------------------- the kernels
def p(t):
    return C.c_void_p(t.data_ptr())


# One workgroup a matrix; the small products of 64 rows in one launch, without and with a contraction dealt to several workgroups, many matrices; tiles 64
# wide in pairs (two and many matrices) and in single steps, tall ones; 128 wide in two groups of waves and in one; 64 wide for the symmetric products and 256 for
# the others; 256 wide for all, in single steps and in pairs.
SIZES = [(1, 64, 256), (2, 50, 200), (3, 200, 30), (1, 64, 300), (1, 64, 5000), (300, 64, 300), (2, 200, 700), (2, 700, 200), (40, 200, 700), (1, 520, 530),
         (2, 130, 65), (2, 1500, 1530), (9, 900, 1000), (100, 200, 260), (200, 200, 260), (200, 200, 520)]


@pytest.mark.gpu
@pytest.mark.parametrize("b,r,c", SIZES)
def test_precision_of_every_kernel(b, r, c):
    from paper_1909_06695_amd import binding as P
    L = P.lib()
    u = gradient(np.random.default_rng(b + r + c), b, r, c)
    g = torch.from_numpy(u).cuda()
    o = torch.full_like(g, float("nan"))
    work = torch.full((L.ouro_op_orthogonalize_scratch(b, r, c),), float("nan"), device="cuda")
    P.check(L.ouro_op_orthogonalize(C.c_void_p(torch.cuda.current_stream().cuda_stream), 0, b, r, c, p(g), c, r * c, None, 0.0, 0, p(o), c, r * c, 1.0, EPS, STEPS, p(work)))
    got = o.cpu().numpy()
    assert np.isfinite(got).all()
    for i in sorted({0, b - 1}):
        fp32, off = errors(u[i], got[i].astype(np.float64))
        print((b, r, c), i, "fp32 %.2e, here %.2e" % (fp32, off))
        assert off <= TIMES * fp32 + 2.0 ** -24, (i, fp32, off)
