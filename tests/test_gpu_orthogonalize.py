"""The orthogonalised update against its definition in 64 bits.

Tolerance, in the Frobenius norm of a matrix: a step maps X to p(X), an odd function of the singular values, and a perturbation of
X by at most its largest slope times that (3.9 for values up to 1.2, where they stay).  A step itself adds at most
eps |X|: operands of 22 bits in three products and a polynomial whose coefficients sum to 10.3 (2^-22 x 3 x 10.3 < 2^-17), and sums of K
terms in fp32, whose errors add up like sqrt(K) 2^-24 x 10.3.  So the result is off by at most sum over the steps of
3.9^(steps after it) eps |X_k|, and by half a step of the type it is stored in.

The 22 bits end at an absolute floor: the lower number of a pair is a multiple of fp16's smallest subnormal, 2^-24, in units in which
X is multiplied by 2^12, so an entry of X is off by up to half of 2^-36 whatever its size, and X in the norm by sqrt(rows cols) 2^-37
more in each step.  It counts where eps is far above |U| alone (|X| is then far below 1)."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

COEF = (3.4445, -4.7750, 2.0315)
HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}


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


def oracle(u, scale, eps, steps):
    """The result for one matrix and the bound on its error's norm, without the storing."""
    tall = u.shape[0] > u.shape[1]
    x = u.T if tall else u
    unit = 2.0 ** -17 + np.sqrt(x.shape[1]) * 2.0 ** -24 * 10.3
    x = x / (np.linalg.norm(x) + eps)
    err = 0.0
    for _ in range(steps):
        err = 3.9 * err + 3.9 * (unit * np.linalg.norm(x) + np.sqrt(x.size) * 2.0 ** -37)
        a = x @ x.T
        x = COEF[0] * x + (COEF[1] * a + COEF[2] * a @ a) @ x
    return scale * (x.T if tall else x), abs(scale) * err


def scratch(batch, rows, cols):
    n = L().ouro_op_orthogonalize_scratch(batch, rows, cols)
    return torch.full((n,), float("nan"), device="cuda")


def run(g, o, m=None, mu=0.0, nesterov=0, scale=1.0, eps=1e-7, steps=5, work=None):
    """g, o, m: tensors [batch, rows, cols] with contiguous columns."""
    b, r, c = g.shape
    work = scratch(b, r, c) if work is None else work
    ok(L().ouro_op_orthogonalize(stream(), int(g.dtype == torch.bfloat16), b, r, c, p(g), g.stride(1), g.stride(0), p(m), mu, nesterov, p(o), o.stride(1),
                                 o.stride(0), scale, eps, steps, p(work)))


def check(u, o, scale=1.0, eps=1e-7, steps=5, dtype=0):
    got = host(o)
    for i in range(len(u)):
        ref, tol = oracle(u[i], scale, eps, steps)
        off = np.linalg.norm(got[i] - ref)
        assert off <= tol + HALF[dtype] * np.linalg.norm(ref), (i, off, tol)


def gradient(rng, b, r, c, noise=1.0):
    k = min(4, r, c)
    return rng.standard_normal((b, r, k)) @ rng.standard_normal((b, k, c)) + noise * rng.standard_normal((b, r, c))


def dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.bfloat16() if dtype else t


SIZES = [(1, 1, 1), (1, 1, 70), (2, 5, 3), (1, 64, 64), (1, 64, 256), (3, 65, 130), (2, 130, 65), (1, 410, 210), (2, 200, 700), (1, 16, 3000), (1, 520, 520),
         (9, 96, 128), (1, 300, 1100), (3, 250, 61), (2, 256, 64), (1, 200, 7), (2, 64, 253)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("b,r,c", SIZES)
def test_against_the_definition(b, r, c, dtype):
    rng = np.random.default_rng(b + r + c)
    g = dev(gradient(rng, b, r, c), dtype)
    o = torch.full_like(g, float("nan"))
    run(g, o, scale=0.7)
    check(host(g), o, scale=0.7, dtype=dtype)


@pytest.mark.parametrize("b,r,c", [(1, 64, 5000), (2, 3000, 200), (3, 100, 2000), (1, 1500, 1530), (2, 1500, 1530), (40, 200, 700), (70, 160, 520), (100, 200, 260),
                                   (200, 200, 260), (300, 64, 300), (9, 900, 1000)])
def test_every_width_of_tiles(b, r, c):
    """Contractions dealt to several workgroups; tiles 64, 128 (one and two groups of waves) and 256 wide, in the symmetric products and the others.
    The first, the last and some of the matrices between."""
    rng = np.random.default_rng(b + r + c)
    g = dev(gradient(rng, b, r, c), 0)
    o = torch.full_like(g, float("nan"))
    run(g, o)
    some = sorted({0, b // 3, b // 2, b - 2 if b > 1 else 0, b - 1})
    check(host(g[some]), o[some])
    assert torch.isfinite(o).all()
    again = torch.full_like(g, float("nan"))
    run(g, again)
    assert torch.equal(o, again)


def test_offsets_beyond_32_bits():
    """Rows and matrices far apart: the last ones behind 2^31 elements."""
    ld, b, r, c = 1 << 24, 2, 70, 80
    wide = torch.empty(b * r * ld, device="cuda").view(b, r, ld)
    assert wide.numel() > 2**31
    g, m, o = (wide[:, :, 1000 * i:1000 * i + c] for i in range(3))
    u = gradient(np.random.default_rng(5), b, r, c)
    g.copy_(dev(u, 0))
    m.fill_(0.5)
    run(g, o, m, mu=1.0)
    assert torch.equal(m, g + 0.5)
    check(host(m), o)


@pytest.mark.parametrize("noise", [0.0, 1e-4, 1e-2])
def test_strong_directions_over_noise(noise):
    """Singular values that five steps bring up from nearly nothing, and a matrix of rank 4."""
    g = dev(gradient(np.random.default_rng(1), 1, 192, 320, noise), 0)
    o = torch.empty_like(g)
    run(g, o)
    check(host(g), o)


@pytest.mark.parametrize("steps", [1, 2, 3, 10])
def test_steps(steps):
    g = dev(gradient(np.random.default_rng(2), 2, 100, 70), 0)
    o = torch.empty_like(g)
    run(g, o, steps=steps)
    check(host(g), o, steps=steps)


def test_singular_values_come_near_one():
    """A well-conditioned matrix: the polynomial keeps values that have arrived within 0.68 and 1.21 (its extremes around 1 are 0.69 and
    1.20 in exact arithmetic)."""
    g = torch.randn(1, 128, 512, device="cuda")
    o = torch.empty_like(g)
    run(g, o)
    s = np.linalg.svd(host(o)[0], compute_uv=False)
    assert s.min() > 0.66 and s.max() < 1.23


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("r,c", [(72, 40), (33, 130)])
def test_momentum(r, c, nesterov, dtype):
    """Two updates in a row; the momentum rounds twice a step (product and sum)."""
    rng = np.random.default_rng(r)
    m = dev(np.zeros((3, r, c)), 0)
    m64 = np.zeros((3, r, c))
    for _ in range(2):
        g = dev(gradient(rng, 3, r, c), dtype)
        o = torch.empty_like(g)
        run(g, o, m, 0.95, nesterov)
        m64 = np.float64(np.float32(0.95)) * m64 + host(g)
        assert np.all(np.abs(host(m) - m64) <= 2.0 ** -22 * (np.abs(m64) + np.abs(host(g))))
        mm = host(m)
        check(host(g) + np.float64(np.float32(0.95)) * mm if nesterov else mm, o, dtype=dtype)


@pytest.mark.parametrize("dtype", [0, 1])
def test_layouts(dtype):
    """Three matrices side by side in wider rows, one element off every alignment, NaN between them, written back in place."""
    rng = np.random.default_rng(4)
    g64 = gradient(rng, 3, 50, 30)
    flat = torch.full((1 + 50 * 101,), float("nan"), dtype=torch.bfloat16 if dtype else torch.float32, device="cuda")
    v = flat[1:].as_strided((3, 50, 30), (31, 101, 1), 1)
    v.copy_(torch.from_numpy(g64.astype(np.float32)))
    u = host(v)
    m = torch.zeros(1 + 50 * 101, device="cuda").as_strided((3, 50, 30), (31, 101, 1), 1)
    run(v, v, m, 0.9, 1)
    check(u + np.float64(np.float32(0.9)) * u, v, dtype=dtype)
    assert int(torch.isnan(flat).sum()) == flat.numel() - 3 * 50 * 30


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e18, 1e36])
def test_gradients_of_any_size(size):
    """The norm is formed in 64 bits; eps counts against it."""
    g = dev(gradient(np.random.default_rng(6), 1, 40, 60) * size, 0)
    o = torch.empty_like(g)
    for eps in (1e-7, 0.0):
        run(g, o, eps=eps)
        check(host(g), o, eps=float(np.float32(eps)))


def test_zero_and_bad_matrices_of_a_batch():
    g = dev(gradient(np.random.default_rng(7), 5, 70, 90), 0)
    good = torch.empty_like(g)
    run(g, good)
    bad = g.clone()
    bad[1] = 0
    bad[2, 3, 4], bad[3, 69, 89] = float("nan"), float("inf")
    o = torch.empty_like(g)
    run(bad, o)
    assert torch.equal(o[0], good[0]) and torch.equal(o[4], good[4])
    assert torch.all(o[1] == 0) and torch.all(torch.isnan(o[2])) and torch.all(torch.isnan(o[3]))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("b,r,c", [(2, 64, 200), (1, 400, 300)])
def test_streams_graphs_and_equal_bits(b, r, c, dtype):
    g = dev(gradient(np.random.default_rng(8), b, r, c), dtype)
    m, m0 = torch.zeros(b, r, c, device="cuda"), torch.zeros(b, r, c, device="cuda")
    work = scratch(b, r, c)
    first, second, third = (torch.empty_like(g) for _ in range(3))
    run(g, first, m, 0.9, 1, work=work)
    m.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(g, second, m, 0.9, 1, work=work)
    torch.cuda.synchronize()
    assert torch.equal(first, second)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(g, third, m, 0.9, 1, work=work)
    for _ in range(3):                                           # the momentum goes on from replay to replay
        g.mul_(-0.5)
        m0.copy_(m)
        graph.replay()
        run(g, first, m0, 0.9, 1)
        torch.cuda.synchronize()
        assert torch.equal(first, third) and torch.equal(m0, m)
