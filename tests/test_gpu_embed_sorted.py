"""The embedding gradient with sorted sums against 64 bits.

Tolerance: a sum of k fp32 terms in any order is off by at most (k - 1) 2^-24 of the sum of their magnitudes; the scale and the
addition onto the matrix round once each.  bf16 gradients convert exactly."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def L():
    import paper_1909_06695_amd as P
    return P.lib()


def stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def ok(rc):
    assert rc == 0, L().ouro_last_error()


def case(rng, N, vocab, d, dtype, hot=0.0, outside=0.0):
    tok = rng.integers(0, vocab, N)
    tok[rng.random(N) < hot] = vocab // 2
    bad = rng.random(N) < outside
    tok[bad] = rng.choice([-1, vocab, vocab + 5, -2**31, 2**31 - 1], bad.sum())
    dh = torch.from_numpy(rng.standard_normal((N, d)).astype(np.float32)).cuda()
    return tok.astype(np.int32), dh.bfloat16() if dtype else dh


def check(tok, dh, got, base, vocab, scale, old):
    x = scale * dh.double().cpu().numpy()
    inside = (tok >= 0) & (tok < vocab)
    ref, mag, k = np.zeros((vocab, x.shape[1])), np.zeros((vocab, x.shape[1])), np.zeros(vocab)
    np.add.at(ref, tok[inside], x[inside])
    np.add.at(mag, tok[inside], np.abs(x[inside]))
    np.add.at(k, tok[inside], 1)
    tol = 2.0 ** -24 * ((k[:, None] + 1) * mag + (np.abs(old) + mag if base else 0))
    assert np.all(np.abs(got - (ref + old if base else ref)) <= tol)


SIZES = [(1, 1, 1), (1, 5, 3), (128, 256, 64), (130, 7, 33), (700, 1, 70), (257, 3000, 410), (4800, 1024, 130), (600, 70000, 24),
         (9000, 300, 36), (5000, 17, 8)]


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,vocab,d", SIZES)
@pytest.mark.parametrize("hot,outside", [(0.0, 0.0), (0.7, 0.1)])
def test_sums(N, vocab, d, dtype, accumulate, hot, outside):
    """Lists of a workgroup from none to all ids (more than it holds at once), tokens spread and nearly all the same."""
    rng = np.random.default_rng(N + vocab + d)
    tok, dh = case(rng, N, vocab, d, dtype, hot, outside)
    old = rng.standard_normal((vocab, d)).astype(np.float32)
    out = torch.from_numpy(old.copy()).cuda() if accumulate else torch.full((vocab, d), float("nan"), device="cuda")
    ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, p(torch.from_numpy(tok).cuda()), p(dh), d, p(out), d, N, d, vocab, 0.5, accumulate))
    check(tok, dh, out.double().cpu().numpy(), accumulate, vocab, 0.5, old.astype(np.float64))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,vocab,d", [(300, 50, 40), (300, 50, 43)])
def test_rows_apart_and_unaligned(N, vocab, d, dtype):
    """Rows with NaN behind them, gradient and matrix one element off every alignment; what lies between rows stays."""
    rng = np.random.default_rng(d)
    tok, dh = case(rng, N, vocab, d, dtype)
    wide = torch.full((N * (d + 5) + 1,), float("nan"), dtype=dh.dtype, device="cuda")
    rows = wide[1:].view(N, d + 5)
    rows[:, :d] = dh
    out = torch.full((vocab * (d + 3) + 1,), 7.0, device="cuda")
    view = out[1:].view(vocab, d + 3)
    ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, p(torch.from_numpy(tok).cuda()), p(rows), d + 5, p(view), d + 3, N, d, vocab, 1.0, 0))
    check(tok, dh, view[:, :d].double().cpu().numpy(), 0, vocab, 1.0, 0.0)
    assert torch.all(view[:, d:] == 7.0) and out[0] == 7.0


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_tokens(dtype):
    out = torch.full((40, 24), 3.0, device="cuda")
    ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, None, None, 0, p(out), 24, 0, 24, 40, 1.0, 1))
    assert torch.all(out == 3.0)
    ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, None, None, 0, p(out), 24, 0, 24, 40, 1.0, 0))
    assert torch.all(out == 0.0)


def test_only_rows_that_occur_are_touched():
    """Infinities and NaN reach the rows of their tokens only; with accumulate other rows keep their bits."""
    tok = np.array([3, 9, 3, 11], np.int32)
    dh = torch.ones(4, 72, device="cuda")
    dh[1], dh[3] = float("inf"), float("nan")
    old = torch.randn(64, 72, device="cuda")
    out = old.clone()
    ok(L().ouro_op_embed_bwd_sorted(stream(), 0, p(torch.from_numpy(tok).cuda()), p(dh), 72, p(out), 72, 4, 72, 64, 2.0, 1))
    assert torch.equal(out[3], old[3] + 4.0) and torch.all(torch.isinf(out[9])) and torch.all(torch.isnan(out[11]))
    rest = [v for v in range(64) if v not in (3, 9, 11)]
    assert torch.equal(out[rest], old[rest])


@pytest.mark.parametrize("dtype", [0, 1])
def test_equal_calls_give_equal_bits(dtype):
    """Also on another stream beside other work, and as a captured graph that is replayed on new values."""
    rng = np.random.default_rng(5)
    N, vocab, d = 6000, 1000, 200
    tok, dh = case(rng, N, vocab, d, dtype, hot=0.4)
    tok = torch.from_numpy(tok).cuda()
    outs = [torch.empty(vocab, d, device="cuda") for _ in range(3)]
    call = lambda o: ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, p(tok), p(dh), d, p(o), d, N, d, vocab, 1.0, 0))
    call(outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[2])
    for _ in range(3):
        perm = torch.randperm(N, device="cuda")
        tok.copy_(tok[perm])
        outs[2].fill_(float("nan"))
        graph.replay()
        call(outs[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^31 elements, a row stride that makes it: the last rows."""
    vocab, d, ldv = 70000, 8, 1 << 15
    out = torch.zeros(vocab * ldv, device="cuda").view(vocab, ldv)
    tok = torch.tensor([vocab - 1, 0, vocab - 1, vocab - 2], dtype=torch.int32, device="cuda")
    dh = torch.arange(32, dtype=torch.float32, device="cuda").view(4, 8)
    ok(L().ouro_op_embed_bwd_sorted(stream(), 0, p(tok), p(dh), 8, p(out), ldv, 4, d, vocab, 1.0, 1))
    assert torch.equal(out[vocab - 1, :8], dh[0] + dh[2]) and torch.equal(out[vocab - 2, :8], dh[3]) and torch.equal(out[0, :8], dh[1])
    assert out.abs().sum() == dh.abs().sum()


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,vocab,d,shares", [(20000, 1000, 130, (0.9, 0.05)), (20001, 40, 3, (0.5, 0.45)), (4096, 9, 64, (1.0, 0.0)), (16385, 9, 64, (1.0, 0.0)), (40000, 100, 7, (0.2, 0.6)), (30000, 50000, 410, (0.3, 0.3)),
                                              (12345, 2, 33, (0.5, 0.5))])
def test_tokens_that_no_list_holds(N, vocab, d, shares, dtype, accumulate):
    """One token and two of thousands of ids, on rows off every alignment; equal calls give equal bits."""
    rng = np.random.default_rng(N + d)
    tok, dh = case(rng, N, vocab, d, dtype, outside=0.02)
    u = rng.random(N)
    tok[u < shares[0]] = vocab - 1
    tok[(u >= shares[0]) & (u < sum(shares))] = vocab // 2
    wide = torch.zeros(N, d + 5, dtype=dh.dtype, device="cuda")[:, 2:2 + d]
    wide.copy_(dh)
    old = rng.standard_normal((vocab, d)).astype(np.float32)
    got = []
    for _ in range(2):
        out = torch.from_numpy(old).cuda()
        ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, p(torch.from_numpy(tok).cuda()), p(wide), d + 5, p(out), d, N, d, vocab, 1.5, accumulate))
        got.append(out)
    check(tok, dh, got[0].double().cpu().numpy(), accumulate, vocab, 1.5, old)
    assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("accumulate", [0, 1])
def test_the_largest_vocabulary(accumulate):
    """2^31 - 1 rows of one column: the first, the last and one of a later workgroup's; everything else is cleared, or left as it was."""
    vocab = 2**31 - 1
    out = torch.ones(vocab, device="cuda")
    tok = torch.tensor([vocab - 1, 0, vocab - 1, 1 << 30, -1], dtype=torch.int32, device="cuda")
    dh = torch.tensor([[2.0], [3.0], [4.0], [5.0], [7.0]], device="cuda")
    ok(L().ouro_op_embed_bwd_sorted(stream(), 0, p(tok), p(dh), 1, p(out), 1, 5, 1, vocab, 0.5, accumulate))
    ref = {0: 1.5, 1 << 30: 2.5, vocab - 1: 3.0}
    for at, value in ref.items():
        assert out[at].item() == value + accumulate
        out[at] = accumulate
    step = 1 << 28
    assert all((out[i:i + step] == accumulate).all() for i in range(0, vocab, step))


def last_of_positions(N, vocab, d, dtype, accumulate, per_class, classes, more=0):
    """Ids of which the last of N is the last of the vocabulary, `per_class` on average those of each of `classes` residues, the others outside the
    vocabulary; `more` ids behind them.

    An entry has N positions at most, and ids behind them are summed after those before: a row that occurs in w such parts gets w sums, each by
    one fma, and each rounds by at most 2^-24 of what the element is then, at most |old| + the sum of magnitudes (|old| is 0 where the matrix is
    written).  The other roundings are those of any sum of k terms, as above.  No list is full before its positions end: it holds 768 entries of each
    of 8 waves, and a class has fewer than 1200 in all."""
    rng = np.random.default_rng(per_class + more)
    tok, dh = case(rng, N + more, vocab, d, dtype)
    tok[rng.random(N + more) >= per_class * classes / N] = -1
    tok[N - 1] = vocab - 1
    old = rng.standard_normal((vocab, d)).astype(np.float32)
    out = torch.from_numpy(old).cuda() if accumulate else torch.full((vocab, d), float("nan"), device="cuda")
    ok(L().ouro_op_embed_bwd_sorted(stream(), dtype, p(torch.from_numpy(tok).cuda()), p(dh), d, p(out), d, N + more, d, vocab, 0.5, accumulate))
    x, inside = 0.5 * dh.double().cpu().numpy(), tok >= 0
    ref, mag, k = np.zeros((vocab, d)), np.zeros((vocab, d)), np.zeros((vocab, 1))
    np.add.at(ref, tok[inside], x[inside])
    np.add.at(mag, tok[inside], np.abs(x[inside]))
    np.add.at(k, tok[inside], 1)
    w = -(-(N + more) // (N - 2048))                             # (a step of 2048 ids before the positions end begins another part)
    base = old.astype(np.float64) if accumulate else np.zeros((vocab, d))
    assert np.all(np.abs(out.double().cpu().numpy() - (base + ref)) <= 2.0 ** -24 * ((k + 1) * mag + w * (np.abs(base) + mag)))


# 2^22 rows go to 2^8 workgroups (2^9 where the sums are added): 14 (13) bits of an entry are the row and 18 (19) the position, and the last id of
# 2^18 (2^19) at the last row would be an entry of ones.
@pytest.mark.parametrize("per_class", [60, 150, 400, 900])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_the_last_row_at_the_last_position(accumulate, dtype, per_class):
    """Lists that are sorted by counting, from runs and by radix."""
    last_of_positions(1 << (18 + accumulate), 1 << 22, 8 if dtype else 4, dtype, accumulate, per_class, 256 << accumulate)


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("more", [1, 3000, 300000])
def test_more_ids_than_an_entry_has_positions(more, accumulate):
    last_of_positions(1 << (18 + accumulate), 1 << 22, 4, 0, accumulate, 300, 256 << accumulate, more)
