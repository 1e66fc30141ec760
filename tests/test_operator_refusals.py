"""What the entry points of the sorted embedding gradient, the recurrence and the orthogonalised update refuse before anything
is enqueued (host only: no GPU is touched), with a message that names the operator."""
import ctypes as C

import pytest

import paper_1909_06695_amd as P

E_ARG = -2
X = C.c_void_p(4096)                                             # an address that is never read


def refused(rc, op):
    assert rc == E_ARG
    assert P.lib().ouro_last_error().startswith(op)


EMBED = dict(dtype=0, tok=X, dh=X, lddh=8, dV=X, ldv=8, N=4, d=8, vocab=16, scale=1.0, accumulate=0)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(dtype=-1), dict(N=-1), dict(N=(1 << 30) + 1), dict(d=0), dict(vocab=0), dict(tok=None),
                                    dict(dh=None), dict(dV=None), dict(lddh=7), dict(ldv=7), dict(d=(1 << 24) + 1, lddh=2**31 - 1, ldv=2**31 - 1)])
def test_embed_bwd_sorted(change):
    a = dict(EMBED, **change)
    refused(P.lib().ouro_op_embed_bwd_sorted(None, *a.values()), b"embed_bwd_sorted")


FWD = dict(dtype=0, B=2, T=4, D=8, z=X, ldz=8, x=X, ldx=8, h0=None, lens=None, h=X, ldh=8, hT=None, states=None, scratch=None)
BWD = dict(dtype=0, B=2, T=4, D=8, z=X, ldz=8, x=X, ldx=8, states=X, lens=None, dh=X, lddh=8, dhT=None, dz=X, lddz=8, dx=X, lddx=8, dh0=None,
           scratch=None)
SIZES = [dict(dtype=2), dict(B=0), dict(T=0), dict(D=0), dict(T=(1 << 30) + 1), dict(D=(1 << 24) + 1, ldz=1 << 30, ldx=1 << 30), dict(z=None), dict(x=None), dict(ldz=7), dict(ldx=7), dict(T=100000),
         dict(T=100000, scratch=C.c_void_p(4104))]


@pytest.mark.parametrize("change", SIZES + [dict(h=None), dict(ldh=7)])
def test_recurrence_fwd(change):
    refused(P.lib().ouro_op_recurrence_fwd(None, *dict(FWD, **change).values()), b"recurrence_fwd")


@pytest.mark.parametrize("change", SIZES + [dict(states=None), dict(dh=None), dict(dz=None), dict(dx=None), dict(lddh=7), dict(lddz=7), dict(lddx=7)])
def test_recurrence_bwd(change):
    refused(P.lib().ouro_op_recurrence_bwd(None, *dict(BWD, **change).values()), b"recurrence_bwd")


def test_recurrence_scratch():
    """No workspace for single tokens or where streams and channels fill the chip; sizes that are refused need none."""
    size = P.lib().ouro_op_recurrence_scratch
    assert size(64, 1, 1024) == 0 and size(64, 1000, 2048) == 0 and size(1, 64, 8) == 0
    assert size(1, 65536, 512) > 0
    assert size(0, 5, 5) == 0 and size(1, 0, 5) == 0 and size(1, 5, 0) == 0 and size(1, 5, (1 << 24) + 1) == 0


ORTHO = dict(dtype=0, batch=2, rows=16, cols=24, g=X, ldg=24, sg=384, momentum=None, mu=0.9, nesterov=0, o=X, ldo=24, so=384, scale=1.0, eps=1e-7,
             steps=5, scratch=X)


@pytest.mark.parametrize("change", [dict(dtype=2), dict(batch=0), dict(batch=65536), dict(rows=0), dict(cols=0), dict(g=None), dict(o=None),
                                    dict(scratch=None), dict(scratch=C.c_void_p(4100)), dict(ldg=23), dict(ldo=23), dict(sg=-1), dict(so=383),
                                    dict(so=0), dict(so=24), dict(so=24, ldo=47), dict(momentum=X, sg=0), dict(momentum=X, sg=100),
                                    dict(o=X, ldo=32, so=512), dict(so=400), dict(eps=-1.0), dict(eps=float("nan")), dict(steps=0), dict(steps=101), dict(rows=32768, cols=32768, ldg=32768, ldo=32768)])
def test_orthogonalize(change):
    refused(P.lib().ouro_op_orthogonalize(None, *dict(ORTHO, **change).values()), b"orthogonalize")


def test_orthogonalize_scratch():
    size = P.lib().ouro_op_orthogonalize_scratch
    assert size(1, 64, 256) > 0 and size(3, 100, 1) > 0 and size(2, 70, 500) == size(2, 500, 70)
    assert size(0, 5, 5) == 0 and size(1, 0, 5) == 0 and size(1, 32768, 32768) == 0
