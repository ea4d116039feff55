"""Layer norm and verification of drafts without a GPU: what they refuse before any HIP call, and the oracle against differences and by hand."""
import ctypes
import os

import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

FAKE = 0x10000          # a non-null, 256-byte aligned "device pointer" that must never be touched
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_24584_amd import build
        build.build()
    return B.lib()


def caller(f, names, ok):
    return lambda **kw: f(*[{**ok, **kw}[n] for n in names.split()], None)


def size(f, *a):
    out = ctypes.c_size_t(0)
    status = f(*a, ctypes.byref(out))
    return status, out.value


def test_layer_norm_rejects_bad_arguments(L):
    call = caller(L.laplex_layer_norm, "x ldx type rows width weight bias eps y ldy mean rstd",
                  dict(x=FAKE, ldx=16, type=B.LAPLEX_F32, rows=4, width=16, weight=FAKE, bias=FAKE, eps=1e-5, y=FAKE, ldy=16, mean=FAKE, rstd=FAKE))
    assert call(x=None) == B.LAPLEX_ERR_NULL and call(y=None) == B.LAPLEX_ERR_NULL
    assert call(type=2) == B.LAPLEX_ERR_VALUE
    for bad in (dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=-1), dict(width=(1 << 20) + 1)):
        assert call(**bad) == B.LAPLEX_ERR_SIZE, bad
    for eps in (0.0, -1e-5, NAN, INF):
        assert call(eps=eps) == B.LAPLEX_ERR_VALUE
    assert call(ldx=15) == B.LAPLEX_ERR_LD and call(ldy=15) == B.LAPLEX_ERR_LD
    for name in ("x", "y", "weight", "bias", "mean", "rstd"):
        assert call(**{name: FAKE + 2}) == B.LAPLEX_ERR_ALIGN
    assert call(x=FAKE + 1, type=B.LAPLEX_BF16) == B.LAPLEX_ERR_ALIGN
    assert call(rows=1 << 30, ldx=1 << 40) == B.LAPLEX_ERR_SIZE
    assert call(rows=0, x=None, y=None, mean=None, rstd=None) == B.LAPLEX_OK


def test_layer_norm_backward_rejects_bad_arguments(L):
    need = size(L.laplex_layer_norm_workspace_bytes, 4, 16)[1]
    call = caller(L.laplex_layer_norm_backward, "x ldx gy ldgy type rows width weight mean rstd gx ldgx gweight gbias ws wsb",
                  dict(x=FAKE, ldx=16, gy=FAKE, ldgy=16, type=B.LAPLEX_F32, rows=4, width=16, weight=FAKE, mean=FAKE, rstd=FAKE, gx=FAKE, ldgx=16, gweight=FAKE,
                       gbias=FAKE, ws=FAKE, wsb=need))
    for name in ("x", "gy", "mean", "rstd", "ws"):
        assert call(**{name: None}) == B.LAPLEX_ERR_NULL, name
    for bad in (dict(rows=-1), dict(width=0)):
        assert call(**bad) == B.LAPLEX_ERR_SIZE, bad
    assert call(type=-1) == B.LAPLEX_ERR_VALUE
    for name in ("ldx", "ldgy", "ldgx"):
        assert call(**{name: 15}) == B.LAPLEX_ERR_LD
    for name in ("x", "gy", "gx", "weight", "mean", "rstd", "gweight", "gbias"):
        assert call(**{name: FAKE + 2}) == B.LAPLEX_ERR_ALIGN
    assert call(ws=FAKE + 64) == B.LAPLEX_ERR_ALIGN and call(wsb=need - 1) == B.LAPLEX_ERR_WORKSPACE
    assert call(gx=None, gweight=None, gbias=None, ws=None, wsb=0) == B.LAPLEX_OK          # nothing is wanted
    f = L.laplex_layer_norm_workspace_bytes
    assert f(4, 16, None) == B.LAPLEX_ERR_NULL and size(f, -1, 16)[0] == B.LAPLEX_ERR_SIZE and size(f, 4, 0)[0] == B.LAPLEX_ERR_SIZE
    for width in (1, 16, 100, 2048, 2049, 4096, 9000, 16384, 16385, 100000):
        sizes = [size(f, rows, width)[1] for rows in (0, 1, 3, 100, 1000, 5000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[-1] <= 1024 * 2 * width * 4


VERIFY = dict(y=FAKE, ldy=12, z=FAKE, ldz=12, type=B.LAPLEX_F32, k=100, batch=12, drafts=FAKE, sequences=3, starts=None, tau=1.0, draft_tau=1.0, chances=FAKE,
              next_chances=FAKE, accepted=FAKE, next=FAKE, logp=FAKE, next_logp=FAKE, ws=FAKE, wsb=1 << 40, flags=0)


def test_verify_rejects_bad_arguments(L):
    call = caller(L.laplex_verify_drafts, "y ldy z ldz type k batch drafts sequences starts tau draft_tau chances next_chances accepted next logp next_logp ws wsb flags",
                  VERIFY)
    for name in ("y", "drafts", "chances", "next_chances", "accepted", "next", "ws"):
        assert call(**{name: None}) == B.LAPLEX_ERR_NULL, name
    for bad in (dict(k=0), dict(k=-1), dict(k=1 << 32), dict(batch=-1), dict(batch=1 << 26), dict(sequences=-1), dict(sequences=(1 << 20) + 1, starts=FAKE),
                dict(batch=13), dict(sequences=0)):
        assert call(**bad) == B.LAPLEX_ERR_SIZE, bad
    assert call(type=3) == B.LAPLEX_ERR_VALUE
    for tau in (0.0, -1.0, NAN, INF):
        assert call(tau=tau) == B.LAPLEX_ERR_VALUE and call(draft_tau=tau) == B.LAPLEX_ERR_VALUE
    assert call(ldy=11) == B.LAPLEX_ERR_LD and call(ldz=11) == B.LAPLEX_ERR_LD
    for flags in (1, 8, 32, 128):
        assert call(flags=flags) == B.LAPLEX_ERR_FLAGS
    for name, off in (("y", 2), ("z", 1), ("drafts", 4), ("starts", 4), ("chances", 4), ("next_chances", 2), ("accepted", 4), ("next", 4), ("logp", 2), ("next_logp", 1),
                      ("ws", 64)):
        assert call(**{name: FAKE + off}) == B.LAPLEX_ERR_ALIGN, name
    need = size(L.laplex_verify_workspace_bytes, 100, 12, 3)[1]
    assert call(wsb=need - 1) == B.LAPLEX_ERR_WORKSPACE
    assert call(sequences=0, batch=0, y=None, z=None, drafts=None, chances=None, next_chances=None, accepted=None, next=None, ws=None, wsb=0) == B.LAPLEX_OK
    f = L.laplex_verify_workspace_bytes
    assert f(10, 1, 1, None) == B.LAPLEX_ERR_NULL and size(f, 0, 1, 1)[0] == B.LAPLEX_ERR_SIZE
    sizes = [size(f, k, t, b)[1] for k, t, b in ((1, 1, 1), (10, 1, 1), (10, 5, 1), (32000, 5, 1), (32000, 40, 8), (32000, 3000, 8), (60000, 50000, 9000), (60000, 1 << 20, 9000))]
    assert sizes == sorted(sizes)


def test_oracle_of_verification_by_hand():
    log = lambda *p: np.log(np.array(p))[:, None]
    y, z = np.repeat(log(0.5, 0.2, 0.3), 2, 1), np.repeat(log(0.25, 0.5, 0.25), 2, 1)
    starts = [0, 2]
    run = lambda x, u, v, **kw: O.verify_drafts(y, kw.pop("z", z), np.array([x, -1]), starts, 1.0, 1.0, np.array([u, 0.0]), np.array([v]), **kw)
    assert run(1, 0.39, 0.6)[:2] == (np.array([1]), np.array([1]))        # kept while u < 0.2 / 0.5; then from p
    a, n, logp, next_logp = run(1, 0.41, 0.83)                            # refused: left are 0.25, 0, 0.05
    assert a[0] == 0 and n[0] == 0 and np.isclose(logp[0], np.log(0.2)) and np.isclose(next_logp[0], np.log(0.5))
    assert run(1, 0.41, 0.84)[1][0] == 2
    assert run(1, 0.21, 0.6, z=None)[0][0] == 0 and run(1, 0.21, 0.6, z=None)[1][0] == 0 and run(1, 0.21, 0.63, z=None)[1][0] == 2
    assert run(7, 0.0, 0.55)[:2] == (np.array([0]), np.array([1]))        # no draft: from p
    assert run(0, 0.9, 0.9, greedy=True)[:2] == (np.array([1]), np.array([0])) and run(2, 0.0, 0.0, greedy=True)[0][0] == 0


def test_oracle_of_the_layer_norm_gradient_against_differences():
    r = np.random.default_rng(5)
    x, gy, w, b = r.normal(size=(3, 11)), r.normal(size=(3, 11)), r.normal(size=11), r.normal(size=11)
    gx, gw, gb = O.layer_norm_backward(x, gy, w, 1e-5)
    f = lambda x, w, b: (O.layer_norm(x, w, b, 1e-5)[0] * gy).sum()
    for which, got in enumerate((gx, gw, gb)):
        for at in np.ndindex(*got.shape):
            ends = []
            for s in (1e-6, -1e-6):
                a = [x.copy(), w.copy(), b.copy()]
                a[which][at] += s
                ends.append(f(*a))
            assert abs((ends[0] - ends[1]) / 2e-6 - got[at]) < 1e-6
