"""The gated delta rule without a GPU: what it refuses before any HIP call, workspaces, and the oracle's gradients against differences."""
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


OK = dict(q=FAKE, ldq=16, k=FAKE, ldk=16, v=FAKE, ldv=16, type=B.LAPLEX_F32, tokens=12, sequences=3, starts=None, lengths=None, heads=2, key_heads=1, dk=16, dv=8,
          rates=FAKE, ldr=2, beta=FAKE, ldb=2, scale=1.0, state_in=FAKE, y=FAKE, ldy=16, state_out=FAKE, ws=FAKE, wsb=1 << 40, flags=0, state=FAKE,
          gy=FAKE, ldgy=16, gstate_out=FAKE, gq=FAKE, ldgq=16, gk=FAKE, ldgk=16, gv=FAKE, ldgv=16, grates=FAKE, ldgr=2, gbeta=FAKE, ldgb=2, gstate_in=FAKE)
COMMON = [(dict(type=7), B.LAPLEX_ERR_VALUE), (dict(sequences=-1), B.LAPLEX_ERR_SIZE), (dict(heads=-1), B.LAPLEX_ERR_SIZE), (dict(heads=65536, key_heads=1), B.LAPLEX_ERR_SIZE),
          (dict(heads=3, key_heads=2), B.LAPLEX_ERR_SIZE), (dict(key_heads=0), B.LAPLEX_ERR_SIZE), (dict(key_heads=-1), B.LAPLEX_ERR_SIZE), (dict(heads=1, key_heads=2), B.LAPLEX_ERR_SIZE),
          (dict(dk=0), B.LAPLEX_ERR_SIZE), (dict(dv=0), B.LAPLEX_ERR_SIZE), (dict(dk=257), B.LAPLEX_ERR_SIZE), (dict(dv=257), B.LAPLEX_ERR_SIZE),
          (dict(scale=0.0), B.LAPLEX_ERR_VALUE), (dict(scale=-1.0), B.LAPLEX_ERR_VALUE), (dict(scale=NAN), B.LAPLEX_ERR_VALUE), (dict(scale=INF), B.LAPLEX_ERR_VALUE),
          (dict(q=None), B.LAPLEX_ERR_NULL), (dict(k=None), B.LAPLEX_ERR_NULL), (dict(v=None), B.LAPLEX_ERR_NULL), (dict(rates=None), B.LAPLEX_ERR_NULL), (dict(beta=None), B.LAPLEX_ERR_NULL),
          (dict(ldq=15), B.LAPLEX_ERR_LD), (dict(ldk=15), B.LAPLEX_ERR_LD), (dict(ldv=15), B.LAPLEX_ERR_LD), (dict(ldr=1), B.LAPLEX_ERR_LD), (dict(ldb=1), B.LAPLEX_ERR_LD),
          (dict(q=FAKE + 2), B.LAPLEX_ERR_ALIGN), (dict(rates=FAKE + 2), B.LAPLEX_ERR_ALIGN), (dict(beta=FAKE + 1), B.LAPLEX_ERR_ALIGN),
          (dict(k=FAKE + 1, type=B.LAPLEX_BF16), B.LAPLEX_ERR_ALIGN)]
PROMPT = [(dict(tokens=-1), B.LAPLEX_ERR_SIZE), (dict(tokens=13), B.LAPLEX_ERR_SIZE), (dict(tokens=1 << 27, sequences=1), B.LAPLEX_ERR_SIZE),
          (dict(sequences=(1 << 20) + 1, starts=FAKE), B.LAPLEX_ERR_SIZE), (dict(sequences=0), B.LAPLEX_ERR_SIZE), (dict(starts=FAKE + 4), B.LAPLEX_ERR_ALIGN),
          (dict(lengths=FAKE + 4), B.LAPLEX_ERR_ALIGN), (dict(state_in=FAKE + 1), B.LAPLEX_ERR_ALIGN), (dict(ws=None), B.LAPLEX_ERR_NULL), (dict(ws=FAKE + 64), B.LAPLEX_ERR_ALIGN),
          (dict(flags=1), B.LAPLEX_ERR_FLAGS), (dict(flags=4), B.LAPLEX_ERR_FLAGS), (dict(flags=16), B.LAPLEX_ERR_FLAGS)]


def need(L, training, **kw):
    a = {**OK, **kw}
    out = ctypes.c_size_t(0)
    status = L.laplex_delta_attention_workspace_bytes(a["type"], a["tokens"], a["sequences"], a["heads"], a["key_heads"], a["dk"], a["dv"], training, ctypes.byref(out))
    assert status == 0
    return out.value


def test_forward_rejects_bad_arguments(L):
    call = caller(L.laplex_delta_attention, "q ldq k ldk v ldv type tokens sequences starts lengths heads key_heads dk dv rates ldr beta ldb scale state_in y ldy state_out ws wsb flags", OK)
    for bad, status in COMMON + PROMPT + [(dict(y=None), B.LAPLEX_ERR_NULL), (dict(ldy=15), B.LAPLEX_ERR_LD), (dict(state_out=FAKE + 2), B.LAPLEX_ERR_ALIGN),
                                          (dict(wsb=need(L, 0) - 1), B.LAPLEX_ERR_WORKSPACE), (dict(wsb=need(L, 1) - 1, flags=B.LAPLEX_SAVE_SCANS), B.LAPLEX_ERR_WORKSPACE)]:
        assert call(**bad) == status, bad
    nothing = dict(q=None, k=None, v=None, y=None, rates=None, beta=None, ws=None, wsb=0)
    assert call(tokens=0, sequences=0, state_in=None, state_out=None, **nothing) == B.LAPLEX_OK
    assert call(heads=0, key_heads=0, **nothing) == B.LAPLEX_OK
    assert call(tokens=0, state_out=None, **nothing) == B.LAPLEX_OK


def test_backward_rejects_bad_arguments(L):
    call = caller(L.laplex_delta_attention_backward, "q ldq k ldk v ldv type tokens sequences starts lengths heads key_heads dk dv rates ldr beta ldb scale state_in gy ldgy gstate_out "
                  "gq ldgq gk ldgk gv ldgv grates ldgr gbeta ldgb gstate_in ws wsb flags", OK)
    for bad, status in COMMON + PROMPT + [(dict(gy=None), B.LAPLEX_ERR_NULL), (dict(ldgy=15), B.LAPLEX_ERR_LD), (dict(ldgq=15), B.LAPLEX_ERR_LD), (dict(ldgk=15), B.LAPLEX_ERR_LD),
                                          (dict(ldgv=15), B.LAPLEX_ERR_LD), (dict(ldgr=1), B.LAPLEX_ERR_LD), (dict(ldgb=0), B.LAPLEX_ERR_LD), (dict(gv=FAKE + 1), B.LAPLEX_ERR_ALIGN),
                                          (dict(grates=FAKE + 2), B.LAPLEX_ERR_ALIGN), (dict(gbeta=FAKE + 2), B.LAPLEX_ERR_ALIGN), (dict(gstate_in=FAKE + 2), B.LAPLEX_ERR_ALIGN),
                                          (dict(gstate_out=FAKE + 1), B.LAPLEX_ERR_ALIGN), (dict(wsb=need(L, 1) - 1), B.LAPLEX_ERR_WORKSPACE)]:
        assert call(**bad) == status, bad
    none = dict(gq=None, gk=None, gv=None, grates=None, gbeta=None, gstate_in=None)
    assert call(**none) == B.LAPLEX_OK          # nothing is wanted
    assert call(tokens=0, q=None, k=None, v=None, gy=None, rates=None, beta=None, ws=None, wsb=0, **none) == B.LAPLEX_OK


def test_step_rejects_bad_arguments(L):
    call = caller(L.laplex_delta_attention_step, "q ldq k ldk v ldv type sequences heads key_heads dk dv rates ldr beta ldb scale state y ldy", OK)
    for bad, status in COMMON:
        assert call(**bad) == status, bad
    assert call(state=None) == B.LAPLEX_ERR_NULL and call(y=None) == B.LAPLEX_ERR_NULL and call(state=FAKE + 2) == B.LAPLEX_ERR_ALIGN
    assert call(sequences=0, q=None, k=None, v=None, y=None, rates=None, beta=None, state=None) == B.LAPLEX_OK


def test_heads_of_keys_without_heads_of_values_are_refused(L):
    """Their gradients would be sums over nothing, which no launch writes."""
    out = ctypes.c_size_t(0)
    bad = dict(heads=0, key_heads=2)
    assert L.laplex_delta_attention_workspace_bytes(0, 12, 3, 0, 2, 16, 8, 1, ctypes.byref(out)) == B.LAPLEX_ERR_SIZE
    for f, names in ((L.laplex_delta_attention, "q ldq k ldk v ldv type tokens sequences starts lengths heads key_heads dk dv rates ldr beta ldb scale state_in y ldy state_out ws wsb flags"),
                     (L.laplex_delta_attention_backward, "q ldq k ldk v ldv type tokens sequences starts lengths heads key_heads dk dv rates ldr beta ldb scale state_in gy ldgy gstate_out "
                      "gq ldgq gk ldgk gv ldgv grates ldgr gbeta ldgb gstate_in ws wsb flags"),
                     (L.laplex_delta_attention_step, "q ldq k ldk v ldv type sequences heads key_heads dk dv rates ldr beta ldb scale state y ldy")):
        call = caller(f, names, {**OK, "ldq": 32, "ldk": 32, "ldgq": 32, "ldgk": 32})
        assert call(**bad) == B.LAPLEX_ERR_SIZE
        assert call(heads=0, key_heads=0) == B.LAPLEX_OK


def test_workspace(L):
    f = L.laplex_delta_attention_workspace_bytes
    out = ctypes.c_size_t(0)
    assert f(0, 12, 3, 2, 1, 16, 8, 0, None) == B.LAPLEX_ERR_NULL and f(3, 12, 3, 2, 1, 16, 8, 0, ctypes.byref(out)) == B.LAPLEX_ERR_VALUE
    for bad in ((-1, 3, 2, 1, 16, 8), (12, -1, 2, 1, 16, 8), (12, 3, 2, 0, 16, 8), (12, 3, 3, 2, 16, 8), (12, 3, 2, 1, 300, 8)):
        assert f(0, *bad, 0, ctypes.byref(out)) == B.LAPLEX_ERR_SIZE, bad
    for type_ in (B.LAPLEX_F32, B.LAPLEX_BF16):
        for training in (0, 1):
            sizes = [need(L, training, type=type_, tokens=n, sequences=b, heads=8, key_heads=8, dk=128, dv=128) for n, b in ((0, 1), (1, 1), (100, 1), (100, 5), (4096, 5), (65536, 5), (65536, 500))]
            assert sizes == sorted(sizes)
    # what the header says it grows by
    more = need(L, 1, type=B.LAPLEX_BF16, tokens=1 << 20, sequences=1, heads=1, key_heads=1, dk=128, dv=128) / (1 << 20)
    assert 3.2 * 1024 < more < 3.6 * 1024
    assert need(L, 0, type=B.LAPLEX_BF16, tokens=1 << 20, sequences=1, heads=1, key_heads=1, dk=128, dv=128) / (1 << 20) < 500


@pytest.mark.parametrize("which", range(6))
def test_oracle_gradients_against_differences(which):
    r = np.random.default_rng(3)
    n, dk, dv = 9, 4, 3
    args = [r.normal(size=(n, dk)), r.normal(size=(n, dk)) / 2, r.normal(size=(n, dv)), r.random(n), r.random(n), r.normal(size=(dk, dv))]
    gy, gs = r.normal(size=(n, dv)), r.normal(size=(dk, dv))

    def loss(q, k, v, rates, beta, state):
        y, last, _ = O.delta_sequence(q, k, v, rates, beta, 0.7, state)
        return (y * gy).sum() + (last * gs).sum()

    got = O.delta_sequence_backward(*args[:5], 0.7, args[5], gy, gs)[0][which]
    for at in np.ndindex(*got.shape):
        ends = []
        for s in (1e-6, -1e-6):
            moved = [a.copy() for a in args]
            moved[which][at] += s
            ends.append(loss(*moved))
        assert abs((ends[0] - ends[1]) / 2e-6 - got[at]) < 1e-6 * max(1.0, np.abs(got).max())
