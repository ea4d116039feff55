"""Operators for token models without a GPU: what they refuse before any HIP call, and the oracle's gradients against differences."""
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


def test_rotary_rejects_bad_arguments(L):
    call = caller(L.laplex_rotary, "x ldx y ldy type tokens heads dim turned positions frequencies magnitude flags",
                  dict(x=FAKE, ldx=32, y=FAKE, ldy=32, type=B.LAPLEX_F32, tokens=4, heads=2, dim=16, turned=8, positions=FAKE, frequencies=FAKE,
                       magnitude=1.0, flags=0))
    for name in ("x", "y", "positions", "frequencies"):
        assert call(**{name: None}) == B.LAPLEX_ERR_NULL
    assert call(type=2) == B.LAPLEX_ERR_VALUE and call(type=-1) == B.LAPLEX_ERR_VALUE
    for bad in (dict(tokens=-1), dict(heads=-1), dict(heads=65536), dict(dim=-2), dict(dim=4098), dict(turned=7), dict(turned=18), dict(turned=-2),
                dict(tokens=1 << 27)):
        assert call(**bad) == B.LAPLEX_ERR_SIZE, bad
    assert call(ldx=31) == B.LAPLEX_ERR_LD and call(ldy=0) == B.LAPLEX_ERR_LD
    for bad in (1, 4, 64, 1 << 31):
        assert call(flags=bad) == B.LAPLEX_ERR_FLAGS
    assert call(magnitude=NAN) == B.LAPLEX_ERR_VALUE and call(magnitude=INF) == B.LAPLEX_ERR_VALUE
    assert call(x=FAKE + 2) == B.LAPLEX_ERR_ALIGN and call(x=FAKE + 1, type=B.LAPLEX_BF16) == B.LAPLEX_ERR_ALIGN
    assert call(positions=FAKE + 4) == B.LAPLEX_ERR_ALIGN and call(frequencies=FAKE + 2) == B.LAPLEX_ERR_ALIGN
    assert call(tokens=0, x=None, y=None, positions=None) == B.LAPLEX_OK
    assert call(heads=0, x=None, y=None) == B.LAPLEX_OK
    f = L.laplex_rotary_frequencies
    assert f(None, 8, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == B.LAPLEX_ERR_NULL
    assert f(FAKE, 7, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == B.LAPLEX_ERR_SIZE
    assert f(FAKE, -2, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == B.LAPLEX_ERR_SIZE
    for bad in ((1e4, 4, 1.0, 0, 0, 0), (1e4, -1, 1.0, 0, 0, 0), (0.0, 0, 1.0, 0, 0, 0), (NAN, 0, 1.0, 0, 0, 0), (INF, 0, 1.0, 0, 0, 0), (1e4, 1, 0.0, 0, 0, 0),
                (1e4, 2, NAN, 0, 0, 0), (1e4, 3, 8.0, 0.0, 1.0, 32.0), (1e4, 3, 8.0, 4096.0, 32.0, 32.0), (1e4, 3, 8.0, 4096.0, NAN, 32.0)):
        assert f(FAKE, 8, *bad, None) == B.LAPLEX_ERR_VALUE, bad
    assert f(None, 0, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == B.LAPLEX_OK


ATTENTION = dict(q=FAKE, ldq=32, k=FAKE, ldk=32, v=FAKE, ldv=16, type=B.LAPLEX_F32, tokens=12, sequences=3, starts=None, heads=2, dk=16, dv=8,
                 rates=FAKE, scale=1.0, state_in=FAKE, y=FAKE, ldy=16, state_out=FAKE, ws=FAKE, wsb=1 << 40)
COMMON = [(dict(type=7), B.LAPLEX_ERR_VALUE), (dict(tokens=-1), B.LAPLEX_ERR_SIZE), (dict(sequences=-1), B.LAPLEX_ERR_SIZE),
          (dict(heads=-1), B.LAPLEX_ERR_SIZE), (dict(heads=65536), B.LAPLEX_ERR_SIZE), (dict(dk=0), B.LAPLEX_ERR_SIZE), (dict(dv=0), B.LAPLEX_ERR_SIZE),
          (dict(dk=257), B.LAPLEX_ERR_SIZE), (dict(dv=257), B.LAPLEX_ERR_SIZE), (dict(scale=0.0), B.LAPLEX_ERR_VALUE), (dict(scale=-1.0), B.LAPLEX_ERR_VALUE),
          (dict(scale=NAN), B.LAPLEX_ERR_VALUE), (dict(scale=INF), B.LAPLEX_ERR_VALUE), (dict(q=None), B.LAPLEX_ERR_NULL), (dict(k=None), B.LAPLEX_ERR_NULL),
          (dict(v=None), B.LAPLEX_ERR_NULL), (dict(rates=None), B.LAPLEX_ERR_NULL), (dict(ldq=31), B.LAPLEX_ERR_LD), (dict(ldk=31), B.LAPLEX_ERR_LD),
          (dict(ldv=15), B.LAPLEX_ERR_LD), (dict(q=FAKE + 2), B.LAPLEX_ERR_ALIGN), (dict(rates=FAKE + 2), B.LAPLEX_ERR_ALIGN),
          (dict(k=FAKE + 1, type=B.LAPLEX_BF16), B.LAPLEX_ERR_ALIGN)]


def need(L, **kw):
    a = {**ATTENTION, **kw}
    out = ctypes.c_size_t(0)
    assert L.laplex_decay_attention_workspace_bytes(a["type"], a["tokens"], a["sequences"], a["heads"], a["dk"], a["dv"], ctypes.byref(out)) == 0
    return out.value


def test_attention_rejects_bad_arguments(L):
    call = caller(L.laplex_decay_attention, "q ldq k ldk v ldv type tokens sequences starts heads dk dv rates scale state_in y ldy state_out ws wsb", ATTENTION)
    for bad, status in COMMON + [(dict(y=None), B.LAPLEX_ERR_NULL), (dict(ldy=15), B.LAPLEX_ERR_LD), (dict(tokens=13), B.LAPLEX_ERR_SIZE),
                                 (dict(sequences=0), B.LAPLEX_ERR_SIZE), (dict(tokens=1 << 27, sequences=1), B.LAPLEX_ERR_SIZE),
                                 (dict(sequences=(1 << 20) + 1, starts=FAKE), B.LAPLEX_ERR_SIZE), (dict(starts=FAKE + 4), B.LAPLEX_ERR_ALIGN),
                                 (dict(state_in=FAKE + 1), B.LAPLEX_ERR_ALIGN), (dict(state_out=FAKE + 2), B.LAPLEX_ERR_ALIGN)]:
        assert call(**bad) == status, bad
    long = dict(tokens=30000, sequences=1)
    if need(L, **long):
        assert call(**long, wsb=need(L, **long) - 1) == B.LAPLEX_ERR_WORKSPACE
        assert call(**long, ws=None) == B.LAPLEX_ERR_NULL and call(**long, ws=FAKE + 64) == B.LAPLEX_ERR_ALIGN
    assert call(tokens=0, sequences=0, q=None, k=None, v=None, y=None, state_in=None, state_out=None, ws=None, wsb=0) == B.LAPLEX_OK
    assert call(heads=0, q=None, k=None, v=None, y=None, rates=None, ws=None, wsb=0) == B.LAPLEX_OK
    assert call(tokens=0, q=None, k=None, v=None, y=None, state_out=None) == B.LAPLEX_OK
    f = L.laplex_decay_attention_workspace_bytes
    out = ctypes.c_size_t(0)
    assert f(0, 12, 3, 2, 16, 8, None) == B.LAPLEX_ERR_NULL
    assert f(3, 12, 3, 2, 16, 8, ctypes.byref(out)) == B.LAPLEX_ERR_VALUE
    assert f(0, -1, 3, 2, 16, 8, ctypes.byref(out)) == B.LAPLEX_ERR_SIZE
    assert f(0, 12, 3, 2, 300, 8, ctypes.byref(out)) == B.LAPLEX_ERR_SIZE


def test_attention_backward_rejects_bad_arguments(L):
    ok = {**ATTENTION, **dict(gy=FAKE, ldgy=16, gstate_out=FAKE, gq=FAKE, ldgq=32, gk=FAKE, ldgk=32, gv=FAKE, ldgv=16, gstate_in=FAKE)}
    call = caller(L.laplex_decay_attention_backward, "q ldq k ldk v ldv type tokens sequences starts heads dk dv rates scale state_in gy ldgy gstate_out "
                  "gq ldgq gk ldgk gv ldgv gstate_in ws wsb", ok)
    for bad, status in COMMON + [(dict(gy=None), B.LAPLEX_ERR_NULL), (dict(ldgy=15), B.LAPLEX_ERR_LD), (dict(ldgq=31), B.LAPLEX_ERR_LD), (dict(ldgk=31), B.LAPLEX_ERR_LD),
                                 (dict(ldgv=15), B.LAPLEX_ERR_LD), (dict(gv=FAKE + 1), B.LAPLEX_ERR_ALIGN), (dict(gstate_in=FAKE + 2), B.LAPLEX_ERR_ALIGN),
                                 (dict(tokens=13), B.LAPLEX_ERR_SIZE)]:
        assert call(**bad) == status, bad
    assert call(gq=None, gk=None, gv=None, gstate_in=None) == B.LAPLEX_OK          # nothing is wanted
    assert call(tokens=0, q=None, k=None, v=None, gy=None, gq=None, gk=None, gv=None, gstate_in=None) == B.LAPLEX_OK


def test_attention_step_rejects_bad_arguments(L):
    ok = {**ATTENTION, "state": FAKE}
    call = caller(L.laplex_decay_attention_step, "q ldq k ldk v ldv type sequences heads dk dv rates scale state y ldy", ok)
    for bad, status in COMMON:
        if "tokens" not in bad:
            assert call(**bad) == status, bad
    assert call(state=None) == B.LAPLEX_ERR_NULL and call(y=None) == B.LAPLEX_ERR_NULL and call(state=FAKE + 2) == B.LAPLEX_ERR_ALIGN
    assert call(sequences=0, q=None, k=None, v=None, y=None, state=None) == B.LAPLEX_OK


def test_logprob_rejects_bad_arguments(L):
    ok = dict(y=FAKE, ldy=4, type=B.LAPLEX_F32, k=100, batch=4, targets=FAKE, tau=1.0, logp=FAKE, lse=FAKE, entropy=FAKE, top=5, top_ids=FAKE, top_logp=FAKE,
              ws=FAKE, wsb=1 << 40)
    call = caller(L.laplex_logprob, "y ldy type k batch targets tau logp lse entropy top top_ids top_logp ws wsb", ok)
    for name in ("y", "targets", "top_ids", "top_logp"):
        assert call(**{name: None}) == B.LAPLEX_ERR_NULL, name
    for bad in (dict(k=-1), dict(batch=-1), dict(top=-1), dict(top=65, k=1000), dict(top=5, k=4), dict(k=1 << 32), dict(batch=1 << 27)):
        assert call(**bad) == B.LAPLEX_ERR_SIZE, bad
    for bad in (dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN), dict(tau=INF), dict(type=2)):
        assert call(**bad) == B.LAPLEX_ERR_VALUE, bad
    assert call(ldy=3) == B.LAPLEX_ERR_LD
    for bad in (dict(y=FAKE + 2), dict(targets=FAKE + 4), dict(logp=FAKE + 1), dict(lse=FAKE + 2), dict(entropy=FAKE + 2), dict(top_ids=FAKE + 4), dict(top_logp=FAKE + 2)):
        assert call(**bad) == B.LAPLEX_ERR_ALIGN, bad
    assert call(logp=None, targets=None, lse=None, entropy=None, top=0, top_ids=None, top_logp=None) == B.LAPLEX_OK     # nothing is wanted
    assert call(batch=0, y=None, targets=None, ws=None, wsb=0) == B.LAPLEX_OK
    out = ctypes.c_size_t(0)
    assert L.laplex_logprob_workspace_bytes(100, 4, 5, None) == B.LAPLEX_ERR_NULL
    assert L.laplex_logprob_workspace_bytes(100, 4, 101, ctypes.byref(out)) == B.LAPLEX_ERR_SIZE
    assert L.laplex_logprob_workspace_bytes(32000, 256, 5, ctypes.byref(out)) == B.LAPLEX_OK
    if out.value:
        assert call(k=32000, batch=256, ldy=256, wsb=out.value - 1) == B.LAPLEX_ERR_WORKSPACE
        assert call(k=32000, batch=256, ldy=256, ws=None) == B.LAPLEX_ERR_NULL
    ok = dict(y=FAKE, ldy=4, type=B.LAPLEX_F32, k=100, batch=4, targets=FAKE, tau=1.0, lse=FAKE, entropy=FAKE, glogp=FAKE, gentropy=FAKE, glse=FAKE, gy=FAKE, ldgy=4)
    call = caller(L.laplex_logprob_backward, "y ldy type k batch targets tau lse entropy glogp gentropy glse gy ldgy", ok)
    for name in ("y", "targets", "lse", "entropy", "gy"):
        assert call(**{name: None}) == B.LAPLEX_ERR_NULL, name
    assert call(ldgy=3) == B.LAPLEX_ERR_LD and call(k=-1) == B.LAPLEX_ERR_SIZE and call(tau=0.0) == B.LAPLEX_ERR_VALUE and call(type=9) == B.LAPLEX_ERR_VALUE
    assert call(gentropy=FAKE + 2) == B.LAPLEX_ERR_ALIGN and call(gy=FAKE + 1) == B.LAPLEX_ERR_ALIGN
    assert call(k=0, y=None, gy=None) == B.LAPLEX_OK


def test_binding_refuses_other_types_and_shapes():
    torch = pytest.importorskip("torch")
    half = torch.zeros(2, 1, 4, dtype=torch.float16)
    with pytest.raises(B.LaplexError) as e:
        B.laplex_rotary(half, torch.zeros(2, dtype=torch.int64), torch.zeros(2), half, stream=0)
    assert e.value.status == B.LAPLEX_ERR_VALUE
    x = torch.zeros(2, 1, 4)
    with pytest.raises(B.LaplexError):
        B.laplex_rotary(x, torch.zeros(2, dtype=torch.int64), torch.zeros(2), x.bfloat16(), stream=0)
    with pytest.raises(AssertionError):
        B.laplex_rotary(x, torch.zeros(2, dtype=torch.int32), torch.zeros(2), x, stream=0)
    with pytest.raises(AssertionError):
        w = torch.zeros(2, 3, 4).transpose(1, 2)
        B.laplex_rotary(w, torch.zeros(2, dtype=torch.int64), torch.zeros(0), w, stream=0)
    with pytest.raises(AssertionError):
        B.laplex_decay_attention_step(x, x, x, torch.zeros(1), torch.zeros(2, 1, 4, 3), x, stream=0)


# --- the oracle's own gradients --------------------------------------------------------------------------------------------

def test_oracle_attention_backward_is_the_derivative():
    r = np.random.default_rng(5)
    n, dk, dv, rate, scale = 9, 3, 4, 0.3, 0.6
    q, k, v, S, gy, G = (r.normal(size=s) for s in ((n, dk), (n, dk), (n, dv), (dk, dv), (n, dv), (dk, dv)))
    grads, _ = O.attention_sequence_backward(q, k, v, rate, scale, S, gy, G)

    def loss(*a):
        y, last, _, _ = O.attention_sequence(a[0], a[1], a[2], rate, scale, a[3])
        return (gy * y).sum() + (G * last).sum()
    for which in range(4):
        for at in np.ndindex(*grads[which].shape):
            def moved(by):
                a = [t.copy() for t in (q, k, v, S)]
                a[which][at] += by
                return loss(*a)
            # the loss is linear in each argument: a central difference has rounding errors only
            assert abs((moved(1e-3) - moved(-1e-3)) / 2e-3 - grads[which][at]) < 1e-9


def test_oracle_logprob_backward_is_the_derivative():
    r = np.random.default_rng(6)
    k, t, tau = 7, 4, 0.8
    y = r.normal(size=(k, t)); y[2, 1] = -np.inf
    targets = np.array([3, 0, -1, 6])
    gl, ge, gs = r.normal(size=(3, t))
    g = O.logprob_backward(y, targets, gl, ge, gs, tau)

    def loss(y):
        f = O.logprob(y, targets, tau)
        return (gl * f["logp"] + ge * f["entropy"] + gs * f["lse"]).sum()
    for at in np.ndindex(k, t):
        a, b = y.copy(), y.copy()
        a[at] += 1e-5; b[at] -= 1e-5
        # third derivatives of these are below 10: the difference is off by at most 1e-10 * 10 / 6, and by rounding / 1e-5
        assert abs((loss(a) - loss(b)) / 2e-5 - g[at]) < 1e-8


def test_oracle_rotary_keeps_lengths_and_turns_by_differences():
    """The product of a turned query and a turned key depends on the difference of their positions alone."""
    r = np.random.default_rng(7)
    q, k = r.normal(size=(2, 1, 1, 10))
    f = np.array([1.0, 0.3, 0.01])
    for pairs in (False, True):
        a = [(O.rotary(q, [p], f, 1.0, pairs)[0] * O.rotary(k, [p - 5], f, 1.0, pairs)[0]).sum() for p in (0, 3, 1000)]
        assert np.ptp(a) < 1e-12
        back = O.rotary(O.rotary(q, [77], f, 1.0, pairs)[0], [77], f, 1.0, pairs, True)[0]
        assert np.abs(back - q).max() < 1e-14
