"""Numerics of the attention with a decay for each head that per-element bounds on the sum of absolute terms do not show.

Tolerances.  U = 2^-24 and H = 2^-8 are the unit roundings of fp32 and bf16.  A bf16 call's factors between its products are two bf16 numbers, off by at most
2^-15 of themselves, and a term passes two of them: 2^-14 of the sum of absolute terms, beside the fp32 sums' 16 sqrt(n + d + 64) U of it and the result's one rounding, H.
In the 2-norm: a result that is off by e before it is rounded is rounded the other way with the probability e / ulp, and is then a whole ulp off: against the exact result
rounded to bf16 the difference is sqrt(e ulp) on average over many.  With e = 2^-15 of the results' size and an ulp of at most 2^-7 that is 2^-11; 2^-10 is allowed.
"""
import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
RATES = np.array([0.03, 0.7, 0.0, 0.002, 3.0, 0.25], np.float32)


def seeded(*what):
    import zlib
    return np.random.default_rng(zlib.crc32(repr(what).encode()))


def dev(v, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(v)).to("cuda").to(dtype)


def host(t):
    return t.double().cpu().numpy()


def within(name, got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: "
                           f"{got[bad][0]} instead of {want[bad][0]}, may be off by {np.broadcast_to(bound, bad.shape)[bad][0]}")


class Problem:
    """Inputs of a forward and a backward call; `starts` is None for equal lengths that are not packed."""

    def __init__(self, lengths, heads, dk, dv, dtype, packed=True, states=True, scale=None, rates=None, what=""):
        r = seeded(what, lengths, heads, dk, dv)
        n, b = int(sum(lengths)), len(lengths)
        self.lengths, self.heads, self.dk, self.dv, self.dtype, self.n, self.b = lengths, heads, dk, dv, dtype, n, b
        of = lambda *s, t=dtype: dev(r.normal(size=s).astype(np.float32), t)
        self.q, self.k, self.v, self.gy = of(n, heads, dk), of(n, heads, dk), of(n, heads, dv), of(n, heads, dv)
        self.state, self.gstate = (of(b, heads, dk, dv, t=F32), of(b, heads, dk, dv, t=F32)) if states else (None, None)
        self.rates = np.resize(RATES if rates is None else np.asarray(rates, np.float32), heads)
        self.scale = float(np.float32(dk ** -0.5 if scale is None else scale))
        self.starts = dev(np.concatenate([[0], np.cumsum(lengths)]), torch.int64) if packed else None

    def workspace(self):
        """Of exactly the size that is asked for; what it holds does not matter."""
        size = B.laplex_decay_attention_workspace_bytes(self.dtype, self.n, self.b, self.heads, self.dk, self.dv)
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def new(self, *s, t=None):
        return torch.full(s, float("nan"), device="cuda", dtype=t or self.dtype)

    def forward(self):
        y, last = self.new(self.n, self.heads, self.dv), self.new(self.b, self.heads, self.dk, self.dv, t=F32)
        B.laplex_decay_attention(self.q, self.k, self.v, dev(self.rates), y, self.workspace(), self.scale, self.b, self.starts, self.state, last)
        return {"y": y, "state": last}

    def backward(self):
        gq, gk, gv = (self.new(self.n, self.heads, d) for d in (self.dk, self.dk, self.dv))
        g0 = self.new(self.b, self.heads, self.dk, self.dv, t=F32)
        B.laplex_decay_attention_backward(self.q, self.k, self.v, dev(self.rates), self.gy, gq, gk, gv, self.workspace(), self.scale, self.b, self.starts,
                                          self.state, self.gstate, g0)
        return {"gq": gq, "gk": gk, "gv": gv, "gstate": g0}

    def each(self, got):
        """(name, what was got, the definition's result in 64 bits, its sum of absolute terms, tokens) for every sequence and head"""
        at = 0
        for i, n in enumerate(self.lengths):
            for h in range(self.heads):
                q, k, v, gy = (host(t[at:at + n, h]) for t in (self.q, self.k, self.v, self.gy))
                S, G = (None if t is None else host(t[i, h]) for t in (self.state, self.gstate))
                want = dict(zip(("y", "state", "|y|", "|state|"), O.attention_sequence(q, k, v, self.rates[h], self.scale, S))) if "y" in got else {}
                if "gq" in got:
                    w, s = O.attention_sequence_backward(q, k, v, self.rates[h], self.scale, S, gy, G)
                    for name, a, b in zip(("gq", "gk", "gv", "gstate"), w, s):
                        want[name], want[f"|{name}|"] = a, b
                for name, t in got.items():
                    yield f"{name}[{i},{h}]", host(t[i, h] if "state" in name else t[at:at + n, h]), want[name], want[f"|{name}|"], n
            at += n


# --- bf16 results are rounded once, whatever the lengths and however the sequences are passed ---------------------------------------

ONCE = [
    ([2] * 64, 2, 64, 64, True), ([2] * 70, 1, 128, 128, True), ([3, 1, 4, 2] * 20, 1, 96, 80, True), ([5, 2] * 30, 1, 190, 256, True),      # packed, over 128 tokens in all
    ([2] * 70, 1, 64, 64, False), ([130, 7], 2, 128, 128, True), ([64], 2, 64, 48, False), ([65, 31, 33], 1, 128, 100, True),
    ([700, 3, 0, 64, 65], 3, 96, 80, True), ([2000], 3, 128, 128, False), ([900, 900], 3, 64, 128, False), ([1100], 2, 256, 256, False), ([600, 40], 2, 192, 130, True),
]


@pytest.mark.parametrize("lengths,heads,dk,dv,packed", ONCE)
@pytest.mark.parametrize("states", [False, True])
def test_bf16_results_are_rounded_once(lengths, heads, dk, dv, packed, states):
    p = Problem(lengths, heads, dk, dv, BF16, packed, states, what="once")
    off, size = {}, {}
    for name, got, want, terms, n in p.each({**p.forward(), **p.backward()}):
        exact = 16 * np.sqrt(n + max(dk, dv) + 64.0) * U * terms
        if "state" in name:
            within(name, got, want, exact)
            continue
        within(name, got, want, exact + 2.0 ** -14 * terms + 1.01 * H * np.abs(want))
        once = host(torch.from_numpy(want).to(BF16))
        kind = name.split("[")[0], name.split(",")[1]
        off[kind] = off.get(kind, 0.0) + ((got - once) ** 2).sum()
        size[kind] = size.get(kind, 0.0) + (want ** 2).sum()
    for kind in off:
        assert off[kind] <= (2.0 ** -10) ** 2 * size[kind], f"{kind}: {np.sqrt(off[kind] / size[kind]):.2e} from the rounded result"


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_short_sequence_has_the_same_bits_in_every_pack(dtype):
    """Alone, of equal lengths, and packed among others."""
    few = Problem([20] * 3, 2, 64, 48, dtype, False, what="pack")
    many = Problem([20] * 40, 2, 64, 48, dtype, True, what="pack of more")
    long = Problem([900, 20, 0, 20, 20, 1500], 2, 64, 48, dtype, True, what="pack with long ones")
    places = {many: (list(range(0, 60, 20)), [0, 1, 2]), long: ([900, 920, 940], [1, 3, 4])}
    for p, (rows, sequences) in places.items():
        for name in ("q", "k", "v", "gy"):
            for i, at in enumerate(rows):
                getattr(p, name)[at:at + 20] = getattr(few, name)[20 * i:20 * i + 20]
        for name in ("state", "gstate"):
            getattr(p, name)[sequences] = getattr(few, name)
        p.scale = few.scale
    want = {**few.forward(), **few.backward()}
    for p, (rows, sequences) in places.items():
        got = {**p.forward(), **p.backward()}
        for name, t in want.items():
            for i, at in enumerate(rows):
                one = got[name][sequences[i]] if "state" in name else got[name][at:at + 20]
                assert torch.equal(one, t[i] if "state" in name else t[20 * i:20 * i + 20]), name


# --- many sequences ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inside", [[], [(7, 900), (39990, 1300)]])
def test_attention_of_tens_of_thousands_of_sequences(dtype, inside):
    """More slots than a grid's second axis takes, empty sequences among them, long ones too or none; states in place."""
    r = seeded("tens of thousands", len(inside))
    lengths = r.integers(0, 4, 40000)
    for i, n in inside:
        lengths[i] = n
    p = Problem([int(n) for n in lengths], 1, 8, 8, dtype, True, rates=[0.1], what="many")
    got = {**p.forward(), **p.backward()}
    some = [0, 1, 2, 7, 8, 32767, 32768, 32769, 39990, 39991, 39999] + [int(i) for i in r.integers(0, 40000, 40)]
    at = np.concatenate([[0], np.cumsum(p.lengths)])
    for i in some:
        one = Problem([p.lengths[i]], 1, 8, 8, dtype, True, rates=[0.1])
        for name in ("q", "k", "v", "gy"):
            setattr(one, name, getattr(p, name)[at[i]:at[i + 1]])
        one.state, one.gstate, one.scale = p.state[i:i + 1], p.gstate[i:i + 1], p.scale
        mine = {name: t[i:i + 1] if "state" in name else t[at[i]:at[i + 1]] for name, t in got.items()}
        for name, g, want, terms, n in one.each(mine):
            exact = 16 * np.sqrt(n + 72.0) * U * terms
            within(f"{i}: {name}", g, want, exact if dtype == F32 or "state" in name else exact + 2.0 ** -14 * terms + 1.01 * H * np.abs(want))
    # in place
    state, y = p.state.clone(), torch.full_like(got["y"], float("nan"))
    B.laplex_decay_attention(p.q, p.k, p.v, dev(p.rates), y, p.workspace(), p.scale, p.b, p.starts, state, state)
    assert torch.equal(y, got["y"]) and torch.equal(state, got["state"])
    empty = torch.from_numpy(lengths == 0).cuda()
    assert torch.equal(state[empty], p.state[empty])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_state_in_place_among_sequences_of_one_stretch_and_of_several(dtype):
    """What several workgroups read and the last of them writes comes through the workspace; what one workgroup does, does not."""
    p = Problem([1, 900, 0, 64, 65, 2000, 3, 700], 2, 130, 72, dtype, True, what="in place")
    want = p.forward()
    for _ in range(3):
        state, y = p.state.clone(), torch.full_like(want["y"], float("nan"))
        B.laplex_decay_attention(p.q, p.k, p.v, dev(p.rates), y, p.workspace(), p.scale, p.b, p.starts, state, state)
        assert torch.equal(y, want["y"]) and torch.equal(state, want["state"])


# --- rates ---------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[70, 3], [1000]])
def test_a_rate_that_is_nan_shows_in_its_head(dtype, lengths):
    """Everything of that head is NaN, and the other heads are the same bits as without it."""
    p = Problem(lengths, 3, 40, 64, dtype, True, rates=[0.1, 0.2, 0.3])
    fine = {**p.forward(), **p.backward()}
    one = [t[:1].clone() for t in (p.q, p.k, p.v)]
    fine_state, fine_y = p.state[:1].clone(), p.new(1, 3, 64)
    B.laplex_decay_attention_step(*one, dev(p.rates), fine_state, fine_y, p.scale)
    p.rates[1] = np.nan
    odd = {**p.forward(), **p.backward()}
    state, y = p.state[:1].clone(), p.new(1, 3, 64)
    B.laplex_decay_attention_step(*one, dev(p.rates), state, y, p.scale)
    fine.update(step=fine_y, step_state=fine_state)
    odd.update(step=y, step_state=state)
    for name, t in odd.items():
        assert torch.isnan(t[:, 1]).all(), name
        assert torch.equal(t[:, [0, 2]], fine[name][:, [0, 2]]), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length", [16, 32, 64, 96, 192, 2048])
def test_nothing_is_left_of_a_state_whose_decay_is_zero(dtype, length):
    """Rates from which exp(-rate) is 0, and 0 over a chunk: of the largest states nothing reaches the tokens behind the first, or the last state."""
    p = Problem([length], 3, 64, 64, dtype, False, rates=[np.inf, 200.0, 1e6], what="zero")
    p.k.zero_(), p.v.zero_()
    p.q.fill_(1.0 / 128.0)                # (q S0 itself has to fit fp32)
    p.state.fill_(3e38)
    got = p.forward()
    assert (got["y"] == 0).all() and (got["state"] == 0).all()


# --- scales --------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[50, 9], [700]])
@pytest.mark.parametrize("scale,size", [(1e-39, 1.0), (1e-38, 1.0), (1e-30, 1e-3), (1e-10, 1e30), (1e-3, 1e35), (2.0 ** -41, 5.0), (1e20, 1e10)])
def test_gradients_of_states_beside_small_and_large_scales(dtype, lengths, scale, size):
    """The gradients are sums of a part that is weighted by the scale and one that is not: neither is lost or infinite for the other's sake."""
    p = Problem(lengths, 2, 48, 40, dtype, True, scale=scale, what="scales")
    p.gstate *= size
    for name, got, want, terms, n in p.each(p.backward()):
        exact = 16 * np.sqrt(n + 112.0) * U * terms + 2.0 ** -126          # (2^-126: results and decayed weights below the smallest normal number have fewer bits)
        within(name, got, want, exact if dtype == F32 or "state" in name else exact + 2.0 ** -14 * terms + 1.01 * H * np.abs(want))


# --- values that are not finite ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv", [(64, 64), (150, 200), (48, 256), (256, 256)])
@pytest.mark.parametrize("lengths,at", [([20, 25, 9], 33), ([100, 900, 40], 500), ([100, 900, 40], 999)])
@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
def test_attention_values_that_are_not_finite_show_and_stay_where_they_reach(dtype, dk, dv, lengths, at, value):
    """One number of one token of the middle sequence, a short one or one in several stretches.  What it is weighted into is not finite, everything else the same bits."""
    p = Problem(lengths, 2, dk, dv, dtype, True, rates=[0.01, 0.03], what="odd")
    first, end, col = lengths[0], lengths[0] + lengths[1], 21
    fine = {**p.forward(), **p.backward()}
    # (result, its rows, its columns) that the number reaches
    every, before, behind = slice(None), slice(first, at + 1), slice(at, end)
    reach = {
        "q": [("y", slice(at, at + 1), every), ("gk", before, col), ("gv", before, every)],
        "k": [("y", behind, every), ("gq", behind, col), ("gv", slice(at, at + 1), every)],
        "v": [("y", behind, col), ("gq", behind, every), ("gk", slice(at, at + 1), every)],
        "gy": [("gq", slice(at, at + 1), every), ("gk", before, every), ("gv", before, col)],
    }
    states = {"q": ("gstate", col, every), "k": ("state", col, every), "v": ("state", every, col), "gy": ("gstate", every, col)}
    for what in reach:
        t = getattr(p, what)
        kept = t[at, 1, col].clone()
        t[at, 1, col] = value
        odd = {**p.forward(), **p.backward()}
        t[at, 1, col] = kept
        for name, rows, columns in reach[what]:
            assert not torch.isfinite(odd[name][rows, 1, columns]).any(), f"{what}: {name}"
            odd[name][rows, 1, columns] = fine[name][rows, 1, columns]
        name, rows, columns = states[what]
        assert not torch.isfinite(odd[name][1, 1, rows, columns]).any(), f"{what}: {name}"
        odd[name][1, 1, rows, columns] = fine[name][1, 1, rows, columns]
        for name, t in odd.items():
            assert torch.equal(t, fine[name]), f"{what}: {name}"
