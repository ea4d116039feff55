"""Linear attention by the gated delta rule against the oracle in 64 bits, token by token; sizes, lengths, heads and values where it can go wrong.

Tolerances.  U = 2^-24 and H = 2^-8 are half a step of fp32 and bf16.  With keys of length 1 and beta from 0 to 1 a token's update is a contraction: what is rounded at one token is not enlarged
by the following ones.  So the errors of a column of the state are those of sums over up to n tokens and dk numbers, with roundings of either sign, of products of
the sizes that the oracle gives: e = 16 sqrt(n + dk + dv + 64) U of the column's size.  A result is a sum of dk of them with a query: e times the query's length; gradients likewise, with
the sizes of the state's gradient.  The gradient of a rate is a sum of up to 64 tokens' terms, six each, with signs: 64 e.  In bf16 results are rounded once (H), and what
enters products of them is carried in 16 bits at least: 2^-15 of the same sizes; states and the gradients of rates, beta and states are fp32 sums whatever the type.
"""
import copy

import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")
NAMES = ("gq", "gk", "gv", "grates", "gbeta", "g0")


def seeded(*what):
    import zlib
    return np.random.default_rng(zlib.crc32(repr(what).encode()))


def dev(v, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(v)).to("cuda").to(dtype)


def host(t):
    return t.double().cpu().numpy()


def within(name, got, want, bound):
    assert got.shape == want.shape, name
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: "
                           f"{got[bad][0]} instead of {want[bad][0]}, may be off by {np.broadcast_to(bound, bad.shape)[bad][0]}")


class Case:
    """Sequences one behind the other; q, k, v inside one matrix, rates and beta inside another, as projections leave them."""

    def __init__(self, r, lengths, heads, key_heads, dk, dv, dtype=F32, states=True, packed=True, read=None, slow=False):
        n, b = int(sum(lengths)), len(lengths)
        self.lengths, self.heads, self.key_heads, self.dk, self.dv, self.dtype, self.packed = list(lengths), heads, key_heads, dk, dv, dtype, packed
        self.n, self.b = n, b
        unit = lambda m: m / np.sqrt((m ** 2).sum(-1, keepdims=True))
        parts = [unit(r.normal(size=(n, key_heads, dk))), unit(r.normal(size=(n, key_heads, dk))), r.normal(size=(n, heads, dv))]
        m = torch.empty(n, 2 * key_heads * dk + heads * dv + 3, device="cuda", dtype=dtype)
        self.q, self.k, self.v = self.split(m, dtype)
        for t, p in zip((self.q, self.k, self.v), parts):
            t.copy_(dev(p, dtype))
        small = torch.empty(n, 2 * heads + 1, device="cuda")
        self.rates, self.beta = small[:, :heads], small[:, heads:2 * heads]
        self.rates.copy_(dev(np.exp(r.uniform(-14 if slow else -8, -5 if slow else 1, size=(n, heads)))))
        self.beta.copy_(dev(1.0 / (1.0 + np.exp(-r.normal(size=(n, heads))))))
        self.state = dev(r.normal(size=(b, heads, dk, dv))) if states else None
        self.gy = dev(r.normal(size=(n, heads, dv)), dtype)
        self.gstate = dev(r.normal(size=(b, heads, dk, dv))) if states else None
        self.scale = float(np.float32(dk ** -0.5))
        self.read = None if read is None else dev(np.array(read), torch.int64)
        self.starts = dev(np.concatenate([[0], np.cumsum(lengths)]), torch.int64) if packed else None

    def split(self, m, dtype):
        kh, h, dk, dv = self.key_heads, self.heads, self.dk, self.dv
        return (m[:, :kh * dk].unflatten(1, (kh, dk)), m[:, kh * dk:2 * kh * dk].unflatten(1, (kh, dk)), m[:, 2 * kh * dk:2 * kh * dk + h * dv].unflatten(1, (h, dv)))

    def workspace(self, training=True):
        return torch.empty(max(1, B.laplex_delta_attention_workspace_bytes(self.dtype, self.n, self.b, self.heads, self.key_heads, self.dk, self.dv, training)),
                           dtype=torch.uint8, device="cuda")

    def forward(self, ws=None, flags=0, state_out=True, state=0):
        y = torch.full((self.n, self.heads, self.dv), NAN, device="cuda", dtype=self.dtype)
        last = torch.full((self.b, self.heads, self.dk, self.dv), NAN, device="cuda") if state_out else None
        B.laplex_delta_attention(self.q, self.k, self.v, self.rates, self.beta, y, self.workspace(bool(flags)) if ws is None else ws, self.scale, self.b, self.starts, self.read,
                                 self.state if isinstance(state, int) else state, last, flags)
        return y, last

    def new_gradients(self):
        m = torch.full((self.n, 2 * self.key_heads * self.dk + self.heads * self.dv + 3), NAN, device="cuda", dtype=self.dtype)
        small = torch.full((self.n, 2 * self.heads + 1), NAN, device="cuda")
        return [*self.split(m, self.dtype), small[:, :self.heads], small[:, self.heads:2 * self.heads],
                torch.full((self.b, self.heads, self.dk, self.dv), NAN, device="cuda")]

    def backward(self, ws=None, flags=0, g=None):
        g = self.new_gradients() if g is None else g
        B.laplex_delta_attention_backward(self.q, self.k, self.v, self.rates, self.beta, self.gy, *g[:5], self.workspace() if ws is None else ws, self.scale, self.b, self.starts,
                                          self.read, self.state, self.gstate, g[5], flags)
        return g

    def sequences(self):
        """(sequence, first row, rows that are read, rows)"""
        at = 0
        for i, n in enumerate(self.lengths):
            yield i, at, n if self.read is None else max(0, min(n, int(self.read[i]))), n
            at += n

    def of(self, i, at, m, h):
        kh = h // (self.heads // self.key_heads)
        return (host(self.q[at:at + m, kh]), host(self.k[at:at + m, kh]), host(self.v[at:at + m, h]), host(self.rates[at:at + m, h]), host(self.beta[at:at + m, h]),
                self.scale, None if self.state is None else host(self.state[i, h]))

    def e(self, m):
        return 16 * np.sqrt(m + self.dk + self.dv + 64.0) * U

    def check_forward(self, y, last, heads=None):
        some, h16 = (2.0 ** -15, H) if self.dtype == BF16 else (0.0, 0.0)
        for i, at, m, n in self.sequences():
            for h in range(self.heads) if heads is None else heads:
                args = self.of(i, at, m, h)
                wy, ws, size = O.delta_sequence(*args)
                query = self.scale * np.sqrt((args[0] ** 2).sum(-1))[:, None]
                within(f"y[{i},{h}]", host(y[at:at + m, h]), wy, (self.e(m) + some) * query * size + 1.01 * h16 * np.abs(wy))
                if last is not None:
                    within(f"state[{i},{h}]", host(last[i, h]), ws, self.e(m) * size)
            assert bool(torch.isnan(y[at + m:at + n]).all())          # rows that are not read: as they were

    def check_backward(self, g):
        some, h16 = (2.0 ** -15, H) if self.dtype == BF16 else (0.0, 0.0)
        group = self.heads // self.key_heads
        for i, at, m, n in self.sequences():
            for kh in range(self.key_heads):
                gq, gk, bq, bk = 0.0, 0.0, 0.0, 0.0
                for h in range(kh * group, (kh + 1) * group):
                    args = self.of(i, at, m, h)
                    gy = host(self.gy[at:at + m, h])
                    _, _, size = O.delta_sequence(*args)
                    want, gsize = O.delta_sequence_backward(*args, gy, None if self.gstate is None else host(self.gstate[i, h]))
                    e, beta = self.e(m), args[4][:, None]
                    S, G, yl = np.sqrt((size ** 2).sum()), np.sqrt((gsize ** 2).sum()), np.sqrt((gy ** 2).sum(-1))[:, None]
                    gq, gk = gq + want[0], gk + want[1]
                    bq, bk = bq + (e + some) * self.scale * yl * S, bk + (e + some) * 3 * S * (G + self.scale * yl)
                    at_h = lambda t: host(t[at:at + m, h])
                    within(f"gv[{i},{h}]", at_h(g[2]), want[2], (e + some) * beta * gsize + 1.01 * h16 * np.abs(want[2]))
                    within(f"grates[{i},{h}]", at_h(g[3]), want[3], 64 * e * S * (G + (self.scale * yl.max() if m else 0.0)))
                    within(f"gbeta[{i},{h}]", at_h(g[4]), want[4], 4 * e * G * (S + np.sqrt((args[2] ** 2).sum(-1))))
                    within(f"g0[{i},{h}]", host(g[5][i, h]), want[5], e * 2 * gsize)
                within(f"gq[{i},{kh}]", host(g[0][at:at + m, kh]), gq if m else np.zeros((0, self.dk)), bq + 1.01 * h16 * np.abs(gq))
                within(f"gk[{i},{kh}]", host(g[1][at:at + m, kh]), gk if m else np.zeros((0, self.dk)), bk + 1.01 * h16 * np.abs(gk))
            for t in g[:5]:
                assert bool(torch.isnan(t[at + m:at + n]).all())


SHAPES = [
    # lengths, heads, key heads, dk, dv, packed
    ([1], 1, 1, 1, 1, False), ([1, 1, 1], 2, 1, 16, 16, False), ([5], 3, 3, 7, 9, False), ([16], 1, 1, 32, 32, False), ([17, 0, 1, 64, 65], 2, 2, 20, 33, True),
    ([63], 2, 1, 64, 64, False), ([64, 64], 2, 2, 64, 64, False), ([130], 1, 1, 128, 128, False), ([200, 3, 0, 0, 129], 4, 2, 96, 80, True),
    ([150], 1, 1, 256, 256, False), ([70], 2, 1, 256, 40, False), ([95], 1, 1, 40, 256, False), ([0, 0], 2, 2, 8, 8, True), ([400, 213], 1, 1, 48, 100, True),
    ([97, 65], 2, 2, 129, 65, True), ([33, 100], 3, 1, 192, 150, True), ([32, 31, 15, 16, 48], 2, 2, 128, 96, True), ([700], 2, 1, 64, 128, False), ([12, 12, 12], 4, 2, 128, 128, False), ([13, 13], 2, 2, 128, 128, False), ([9] * 3, 2, 1, 256, 33, False), ([11], 1, 1, 100, 256, False),
    ([10] * 70, 4, 4, 64, 64, False),
    ([40, 0], 2, 1, 32, 48, True), ([0, 130, 0, 0], 2, 2, 64, 64, True), ([2100, 0, 0], 1, 1, 64, 64, True),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv,packed", SHAPES)
@pytest.mark.parametrize("states", [False, True])
def test_delta(dtype, lengths, heads, key_heads, dk, dv, packed, states):
    c = Case(seeded("delta", lengths, heads, dk, dv), lengths, heads, key_heads, dk, dv, dtype, states, packed)
    c.check_forward(*c.forward())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv,packed", SHAPES)
@pytest.mark.parametrize("states", [False, True])
def test_delta_backward(dtype, lengths, heads, key_heads, dk, dv, packed, states):
    c = Case(seeded("delta backward", lengths, heads, dk, dv), lengths, heads, key_heads, dk, dv, dtype, states, packed)
    g = c.backward()
    c.check_backward(g)
    # what a forward call has kept gives the same bits, and so does leaving gradients out
    ws = c.workspace()
    y, last = c.forward(ws, B.LAPLEX_SAVE_SCANS)
    c.check_forward(y, last)
    for t, full in zip(c.backward(ws, B.LAPLEX_SAVE_SCANS), g):
        assert torch.equal(t.nan_to_num(), full.nan_to_num())
    for left in range(6):
        some = c.backward(g=[None if i == left else t for i, t in enumerate(c.new_gradients())])
        for t, full in zip(some, g):
            assert t is None or torch.equal(t.nan_to_num(), full.nan_to_num())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("packed", [False, True])
def test_only_the_first_tokens_are_read(dtype, packed):
    r = seeded("lengths")
    c = Case(r, [70] * 6, 2, 1, 32, 48, dtype, packed=packed, read=[0, 1, 64, 65, 700, -3])
    c.check_forward(*c.forward())
    c.check_backward(c.backward())
    short = Case(r, [5] * 7, 4, 2, 64, 64, dtype, packed=packed, read=[0, 1, 2, 3, 4, 5, 9])
    short.check_forward(*short.forward())
    short.check_backward(short.backward())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sequences,heads,key_heads,dk,dv", [(1, 1, 1, 1, 1), (1, 16, 8, 128, 128), (3, 2, 2, 20, 33), (5, 1, 1, 256, 256), (70, 8, 4, 64, 64), (2, 3, 1, 96, 80), (9, 2, 2, 129, 130),
                                                             (600, 1, 1, 32, 40)])
def test_step(dtype, sequences, heads, key_heads, dk, dv):
    c = Case(seeded("step", sequences, heads, dk, dv), [1] * sequences, heads, key_heads, dk, dv, dtype, packed=False)
    state, y = c.state.clone(), torch.full((sequences, heads, dv), NAN, device="cuda", dtype=dtype)
    B.laplex_delta_attention_step(c.q, c.k, c.v, c.rates, c.beta, state, y, c.scale)
    c.check_forward(y, state)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_then_steps_and_drafts_is_the_longer_prompt(dtype):
    """A state handed from a prompt to steps, to some of a few drafted tokens, and to a second prompt (in place) ends where one prompt over all tokens ends."""
    r = seeded("hand over")
    first, steps, drafts, second = 133, 3, 4, 70
    n = first + steps + drafts + second
    c = Case(r, [n], 2, 1, 48, 64, dtype, states=False, packed=False)
    y, last = c.forward()
    state, got = torch.empty(1, 2, 48, 64, device="cuda"), torch.full_like(y, NAN)
    ws = c.workspace(False)
    cut = lambda a, b: [t[a:b] for t in (c.q, c.k, c.v, c.rates, c.beta)]
    B.laplex_delta_attention(*cut(0, first), got[:first], ws, c.scale, state_out=state)
    for t in range(first, first + steps):
        B.laplex_delta_attention_step(*cut(t, t + 1), state, got[t:t + 1], c.scale)
    at = first + steps
    # two of the drafts, then the other two
    B.laplex_delta_attention(*cut(at, at + drafts), got[at:at + drafts], ws, c.scale, lengths=dev([2], torch.int64), state_in=state, state_out=state)
    assert bool(torch.isnan(got[at + 2:at + drafts]).all())
    B.laplex_delta_attention(*cut(at + 2, at + drafts), got[at + 2:at + drafts], ws, c.scale, state_in=state, state_out=state)
    B.laplex_delta_attention(*cut(at + drafts, n), got[at + drafts:], ws, c.scale, state_in=state, state_out=state)
    c.check_forward(got, state)
    c.check_forward(y, last)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[3000], [1, 0, 2000, 700, 2, 300]])
def test_long_sequences_with_slow_decays(dtype, lengths):
    """Rates of 1e-6 to 7e-3: states that hold thousands of tokens; the state in place; relative errors over all."""
    c = Case(seeded("slow", lengths), lengths, 2, 2, 64, 64, dtype, slow=True)
    y, last = c.forward()
    c.check_forward(y, last)
    g = c.backward()
    c.check_backward(g)
    same, z = c.state.clone(), torch.full_like(y, NAN)
    B.laplex_delta_attention(c.q, c.k, c.v, c.rates, c.beta, z, c.workspace(False), c.scale, c.b, c.starts, None, same, same)
    assert torch.equal(z, y) and torch.equal(same, last)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rates_and_weights_at_their_ends(dtype):
    """Rates of 0, of 200, 1e5, 1e30 and infinite ones; weights of 0 and 1; the same key again and again."""
    r = seeded("ends")
    c = Case(r, [150, 40], 3, 3, 32, 48, dtype)
    c.rates[:, 0] = 0.0
    c.rates[::7, 1] = INF
    c.rates[3::7, 1] = 1e30
    c.rates[5::11, 2] = 200.0
    c.rates[6::11, 2] = 1e5
    c.beta[:, 0] = 1.0
    c.beta[::3, 1] = 0.0
    c.k[20:90] = c.k[20].clone()
    y, last = c.forward()
    c.check_forward(y, last)
    g = c.backward()
    keep, c.rates = c.rates, c.rates.clamp(max=1e30)
    c.check_backward(g)
    # a token at a time
    c = Case(r, [1] * 6, 3, 3, 32, 48, dtype, packed=False)
    c.rates[:, 0], c.rates[::2, 1], c.beta[:, 2] = 0.0, INF, 0.0
    state, z = c.state.clone(), torch.empty(6, 3, 48, device="cuda", dtype=dtype)
    B.laplex_delta_attention_step(c.q, c.k, c.v, c.rates, c.beta, state, z, c.scale)
    c.check_forward(z, state)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("what", ["q", "k", "v", "rates", "beta"])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("lengths,packed", [([100, 90, 40], True), ([8] * 30, False)])
def test_values_that_are_not_finite_stay_behind_their_token(dtype, what, value, lengths, packed):
    """Rows before the token, other sequences and other heads are the same bits as without it."""
    if what == "rates" and value == INF:
        pytest.skip("nothing is left of the state: a number like others")
    c = Case(seeded("odd", what), lengths, 2, 2, 64, 64, dtype, packed=packed)
    y, last = c.forward()
    sequence = 1
    at = int(sum(lengths[:sequence])) + (37 if packed else 5)
    t = getattr(c, what)
    if what in ("rates", "beta"):
        t[at, 1] = value
    else:
        t[at, 1, 21] = value
    z, last2 = c.forward()
    end = int(sum(lengths[:sequence + 1]))
    assert torch.equal(z[:at], y[:at]) and torch.equal(z[end:], y[end:]) and torch.equal(z[:, 0], y[:, 0])
    assert not bool(torch.isfinite(z[at, 1]).all())
    others = [i for i in range(c.b) if i != sequence]
    assert torch.equal(last2[others], last[others]) and torch.equal(last2[:, 0], last[:, 0])
    if what == "q":
        assert torch.equal(z[at + 1:], y[at + 1:]) and torch.equal(last2, last)
    else:
        assert not bool(torch.isfinite(last2[sequence, 1]).all())
    g = c.backward()
    for got in g[:5]:
        assert bool(torch.isfinite(got[:int(sum(lengths[:sequence]))]).all()) and bool(torch.isfinite(got[end:]).all()) and bool(torch.isfinite(got[:, 0]).all())


@pytest.mark.parametrize("starts", [[0, 90, 40, 200, 230], [50, 50, 50, 50, 50], [-30, 1000, 1 << 40, 70, 230], [230, 200, 100, 50, 0]])
def test_starts_out_of_order_touch_nothing_else(starts):
    c = Case(seeded("bad starts"), [60, 60, 60, 50], 2, 1, 32, 32, BF16)
    c.starts = dev(np.array(starts), torch.int64)
    c.forward()
    c.backward()
    torch.cuda.synchronize()


def test_rows_aligned_to_nothing():
    """Matrices whose rows lie any number of numbers apart and begin anywhere give the bits of whole ones."""
    r = seeded("unaligned")
    for dtype in (F32, BF16):
        c = Case(r, [77, 64, 3], 2, 1, 64, 128, dtype)
        y, last = c.forward()
        g = c.backward()
        for off in (1, 2, 3):
            m = torch.zeros(c.n, 2 * 64 + 2 * 128 + 7, device="cuda", dtype=dtype)[:, off:]
            parts = c.split(m, dtype)
            for to, t in zip(parts, (c.q, c.k, c.v)):
                to.copy_(t)
            kept, (c.q, c.k, c.v) = (c.q, c.k, c.v), parts
            y2, last2 = c.forward()
            assert torch.equal(y2, y) and torch.equal(last2, last)
            for a, b in zip(c.backward(), g):
                assert torch.equal(a, b)
            c.q, c.k, c.v = kept


def test_captured_and_replayed():
    """A training step's two calls in a graph, replayed between eager calls with a workspace of their own."""
    r = seeded("graph")
    c = Case(r, [200, 100, 0, 57], 4, 2, 64, 64, BF16)
    ws, g, y, last = c.workspace(), c.new_gradients(), torch.zeros(c.n, 4, 64, device="cuda", dtype=BF16), torch.zeros(c.b, 4, 64, 64, device="cuda")
    short = Case(r, [4] * 9, 4, 2, 64, 64, BF16, packed=False, read=[1, 2, 3, 4, 0, 1, 2, 3, 4])
    ws2, y2, last2 = short.workspace(False), torch.zeros(36, 4, 64, device="cuda", dtype=BF16), torch.zeros(9, 4, 64, 64, device="cuda")

    def call():
        B.laplex_delta_attention(c.q, c.k, c.v, c.rates, c.beta, y, ws, c.scale, c.b, c.starts, None, c.state, last, B.LAPLEX_SAVE_SCANS)
        c.backward(ws, B.LAPLEX_SAVE_SCANS, g)
        B.laplex_delta_attention(short.q, short.k, short.v, short.rates, short.beta, y2, ws2, short.scale, 9, None, short.read, short.state, last2)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        c.v.copy_(dev(r.normal(size=c.v.shape), BF16))
        short.v.copy_(dev(r.normal(size=short.v.shape), BF16))
        want, want_last = c.forward()
        want_g = c.backward()
        want2, want_last2 = short.forward()
        y.zero_(), last.zero_(), y2.zero_(), last2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(last, want_last) and torch.equal(last2, want_last2) and torch.equal(y2, want2.nan_to_num())
        for a, b in zip(g, want_g):
            assert torch.equal(a, b)


def test_two_calls_at_once():
    """On two streams, with a workspace each."""
    r = seeded("streams")
    cases = [Case(r, [300, 41], 4, 2, 64, 64, BF16), Case(r, [129, 300, 7], 4, 4, 64, 64, BF16)]
    want = [c.forward() + tuple(c.backward()) for c in cases]
    spaces = [c.workspace() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i] = c.forward(spaces[i], B.LAPLEX_SAVE_SCANS) + tuple(c.backward(spaces[i], B.LAPLEX_SAVE_SCANS))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv,packed,read", [
    ([2600], 2, 1, 64, 64, False, None), ([1, 2000, 0, 900], 4, 2, 96, 80, True, None), ([1500, 1500], 2, 2, 20, 130, False, None), ([1300], 1, 1, 200, 256, False, None),
    ([1100, 1100, 1100], 2, 2, 48, 48, False, [1100, 77, 1027]), ([40, 1500, 30, 2000], 2, 2, 128, 128, True, [40, 1501, 7, 1025]), ([769, 5, 1025], 1, 1, 256, 64, True, None),
    ([384, 385, 768, 769], 2, 1, 64, 48, True, None), ([769, 769], 2, 2, 32, 64, False, [768, 769])])
def test_sequences_in_stretches(dtype, lengths, heads, key_heads, dk, dv, packed, read):
    """Sequences that are cut, with lengths that end inside, at and behind the edges of stretches; the state in place."""
    c = Case(seeded("stretches", lengths, heads, dk, dv), lengths, heads, key_heads, dk, dv, dtype, True, packed, read)
    y, last = c.forward()
    c.check_forward(y, last, [heads - 1])
    ws = c.workspace()
    z, last2 = c.forward(ws, B.LAPLEX_SAVE_SCANS)
    assert torch.equal(z.nan_to_num(), y.nan_to_num()) and torch.equal(last2, last)
    g = c.backward(ws, B.LAPLEX_SAVE_SCANS)
    c.check_backward(g)
    for a, b in zip(c.backward(), g):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())
    same = c.state.clone()
    B.laplex_delta_attention(c.q, c.k, c.v, c.rates, c.beta, z, c.workspace(False), c.scale, c.b, c.starts, c.read, same, same)
    assert torch.equal(z.nan_to_num(), y.nan_to_num()) and torch.equal(same, last)

@pytest.mark.parametrize("dtype", [F32, BF16])
def test_growing_states_of_a_few_numbers(dtype):
    """Rates below 0 in sequences that are cut: e^0.045 a token is e^92 over a stretch of 2048 tokens, more than fp32 holds, while keys of one number and weights near 1 take a tenth of the
    state from token to token.  What lies beside that number of a key, as far as tiles are padded, may not grow.  A chunk's maps hold factors of up to exp(63 * 0.045) = 17, which
    enlarge its roundings."""
    c = Case(seeded("growing"), [8192], 64, 64, 1, 24, dtype, packed=False)
    c.rates.fill_(-0.045)
    c.beta.fill_(0.9)
    one = copy.copy(c)                                          # the last head by itself
    one.heads = one.key_heads = 1
    for name in ("q", "k", "v", "rates", "beta", "gy"):
        setattr(one, name, getattr(c, name)[:, -1:])
    one.state, one.gstate = c.state[:, -1:], c.gstate[:, -1:]
    one.e = lambda m: 17 * Case.e(one, m)
    ws = c.workspace()
    y, last = c.forward(ws, B.LAPLEX_SAVE_SCANS)
    g = c.backward(ws, B.LAPLEX_SAVE_SCANS)
    assert all(bool(torch.isfinite(t).all()) for t in (y, last, *g))
    one.check_forward(y[:, -1:], last[:, -1:])
    one.check_backward([t[:, -1:] for t in g])
