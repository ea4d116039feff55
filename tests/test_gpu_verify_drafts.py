"""Verification of drafted tokens against the oracle: whole numbers are equal (everything that is compared is in 64 bits on both sides; chances that lie
within 1e-11 of a border would be the exception, and there are none among these), log probabilities are off by one fp32 rounding and the 64-bit
sums' errors: 2^-24 (|logp| + 1)."""
import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def seeded(*what):
    import zlib
    return np.random.default_rng(zlib.crc32(repr(what).encode()))


def dev(v, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(v)).to("cuda").to(dtype)


def host(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, r, k, lengths, dtype=F32, logits=True, near=0.5, spread=2.0, packed=True, pad=0):
        t = int(sum(lengths))
        self.k, self.lengths, self.packed, self.b = k, lengths, packed, len(lengths)
        z = spread * r.normal(size=(k, t + pad))
        y = z + near * r.normal(size=(k, t + pad))
        self.y = dev(y, dtype)[:, :t]
        self.z = dev(z, dtype)[:, :t] if logits else None
        noise = -np.log(-np.log(r.random((k, t)).clip(1e-300, 1.0 - 1e-16)))
        source = host(self.z if logits else self.y)
        drafts = (source + noise).argmax(0) if t else np.zeros(0, np.int64)
        drafts[r.random(t) < 0.04] = -1
        drafts[r.random(t) < 0.02] = k
        self.drafts = dev(drafts, torch.int64)
        self.chances, self.next_chances = dev(r.random(t), torch.float64), dev(r.random(self.b), torch.float64)

    @property
    def starts(self):
        return np.concatenate([[0], np.cumsum(self.lengths)]).astype(np.int64)

    def run(self, tau=1.0, draft_tau=1.0, greedy=False, log=True):
        t = self.y.shape[1]
        ws = torch.empty(max(1, B.laplex_verify_workspace_bytes(self.k, t, self.b)), dtype=torch.uint8, device="cuda")
        accepted, following = torch.full((self.b,), -7, device="cuda"), torch.full((self.b,), -7, device="cuda")
        logp, next_logp = (torch.full((n,), NAN, device="cuda") for n in (t, self.b)) if log else (None, None)
        B.laplex_verify_drafts(self.y, None if greedy else self.z, self.drafts, None if greedy else self.chances, None if greedy else self.next_chances, accepted,
                               following, ws, logp, next_logp, tau, draft_tau, self.b, dev(self.starts, torch.int64) if self.packed else None,
                               B.LAPLEX_VERIFY_GREEDY if greedy else 0)
        return accepted, following, logp, next_logp

    def check(self, tau=1.0, draft_tau=1.0, greedy=False):
        accepted, following, logp, next_logp = self.run(tau, draft_tau, greedy)
        of = lambda v: float(np.float32(v))
        want = O.verify_drafts(host(self.y), None if self.z is None or greedy else host(self.z), host(self.drafts).astype(np.int64), self.starts, of(tau), of(draft_tau),
                               host(self.chances), host(self.next_chances), greedy)
        assert accepted.tolist() == want[0].tolist()
        assert following.tolist() == want[1].tolist()
        for got, w in ((host(logp), want[2]), (host(next_logp), want[3])):
            # (results are fp32 numbers: what is below -(2 - 2^-24) 2^127, half a step beyond the last one, rounds to -inf)
            w = np.where(w <= -(2.0 - 2.0 ** -24) * 2.0 ** 127, -INF, w)
            assert np.array_equal(np.isnan(got), np.isnan(w)) and np.array_equal(np.isinf(got), np.isinf(w))
            f = np.isfinite(w)
            assert (np.abs(got - w)[f] <= U * (np.abs(w[f]) + 1.0)).all()
        return want


SHAPES = [(1, [1]), (1, [3, 2]), (2, [1, 2]), (7, [5]), (10, [1] * 9), (33, [4, 0, 1, 9, 0, 2]), (300, [2, 7, 3, 1]), (1000, [5] * 40), (2049, [3] * 23),
          (5000, [17, 1, 300, 0, 4]), (32000, [5]), (513, [4] * 300), (70001, [2, 3])]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rule", ["logits", "sure", "greedy"])
@pytest.mark.parametrize("k,lengths", SHAPES)
def test_verify(dtype, rule, k, lengths):
    r = seeded("verify", k, lengths, rule)
    c = Case(r, k, lengths, dtype, rule == "logits", packed=len(set(lengths)) > 1)
    if rule == "greedy":
        best = c.y.argmax(0)
        c.drafts = torch.where(dev(r.random(len(best))) < 0.7, best, c.drafts)
    c.check(0.9, 1.1, rule == "greedy")
    c.check(greedy=rule == "greedy")


def test_what_is_kept_is_kept_in_every_way():
    """All drafts kept, none kept, and something between, over many columns of one sequence."""
    r = seeded("ways")
    c = Case(r, 50, [700, 1, 300])
    c.drafts = c.y.argmax(0)
    c.chances.zero_()
    want = c.check()
    assert want[0].tolist() == [699, 0, 299]
    c.chances[600] = 1.0 - 2.0 ** -53
    c.z[:, 600] = -50.0
    c.z[int(c.drafts[600]), 600] = 50.0
    assert c.check()[0].tolist() == [600, 0, 299]
    c.chances.fill_(1.0 - 2.0 ** -53)
    c.check()


def test_emitted_tokens_have_the_target_distribution():
    """20000 sequences of one draft each over nine tokens: what is written first is distributed as the target says (five standard deviations)."""
    r = seeded("law")
    n, k = 20000, 9
    z, y = 1.5 * r.normal(size=k), 1.5 * r.normal(size=k)
    p, q = (np.exp(v - v.max()) / np.exp(v - v.max()).sum() for v in (y, z))
    for logits in (True, False):
        c = Case(r, k, [2] * n, F32, logits, packed=False)
        c.y = dev(np.repeat(y[:, None], 2 * n, 1))
        if logits:
            c.z = dev(np.repeat(z[:, None], 2 * n, 1))
        c.drafts = dev(r.choice(k, size=2 * n, p=q) if logits else np.full(2 * n, 4), torch.int64)
        accepted, following, _, _ = c.run()
        first = torch.where(accepted > 0, c.drafts[::2], following)
        share = np.bincount(first.cpu().numpy(), minlength=k) / n
        assert (np.abs(share - p) < 5 * np.sqrt(p * (1 - p) / n)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rule", ["logits", "sure", "greedy"])
def test_masks_and_values_that_are_not_finite(dtype, rule):
    r = seeded("masks", rule)
    c = Case(r, 400, [4] * 30, dtype, rule == "logits", packed=False)
    c.y[dev(r.random((400, 120))) < 0.3] = -INF
    c.y[:, 5] = -INF                                           # no distribution
    c.y[17, 20] = NAN
    c.y[18, 33] = INF
    c.y[:, 44] = -INF
    c.y[9, 44] = 1.0                                           # one token alone
    c.y[:, 49] = torch.finfo(dtype).min                        # the type's lowest value everywhere: all alike
    c.y[:200, 53] = torch.finfo(dtype).min
    if c.z is not None:
        c.z[:, 60] = -INF
        c.z[3, 65] = NAN
        c.z[4, 70] = INF
        c.z[:, 73] = torch.finfo(dtype).min
    if rule == "greedy":
        c.drafts = torch.where(dev(r.random(120)) < 0.7, c.y.nan_to_num(nan=-9.0).argmax(0), c.drafts)
    want = c.check(greedy=rule == "greedy")
    assert want[1][1] == -1 or want[0][1] == 0
    c.check(3.0, 0.5, rule == "greedy")


def test_equal_logits_go_to_the_lowest_row():
    r = seeded("ties")
    c = Case(r, 900, [3] * 20, packed=False)
    c.y = dev(np.round(host(c.y)))
    c.y[::3] = 9.0
    c.y[0] = -INF
    c.drafts = torch.full_like(c.drafts, 3)
    assert c.check(greedy=True)[1].tolist() == [3] * 20
    c.y.zero_()
    c.y.mul_(-1.0)                                             # -0 and +0 are equal
    c.y[5:] = 0.0
    c.drafts.fill_(1)
    assert c.check(greedy=True)[1].tolist() == [0] * 20


def test_columns_apart_and_results_not_asked_for():
    """Columns inside a wider matrix; without log probabilities the same tokens."""
    r = seeded("apart")
    c = Case(r, 777, [4] * 33, pad=9, packed=False)
    c.check()
    accepted, following, _, _ = c.run()
    a2, f2, _, _ = c.run(log=False)
    assert torch.equal(accepted, a2) and torch.equal(following, f2)


def test_equal_distributions_keep_every_draft():
    r = seeded("same")
    c = Case(r, 1000, [6] * 50, near=0.0, packed=False)
    c.drafts = c.drafts.clamp(0, 999)
    assert c.check()[0].tolist() == [5] * 50


def test_no_columns():
    c = Case(seeded("none"), 10, [0, 0, 0])
    c.check()


@pytest.mark.parametrize("starts", [[0, 9, 4, 20, 31], [5, 5, 5, 5, 5], [-3, 100, 1 << 40, 7, 31], [31, 20, 10, 5, 0]])
def test_starts_out_of_order_touch_nothing_else(starts):
    r = seeded("bad starts")
    c = Case(r, 60, [8, 8, 8, 7])
    ws = torch.empty(B.laplex_verify_workspace_bytes(60, 31, 4), dtype=torch.uint8, device="cuda")
    out = torch.full((4 + 8,), -7, device="cuda")
    B.laplex_verify_drafts(c.y, c.z, c.drafts, c.chances, c.next_chances, out[:4], out[4:8], ws, sequences=4, starts=dev(np.array(starts), torch.int64))
    assert out[8:].tolist() == [-7] * 4 and ((out[4:8] >= -1) & (out[4:8] < 60)).all()


def test_chances_at_their_ends():
    """0 takes the first row that has any weight, the largest number below 1 the last."""
    r = seeded("ends")
    c = Case(r, 3000, [1] * 6, packed=False)
    c.y[:40] = -INF
    c.y[2900:] = -INF
    c.next_chances.zero_()
    assert c.check()[1].tolist() == [40] * 6
    c.next_chances.fill_(1.0 - 2.0 ** -53)
    _, following, _, _ = c.run()
    assert following.tolist() == [2899] * 6
    c.next_chances.fill_(NAN)
    assert ((c.run()[1] >= 40) & (c.run()[1] < 2900)).all()


def test_captured_and_replayed():
    r = seeded("graph")
    c = Case(r, 5000, [5] * 12, packed=False)
    ws = torch.empty(B.laplex_verify_workspace_bytes(5000, 60, 12), dtype=torch.uint8, device="cuda")
    accepted, following = torch.zeros(12, dtype=torch.int64, device="cuda"), torch.zeros(12, dtype=torch.int64, device="cuda")
    logp, next_logp = torch.zeros(60, device="cuda"), torch.zeros(12, device="cuda")
    call = lambda: B.laplex_verify_drafts(c.y, c.z, c.drafts, c.chances, c.next_chances, accepted, following, ws, logp, next_logp, 0.8, 1.0, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        c.chances.copy_(dev(r.random(60), torch.float64))
        c.next_chances.copy_(dev(r.random(12), torch.float64))
        want = c.run(0.8)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((accepted, following, logp, next_logp), want):
            assert torch.equal(got, w)

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rule", ["logits", "sure", "greedy"])
@pytest.mark.parametrize("size,tau", [(1.0, 1e6), (1.0, 1e9), (1.0, 1e20), (1.0, 1e38), (1e4, 1.0), (1e4, 1e6), (1e10, 1.0), (1e30, 1.0), (1e30, 1e38), (1e-30, 1e30), (1e-38, 1.0)])
def test_inverse_temperatures_and_logits_of_any_size(dtype, rule, size, tau):
    """Where a step of a logit is more than a probability can fall: the likeliest tokens alone have weight, equal ones the same."""
    r = seeded("any size", rule, size, tau)
    c = Case(r, 5000, [4, 1, 0, 7, 3], dtype, rule == "logits")
    for m in (c.y, c.z):
        if m is not None:
            m.mul_(size)
    c.y[dev(r.random((5000, 15))) < 0.05] = -INF               # banned entries
    c.y[:300, 3:6] = -INF
    c.y[7:9, 9] = 9.0 * size                                    # two likeliest tokens
    c.drafts = torch.where(dev(r.random(15)) < 0.6, c.y.argmax(0), c.drafts)
    want = c.check(tau, tau, rule == "greedy")
    assert (want[1][[0, 1, 3, 4]] >= 0).all()
    c.check(tau, 1.0, rule == "greedy")
    c.check(1.0, tau, rule == "greedy")

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,sequences", [(3000, 64), (3000, 3), (70000, 1)])
def test_certain_draft_that_is_alone_in_its_part_of_the_rows(dtype, k, sequences):
    """A refused draft with nothing but banned entries around it, before and behind all others: at either end of the chances the next token is the first or the last of the others."""
    r = seeded("alone", k, sequences)
    for at, chance in ((5, 0.0), (k - 9, 1.0 - 2.0 ** -53), (5, 0.5), (k - 9, 0.5)):
        c = Case(r, k, [2] * sequences, dtype, False, spread=1.0, packed=False)
        c.y[:600] = -INF
        c.y[k - 600:] = -INF
        c.y[at] = dev(r.normal(size=2 * sequences), dtype)
        c.drafts.fill_(at)
        c.chances.fill_(1.0 - 2.0 ** -53)
        c.next_chances.fill_(chance)
        want = c.check()
        assert not want[0].any() and ((want[1] >= 600) & (want[1] < k - 600)).all()
        assert chance == 0.5 or set(want[1]) == {600 if chance == 0.0 else k - 601}


@pytest.mark.parametrize("rule", ["sure", "none"])
def test_weights_at_the_end_of_the_numbers(rule):
    """A part of the rows whose weights are the smallest number there is, which a division by the sum of all takes away: some token of those that are not banned is drawn."""
    c = Case(seeded("smallest"), 4000, [2] * 40, F32, False, packed=False)
    c.y.fill_(-INF)
    c.y[:100] = -744.4                                          # e^-744.4 is 1.03 times 2^-1074
    c.y[2000:2008] = 0.0
    c.drafts.fill_(50 if rule == "sure" else -1)
    c.chances.fill_(1.0 - 2.0 ** -53)
    for chance in (0.0, 0.5, 1.0 - 2.0 ** -53):
        c.next_chances.fill_(chance)
        accepted, following, _, _ = c.run()
        some = following.cpu().numpy()
        assert not accepted.any() and (((some >= 0) & (some < 100)) | ((some >= 2000) & (some < 2008))).all()


def test_certain_draft_that_has_nearly_all_the_weight():
    """What the others weigh is formed from them: as the difference of two numbers near 1 it would be off by up to a tenth here."""
    r = seeded("nearly all")
    c = Case(r, 2500, [2] * 200, F32, False, spread=1.0, packed=False)
    c.y[1200] = 41.0                                            # the others: some 4000 e^-41 = 6e-15
    c.drafts.fill_(1200)
    c.chances.fill_(1.0 - 2.0 ** -53)
    assert not c.check()[0].any()

def test_entries_that_are_as_likely_under_both_are_never_drawn():
    """Target and drafts differ in two entries that have changed places: what is left of a refused draft is one of them alone, up to the last chance."""
    r = seeded("changed places")
    for k in (40, 3000, 20000):
        c = Case(r, k, [2] * 64, F32, spread=1.0, near=0.0, packed=False)
        c.y[0], c.y[1] = 1.0, 2.0
        c.z.copy_(c.y)
        c.z[0], c.z[1] = 2.0, 1.0
        c.drafts.fill_(0)
        c.chances.fill_(1.0 - 2.0 ** -53)
        for chance in (0.0, 0.5, 1.0 - 2.0 ** -53):
            c.next_chances.fill_(chance)
            accepted, following, _, _ = c.run(0.9, 0.9)
            assert not bool(accepted.any()) and following.tolist() == [1] * 64

@pytest.mark.parametrize("rule", ["logits", "sure", "greedy"])
def test_columns_of_no_sequence(rule):
    """Columns before the first sequence and behind the last one have no draft: their log probability is 0, whatever stood there; also where there is no sequence at all."""
    r = seeded("outside", rule)
    c = Case(r, 700, [12], F32, rule == "logits")
    for starts in ([2, 5, 5, 9], [0, 0], [12, 12, 12], [4]):
        b = len(starts) - 1
        ws = torch.empty(max(1, B.laplex_verify_workspace_bytes(700, 12, b)), dtype=torch.uint8, device="cuda")
        accepted, following = torch.full((b,), -7, device="cuda"), torch.full((b,), -7, device="cuda")
        logp, next_logp = torch.full((12,), NAN, device="cuda"), torch.full((b,), NAN, device="cuda")
        chances, next_chances = c.chances, dev(r.random(b), torch.float64)
        B.laplex_verify_drafts(c.y, c.z, c.drafts, chances, next_chances, accepted, following, ws, logp, next_logp, sequences=b, starts=dev(np.array(starts), torch.int64),
                               flags=B.LAPLEX_VERIFY_GREEDY if rule == "greedy" else 0)
        want = O.verify_drafts(host(c.y), None if c.z is None else host(c.z), host(c.drafts).astype(np.int64), starts, 1.0, 1.0, host(chances), host(next_chances), rule == "greedy")
        assert accepted.tolist() == want[0].tolist() and following.tolist() == want[1].tolist()
        outside = [t for t in range(12) if t < starts[0] or t >= starts[-1]]
        assert host(logp)[outside].tolist() == [0.0] * len(outside)
        for got, w in ((host(logp), want[2]), (host(next_logp), want[3])):
            assert (np.abs(got - w) <= U * (np.abs(w) + 1.0)).all()
