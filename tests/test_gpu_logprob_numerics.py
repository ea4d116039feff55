"""Numerics of the log probabilities and their gradient where bounds that grow with the logits do not show them: what depends on the differences of a column's
logits alone has to be as good at logits of thousands, or of the type's lowest value, as it is around zero.

Tolerances, U = 2^-24 and H = 2^-8 the unit roundings of fp32 and bf16.  A difference from the column's maximum is rounded once, and so are its product and the sum with the
logarithm; the sums over the column are off by 64 U: a log probability is off by U (64 + 8 |log p|), the entropy by U (64 + 16 H).  In the gradient columns up to |lse| = 64 may use
lse as it was rounded, 64 U more; the terms' sizes are multiplied by that.
"""
import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16


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


def forward(y, targets, tau, top=0):
    k, t = y.shape
    new = lambda *s, d=F32: torch.full(s, -77, device="cuda", dtype=d)
    out = dict(logp=new(t), lse=new(t), entropy=new(t))
    ids, values = (new(top, t, d=torch.int64), new(top, t)) if top else (None, None)
    ws = torch.full((B.laplex_logprob_workspace_bytes(k, t, top),), 0xFF, dtype=torch.uint8, device="cuda")     # what it holds does not matter
    B.laplex_logprob(y, dev(targets, torch.int64), out["logp"], out["lse"], out["entropy"], ids, values, ws, tau)
    return {**out, "top_ids": ids, "top_logp": values} if top else out


def oracle(hy, targets, tau, top=0):
    """Of the differences from each column's maximum: 64 bits do not hold the logarithm of a sum beside 1e30 either.  (results with lse in place, the differences)"""
    most = np.where(np.isfinite(hy), hy, -np.inf).max(axis=0)
    most = np.where(np.isfinite(most), most, 0.0)
    o = O.logprob(hy - most, targets, tau, top)
    return {**o, "own_lse": o["lse"], "lse": o["lse"] + tau * most}, hy - most


def shifted(r, k, t, dtype):
    """Columns of ordinary differences around all kinds of values."""
    at = np.resize([0.0, 60.0, 64.5, 70.0, 300.0, -1000.0, 3e4, -1e6, 1e30, -40.0], t)
    return dev((3.0 * r.normal(size=(k, t)) + at).astype(np.float32), dtype)


def odd_masks(k, t, dtype):
    """Columns of nothing but the type's lowest value, or of it beside a few others."""
    low = float(torch.finfo(dtype).min)
    y = torch.full((k, t), low, device="cuda", dtype=dtype)
    y[: k // 2, 1::4] = 0.25 * low
    y[k // 3, 2::4] = 5.0
    y[:, 3::4] = -float("inf")
    return y


def check_gradient(y, targets, tau, which=(True, True, True), in_place=False):
    hy = host(y)
    k, t = hy.shape
    tau = float(np.float32(tau))
    r = seeded("weights", k, t)
    glogp, gent, glse = (r.normal(size=t).astype(np.float32) if w else np.zeros(t, np.float32) for w in which)
    give = lambda g, w: dev(g) if w else None
    f = forward(y, targets, tau)
    gy = y if in_place else torch.full_like(y, float("nan"))
    B.laplex_logprob_backward(y, dev(targets, torch.int64), f["lse"], f["entropy"], give(glogp, which[0]), give(gent, which[1]), give(glse, which[2]), gy, tau)
    o, away = oracle(hy, targets, tau)
    want = O.logprob_backward(away, targets, glogp, gent, glse, tau)
    with np.errstate(all="ignore"):
        logp = tau * away - o["own_lse"]
        p = np.where(np.isfinite(o["lse"]) & (logp > -200), np.exp(logp), 0.0)
    logp = np.where(p > 0, logp, 0.0)
    size = tau * p * (np.abs(glogp) + np.abs(gent) * (np.abs(logp) + np.abs(o["entropy"]) + 1.0) + np.abs(glse))
    for c in range(t):
        if 0 <= targets[c] < k and np.isfinite(o["lse"][c]):
            size[targets[c], c] += tau * abs(glogp[c])
    within("gy", host(gy), want, U * (192 + 8 * np.abs(logp) + 16 * np.abs(o["entropy"])) * size + (H * np.abs(want) if y.dtype == BF16 else 0.0) + 1e-36)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(10, 13), (500, 1), (500, 3), (257, 300), (5001, 21), (32000, 6)])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_log_probabilities_do_not_depend_on_where_the_logits_lie(dtype, k, batch, tau):
    r = seeded("shifted", k, batch)
    y = shifted(r, k, batch, dtype)
    hy, targets = host(y), r.integers(0, k, batch)
    f, tau = forward(y, targets, tau, min(k, 7)), float(np.float32(tau))
    o, _ = oracle(hy, targets, tau, min(k, 7))
    within("logp", host(f["logp"]), o["logp"], U * (64 + 8 * np.abs(o["logp"])))
    within("top_logp", host(f["top_logp"]), o["top_logp"], U * (64 + 8 * np.abs(o["top_logp"])))
    within("entropy", host(f["entropy"]), o["entropy"], U * (64 + 16 * o["entropy"]))
    within("lse", host(f["lse"]), o["lse"], U * (64 + 4 * np.abs(o["lse"])))
    assert np.array_equal(f["top_ids"].cpu().numpy(), o["top_ids"])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(10, 13), (500, 1), (500, 3), (257, 300), (5001, 21), (32000, 6)])
@pytest.mark.parametrize("in_place", [False, True])
def test_the_gradient_does_not_depend_on_where_the_logits_lie(dtype, k, batch, in_place):
    r = seeded("shifted backward", k, batch)
    y = shifted(r, k, batch, dtype)
    targets = r.integers(0, k, batch); targets[::6] = -1
    check_gradient(y, targets, 0.7, in_place=in_place)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(37, 4096), (300, 4099), (1100, 5000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_the_gradient_of_thousands_of_columns(dtype, k, batch, in_place):
    """Enough columns that those far from zero are taken sixteen at a time, some of them in every sixteen, and stretches with none and with nothing else."""
    r = seeded("thousands", k, batch)
    y = shifted(r, k, batch, dtype)
    y[:, 1000:1500] = dev((3.0 * r.normal(size=(k, 500))).astype(np.float32), dtype)
    y[:, 2000:2500] = dev((3.0 * r.normal(size=(k, 500)) + 300.0).astype(np.float32), dtype)
    y[:, 3001:3040] = -float("inf")
    targets = r.integers(0, k, batch); targets[::6] = -1
    check_gradient(y, targets, 1.0, in_place=in_place)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(8, 3), (500, 9), (5001, 17)])
@pytest.mark.parametrize("tau", [1.0, 1.3, 0.5])
@pytest.mark.parametrize("which", [(True, True, True), (True, False, False), (False, True, False), (False, False, True)])
def test_the_gradient_of_masks_of_the_lowest_value(dtype, k, batch, tau, which):
    """Where all logits are the type's lowest value all are as likely, also where tau times it is beyond the type."""
    y = odd_masks(k, batch, dtype)
    for targets in (np.zeros(batch, np.int64), np.full(batch, k - 1), np.full(batch, -1)):
        check_gradient(y, targets, tau, which)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_column_of_the_gradient_does_not_depend_on_its_neighbours(dtype):
    """Columns far from zero beside others, and those alone: the same bits."""
    r = seeded("neighbours")
    k, batch = 700, 29
    y = dev((3.0 * r.normal(size=(k, batch))).astype(np.float32), dtype)
    targets = r.integers(0, k, batch)
    w = [dev(r.normal(size=batch).astype(np.float32)) for _ in range(3)]

    def gradient(y):
        f = forward(y, targets, 1.0)
        gy = torch.full_like(y, float("nan"))
        B.laplex_logprob_backward(y, dev(targets, torch.int64), f["lse"], f["entropy"], *w, gy)
        return gy
    want = gradient(y)
    far = y.clone()
    moved = [2, 11, 12, 28]
    far[:, moved] += 512.0
    got = gradient(far)
    rest = [c for c in range(batch) if c not in moved]
    assert torch.equal(got[:, rest], want[:, rest])
    odd = far.clone()
    odd[5, 3], odd[6, 13], odd[7, 2] = float("nan"), float("inf"), float("nan")
    got_odd = gradient(odd)
    assert torch.isnan(got_odd[:, [3, 13, 2]]).all()
    rest = [c for c in range(batch) if c not in (3, 13, 2)]
    assert torch.equal(got_odd[:, rest], got[:, rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(9, 2), (300, 7), (3000, 5)])
@pytest.mark.parametrize("tau", [3e38, 3.4e38, 2.5e38, 1e30, 1e-30, 1e-38])
def test_inverse_temperatures_at_their_ends(dtype, k, batch, tau):
    """All that is positive and finite is accepted: the largest logits have all of the probability, or all logits have the same."""
    r = seeded("tau", k, batch)
    y = dev(np.round(r.normal(size=(k, batch)) * 8.0).astype(np.float32) / 8.0, dtype)
    y[1:, 0] = -float("inf")
    hy = host(y)
    targets = hy.argmax(axis=0)
    f = forward(y, targets, tau, 3)
    n = (hy == hy.max(axis=0)).sum(axis=0) if tau > 1 else np.isfinite(hy).sum(axis=0)
    within("logp", host(f["logp"]), -np.log(n), 64 * U * (1 + np.log(n)))
    within("entropy", host(f["entropy"]), np.log(n), 64 * U * (1 + np.log(n)))
    within("top_logp", host(f["top_logp"])[0], -np.log(n), 64 * U * (1 + np.log(n)))
    gy = torch.full_like(y, float("nan"))
    ones = torch.ones(batch, device="cuda")
    B.laplex_logprob_backward(y, dev(targets, torch.int64), f["lse"], f["entropy"], None, None, ones / k * 1e-3, gy, tau)
    likely = (hy == hy.max(axis=0)) if tau > 1 else np.isfinite(hy)
    want = float(np.float32(tau)) * np.where(likely, 1.0 / n, 0.0) * float(np.float32(1.0) / np.float32(k) * np.float32(1e-3))
    within("gy", host(gy), want, (H if dtype == BF16 else 0.0) * want + 128 * U * want + 1e-37)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(50, 3), (2000, 6), (40000, 2)])
def test_entropy_of_logits_as_large_as_the_type_at_a_small_inverse_temperature(dtype, k, batch):
    """Sums of differences times probabilities beyond the type, whose product with tau is of ordinary size (the differences themselves are within it)."""
    r = seeded("large logits", k, batch)
    y = dev((r.normal(size=(k, batch)).clip(-5.0, 5.0) * 3e37).astype(np.float32), dtype)
    hy, targets, tau = host(y), r.integers(0, k, batch), float(np.float32(2.0 ** -125))
    f = forward(y, targets, tau)
    o, _ = oracle(hy, targets, tau)
    within("logp", host(f["logp"]), o["logp"], U * (64 + 8 * np.abs(o["logp"])))
    within("entropy", host(f["entropy"]), o["entropy"], U * (64 + 16 * o["entropy"]))
    within("lse", host(f["lse"]), o["lse"], U * (64 + 4 * np.abs(o["lse"])))


# --- alternatives: several slabs of columns, several stretches of rows, more equal values than there is room for -------------------------

def check_alternatives(y, top):
    hy = y.float().cpu().numpy()
    k, t = hy.shape
    f = forward(y, np.zeros(t, np.int64), 1.0, top)
    with np.errstate(invalid="ignore"):
        for c in range(t):
            # NaN first, then by value, of equal ones the lowest row
            order = np.lexsort((np.arange(k), -np.nan_to_num(hy[:, c], nan=0.0, posinf=np.inf, neginf=-np.inf), ~np.isnan(hy[:, c])))[:top]
            assert np.array_equal(f["top_ids"][:, c].cpu().numpy(), order), f"column {c}"
    logp = torch.gather(y.double(), 0, f["top_ids"]) - f["lse"].double()
    empty = f["lse"] == -float("inf")
    logp[:, empty] = -float("inf")
    got = f["top_logp"].double()
    assert torch.equal(torch.isnan(got), torch.isnan(logp))
    some = torch.isfinite(logp)
    assert torch.equal(got[~some & ~torch.isnan(logp)], logp[~some & ~torch.isnan(logp)])
    assert ((got - logp).abs()[some] <= U * (128 + 16 * logp.abs()[some] + 4 * f["lse"].double().abs().expand_as(logp)[some])).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,batch", [(1025, 257), (1500, 300), (3000, 700), (20000, 260)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_alternatives_of_many_columns(dtype, k, batch, top):
    r = seeded("many columns", k, batch)
    y = (3.0 * r.normal(size=(k, batch))).astype(np.float32)
    y[:, 1::7] = r.integers(0, 4, size=y[:, 1::7].shape)                   # many equal values
    y[r.random((k, batch)) < 0.05] = -np.inf
    y[:, 256] = -np.inf
    y[k - 1, 2::9] = 50.0
    check_alternatives(dev(y, dtype), top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [131072, 131073, 140001, 262147])
@pytest.mark.parametrize("top", [1, 13, 64])
def test_alternatives_of_several_stretches_of_rows(dtype, k, top):
    """131072 rows are looked at at a time: equal values, NaN and -inf on either side of that."""
    r = seeded("stretches of rows", k)
    edge = 131072
    c = [np.full(k, -np.inf), np.zeros(k), r.integers(0, 3, k), r.integers(0, 50, k), 3.0 * r.normal(size=k), np.sort(3.0 * r.normal(size=k)), -np.sort(3.0 * r.normal(size=k))]
    few = r.normal(size=k); few[max(0, edge - 5):edge + 5] = 9.0; c.append(few)              # equal values across the edge
    nan = r.integers(0, 3, k).astype(float); nan[[3, edge - 1, min(edge, k - 1), k - 1]] = np.nan; c.append(nan)
    late = np.full(k, -np.inf); late[-3:] = 1.0; c.append(late)                                # all but a few banned
    both = np.where(r.random(k) < 0.999, -np.inf, 2.0); both[edge - 1:edge + 1] = 7.0; c.append(both)
    low = np.full(k, float(torch.finfo(dtype).min)); low[-1] = 0.0; c.append(low)
    y = dev(np.stack(c, axis=1).astype(np.float32), dtype)
    check_alternatives(y, top)
    check_alternatives(y[:, 2:4].contiguous(), top)
    check_alternatives(y[:, 8:9].contiguous(), top)


def test_a_vector_of_logits_whose_numbers_lie_apart():
    r = seeded("apart")
    m = dev(r.normal(size=(600, 5)).astype(np.float32))
    y, target = m[:, 3], dev(np.array([17]), torch.int64)
    new = lambda: torch.full((1,), float("nan"), device="cuda")
    logp, lse, entropy = new(), new(), new()
    ws = torch.empty(B.laplex_logprob_workspace_bytes(600, 1), dtype=torch.uint8, device="cuda")
    B.laplex_logprob(y, target, logp, lse, entropy, None, None, ws)
    o = O.logprob(host(y)[:, None], [17])
    within("logp", host(logp), o["logp"], U * (64 + 8 * np.abs(o["logp"])))
    g, kept = torch.zeros(600, 5, device="cuda"), m.clone()
    B.laplex_logprob_backward(y, target, lse, entropy, torch.ones(1, device="cuda"), None, None, g[:, 2])
    want = O.logprob_backward(host(y)[:, None], [17], [1.0], [0.0], [0.0])
    within("gy", host(g[:, 2]), want[:, 0], 300 * U * np.maximum(np.abs(want[:, 0]), 1e-3))
    assert torch.equal(m, kept) and (g[:, [0, 1, 3, 4]] == 0).all()
