"""Layer norm and its gradient against the oracle in 64 bits.

Tolerances.  U = 2^-24 and H = 2^-8 are half a step of fp32 and bf16.  A row's sums are at most 64 numbers in a thread's order, then a tree: 80 U of the sum of
absolute values.  The centred value is off by that mean's error and its own rounding, a variance by twice as much as its squares, the root and
the products by a few roundings more: delta() below, in units of the normalised value.  A column's sums over n rows, with roundings of either
sign: 16 sqrt(n + 64) U of the sum of absolute values.  bf16 results are rounded once: H of the value.
"""
import numpy as np
import pytest

from oracle import token_oracle as O
from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
EPS = float(np.float32(1e-5))


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


def delta(x, mean, rstd):
    """How far a normalised value may be off."""
    size = np.abs(x).mean(-1, keepdims=True)
    m, r = mean[..., None], rstd[..., None]
    return 84 * U * r * size + 4 * U * r * np.abs(x - m) + 100 * U * np.abs(x - m) * r


def inputs(r, rows, width, dtype, affine, far=0.0):
    x = dev(r.normal(size=(rows, width)) * (0.3 + r.random((rows, 1))) + r.normal(size=(rows, 1)) + far, dtype)
    gy = dev(r.normal(size=(rows, width)), dtype)
    weight, bias = (dev(1.0 + 0.3 * r.normal(size=width)), dev(r.normal(size=width))) if affine else (None, None)
    return x, gy, weight, bias


def check(x, gy, weight, bias, dtype, y, mean, rstd, gx=None, gweight=None, gbias=None, eps=EPS):
    hx, hg = host(x), host(gy)
    w = np.ones(hx.shape[-1]) if weight is None else host(weight)
    want, wm, wr = O.layer_norm(hx, w, None if bias is None else host(bias), eps)
    d = delta(hx, wm, wr)
    hat = (hx - wm[:, None]) * wr[:, None]
    h = H if dtype == BF16 else 0.0
    if y is not None:
        within("mean", host(mean), wm, 81 * U * np.abs(hx).mean(-1))
        within("rstd", host(rstd), wr, 100 * U * wr)
        within("y", host(y), want, np.abs(w) * d + 4 * U * (np.abs(want) + (0.0 if bias is None else np.abs(host(bias)))) + h * 1.01 * np.abs(want))
    if gx is not None or gweight is not None:
        wx, ww, wb = O.layer_norm_backward(hx, hg, w, eps)
        g = np.abs(hg * w)
        n = len(hx)
        c1, c2 = g.mean(-1, keepdims=True), (g * np.abs(hat)).mean(-1, keepdims=True)
        size = wr[:, None] * (g + c1 + np.abs(hat) * c2)
        off = 200 * U * size + wr[:, None] * (d * c2 + np.abs(hat) * (g * d).mean(-1, keepdims=True))
        if gx is not None:
            within("gx", host(gx), wx, off + h * 1.01 * np.abs(wx))
        if gweight is not None:
            within("gweight", host(gweight), ww, 16 * np.sqrt(n + 64.0) * U * np.abs(hg * hat).sum(0) + (np.abs(hg) * d).sum(0))
        if gbias is not None:
            within("gbias", host(gbias), wb, 16 * np.sqrt(n + 64.0) * U * np.abs(hg).sum(0))


def run(x, gy, weight, bias, backward=True, eps=EPS):
    rows, width = x.shape
    nan = lambda *s, t=F32: torch.full(s, float("nan"), device="cuda", dtype=t)
    y, mean, rstd = nan(rows, width, t=x.dtype), nan(rows), nan(rows)
    B.laplex_layer_norm(x, weight, bias, y, mean, rstd, eps)
    if not backward:
        return y, mean, rstd
    gx, gw, gb = nan(rows, width, t=x.dtype), nan(width), nan(width)
    ws = torch.empty(B.laplex_layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
    B.laplex_layer_norm_backward(x, gy, weight, mean, rstd, gx, gw, gb, ws)
    return y, mean, rstd, gx, gw, gb


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 2), (5, 7), (64, 8), (2, 9), (67, 16), (130, 33), (33, 64), (1, 100), (700, 128), (9, 200), (257, 255), (70, 512),
                                        (5, 513), (31, 1000), (2, 2048), (2051, 2050), (3, 4096), (2100, 300), (17, 4100), (2, 8192), (3, 8200), (5, 16384), (4, 16400),
                                        (70, 20001), (1030, 40)])
def test_layer_norm(dtype, affine, rows, width):
    r = seeded("norm", rows, width)
    x, gy, weight, bias = inputs(r, rows, width, dtype, affine)
    check(x, gy, weight, bias, dtype, *run(x, gy, weight, bias))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_rows(dtype):
    """More rows than workgroups of the gradient."""
    r = seeded("many")
    x, gy, weight, bias = inputs(r, 40000, 24, dtype, True)
    check(x, gy, weight, bias, dtype, *run(x, gy, weight, bias))


def test_means_far_from_zero():
    """A variance about the mean: rows around 1000 keep what the mean's own rounding leaves."""
    r = seeded("far")
    x, gy, weight, bias = inputs(r, 50, 300, F32, True, far=1000.0)
    check(x, gy, weight, bias, F32, *run(x, gy, weight, bias))


def test_equal_numbers_and_one_number():
    """No variance: the result is the bias, the gradient 0, and nothing is NaN."""
    x = torch.full((7, 60), 3.0, device="cuda")
    gy = dev(seeded("equal").normal(size=(7, 60)))
    bias = dev(np.arange(60.0))
    y, mean, rstd, gx, gw, gb = run(x, gy, None, bias)
    assert torch.equal(y, bias.expand(7, 60)) and torch.equal(mean, torch.full_like(mean, 3.0)) and bool(torch.isfinite(gx).all())
    assert torch.equal(gw, torch.zeros_like(gw))
    y, mean, rstd, gx, gw, gb = run(x[:, :1].contiguous(), gy[:, :1].contiguous(), None, None)
    assert torch.equal(y, torch.zeros_like(y)) and torch.equal(gx, torch.zeros_like(gx))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width,pad,rows", [(40, 3, 37), (513, 7, 9), (4096, 1, 5), (20000, 5, 3)])
def test_parts_of_a_matrix_and_in_place(dtype, width, pad, rows):
    """Rows that lie apart, aligned to nothing; results over their inputs; what lies beside them stays."""
    r = seeded("parts", width)
    m = dev(r.normal(size=(rows, width + 2 * pad)), dtype)
    x, gy = m[:, pad:pad + width], dev(r.normal(size=(rows, width + 1)), dtype)[:, 1:]
    weight, bias = dev(r.normal(size=width)), dev(r.normal(size=width))
    y, mean, rstd, gx, gw, gb = run(x.contiguous(), gy.contiguous(), weight, bias)
    beside = m.clone()
    ws = torch.empty(B.laplex_layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
    over, w2, b2 = gy.clone(), torch.empty_like(gw), torch.empty_like(gb)
    wide = torch.zeros(rows, width + 3, device="cuda", dtype=dtype)
    wide[:, :width] = gy
    B.laplex_layer_norm_backward(x, wide[:, :width], weight, mean, rstd, wide[:, :width], w2, b2, ws)
    assert torch.equal(wide[:, :width], gx) and torch.equal(w2, gw) and torch.equal(b2, gb)
    kept = x.clone()
    B.laplex_layer_norm(x, weight, bias, x, None, None)
    assert torch.equal(x, y)
    x.copy_(kept)
    B.laplex_layer_norm_backward(x, gy, weight, mean, rstd, x, w2, b2, ws)
    assert torch.equal(x, gx) and torch.equal(w2, gw) and torch.equal(b2, gb)
    assert torch.equal(m[:, :pad], beside[:, :pad]) and torch.equal(m[:, pad + width:], beside[:, pad + width:])
    # whatever is not asked for changes nothing of the rest
    for left in range(3):
        some = [None if i == left else torch.full_like(t, float("nan")) for i, t in enumerate((gx, gw, gb))]
        B.laplex_layer_norm_backward(kept, gy, weight, mean, rstd, *some, ws)
        for t, full in zip(some, (gx, gw, gb)):
            assert t is None or torch.equal(t, full)
    only = torch.empty_like(gx)
    B.laplex_layer_norm_backward(kept, gy, weight, mean, rstd, only, None, None, None)
    assert torch.equal(only, gx)


def test_heads_of_tokens():
    """Heads of a (tokens, heads, numbers) tensor are rows; with weight width^-1/2 they have length 1."""
    r = seeded("heads")
    x = dev(r.normal(size=(21, 6, 64)))
    y, mean, rstd = torch.empty_like(x), torch.empty(21, 6, device="cuda"), torch.empty(21, 6, device="cuda")
    B.laplex_layer_norm(x, torch.full((64,), 64 ** -0.5, device="cuda"), None, y, mean, rstd)
    within("length", host(y.square().sum(-1)), np.ones((21, 6)), 1e-4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("width", [24, 300, 5000, 20000])
def test_values_that_are_not_finite_stay_in_their_row(dtype, value, width):
    r = seeded("odd", width)
    x, gy, weight, bias = inputs(r, 19, width, dtype, True)
    y, mean, rstd, gx, gw, gb = run(x, gy, weight, bias)
    x[7, width // 2] = value
    y2, mean2, rstd2, gx2, gw2, gb2 = run(x, gy, weight, bias)
    rows = [i for i in range(19) if i != 7]
    assert torch.equal(y2[rows], y[rows]) and torch.equal(gx2[rows], gx[rows]) and torch.equal(mean2[rows], mean[rows]) and torch.equal(gb2, gb)
    assert bool(torch.isnan(y2[7]).all()) and bool(torch.isnan(gx2[7]).all()) and bool(torch.isnan(gw2).all())


def test_no_rows():
    gw, gb = torch.full((9,), float("nan"), device="cuda"), torch.full((9,), float("nan"), device="cuda")
    e = torch.empty(0, 9, device="cuda")
    B.laplex_layer_norm(e, None, None, e)
    ws = torch.empty(max(1, B.laplex_layer_norm_workspace_bytes(0, 9)), dtype=torch.uint8, device="cuda")
    B.laplex_layer_norm_backward(e, e, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), None, gw, gb, ws)
    assert not bool(gw.any()) and not bool(gb.any())


def test_gradients_against_differences():
    r = seeded("differences")
    x, gy, weight, bias = inputs(r, 4, 37, F32, True)
    _, _, _, gx, gw, gb = run(x, gy, weight, bias)
    of = lambda x, w, b: float((O.layer_norm(x, w, b, EPS)[0] * host(gy)).sum())
    base, step = [host(x), host(weight), host(bias)], 1e-5
    for which, got in enumerate((gx, gw, gb)):
        for _ in range(12):
            at = tuple(int(r.integers(n)) for n in base[which].shape)
            ends = []
            for s in (step, -step):
                moved = [b.copy() for b in base]
                moved[which][at] += s
                ends.append(of(*moved))
            assert abs((ends[0] - ends[1]) / (2 * step) - float(got[at])) < 1e-4 * max(1.0, float(got.abs().max()))


def test_captured_and_replayed():
    """A forward and a backward call in a graph, with eager calls between the replays."""
    r = seeded("graph")
    x, gy, weight, bias = inputs(r, 600, 700, BF16, True)
    rows, width = x.shape
    new = lambda *s, t=F32: torch.zeros(*s, device="cuda", dtype=t)
    y, mean, rstd, gx, gw, gb = new(rows, width, t=BF16), new(rows), new(rows), new(rows, width, t=BF16), new(width), new(width)
    ws = torch.empty(B.laplex_layer_norm_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")

    def call():
        B.laplex_layer_norm(x, weight, bias, y, mean, rstd)
        B.laplex_layer_norm_backward(x, gy, weight, mean, rstd, gx, gw, gb, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.copy_(dev(r.normal(size=(rows, width)), BF16))
        want = run(x, gy, weight, bias)
        for t in (y, mean, rstd, gx, gw, gb):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((y, mean, rstd, gx, gw, gb), want):
            assert torch.equal(got, w), i
