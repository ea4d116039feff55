"""Layer norm, the gated delta rule and the verification of drafts where numbers lie more than 2^32 elements from the first: the last rows, sequences or columns of a large call
against a call on them alone.  The same numbers are added in the same order in both unless a test says otherwise."""
import pytest

from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def released():
    torch.cuda.manual_seed(5)
    yield
    torch.cuda.empty_cache()


def workspace(size):
    return torch.empty(max(1, size), dtype=torch.uint8, device="cuda")


def test_layer_norm():
    rows, width, few = (1 << 20) + 3, 4096, 7
    x = torch.empty(rows, width, device="cuda", dtype=BF16).normal_()
    weight, bias = torch.randn(width, device="cuda"), torch.randn(width, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.laplex_layer_norm(x, weight, bias, y, mean, rstd)
    x1 = x[-few:].clone()
    y1, mean1, rstd1 = torch.empty_like(x1), torch.empty(few, device="cuda"), torch.empty(few, device="cuda")
    B.laplex_layer_norm(x1, weight, bias, y1, mean1, rstd1)
    assert torch.equal(y[-few:], y1) and torch.equal(mean[-few:], mean1) and torch.equal(rstd[-few:], rstd1)
    # the results as gradients, and in their place
    B.laplex_layer_norm_backward(x, y, weight, mean, rstd, y, None, None, None)
    B.laplex_layer_norm_backward(x1, y1, weight, mean1, rstd1, y1, None, None, None)
    assert torch.equal(y[-few:], y1)


def test_delta_attention():
    """Rows 8200 numbers apart, a long sequence of zeros and a short one behind it."""
    n, short, d, apart = 530000, 200, 64, 8200
    m = torch.zeros(n, apart, device="cuda", dtype=BF16)
    q, k, v = (m[:, 8000 + i * d:8000 + (i + 1) * d].unflatten(1, (1, d)) for i in range(3))
    for t in (q, k, v):
        t[-short:] = torch.nn.functional.normalize(torch.randn(short, 1, d, device="cuda"), dim=-1).to(BF16)
    rates, beta = torch.full((n, 1), 0.01, device="cuda"), torch.full((n, 1), 0.7, device="cuda")
    starts = torch.tensor([0, n - short, n], device="cuda")
    gm = torch.empty_like(m)
    y, gq, gk, gv = (gm[:, 7900 + i * d:7900 + (i + 1) * d].unflatten(1, (1, d)) for i in range(4))
    gr, gb = torch.empty_like(rates), torch.empty_like(beta)
    ws = workspace(B.laplex_delta_attention_workspace_bytes(BF16, n, 2, 1, 1, d, d, True))
    B.laplex_delta_attention(q, k, v, rates, beta, y, ws, starts=starts, flags=B.LAPLEX_SAVE_SCANS)
    B.laplex_delta_attention_backward(q, k, v, rates, beta, v, gq, gk, gv, gr, gb, ws, starts=starts, flags=B.LAPLEX_SAVE_SCANS)
    q1, k1, v1, r1, b1 = (t[-short:].contiguous() for t in (q, k, v, rates, beta))
    y1, gq1, gk1, gv1 = (torch.empty_like(q1) for _ in range(4))
    gr1, gb1 = torch.empty_like(r1), torch.empty_like(b1)
    ws1 = workspace(B.laplex_delta_attention_workspace_bytes(BF16, short, 1, 1, 1, d, d, True))
    B.laplex_delta_attention(q1, k1, v1, r1, b1, y1, ws1)
    B.laplex_delta_attention_backward(q1, k1, v1, r1, b1, v1, gq1, gk1, gv1, gr1, gb1, ws1)
    for large, alone in ((y, y1), (gq, gq1), (gk, gk1), (gv, gv1), (gr, gr1), (gb, gb1)):
        assert torch.equal(large[-short:], alone)
    assert float(y[:-short].abs().max()) == 0.0


def test_delta_attention_step():
    """States of 7e4 sequences.  Alone a thread has other rows of a state: sums of 128 products with half a step of fp32 each, twice, 128 2^-23 = 1.5e-5 of their sizes at most."""
    b, h, d, few = 70000, 16, 64, 3
    q, k, v = (torch.nn.functional.normalize(torch.randn(b, h, d, device="cuda"), dim=-1).to(BF16) for _ in range(3))
    rates, beta = torch.rand(b, h, device="cuda"), torch.rand(b, h, device="cuda")
    state = torch.zeros(b, h, d, d, device="cuda")
    state[-few:].normal_()
    start, y = state[-few:].clone(), torch.empty_like(v)
    assert state.numel() > 1 << 32
    B.laplex_delta_attention_step(q, k, v, rates, beta, state, y)
    y1 = torch.empty(few, h, d, device="cuda", dtype=BF16)
    B.laplex_delta_attention_step(q[-few:], k[-few:], v[-few:], rates[-few:].contiguous(), beta[-few:].contiguous(), start, y1)
    size = float(start.norm(dim=-2).max())
    assert float((state[-few:] - start).abs().max()) <= 1.5e-5 * size
    assert float((y[-few:].float() - y1.float()).abs().max()) <= (1.5e-5 + 2.0 ** -7) * size      # (either may be rounded to the neighbour)


def test_verify_drafts():
    """Alone the rows are cut into more parts: sums in 64 bits in another order, 1e-13 off at most, which no chance here is near."""
    k, sequences, each, few = 70000, 16384, 4, 8
    t = sequences * each
    y = torch.empty(k, t, device="cuda", dtype=BF16).normal_()
    assert y.numel() > 1 << 32
    drafts = torch.randint(0, k, (t,), device="cuda")
    drafts[::3] = y[:, ::3].argmax(0)
    chances, following_chances = torch.rand(t, device="cuda", dtype=torch.float64) * 1e-3, torch.rand(sequences, device="cuda", dtype=torch.float64)
    accepted, following = (torch.empty(sequences, device="cuda", dtype=torch.int64) for _ in range(2))
    B.laplex_verify_drafts(y, None, drafts, chances, following_chances, accepted, following, workspace(B.laplex_verify_workspace_bytes(k, t, sequences)), tau=2.0, sequences=sequences)
    at = few * each
    a1, f1 = (torch.empty(few, device="cuda", dtype=torch.int64) for _ in range(2))
    B.laplex_verify_drafts(y[:, -at:].contiguous(), None, drafts[-at:], chances[-at:], following_chances[-few:], a1, f1, workspace(B.laplex_verify_workspace_bytes(k, at, few)), tau=2.0,
                           sequences=few)
    assert torch.equal(accepted[-few:], a1) and torch.equal(following[-few:], f1)
    assert 0 < int(accepted.sum()) < sequences * (each - 1)
