"""What the binding makes of tensors that are not contiguous.  No GPU: refusals come before any call, leading dimensions are arithmetic."""
import pytest

from paper_2605_24584_amd import binding as B

torch = pytest.importorskip("torch")


def test_leading_dimension_of_rows_and_vectors():
    m = torch.zeros(6, 8)
    assert B._ld(m) == 8 and B._ld(m[:, :3]) == 8 and B._ld(m[::2]) == 16 and B._ld(m[:, :1]) == 8
    assert B._ld(m[:1]) == 8 and B._ld(m[:1, :5]) == 5 and B._ld(m[:0]) == 8 and B._ld(m[:, :0]) == 1
    assert B._ld(None) == 0
    # vectors whose numbers lie apart
    assert B._ld(m[:, 2]) == 8 and B._ld(torch.zeros(10)[::3]) == 3 and B._ld(torch.zeros(10)) == 1
    assert B._ld(torch.zeros(10)[::3][:1]) == 1 and B._ld(torch.zeros(0)) == 1


def test_columns_that_lie_apart_are_refused():
    m = torch.zeros(6, 8)
    for t in (m[:, ::2], m[:1, ::2], m.T[:2, :3], m.T[:1, :3]):
        with pytest.raises(AssertionError):
            B._ld(t)
    out = torch.zeros(4)
    with pytest.raises(AssertionError):
        B.laplex_logprob(m[:1, ::2], None, None, out, None, None, None, None, stream=0)
    with pytest.raises(AssertionError):
        B.laplex_logprob_backward(m[:1, ::2], None, out, None, None, None, None, torch.zeros(1, 4), stream=0)


def test_vectors_that_are_one_number_over_and_over_are_refused():
    """A leading dimension of 0 is refused by the library."""
    with pytest.raises(B.LaplexError) as e:
        B.laplex_logprob(torch.zeros(1).expand(7), None, None, torch.zeros(1), None, None, None, None, stream=0)
    assert e.value.status == B.LAPLEX_ERR_LD
