"""Logits and their gradient as columns of one buffer: rows side by side do not overlap.  No GPU: no call with rows is launched."""
import pytest

from paper_2606_18967_amd import sdrl
from test_logits_host import INVAL, PTR


def status(x, ld, out, out_ld, V, rows=4):
    """The check of logits and gradient alone: a NULL norm is refused after it."""
    L = sdrl.lib()
    assert L.sd_token_logprobs_grad(0, rows, V, x, ld, PTR, 1.0, None, PTR, None, None, out, out_ld, None) == INVAL
    return L.sd_last_error().decode()


@pytest.mark.parametrize("ld,at", [(200, 100), (250, 100), (250, 150), (250, -100), (250, -150), (250, 600), (250, -650)])
def test_rows_side_by_side(ld, at):
    assert "norm" in status(PTR + 4096, ld, PTR + 4096 + 4 * at, ld, 100)


@pytest.mark.parametrize("ld,out_ld,at", [(200, 200, 99), (200, 200, 101), (250, 250, 151), (250, 250, -99), (250, 250, 349), (250, 250, 250),
                                          (250, 250, -250), (250, 251, 100), (200, 100, 100), (200, 400, 100)])
def test_rows_that_overlap(ld, out_ld, at):
    """Or that may, at strides that differ."""
    assert "overlap" in status(PTR + 4096, ld, PTR + 4096 + 4 * at, out_ld, 100)
