"""Norms in place, on the host: a tensor that is written may be one that is read element for element, and is refused where other rows would read what is written."""
import pytest

from test_host_i8 import EINVAL, ESHAPE, P, norm

H, BLOCK, BLOCK_GAIN, GATE, GAIN, H_OUT, OUT = (P * n for n in range(1, 8))


@pytest.mark.parametrize("bad", [
    dict(h_out=H, h_row=0), dict(h_out=H, h_row=128), dict(h_out=H, h_out_row=128), dict(h_out=BLOCK, block_row=0), dict(h_out=BLOCK, block_row=65), dict(out=H, h_row=0),
    dict(out=H, out_row=80), dict(out=BLOCK, block_row=128), dict(out=BLOCK, h_out=H, block_row=0), dict(out=GATE, gate_row=0), dict(h_out=GATE, gate_row=0), dict(out=GAIN),
    dict(h_out=GAIN), dict(out=BLOCK_GAIN), dict(h_out=BLOCK_GAIN), dict(block=None, block_gain=None, gate=None, h_out=None, out=H, h_row=0)])
def test_rows_that_would_read_what_others_write_are_refused(bad):
    assert norm(**bad) == EINVAL


@pytest.mark.parametrize("good", [dict(h_out=H), dict(h_out=BLOCK), dict(out=H), dict(out=BLOCK, h_out=H), dict(out=H, h_out=BLOCK), dict(rows=1, h_out=H, h_row=0), dict(rows=1, out=BLOCK, out_row=0)])
def test_in_place_is_not_refused(good):
    """With a width that is refused for itself, so that nothing is launched: the status is that one's."""
    assert norm(**good, K=65537) == ESHAPE
