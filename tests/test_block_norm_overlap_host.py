"""The norm's output in the place of its branch: refused where their rows would not lie on one another."""

import pytest

from paper_2605_28803_gb300 import qvla as Q


class At:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("quant", [False, True])
def test_h_in_the_place_of_y(quant):
    norm = Q.BlockNorm(Q.NORM_RMS, Q.BF16)
    r, y, r_out, q, s = (At(i << 30) for i in range(1, 6))
    more = (1, Q.MXFP4, None, q, s) if quant else ()
    call = Q.qvla_block_norm_fp4 if quant else Q.qvla_block_norm
    with pytest.raises(Q.QvlaError, match="y_stride") as e:
        call(norm, r, Q.BF16, 256, y, 264, 3, 256, r_out, y, *more)
    assert e.value.status == 1
    call(norm, r, Q.BF16, 256, y, 256, 0, 256, r_out, y, *more)  # (no rows: nothing is launched)
