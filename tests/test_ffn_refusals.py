"""More of what the feed-forward calls refuse before they touch the device; no GPU."""
from __future__ import annotations

import pytest

from paper_2606_30634_gb300 import dpo
from test_ffn_oracle import addr, ffn_args, ffn_back_args, norm_args, packed, refused


@pytest.mark.parametrize("ld,shift", [(516, 0), (512, 4), (520, 1)])
def test_codes_of_the_backward_are_8_byte_aligned(ld, shift):
    p = dpo.dpo_packed8(addr(7) + shift, addr(8), ld, 16)
    refused("dpo_ffn_backward", ffn_back_args(gate8=p, up8=packed(9, ld, 16)), dpo.DPO_EALIGN)


# x is the left half of rows of 16384 bytes, 8192 of them its own; a block beside it has to
# begin there and end with the row.
@pytest.mark.parametrize("shift", [8192 - 2, 8192 + 2, 16384 - 8190, 3 * 16384 + 8192 - 2, 16384 * 7 + 8190,
                                   -2, -8190, -16384, -16384 + 2])
def test_columns_that_overlap_in_part(shift):
    args = norm_args(ld_x=8192, residual=None, y=addr(0) + shift, ld_y=8192)
    refused("dpo_rmsnorm", args, dpo.DPO_EINVAL)


@pytest.mark.parametrize("shift", [512 - 16, 512 + 16, 1024 * 7 + 512 - 16, -512 + 16, -512 - 16])
def test_columns_of_the_block_that_overlap_in_part(shift):
    refused("dpo_ffn_forward", ffn_args(ld_x=512, out=addr(0) + shift, ld_out=512), dpo.DPO_EINVAL)
    refused("dpo_ffn_backward", ffn_back_args(ld_dout=512, dx=addr(0) + shift, ld_dx=512),
            dpo.DPO_EINVAL)
    # other pitches: what lies between the rows counts
    refused("dpo_ffn_forward", ffn_args(ld_x=512, out=addr(0) + 512, ld_out=520), dpo.DPO_EINVAL)
