"""More of what the feed-forward calls refuse before they touch the device; no GPU."""
from __future__ import annotations

import pytest

from paper_2606_30634_gb300 import dpo
from test_ffn_oracle import addr, ffn_back_args, packed, refused


@pytest.mark.parametrize("ld,shift", [(516, 0), (512, 4), (520, 1)])
def test_codes_of_the_backward_are_8_byte_aligned(ld, shift):
    p = dpo.dpo_packed8(addr(7) + shift, addr(8), ld, 16)
    refused("dpo_ffn_backward", ffn_back_args(gate8=p, up8=packed(9, ld, 16)), dpo.DPO_EALIGN)
