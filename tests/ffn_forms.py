"""Sizes of the feed-forward tests and the forms that they are there for."""
from __future__ import annotations

from paper_2606_30634_gb300 import dpo

GATE, DOWN, BACK, DX, LIST = range(5)   # dpo_ffn_test_forms
KEEP = {"none": dpo.DPO_KEEP_NONE, "8bit": dpo.DPO_KEEP_8BIT, "bf16": dpo.DPO_KEEP_BF16}
# What a GB300 holds at once: CTA pairs, single CTAs, clusters of 1, 2, 4, 8. The larger clusters'
# numbers go by how a chip's SMs are spread, so the sizes of the GPU tests split their products
# with a few more or less too (all but DX of ROUNDS).
GB300 = (76, 152, 152, 76, 36, 15)
NEAR = [(76, 152, 152, 76, s4, s8) for s4 in (33, 36, 38) for s8 in (13, 15, 16, 18)]

# (tokens, dim, hidden): {product: (shares of K, a tile's columns)}. Widths end inside a stage
# of 64 of K and inside a tile; 32, 64 or 128 rows of A.
SPLIT = {
    (14, 1672, 2320): {GATE: (2, 64)},
    (51, 2088, 2552): {GATE: (2, 128)},
    (572, 2056, 456): {GATE: (2, 64)},
    (48, 1416, 536): {GATE: (4, 64)},
    (19, 1648, 1160): {GATE: (4, 128)},
    (261, 1448, 392): {GATE: (4, 128)},
    (39, 2560, 528): {GATE: (8, 128)},
    (135, 1408, 256): {GATE: (8, 128)},
    (69, 1416, 8): {GATE: (8, 64), BACK: (8, 64)},
    (570, 2064, 920): {BACK: (2, 64)},
    (397, 1560, 584): {BACK: (4, 128)},
    (14, 1824, 4880): {BACK: (2, 128)},
    (462, 2296, 1280): {BACK: (2, 128)},
    (47, 1456, 1048): {BACK: (4, 64)},
    (19, 1544, 2320): {BACK: (4, 128)},
    (19, 1808, 976): {BACK: (8, 128)},
    (134, 1320, 560): {BACK: (8, 128)},
}
# More tiles than clusters, so that a cluster's exchange and rings go round again; and one
# share of K, the split form's own epilogue on whole tiles.
ROUNDS = {
    (29, 1704, 10056): {GATE: (2, 128)},
    (29, 3984, 5048): {GATE: (4, 128)},
    (4, 4008, 9816): {BACK: (4, 128)},
    (552, 1928, 6072): {DOWN: (4, 128)},
    (438, 1264, 3232): {DX: (8, 128)},
}
WHOLE = {(26, 4152, 7056): {GATE: (1, 128)}}


def forms(size, keep, slots=GB300):
    return dpo.dpo_ffn_test_forms(*size, KEEP[keep], slots)


def rounds(form):
    return -(-form.tiles // form.slots)
