"""Which forms the feed-forward products take (dpo_ffn_test_forms) where as much is resident
as on a GB300, without one: the sizes of the GPU tests take the forms that those are
about, so a change of the estimates that empties one shows here first."""
from __future__ import annotations

import pytest

from ffn_forms import BACK, DOWN, DX, GATE, GB300, KEEP, LIST, NEAR, ROUNDS, SPLIT, WHOLE, forms, rounds
from paper_2606_30634_gb300 import dpo
from test_ffn_forms_gpu import SIZES

ALL = {**SPLIT, **ROUNDS, **WHOLE}


@pytest.mark.parametrize("size", ALL)
@pytest.mark.parametrize("keep", ["8bit", "bf16"])
def test_sizes_of_the_split_tests(size, keep):
    got = forms(size, keep)
    for product, (split, cols) in ALL[size].items():
        if keep == "bf16" and size[0] <= 8 and product in (GATE, DOWN):
            continue
        f = got[product]
        assert (f.kind, f.split, f.cols) == (dpo.DPO_FFN_SPLIT, split, cols), product
        assert (rounds(f) > 1) == (size in ROUNDS)


@pytest.mark.parametrize("slots", NEAR)
def test_the_gpu_tests_split_on_a_chip_with_other_clusters(slots):
    for sizes in (SPLIT, ROUNDS, WHOLE):
        for size, products in sizes.items():
            for keep in ("8bit", "bf16"):
                got = forms(size, keep, slots)
                for p in set(products) - {DX}:
                    if keep == "bf16" and size[0] <= 8 and p in (GATE, DOWN):
                        continue
                    assert got[p].kind == dpo.DPO_FFN_SPLIT and (rounds(got[p]) > 1) >= (sizes is ROUNDS)
    got = forms((20, 512, 4096), "8bit", slots)   # test_ffn_abi_gpu.py
    assert got[DOWN].kind == got[DX].kind == dpo.DPO_FFN_SPLIT
    for size in ((70, 1032, 264), (300, 200, 328), (2600, 136, 264)):
        assert forms(size, "8bit", slots)[DX].kind == dpo.DPO_FFN_NO_LAUNCH


def test_the_split_tests_reach_every_split():
    for product in (GATE, BACK):
        want = {(s, c) for s in (2, 4, 8) for c in (64, 128)}
        have = {v for sizes in (SPLIT, ROUNDS) for w in sizes.values() for p, v in w.items()
                if p == product}
        assert have == want
    # and stages of 32, 64 and 128 rows of A
    for product in (GATE, BACK):
        t = [s[0] for s, w in SPLIT.items() if product in w]
        assert min(t) <= 32 and any(32 < v <= 64 for v in t) and max(t) > 64


def test_sizes_of_the_other_forms():
    got = [forms(s, "8bit") for s in SIZES]
    assert {f[GATE].kind for f in got} == {dpo.DPO_FFN_SINGLE, dpo.DPO_FFN_PAIRS}
    assert {(f[DOWN].kind, f[DOWN].cols) for f in got} >= {(dpo.DPO_FFN_SPLIT, 64),
                                                           (dpo.DPO_FFN_SPLIT, 128)}
    assert {f[DX].kind for f in got} == {dpo.DPO_FFN_NO_LAUNCH, dpo.DPO_FFN_SPLIT}
    assert {f[LIST].kind for f in got} == {dpo.DPO_FFN_SINGLE, dpo.DPO_FFN_PAIRS}
    assert max(rounds(f[LIST]) for f in got) > 1
    pairs = forms((2600, 1048, 4136), "8bit")   # test_ffn_by_cta_pairs
    assert all(pairs[p].kind == dpo.DPO_FFN_PAIRS for p in (GATE, BACK, LIST))
    assert all(rounds(pairs[p]) > 2 for p in (GATE, BACK, LIST))


@pytest.mark.parametrize("tokens,keep,streamed", [(1, "none", True), (8, "bf16", True),
                                                  (8, "8bit", False), (9, "none", False)])
def test_few_tokens_stream_the_weights(tokens, keep, streamed):
    got = forms((tokens, 4096, 11008), keep)
    assert all((got[p].kind == dpo.DPO_FFN_STREAM) == streamed for p in (GATE, DOWN))


@pytest.mark.parametrize("args", [(0, 64, 64, 1), (-1, 64, 64, 1), (4, 60, 64, 1), (4, 64, 64, 3),
                                  (1 << 40, 64, 64, 1)])
def test_bad_arguments(args):
    with pytest.raises(dpo.DpoError) as e:
        dpo.dpo_ffn_test_forms(*args, GB300)
    assert e.value.code == dpo.DPO_EINVAL


def test_bad_slots():
    with pytest.raises(dpo.DpoError):
        dpo.dpo_ffn_test_forms(4, 64, 64, KEEP["none"], (76, 152, 152, 76, 0, 15))
    assert dpo.load().dpo_ffn_test_forms(4, 64, 64, 0, None, None) == dpo.DPO_EINVAL
