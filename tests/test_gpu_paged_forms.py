"""The forms attention over the paged cache takes: an item (sequence, key head, one or two row tiles) left to one workgroup, or its steps
divided among several whose parts are joined.  Which one is chosen goes by how long sequences may be: a page table with room for many more
slots sends the same calls to the divided form.  Everything is compared with the definition in 64 bits, as where it fits one workgroup."""
import numpy as np
import pytest

import paged_reference as R
import test_gpu_paged as base

pytestmark = pytest.mark.gpu


@pytest.fixture
def roomy(monkeypatch):
    """Caches whose tables have room for 2^17 slots more a sequence, without pages."""
    plain = R.Cache.__init__

    def init(self, *args, **kwargs):
        plain(self, *args, **kwargs)
        self.table = np.pad(self.table, ((0, 0), (0, (1 << 17) // self.page)), constant_values=-1)
    monkeypatch.setattr(R.Cache, "__init__", init)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("dh,heads,kv,page,rows,lengths", [
    (128, 2, 2, 16, 1, [0]), (128, 4, 2, 16, 1, [15, 16, 31, 32]), (128, 2, 1, 32, 16, [97]), (128, 1, 1, 16, 17, [40, 3]),
    (64, 6, 2, 128, 26, [300]), (128, 8, 1, 64, 33, [129, 64]), (128, 1, 1, 256, 64, [5, 260]), (64, 2, 2, 16, 64, [1000]),
    (128, 16, 1, 64, 60, [90]), (64, 64, 1, 16, 1, [257]), (128, 2, 1, 64, 20, [3000, 17, 1200]), (64, 3, 1, 64, 5, [4000])])
def test_causal_rows_divided(roomy, bf16, dh, heads, kv, page, rows, lengths):
    base.test_attention_of_causal_rows(bf16, dh, heads, kv, page, rows, lengths)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("topk,widths,lengths,per_seq", [([4, 2, 2, 1, 1], [1, 4, 8, 6, 4, 3], [100, 37], False),
                                                         ([10, 5, 3, 2], [1, 10, 20, 18, 15], [7, 0, 250], True)])
def test_trees_divided(roomy, bf16, topk, widths, lengths, per_seq):
    base.test_attention_of_trees(bf16, topk, widths, lengths, per_seq)


@pytest.mark.parametrize("bf16", [True, False])
def test_masks_that_leave_nothing_divided(roomy, bf16):
    base.test_rows_whose_mask_leaves_nothing_and_masks_of_any_form(bf16)


@pytest.mark.parametrize("bf16", [True, False])
def test_not_a_number_divided(roomy, bf16):
    base.test_not_a_number_reaches_the_rows_that_see_it_and_no_other(bf16)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("lo,hi", [(27, 60), (95, 112), (200, 230), (27, 230)])
def test_values_of_any_magnitude_divided(roomy, bf16, lo, hi):
    base.test_values_of_any_magnitude(bf16, lo, hi)


def test_a_dominant_late_key_and_many_sequences_divided(roomy):
    base.test_a_dominant_late_key_and_scores_far_apart()
    base.test_more_sequences_than_a_wave_has_lanes()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
def test_two_row_tiles_in_one_workgroup(bf16, dh):
    """More items of one tile than the chip has compute units: 40 sequences of 4 key heads and 20 rows."""
    rng = np.random.default_rng(dh)
    lengths = [int(v) for v in rng.integers(0, 130, 40)]
    ref = R.Cache(rng, 1, 40, 4, 16, dh, lengths, 20)
    q = base.rounded(rng.standard_normal((40, 20, 4, dh)), bf16).astype(np.float64)
    want = ref.attend(0, q, base.causal(40, 20), 0.1)
    got = base.run_attend(ref, q, bf16, scale=0.1)
    assert base.agrees(ref, 0, q, 0.1, bf16, got, want).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_items_in_more_than_one_round(bf16):
    rng = np.random.default_rng(21)
    lengths = [int(v) for v in rng.integers(0, 300, 150)]
    ref = R.Cache(rng, 1, 150, 4, 16, 64, lengths, 1)
    q = base.rounded(rng.standard_normal((150, 1, 8, 64)), bf16).astype(np.float64)
    want = ref.attend(0, q, base.causal(150, 1), 0.125)
    got = base.run_attend(ref, q, bf16, scale=0.125)
    assert base.agrees(ref, 0, q, 0.125, bf16, got, want).all()
