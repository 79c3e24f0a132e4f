"""Page numbers outside the pool in what meda_page_tables moves: recorded, passed on as -1, never used as a page."""
import numpy as np
import pytest
import torch

import test_gpu_pages as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("bad", [-1, 8, 1 << 30, -(1 << 31)])
def test_an_entry_given_back_goes_onto_the_list_as_nothing_and_is_recorded_again(B, bad):
    table = np.array([[2, bad, 4], [1, -3, -3]])
    free = np.array([9, 9, 9, 9, 0, 3, 5, 6])                      # in front of 4: nothing
    got, status = T.run_tables(B, [40, 16], [10, 16], 16, 3, 8, 4, table, free, 4)
    assert status == B.MEDA_ERR_INVALID_ARG
    t, f, top, cu, slots = got
    assert top == 2 and f.tolist() == [9, 9, 4, -1, 0, 3, 5, 6] and cu.tolist() == [0, 0, 0] and (slots == -1).all()
    np.testing.assert_array_equal(t, table)
    # the next call takes -1 and 4 (in the list's order) and says so
    got, status = T.run_tables(B, [10, 16], [10, 40], 16, 3, 8, 2, t, f, 30)
    assert status == B.MEDA_ERR_INVALID_ARG
    t, _, top, cu, slots = got
    assert top == 4 and t[1].tolist() == [1, 4, -1] and cu.tolist() == [0, 0, 24]
    assert slots.tolist() == [4 * 16 + r for r in range(16)] + [-1] * 14


@pytest.mark.parametrize("bad", [-1, 8, 1 << 30, -(1 << 31)])
def test_an_entry_handed_on_taken_or_grown_into(B, bad):
    table = np.array([[2, bad, -3], [bad, -3, -3], [7, -3, -3]])
    free = np.array([9, 9, 9, 9, bad, 3, 5, 6])
    # sequence 0 gives `bad` to sequence 1, whose open page is bad too; sequence 2 takes the list's bad entry
    got, status = T.run_tables(B, [20, 9, 16], [16, 18, 17], 16, 3, 8, 4, table, free, 12)
    assert status == B.MEDA_ERR_INVALID_ARG
    t, f, top, cu, slots = got
    assert t[1, 1] == -1 and t[1, 0] == bad and t[2, 1] == -1 and top == 5
    assert cu.tolist() == [0, 0, 9, 10] and (slots == -1).all()
    np.testing.assert_array_equal(f, free)
    # appending to those slots touches nothing
    pg = T.make(B, page_size=16, n_pages=8, max_seqs=3, max_seq_pages=3)
    kp = torch.full((8, 2, 16, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    vp, k = kp.clone(), torch.ones((12, 2, 64), dtype=torch.bfloat16, device="cuda")
    pg.rope_append(None, k, k, None, torch.tensor(slots, device="cuda"), None, kp, vp)
    pg.check()
    assert (kp == 3).all() and (vp == 3).all()
    pg.close()
