"""Values that are infinite: a softmax weight is above 0, so they reach the output as infinities of their sign, in their own
dimension only; both signs in one dimension, or a NaN, make it NaN."""
import math

import numpy as np
import pytest
import torch

import parity as P
import test_gpu_pages as T
from oracle import pages_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


# lengths around the tiles' and the four-row groups' borders, and long ones that many blocks share
LENS = [1, 2, 4, 5, 8, 13, 15, 16, 17, 32, 33, 47, 64, 65, 200, 209]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,lens,flat", [(2, 1, 64, LENS, False), (28, 4, 128, LENS, False), (16, 1, 128, LENS, False), (7, 1, 256, LENS, False),
                                                (4, 1, 64, LENS, True), (3, 1, 128, LENS, True), (2, 2, 256, LENS, True), (7, 1, 128, [5003, 3000], False),
                                                (2, 1, 256, [4001], True)])
def test_infinite_values(B, dtype, hq, hkv, d, lens, flat):
    page = 16
    # logits of unit spread (or all equal: every weight is 1, the low half of which is 0): no weight is anywhere near 2^-126
    pg, q, kp, vp, table, out, lse = T.attention_case(B, lens, hq, hkv, d, dtype, page, seed=41, q_std=0.0 if flat else 1.0)
    def cell(i, row):
        return vp[int(table[i, row // page]), :, row % page]
    t, n = T.i32(table.tolist()), T.i32(lens)
    pg.paged_attention(q, kp, vp, t, n, out, lse)                  # the finite case: what all other dimensions have to stay
    finite, finite_lse = out.clone(), lse.clone()
    want = P.np64(out)
    for i, m in enumerate(lens):
        cell(i, m - 1)[:, 3] = math.inf                            # the last row, which a ragged tile meets more than once
        cell(i, 0)[:, 5] = -math.inf
        cell(i, m // 2)[:, 8] = math.inf
        want[i, :, 3], want[i, :, 5], want[i, :, 8] = np.inf, -np.inf, np.inf
        if m > 1:
            cell(i, 0)[:, 11] = math.inf                           # both signs
            cell(i, m - 1)[:, 11] = -math.inf
            cell(i, m - 1)[:, 14] = math.nan
            want[i, :, 11] = want[i, :, 14] = np.nan
    pg.paged_attention(q, kp, vp, t, n, out, lse)
    pg.check()
    np.testing.assert_array_equal(P.np64(out), want)
    assert torch.equal(lse, finite_lse)
    # the last row's infinities are gone with the row
    shorter = [m - 1 for m in lens]
    pg.paged_attention(q, kp, vp, t, T.i32(shorter), out, lse)
    pg.check()
    for i, m in enumerate(shorter):
        if m:
            keep = torch.tensor([x for x in range(d) if x not in (3, 5, 8, 11, 14)], device="cuda")
            got = out[i][:, keep]
            assert got.isfinite().all()
            assert (out[i, :, 3].isfinite() & out[i, :, 14].isfinite()).all() and (out[i, :, 5] == -math.inf).all()
            assert (out[i, :, 11] == math.inf).all()
    pg.close()
