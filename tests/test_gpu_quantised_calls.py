"""Calls on quantised pages that the documentation allows, or has to refuse, beside those of test_gpu_quantised.py."""
import numpy as np
import pytest
import torch

import parity as P
import test_gpu_pages as T
import test_gpu_quantised as Q
from oracle import pages_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_load_into_rows_side_by_side_and_not_into_the_same(B, bits, dtype):
    """k and v of one buffer, in every nesting of (keys or values, sequence, head); on top of each other in whole or in part is refused."""
    n, hkv, cap, d, page = 3, 4, 20, 64, 16
    pg = T.make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=6, max_seqs=n, max_seq_pages=2, cache_bits=bits)
    dt = T.DT[dtype]
    shape = (6, hkv, pg.page_bytes()) if bits else (6, hkv, page, d)
    kp, vp = (torch.zeros(shape, dtype=torch.uint8 if bits else dt, device="cuda") for _ in range(2))
    t, lens = T.i32([[0, 1], [2, 3], [4, 5]]), T.i32([20, 17, 3])
    k, v = T.normal((n, hkv, cap, d), dt, 1), T.normal((n, hkv, cap, d), dt, 2)
    pg.page_store(k, v, lens, t, kp, vp)
    want = torch.full((2, n, hkv, cap, d), 7.0, dtype=dt, device="cuda")
    pg.page_load(kp, vp, t, lens, want[0], want[1])
    new = lambda *s: torch.full(s, 7.0, dtype=dt, device="cuda")
    a, b, c, e = new(n, 2, hkv, cap, d), new(n, hkv, 2, cap, d), new(hkv, n, 2, cap, d), new(2, hkv, n, cap, d)
    wide = new(n, 2 * hkv, cap, d)
    every = new(n, 3 * hkv, cap, d)
    for x, y in ((a[:, 0], a[:, 1]), (a[:, 1], a[:, 0]), (b[:, :, 0], b[:, :, 1]), (c[:, :, 0].transpose(0, 1), c[:, :, 1].transpose(0, 1)),
                 (e[0].transpose(0, 1), e[1].transpose(0, 1)), (wide[:, ::2], wide[:, 1::2]), (wide[:, hkv:], wide[:, :hkv]),
                 (every[:, 0:2 * hkv:2], every[:, 3:2 * hkv + 3:2])):
        pg.page_load(kp, vp, t, lens, x, y)
        pg.check()
        assert torch.equal(x, want[0]) and torch.equal(y, want[1])
        x.fill_(7.0), y.fill_(7.0)
    launches = pg.launch_count()
    long = new(n, hkv, 2 * cap, d)
    for x, y in ((k, k), (wide[:, :hkv], wide[:, 1:hkv + 1]), (wide[:, 1:hkv + 1], wide[:, :hkv]), (every[:, 0:2 * hkv:2], every[:, 2:2 * hkv + 2:2]),
                 (long[:, :, :cap], long[:, :, cap - 1:2 * cap - 1]), (long[:, :, 8:8 + cap], long[:, :, :cap])):
        with pytest.raises(ValueError):
            pg.page_load(kp, vp, t, lens, x, y)
    assert pg.launch_count() == launches
    pg.page_load(kp, vp, t, T.i32([0, 0, 0]), k[:, :, :0], k[:, :, :0])    # no rows, nothing to overlap
    pg.check()
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,lens,keep", [(28, 4, 128, 16, [5000, 17, 0, 300, 641], 40), (4, 4, 64, 64, [2000, 64, 1], 7), (16, 1, 256, 32, [3000, 100], 30)])
def test_chosen_pages_in_any_order(B, bits, dtype, hq, hkv, d, page, lens, keep):
    """Ragged sequences, the chosen pages of each backwards and shuffled: its last page, partly filled, stands anywhere in the list."""
    pg, q, kp, vp, table, out, lse = Q.attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=31)
    rng = np.random.default_rng(d)
    t, n = T.i32(table.tolist()), T.i32(lens)
    for turn in range(2):
        sel = np.full((len(lens), hkv, keep), 1 << 29, np.int32)   # behind min(keep, pages): never read
        for i, m in enumerate(lens):
            c = O.n_pages_of(m, page)
            for g in range(hkv):
                pick = np.sort(rng.permutation(c)[:min(keep, c)])
                pick[-1:] = c - 1                                  # (the last page always: where it was not chosen, for the largest one)
                sel[i, g, :len(pick)] = pick[::-1] if turn == 0 else rng.permutation(pick)
        pg.paged_attention(q, kp, vp, t, n, out, lse, sel=T.i32(sel.tolist()))
        pg.check()
        Q.check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype, sel, keep)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
def test_append_does_not_go_by_the_table(B, bits):
    """An append into a page that a bad table does not name is there all the same: rows go by their slots, and a read by that table reports the page and
    leaves its rows out."""
    hkv, d, page = 2, 64, 16
    pg = T.make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=4, max_seqs=1, max_seq_pages=2, cache_bits=bits)
    kp, vp = (torch.zeros((4, hkv, pg.page_bytes()), dtype=torch.uint8, device="cuda") for _ in range(2))
    k, v = T.normal((20, hkv, d), torch.bfloat16, 1), T.normal((20, hkv, d), torch.bfloat16, 2)
    slots = torch.tensor([2 * page + r if r < page else 1 * page + r - page for r in range(20)], device="cuda")
    pg.rope_append(None, k, v, None, slots, None, kp, vp)
    pg.check()
    back = torch.full((2, 1, hkv, 20, d), 7.0, dtype=torch.bfloat16, device="cuda")
    pg.page_load(kp, vp, T.i32([[2, 77]]), T.i32([20]), back[0], back[1])
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    held = [Q.rounded(O.held(*O.quantise(P.np64(x).astype(np.float32), bits)), "bf16").transpose(1, 0, 2) for x in (k, v)]
    for x, y in zip(back, held):
        np.testing.assert_array_equal(P.np64(x[0, :, :page]), y[:, :page])
        assert (x[0, :, page:] == 7).all()
    pg.page_load(kp, vp, T.i32([[2, 1]]), T.i32([20]), back[0], back[1])
    pg.check()
    for x, y in zip(back, held):
        np.testing.assert_array_equal(P.np64(x[0]), y)
    pg.close()
