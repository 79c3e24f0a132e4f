"""Every row of a cache counts once, and the decoder's choice of pages: tests that one lost or doubled tile, or one stale bound, fails.

With queries of zero every logit is 0 and every weight exactly 1 (2^0 has no rounding), so a softmax sum is the number of rows, exact
below 2^24, and lse = log(rows): log2 is off by one unit in the last place at most (2^-23 relative), the constant by 2^-24 and the
product by 2^-24, together below 2^-22 of it.  One row of n missing moves it by 1 / n.  Values that are 1 in one dimension of a row and 0
elsewhere make an output element the share of the rows with that code: sums of ones, exact, then the reciprocal and a product (2^-24
each) and the rounding to the type."""
import math

import numpy as np
import pytest
import torch

import paged_steps as S
import test_gpu_pages as T
from oracle import pages_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def codes(lens, d):
    """Row number -> dimension, three ways: by tile modulo d, by runs of tiles, by row modulo d."""
    tiles = max(1, -(-max(lens) // 16))
    return {"tile": lambda r: r // 16 % d, "run": lambda r: r // 16 // -(-tiles // d), "row": lambda r: r % d}


RAGGED = [0, 0] + [int(round(36 * (18_944 / 36) ** (i / 61))) for i in range(62)]
CASES = [("bf16", 28, 4, 128, 64, [129_072]), ("bf16", 28, 4, 128, 16, RAGGED), ("bf16", 4, 4, 64, 32, [20_000, 3, 9000]), ("bf16", 7, 1, 128, 16, [40_001, 17]),
         ("bf16", 16, 1, 128, 16, [30_011]), ("bf16", 16, 2, 64, 16, [3000, 1999, 501, 16]), ("bf16", 8, 1, 256, 16, [9001, 100]), ("bf16", 11, 1, 256, 64, [5000, 777, 1]),
         ("f32", 4, 4, 64, 32, [6000, 1, 0, 12_345]), ("f32", 7, 1, 128, 32, [7001, 4000]), ("f32", 12, 1, 128, 16, [2500, 37]), ("f32", 4, 1, 256, 16, [4001]),
         ("f32", 16, 1, 256, 16, [1500, 90])]


@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", CASES)
@pytest.mark.parametrize("chosen", [False, True])
def test_every_row_counts_once(B, dtype, hq, hkv, d, page, lens, chosen):
    pg, q, kp, vp, table, out, lse = T.attention_case(B, lens, hq, hkv, d, dtype, page, seed=51, q_std=0.0)
    t, n, group = T.i32(table.tolist()), T.i32(lens), hq // hkv
    sel = None
    if chosen:                                                     # all pages, in an order of their own for every head
        rng = np.random.default_rng(7)
        sel = np.full((len(lens), hkv, table.shape[1]), 1 << 30, np.int64)
        for i, m in enumerate(lens):
            for g in range(hkv):
                sel[i, g, :O.n_pages_of(m, page)] = rng.permutation(O.n_pages_of(m, page))
        sel = torch.tensor(sel, dtype=torch.int32, device="cuda")
    for name, code in codes(lens, d).items():
        vp.fill_(math.nan)
        want = np.zeros((len(lens), hq, d))
        for i, m in enumerate(lens):
            if m == 0:
                continue
            rows = np.arange(m)
            for g in range(hkv):                                   # heads differ, so that one's rows cannot stand in for another's
                at = (code(rows) + 5 * g) % d
                counts = np.bincount(at, minlength=d)
                want[i, g * group:(g + 1) * group] = counts / m
                if name != "row" and m >= 16:                      # a tile more or less in any dimension is seen
                    assert 16 / counts.max() > 2 * T.HALF_STEP[dtype] * 1.01 + 2.0 ** -21
                hot = torch.zeros((O.n_pages_of(m, page) * page, d), dtype=vp.dtype, device="cuda")
                hot[torch.as_tensor(rows, device="cuda"), torch.as_tensor(at, device="cuda")] = 1.0
                hot[m:] = math.nan
                vp[t[i, :O.n_pages_of(m, page)].long(), g] = hot.view(-1, page, d)
        out.fill_(math.nan)
        lse.fill_(math.nan)
        pg.paged_attention(q, kp, vp, t, n, out, lse, sel=sel)
        pg.check()
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        bound = (T.HALF_STEP[dtype] * 1.01 + 2.0 ** -22) * want
        assert (np.abs(got - want) <= bound).all(), (name, float((np.abs(got - want) - bound).max()))
        for i, m in enumerate(lens):
            if m == 0:
                assert (got_lse[i] == -np.inf).all()
                continue
            assert (np.abs(got_lse[i] - math.log(m)) <= 2.0 ** -22 * math.log(m)).all(), (i, m)
            assert m == 1 or 2.0 ** -22 * math.log(m) < 0.5 / m    # one row more or less is seen
    pg.close()


LONG = [("bf16", 28, 4, 128, 64, [129_072]), ("bf16", 7, 1, 128, 16, [40_001, 17]), ("bf16", 28, 4, 128, 16, RAGGED), ("bf16", 16, 1, 64, 16, [30_011]),
        ("bf16", 8, 1, 256, 16, [9001, 100]), ("f32", 7, 1, 128, 32, [7001, 4000]), ("f32", 4, 1, 256, 16, [4001]), ("f32", 4, 4, 64, 32, [6000, 1, 0, 12_345])]


@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", LONG)
def test_long_caches_with_random_queries(B, dtype, hq, hkv, d, page, lens):
    """The sums over the rows are short chains: a warp adds its own tiles (six roundings of 2^-22 at most for each: two additions, a
    change of the maximum with its exponential, factor and product, and the weights' own), at most 16 warps are joined in a block, at most a
    block per SM in the end (two roundings each).  Tiles are dealt evenly to the blocks, 20 more for each segment counted, of eight tiles
    per block at least, and to no fewer than eight warps (a warp may have one more).  The rest is attention_tolerance's."""
    pg, q, kp, vp, table, out, lse = T.attention_case(B, lens, hq, hkv, d, dtype, page, seed=61)
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse)
    pg.check()
    sms, group = torch.cuda.get_device_properties(0).multi_processor_count, hq // hkv
    segments = hkv * -(-group // 4) * len(lens)                    # four query heads to a segment at least (fewer only where the group is smaller)
    tiles = sum(-(-m // 16) for m in lens) * (segments // len(lens)) + 20 * segments
    chain = (6 * (-(-max(8, tiles // sms + 1) // 8) + 1) + 2 * 16 + 2 * sms) * 2.0 ** -22
    got, got_lse, qh = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    for i, m in enumerate(lens):
        pages = torch.as_tensor(table[i, :O.n_pages_of(m, page)].astype(np.int64), device="cuda")
        for g in range(hkv):
            k, v = (x[pages, g].double().cpu().numpy().reshape(-1, d)[:m] for x in (kp, vp))
            heads = slice(g * group, (g + 1) * group)
            want, want_lse, aux = O.attention(qh[i, heads], k, v)
            if m == 0:
                assert (got[i, heads] == 0).all()
                continue
            delta = (d + 16) * 2.0 ** -22 * aux["mag"]
            rel = 2 * delta * (1 + delta) + chain + 2.0 ** -16
            assert (np.abs(got[i, heads] - want) <= aux["spread"] * rel[:, None] + T.HALF_STEP[dtype] * np.abs(want) * 1.01).all(), (i, g)
            assert (np.abs(got_lse[i, heads] - want_lse) <= delta + chain + 2.0 ** -22 * np.abs(want_lse) + 1e-6).all(), (i, g)
    pg.close()


@pytest.mark.parametrize("graph", [False, True])
def test_decoding_over_chosen_pages(B, graph):
    """Steps with a choice of pages while requests come and go: after every step the bounds of all pages in use are those of the pool's
    rows, the choice is the one they give, and the outputs are the attention over the chosen pages."""
    wl = S.workload()
    cps = [S.compressed(wl), S.compressed(wl.with_(seed=9))]
    dec = S.decoder(wl, 120, 3, 400, keep_pages=6)
    st = S.Steps(wl, dec)
    st.admit(0, cps[0])
    run = None
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            st.step([0])                                           # loads the kernels
        side.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            st.body()
        run = captured.replay
    left_out = 0
    for n in range(30):
        if n == 2:
            st.admit(2, cps[1])
        if n == 12:
            st.release(0)                                          # its pages serve others from here on
        if n == 14:
            st.admit(1, cps[0])
        if n == 19:
            st.admit(2, cps[0])                                    # replaced
        live = sorted({r for r, _ in st.rows})
        st.step(live, run)
        dec.check()
        st.check_caches(live)
        st.check_outputs(live)
        left_out += st.check_choice(live)
    assert left_out > 100
    dec.close()
    for cp in cps:
        cp.close()
