"""The paged-cache operators on the device against the fp64 / integer oracle (oracle/pages_oracle.py), operator by
operator and as a run of them.

Tolerances.  Integers (tables, slots, lists, bounds of bf16 and fp32 keys, copied rows) are compared exactly.  Rotary: one
rounding to the output's type (half a step: 2^-8 relative in bf16, 2^-24 in fp32), and for the sine and cosine an error
of at most 2^-20 of |a| + |b|: the fraction of a turn is rounded to fp32 (pi * 2^-24 of the angle at most half a turn), sincospi
is off by 2^-23 at most, and three fp32 operations follow.  Attention: see attention_tolerance."""
import math

import numpy as np
import pytest
import torch

import parity as P
from oracle import pages_oracle as O
from paper_2502_17599_b200 import workloads as W

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def make(B, **kw):
    base = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", page_size=16, n_pages=64, max_seqs=64, max_seq_pages=16)
    base.update(kw)
    return B.Pages(**base)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def normal(shape, dtype, seed, mean=0.0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def table_for(lens, page, width, n_pages, seed):
    """Pages handed out in a shuffled order; unused entries hold a page number far outside the pool."""
    rng = np.random.default_rng(seed)
    order = rng.permutation(n_pages)
    table = np.full((len(lens), width), 1 << 30, np.int32)
    at = 0
    for i, n in enumerate(lens):
        c = O.n_pages_of(n, page)
        table[i, :c] = order[at:at + c]
        at += c
    return table


# ------------------------------------------------------------------------------------------------ tables

def run_tables(B, lens, new, page, width, n_pages, top, table, free, capacity, stride=1):
    pg = make(B, page_size=page, n_pages=n_pages, max_seqs=max(1, len(new)), max_seq_pages=width)
    spread = lambda x: torch.stack([i32(x)] + [torch.full((len(x),), -7, dtype=torch.int32, device="cuda")] * (stride - 1), 1)[:, 0]
    d_table, d_free = i32(table.tolist()).view(len(new), width), i32(free.tolist())
    top_in, top_out, cu = i32([top]), i32([-5]), i32([-5] * (len(new) + 1))
    slots = torch.full((capacity,), -9, dtype=torch.int64, device="cuda")
    pg.page_tables(None if lens is None else spread(lens), spread(new), d_free, top_in, top_out, d_table, cu, slots)
    status = pg.poll_status()
    got = (d_table.cpu().numpy(), d_free.cpu().numpy(), int(top_out), cu.cpu().numpy(), slots.cpu().numpy())
    assert int(top_in) == top
    pg.close()
    return got, status


def same_tables(got, want):
    for a, b, what in zip(got, want, ("table", "free_pages", "free_top", "cu_new", "slots")):
        np.testing.assert_array_equal(np.asarray(a, np.int64), np.asarray(b, np.int64), err_msg=what)


@pytest.mark.parametrize("n,page,hi,stride,seed", [(1, 16, 40, 1, 0), (1, 256, 600, 1, 1), (7, 16, 100, 3, 2), (33, 32, 257, 1, 3),
                                                   (300, 16, 90, 2, 4), (513, 64, 500, 1, 5), (2000, 16, 70, 1, 6), (1100, 16, 1300, 3, 7)])
def test_page_tables_against_the_oracle(B, n, page, hi, stride, seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, hi + 1, n)
    new = np.where(rng.random(n) < 0.2, 0, np.where(rng.random(n) < 0.3, rng.integers(0, hi + 1, n), np.minimum(lens + 1, hi)))
    width = O.n_pages_of(hi, page) + 1
    used = sum(O.n_pages_of(int(x), page) for x in lens)
    need = sum(O.n_pages_of(int(x), page) for x in new)
    n_pages = max(used, need) + 5
    table = table_for(lens, page, width, used, seed)
    perm = rng.permutation(n_pages)
    held = table[table < (1 << 30)]
    free = np.concatenate([np.full(used, 999999), np.setdiff1d(perm, held)]).astype(np.int64)[:n_pages]
    capacity = int(np.maximum(new - lens, 0).sum()) + 3
    want = O.page_tables(lens, new, free, used, table, page, capacity)
    assert want[5]
    got, status = run_tables(B, lens.tolist(), new.tolist(), page, width, n_pages, used, table, free, capacity, stride)
    assert status == 0
    same_tables(got, want)


def test_page_tables_from_nothing_and_without_a_slot_map(B):
    lens = [0, 17, 64, 1, 0, 33]
    table = np.full((6, 4), -3, np.int32)
    free = np.random.default_rng(0).permutation(20)
    want = O.page_tables(None, lens, free, 0, table, 16, 120)
    got, status = run_tables(B, None, lens, 16, 4, 20, 0, table, free, 120)
    assert status == 0
    same_tables(got, want)
    got, status = run_tables(B, None, lens, 16, 4, 20, 0, table, free, 0)
    assert status == 0
    same_tables(got[:4], want[:4])
    # no sequence at all: the list's front is passed on
    got, status = run_tables(B, None, [], 16, 4, 20, 7, table[:0], free, 3)
    assert status == 0 and got[2] == 7 and got[3].tolist() == [0] and (got[4] == -1).all()


@pytest.mark.parametrize("case", ["pool", "capacity", "negative", "too_long", "front", "front_negative"])
def test_page_tables_refuses_and_changes_nothing(B, case):
    lens, new, page, width, n_pages, top, capacity = [16, 0], [40, 20], 16, 4, 6, 1, 44
    code = B.MEDA_ERR_INVALID_ARG
    if case == "pool":
        n_pages, code = 4, B.MEDA_ERR_WORKSPACE
    elif case == "capacity":
        capacity, code = 43, B.MEDA_ERR_WORKSPACE
    elif case == "negative":
        lens = [16, -1]
    elif case == "too_long":
        new = [40, 65]
    elif case == "front":
        top = 7
    else:
        top = -1
    table = np.full((2, width), 3, np.int32)
    free = np.arange(n_pages)
    want = O.page_tables(lens, new, free, top, table, page, capacity)
    assert not want[5]
    got, status = run_tables(B, lens, new, page, width, n_pages, top, table, free, capacity)
    assert status == code
    same_tables(got, want)


def test_page_tables_steps_never_share_a_page(B):
    """Two hundred random changes: no page has two owners, and list and tables together hold every page."""
    rng = np.random.default_rng(3)
    n, page, width, n_pages = 37, 16, 9, 200
    pg = make(B, page_size=page, n_pages=n_pages, max_seqs=n, max_seq_pages=width)
    table, free = i32(np.full((n, width), -1).tolist()), i32(rng.permutation(n_pages).tolist())
    top, out, cu = i32([0]), i32([0]), i32([0] * (n + 1))
    slots = torch.empty(n * width * page, dtype=torch.int64, device="cuda")
    lens = np.zeros(n, np.int64)
    moved = 0
    for step in range(200):
        new = np.where(rng.random(n) < 0.15, rng.integers(0, width * page + 1, n), np.minimum(lens + 1, width * page))
        new = np.where(rng.random(n) < 0.05, 0, new)
        pg.page_tables(i32(lens.tolist()), i32(new.tolist()), free, top, out, table, cu, slots)
        status = pg.poll_status()
        fits = sum(O.n_pages_of(int(x), page) for x in new) <= n_pages
        assert status == (0 if fits else B.MEDA_ERR_WORKSPACE)
        top.copy_(out)
        if fits:
            lens = new
            moved += 1
        t = table.cpu().numpy()
        held = [int(t[i, p]) for i in range(n) for p in range(O.n_pages_of(int(lens[i]), page))]
        rest = free.cpu().numpy()[int(top):].tolist()
        assert sorted(held + rest) == list(range(n_pages)), step
    assert moved > 20
    pg.close()


def test_page_tables_largest_batch(B):
    """8,192 sequences (all the shared memory the scans take), most of them untouched."""
    rng = np.random.default_rng(9)
    n, page, width = 8192, 16, 6
    lens = rng.integers(0, 90, n)
    new = np.where(rng.random(n) < 0.9, lens, rng.integers(0, 97, n))
    used = sum(O.n_pages_of(int(x), page) for x in lens)
    table = table_for(lens, page, width, used, 1)
    n_pages = used + 9000
    free = np.concatenate([np.zeros(used), np.arange(used, n_pages)]).astype(np.int64)
    capacity = int(np.maximum(new - lens, 0).sum()) + 1000
    want = O.page_tables(lens, new, free, used, table, page, capacity)
    got, status = run_tables(B, lens.tolist(), new.tolist(), page, width, n_pages, used, table, free, capacity)
    assert want[5] and status == 0
    same_tables(got, want)


# ------------------------------------------------------------------------------------------------- store

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 128), (128, 16), (128, 64), (256, 32), (256, 256)])
def test_page_store_and_bounds(B, dtype, d, page):
    hkv, cap = 3, 300
    lens = [0, 1, 15, 16, 17, 255, 256, 257, 300, 299]
    n, width = len(lens), O.n_pages_of(cap, page)
    need = sum(O.n_pages_of(x, page) for x in lens)
    n_pages = need + 4
    table = table_for(lens, page, width, n_pages, d + page)
    pg = make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=n, max_seq_pages=width)
    # heads and sequences strided: every other head of a larger cache; rows behind a length are NaN
    base = normal((n, 2 * hkv, cap + 2, d), DT[dtype], 5, 0.5)
    both = torch.stack([base, base * -1.5])
    k, v = both[0, :, ::2, :cap], both[1, :, ::2, :cap]
    for i, m in enumerate(lens):
        both[:, i, :, m:] = math.nan
    kp = torch.full((n_pages, hkv, page, d), 7.0, dtype=DT[dtype], device="cuda")
    vp, bd = torch.full_like(kp, 8.0), torch.full((n_pages, hkv, 2, d), 9.0, dtype=DT[dtype], device="cuda")
    want_k, want_v, want_b = P.np64(kp), P.np64(vp), P.np64(bd)
    kh, vh = P.np64(k), P.np64(v)
    for i, m in enumerate(lens):
        for c in range(O.n_pages_of(m, page)):
            r0, r1 = c * page, min(m, c * page + page)
            want_k[table[i, c], :, :r1 - r0] = kh[i, :, r0:r1]
            want_v[table[i, c], :, :r1 - r0] = vh[i, :, r0:r1]
            for g in range(hkv):
                want_b[table[i, c], g] = O.page_bounds(kh[i, g, r0:r1])
    t = i32(table.tolist())
    pg.page_store(k, v, i32(lens), t, kp, vp, bd)
    pg.check()
    np.testing.assert_array_equal(P.np64(kp), want_k)              # rows behind a length keep what they held
    np.testing.assert_array_equal(P.np64(vp), want_v)
    np.testing.assert_array_equal(P.np64(bd), want_b)
    # the bounds alone, over all pages, and only over those that a range of rows touches
    again = torch.full_like(bd, 9.0)
    pg.page_bounds(kp, t, None, i32(lens), again)
    pg.check()
    np.testing.assert_array_equal(P.np64(again), want_b)
    part = torch.full_like(bd, 9.0)
    start = [max(0, m - 3) for m in lens]
    start[3] = lens[3]                                             # nothing new
    pg.page_bounds(kp, t, i32(start), i32(lens), part)
    pg.check()
    want_part = np.full_like(want_b, 9.0)
    for i, m in enumerate(lens):
        if start[i] < m:
            for c in range(start[i] // page, O.n_pages_of(m, page)):
                want_part[table[i, c]] = want_b[table[i, c]]
    np.testing.assert_array_equal(P.np64(part), want_part)
    pg.close()


def test_page_store_skips_what_does_not_fit_and_keeps_nan_keys(B):
    hkv, d, page, cap = 2, 64, 16, 40
    lens = [33, 41, 20]                                            # the second is longer than its source
    table = np.array([[5, 2, 1], [3, 4, 0], [6, 99, 7]], np.int32)   # the third's second page is outside the pool
    pg = make(B, n_q_heads=2, n_kv_heads=hkv, head_dim=d, dtype="f32", page_size=page, n_pages=8, max_seqs=3, max_seq_pages=3)
    k, v = normal((3, hkv, cap, d), torch.float32, 1), normal((3, hkv, cap, d), torch.float32, 2)
    k[0, 1, 35 - 3, 7] = math.nan
    kp = torch.zeros((8, hkv, page, d), device="cuda")
    vp, bd = torch.zeros_like(kp), torch.zeros((8, hkv, 2, d), device="cuda")
    pg.page_store(k, v, i32(lens), i32(table.tolist()), kp, vp, bd)
    assert pg.poll_status() in (B.MEDA_ERR_WORKSPACE, B.MEDA_ERR_INVALID_ARG)
    assert pg.poll_status() == 0
    assert (kp[[0, 3, 4, 7]] == 0).all() and (bd[[0, 3, 4, 7]] == 0).all()
    assert torch.equal(kp[6], k[2, :, :16]) and torch.equal(vp[2], v[0, :, 16:32])
    assert bd[1, 1, :, 7].isnan().all() and bd[1, 0].isnan().sum() == 0 and bd[1, 1].isnan().sum() == 2
    # lengths outside [0, capacity of a table row]: the store skips them, the bounds take the nearest
    kp.zero_()
    pg.page_store(k, v, i32([-4, 0, 49]), i32(table.tolist()), kp, vp)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG and (kp == 0).all()
    pg.close()


# ------------------------------------------------------------------------------------------------- rotary

ROPES = [((32, 0, 0), 0), ((8, 12, 12), 0), ((12, 10, 10), 1), ((4, 2, 2), 1), ((0, 16, 16), 0), ((16, 8, 0), 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("sections,order", ROPES)
@pytest.mark.parametrize("d,t", [(64, 1), (128, 37), (256, 5)])
def test_rope_append(B, dtype, pairing, sections, order, d, t):
    hq, hkv, page, n_pages = 6, 2, 16, t + 2
    half = sum(sections)
    pg = make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, rope_theta=1e6,
              rope_sections=sections, rope_order=order, rope_pairing=pairing)
    rng = np.random.default_rng(t)
    qkv = normal((t, hq + 2 * hkv + 1, d), DT[dtype], 3, 0.1, 2.0)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
    pos = rng.integers(0, 1_000_000, (3, t + 5)).astype(np.int32)
    pos[:, 0] = [2 ** 31 - 1, -17, 0]
    slots = rng.permutation(n_pages * page)[:t]
    slots[1::4] = -1
    q_out = torch.full((t, hq, d), 5.0, dtype=DT[dtype], device="cuda")
    kp = torch.full((n_pages, hkv, page, d), 6.0, dtype=DT[dtype], device="cuda")
    vp = torch.full_like(kp, 7.0)
    d_pos = i32(pos.tolist())[:, :t]                               # axes farther apart than the tokens
    pg.rope_append(q, k, v, d_pos, torch.tensor(slots, device="cuda"), q_out, kp, vp)
    pg.check()
    live = slots >= 0
    p64 = pos[:, :t].astype(np.int64)
    for x, got in ((P.np64(q), P.np64(q_out)), (P.np64(k), None)):
        want = O.rope(x, p64, sections, order, pairing, 1e6)
        if got is None:
            cells = P.np64(kp).transpose(0, 2, 1, 3).reshape(-1, hkv, d)
            got = np.full_like(want, 6.0)
            got[live] = cells[slots[live]]
            others = np.setdiff1d(np.arange(n_pages * page), slots[live])
            assert (cells[others] == 6.0).all()
            fill = 6.0
        else:
            fill = 5.0
        assert (got[~live] == fill).all()
        a, b = (np.arange(half), np.arange(half) + half) if pairing == 0 else (2 * np.arange(half), 2 * np.arange(half) + 1)
        mag = np.zeros_like(x)
        mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        # 64-bit angles of the oracle at position 2^31 are themselves off by 2^31 * 2^-52
        tol = HALF_STEP[dtype] * np.abs(want) * 1.001 + mag * (2.0 ** -20)
        err = np.abs(got - want)[live]
        assert (err <= tol[live]).all(), float((err - tol[live]).max())
        assert (got[..., 2 * half:][live] == x[..., 2 * half:][live]).all()
    cells = P.np64(vp).transpose(0, 2, 1, 3).reshape(-1, hkv, d)
    assert (cells[slots[live]] == P.np64(v)[live]).all() and (cells == 7.0).all(-1).sum() == (n_pages * page - live.sum()) * hkv
    pg.close()


def test_rope_append_in_place_without_queries_without_rotation_and_bad_slots(B):
    hq, hkv, d, page, t = 4, 2, 128, 32, 2500                      # several tokens per block
    pg = make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=100)
    q, k, v = normal((t, hq, d), DT["bf16"], 1), normal((t, hkv, d), DT["bf16"], 2), normal((t, hkv, d), DT["bf16"], 3)
    pos = torch.arange(3 * t, dtype=torch.int32, device="cuda").view(3, t)
    slots = torch.randperm(100 * page, generator=torch.Generator().manual_seed(1))[:t].cuda()
    pools = lambda: (torch.zeros((100, hkv, page, d), dtype=DT["bf16"], device="cuda"), torch.zeros((100, hkv, page, d), dtype=DT["bf16"], device="cuda"))
    q_out, (kp, vp) = torch.empty_like(q), pools()
    pg.rope_append(q, k, v, pos, slots, q_out, kp, vp)
    q2, (kp2, vp2) = q.clone(), pools()
    pg.rope_append(q2, k, v, pos, slots, q2, kp2, vp2)             # q_out is q
    assert torch.equal(q2, q_out) and torch.equal(kp, kp2) and torch.equal(vp, vp2)
    kp3, vp3 = pools()
    pg.rope_append(None, k, v, pos, slots, None, kp3, vp3)         # keys and values alone
    assert torch.equal(kp, kp3) and torch.equal(vp, vp3)
    kp4, vp4 = pools()
    pg.rope_append(q, k, v, None, slots, q_out, kp4, vp4)          # nothing rotated
    cells = kp4.transpose(1, 2).reshape(-1, hkv, d)
    assert torch.equal(q_out, q) and torch.equal(cells[slots], k) and torch.equal(vp4, vp)
    pg.check()
    bad = slots.clone()
    bad[3], bad[2000] = 100 * page, -2
    kp5, vp5 = pools()
    pg.rope_append(None, k, v, pos, bad, None, kp5, vp5)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[3] = keep[2000] = False
    a, b = (x.transpose(1, 2).reshape(-1, hkv, d) for x in (kp, kp5))
    assert torch.equal(a[slots[keep]], b[slots[keep]]) and (b[slots[~keep]] == 0).all()
    pg.close()


# ----------------------------------------------------------------------------------------------- attention

def attention_tolerance(want, aux, d, rows, dtype):
    """Absolute bound on |out - want|.  A logit is a sum of d products accumulated in fp32 (2^-22 per step, which also covers an
    accumulator that truncates): off by at most delta = (d + 16) 2^-22 max_j sum |q k| / sqrt(d), which moves a
    probability by exp(delta) and its normaliser by as much: 2 delta (1 + delta) relative.  exp2 is off by 2^-22, a probability enters
    the product with 16 bits of mantissa in the bf16 path (2^-16, generous), sums of `rows` terms by rows 2^-22.  All
    of that is relative to sum p |v|.  The result is rounded once."""
    delta = (d + 16) * 2.0 ** -22 * aux["mag"]
    rel = 2 * delta * (1 + delta) + (rows + 64) * 2.0 ** -22 + 2.0 ** -16
    return aux["spread"] * rel[:, None] + HALF_STEP[dtype] * np.abs(want) * 1.01 + 1e-30


def lse_tolerance(lse, aux, d, rows):
    return (d + 16) * 2.0 ** -22 * aux["mag"] + (rows + 64) * 2.0 ** -22 + 2.0 ** -21 * np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 1e-6


def check_attention(out, lse, q, kp, vp, table, lens, page, dtype, sel=None, keep=0):
    n, hq, d = q.shape
    hkv = kp.shape[1]
    group = hq // hkv
    got, got_lse = P.np64(out), P.np64(lse) if lse is not None else None
    qh = P.np64(q)
    for i, m in enumerate(lens):
        c = O.n_pages_of(m, page)
        pages = torch.as_tensor(table[i, :c].astype(np.int64), device="cuda")
        for g in range(hkv):
            kr, vr = P.np64(kp[pages, g]).reshape(-1, d)[:m], P.np64(vp[pages, g]).reshape(-1, d)[:m]
            if sel is not None:
                rows = np.concatenate([np.arange(x * page, min(m, x * page + page)) for x in sel[i, g, :min(keep, c)]]) if c else np.arange(0)
                kr, vr = kr[rows.astype(np.int64)], vr[rows.astype(np.int64)]
            heads = slice(g * group, (g + 1) * group)
            want, want_lse, aux = O.attention(qh[i, heads], kr, vr)
            tol = attention_tolerance(want, aux, d, len(kr), dtype)
            assert (np.abs(got[i, heads] - want) <= tol).all(), (i, g, m, float((np.abs(got[i, heads] - want) - tol).max()))
            if got_lse is not None:
                if len(kr) == 0:
                    assert (got_lse[i, heads] == -np.inf).all()
                else:
                    assert (np.abs(got_lse[i, heads] - want_lse) <= lse_tolerance(want_lse, aux, d, len(kr))).all(), (i, g, m)


def attention_case(B, lens, hq, hkv, d, dtype, page, seed=0, n_pages=None, q_std=2.0):
    width = max(1, max(O.n_pages_of(x, page) for x in lens) + 1)
    n_pages = n_pages or sum(O.n_pages_of(x, page) for x in lens) + 3
    table = table_for(lens, page, width, n_pages, seed)
    pg = make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=len(lens), max_seq_pages=width)
    kp, vp = normal((n_pages, hkv, page, d), DT[dtype], seed + 1, 0.3), normal((n_pages, hkv, page, d), DT[dtype], seed + 2, 0.5)
    # whatever no sequence owns is NaN: it must never reach a result
    owned = np.zeros((n_pages, page), bool)
    for i, m in enumerate(lens):
        for c in range(O.n_pages_of(m, page)):
            owned[table[i, c], :min(page, m - c * page)] = True
    dead = torch.as_tensor(~owned, device="cuda")[:, None, :, None]
    kp.masked_fill_(dead, math.nan)
    vp.masked_fill_(dead, math.nan)
    q = normal((len(lens), hq, d), DT[dtype], seed + 3, 0.0, q_std)
    out = torch.full((len(lens), hq, d), math.nan, dtype=DT[dtype], device="cuda")
    lse = torch.full((len(lens), hq), math.nan, device="cuda")
    return pg, q, kp, vp, table, out, lse


EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 127, 128, 129, 0, 200]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page", [(1, 1, 64, 16), (4, 2, 64, 32), (6, 2, 128, 16), (7, 1, 128, 64), (8, 8, 128, 128), (28, 4, 128, 16),
                                           (8, 1, 64, 256), (9, 1, 64, 16), (16, 1, 128, 16), (24, 2, 128, 32), (2, 2, 256, 16), (10, 2, 256, 32),
                                           (16, 1, 256, 64), (11, 1, 256, 16)])
def test_paged_attention_edges(B, dtype, hq, hkv, d, page):
    pg, q, kp, vp, table, out, lse = attention_case(B, EDGES, hq, hkv, d, dtype, page, seed=hq + d)
    pg.paged_attention(q, kp, vp, i32(table.tolist()), i32(EDGES), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, EDGES, page, dtype)
    # again without lse, strided lengths, another stream: the same bits
    lens3 = torch.stack([i32(EDGES), i32([9999] * len(EDGES))], 1)[:, 0]
    out2 = torch.full_like(out, math.nan)
    t = i32(table.tolist())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pg.paged_attention(q, kp, vp, t, lens3, out2, stream=s)
    s.synchronize()
    assert torch.equal(out, out2)
    pg.close()


@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", [
    ("bf16", 7, 1, 128, 16, [5003]), ("bf16", 28, 4, 128, 64, [40001]), ("bf16", 4, 4, 64, 32, [20000, 3, 9000]),
    ("bf16", 16, 1, 128, 16, [30011]), ("f32", 7, 1, 128, 32, [7001]), ("f32", 3, 1, 64, 16, [6000, 1, 0, 12345]),
    ("bf16", 8, 1, 256, 16, [9001, 100]), ("f32", 4, 1, 256, 16, [4001])])
def test_paged_attention_split_over_many_blocks(B, dtype, hq, hkv, d, page, lens):
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, seed=11)
    t, n = i32(table.tolist()), i32(lens)
    pg.paged_attention(q, kp, vp, t, n, out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, dtype)
    for _ in range(5):                                             # joined in a fixed order: the same bits every time
        out2, lse2 = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
        pg.paged_attention(q, kp, vp, t, n, out2, lse2)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
    pg.close()


def test_paged_attention_many_short_sequences(B):
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 60, 1500).tolist()
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 4, 2, 64, "bf16", 16, seed=3)
    pg.paged_attention(q, kp, vp, i32(table.tolist()), i32(lens), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, 16, "bf16")
    pg.close()


def test_paged_attention_large_logits_infinities_and_nan(B):
    """A logit of 1e4 decides alone; an infinite logit or a NaN key gives NaN, in its own sequence only; rows whose logits
    are all -inf give 0."""
    lens, page, d = [40, 40, 40, 40], 16, 64
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 2, 1, d, "bf16", page, seed=5)
    q.fill_(0.0)
    q[:, 0, 0], q[:, 1, 1] = 1.0, 1.0                              # head 0 looks at dimension 0, head 1 at dimension 1
    for i in range(4):
        for c in range(3):
            kp[table[i, c], 0, :min(page, 40 - c * page), :2] = 0.0
    kp[table[0, 1], 0, 3, 0] = 80000.0                             # row 19 of sequence 0
    kp[table[1, 2], 0, 7, 0] = math.nan                            # row 39 of sequence 1
    for c in range(3):
        kp[table[2, c], 0, :min(page, 40 - c * page), 0] = -math.inf
    kp[table[3, 0], 0, 0, 1] = math.inf
    pg.paged_attention(q, kp, vp, i32(table.tolist()), i32(lens), out, lse)
    pg.check()
    assert torch.equal(out[0, 0], vp[table[0, 1], 0, 3])
    assert not out[0].isnan().any() and out[1].isnan().all()
    # 0 * -inf and 0 * inf are NaN too: head 1 of sequence 2 and head 0 of sequence 3 see one
    assert (lse[2, 0] == -math.inf) and (out[2, 0] == 0).all() and out[2, 1].isnan().all()
    assert out[3, 0].isnan().all() and out[3, 1].isnan().all()
    pg.close()


def test_paged_attention_bad_pages_and_lengths_are_reported_and_skipped(B):
    page, d, lens = 16, 64, [48, 33]
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 2, 1, d, "bf16", page, seed=8)
    bad = table.copy()
    bad[0, 1] = -1
    bad[1, 0] = 5000
    pg.paged_attention(q, kp, vp, i32(bad.tolist()), i32(lens), out, lse)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    for i, rows in ((0, [0, 2]), (1, [1, 2])):
        k = torch.cat([kp[bad[i, c], 0, :min(page, lens[i] - c * page)] for c in rows])
        v = torch.cat([vp[bad[i, c], 0, :min(page, lens[i] - c * page)] for c in rows])
        want, _, aux = O.attention(P.np64(q[i]), P.np64(k), P.np64(v))
        assert (np.abs(P.np64(out[i]) - want) <= attention_tolerance(want, aux, d, 48, "bf16")).all()
    # lengths are cut to the table's width; negative ones are 0
    width = table.shape[1]
    full = np.zeros((2, width), np.int32)
    pg2 = make(B, n_q_heads=2, n_kv_heads=1, head_dim=d, page_size=page, n_pages=kp.shape[0], max_seqs=2, max_seq_pages=width)
    kp.nan_to_num_(0.0)
    vp.nan_to_num_(0.0)
    pg2.paged_attention(q, kp, vp, i32(full.tolist()), i32([width * page + 1, -3]), out, lse)
    assert pg2.poll_status() == B.MEDA_ERR_INVALID_ARG
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all() and out[0].isfinite().all()
    pg.close()
    pg2.close()


def test_pools_beyond_four_gib(B):
    """Pages whose byte offsets and element offsets pass 2^32."""
    hkv, d, page = 4, 128, 16
    n_pages = 560_000                                              # 16 KiB each: 9.2 GB, 4.6e9 elements
    lens = [50, 2000]
    pg = make(B, n_q_heads=28, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_seqs=2, max_seq_pages=125)
    kp = torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device="cuda")
    vp = torch.empty_like(kp)
    bd = torch.empty((n_pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    table = np.full((2, 125), 1 << 30, np.int32)
    table[0, :4] = [n_pages - 1, 3, 262_144, n_pages - 2]
    table[1] = n_pages - 3 - 4000 * np.arange(125)
    k, v = normal((2, hkv, 2000, d), torch.bfloat16, 1, 0.3), normal((2, hkv, 2000, d), torch.bfloat16, 2, 0.5)
    q, out, lse = normal((2, 28, d), torch.bfloat16, 3), torch.empty((2, 28, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 28), device="cuda")
    t = i32(table.tolist())
    pg.page_store(k, v, i32([49, 2000]), t, kp, vp, bd)
    row, val = normal((1, hkv, d), torch.bfloat16, 4), normal((1, hkv, d), torch.bfloat16, 5)
    pg.rope_append(None, row, val, None, torch.tensor([int(table[0, 3]) * page + 1], device="cuda"), None, kp, vp)
    pg.page_bounds(kp, t, i32([49, 2000]), i32(lens), bd)
    pg.paged_attention(q, kp, vp, t, i32(lens), out, lse)
    pg.check()
    assert torch.equal(kp[n_pages - 2, :, 1], row[0]) and torch.equal(vp[n_pages - 2, :, 1], val[0])
    assert torch.equal(kp[n_pages - 1], k[0, :, :16])
    assert torch.equal(bd[n_pages - 2, :, 1], torch.maximum(k[0, :, 48], row[0]))
    check_attention(out, lse, q, kp, vp, table, lens, page, "bf16")
    sel = torch.full((2, hkv, 3), -1, dtype=torch.int32, device="cuda")
    pg.select_pages(q, bd, t, i32(lens), 1, 1, sel)
    pg.check()
    check_selection(sel, q, bd, table, lens, page, 3, 1, 1)
    pg.close()


# ----------------------------------------------------------------------------------------------- selection

def check_selection(sel, q, bd, table, lens, page, keep, first, last):
    hkv = sel.shape[1]
    group = q.shape[1] // hkv
    got, qh = sel.cpu().numpy(), P.np64(q)
    for i, m in enumerate(lens):
        c = O.n_pages_of(m, page)
        b = P.np64(bd[torch.as_tensor(table[i, :c].astype(np.int64), device="cuda")])
        for g in range(hkv):
            want = O.select_pages(O.page_scores(qh[i, g * group:(g + 1) * group], b[:, g]), keep, first, last) if c else np.arange(0)
            np.testing.assert_array_equal(got[i, g, :len(want)], want)
            assert (got[i, g, len(want):] == -1).all()             # entries behind the kept pages stay as they were


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,lens,keep,first,last", [
    (2, 2, 64, 16, [1, 16, 500, 0, 77], 4, 1, 1), (7, 1, 128, 16, [3000, 5], 20, 1, 2), (28, 4, 128, 16, [20000], 60, 0, 0),
    (16, 1, 64, 32, [9000, 4000, 31], 9, 2, 7), (3, 1, 256, 16, [2500], 30, 1, 1), (4, 2, 128, 64, [640] * 40, 5, 0, 1),
    (8, 1, 128, 16, [70000], 500, 4, 16), (1, 1, 64, 16, [40000, 39999, 12], 2047, 0, 3)])
def test_select_pages_and_attend_to_them(B, dtype, hq, hkv, d, page, lens, keep, first, last):
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, seed=21)
    t, n = i32(table.tolist()), i32(lens)
    bd = torch.full((kp.shape[0], hkv, 2, d), math.nan, dtype=DT[dtype], device="cuda")
    sel = torch.full((len(lens), hkv, keep), -1, dtype=torch.int32, device="cuda")
    pg.page_bounds(kp, t, None, n, bd)
    pg.select_pages(q, bd, t, n, first, last, sel)
    pg.paged_attention(q, kp, vp, t, n, out, lse, sel=sel)
    pg.check()
    check_selection(sel, q, bd, table, lens, page, keep, first, last)
    check_attention(out, lse, q, kp, vp, table, lens, page, dtype, sel.cpu().numpy(), keep)
    pg.close()


def test_select_pages_ties_zeros_and_nan(B):
    page, d, hkv = 16, 64, 1
    lens = [16 * 700, 16 * 700, 16 * 700, 16 * 700]
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 2, hkv, d, "f32", page, seed=2)
    bd = torch.zeros((kp.shape[0], hkv, 2, d), device="cuda")
    t, n = i32(table.tolist()), i32(lens)
    q[0] = 0.0                                                     # every score is 0: the lowest pages
    bd[t[1].long()[:700], 0, 0, :], bd[t[1].long()[:700], 0, 1, :] = -1.0, 1.0
    bd[int(t[1, 650]), 0, 1] = 1.5                                 # equal scores but one
    bd[t[2].long()[:700], 0, 1, 0] = torch.arange(700, device="cuda").float() // 7
    q[2] = 0.0
    q[2, :, 0] = torch.tensor([1.0, 0.5], device="cuda")           # a page's score is its number // 7
    bd[t[3].long()[:700], 0, 1, 0] = torch.arange(700, device="cuda").float()
    q[3] = 0.0
    q[3, :, 0] = 1.0
    for c in (5, 300, 301):
        bd[int(t[3, c]), 0, 1, 1] = math.nan                       # NaN ranks highest, behind the forced pages
    bd[int(t[0, 30]), 0, 0, 3] = -0.0
    sel = torch.full((4, hkv, 45), -1, dtype=torch.int32, device="cuda")
    pg.select_pages(q, bd, t, n, 2, 3, sel)
    pg.check()
    check_selection(sel, q, bd, table, lens, page, 45, 2, 3)
    assert {5, 300, 301, 0, 1, 697, 698, 699} <= set(sel[3, 0].tolist()) and sel[0, 0].tolist() == list(range(42)) + [697, 698, 699]
    # with only the forced pages wanted, NaN pages do not displace them
    five = torch.full((4, hkv, 5), -1, dtype=torch.int32, device="cuda")
    pg.select_pages(q, bd, t, n, 2, 3, five)
    assert five[3, 0].tolist() == [0, 1, 697, 698, 699]
    # entries outside the sequence's pages are reported and skipped
    five[1, 0, 2] = 700
    pg.paged_attention(q, kp, vp, t, n, out, lse, sel=five)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    rows = np.concatenate([np.arange(x * 16, x * 16 + 16) for x in (0, 1, 698, 699)])
    pages = t[1].long()[:700]
    want, _, aux = O.attention(P.np64(q[1]), P.np64(kp[pages, 0]).reshape(-1, d)[rows], P.np64(vp[pages, 0]).reshape(-1, d)[rows])
    assert (np.abs(P.np64(out[1]) - want) <= attention_tolerance(want, aux, d, 64, "f32")).all()
    pg.close()


def test_select_pages_many_rounds_and_many_pairs(B):
    """More pages than a block holds at once (one large block per pair, and small blocks for many pairs), and more sequences than
    the scratch holds scores of at once."""
    for lens, hq, hkv, d, keep in (([150_011], 2, 1, 64, 700), ([41_000] * 38 + [3, 0], 8, 4, 64, 37)):
        pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, "bf16", 16, seed=31)
        t, n = i32(table.tolist()), i32(lens)
        bd = torch.zeros((kp.shape[0], hkv, 2, d), dtype=torch.bfloat16, device="cuda")
        sel = torch.full((len(lens), hkv, keep), -1, dtype=torch.int32, device="cuda")
        pg.page_bounds(kp, t, None, n, bd)
        pg.select_pages(q, bd, t, n, 1, 2, sel)
        pg.check()
        check_selection(sel, q, bd, table, lens, 16, keep, 1, 2)
        # the same query everywhere 0: every page ties, the 64-bit path decides by the page's number
        q.zero_()
        sel.fill_(-1)
        pg.select_pages(q, bd, t, n, 1, 2, sel)
        pg.check()
        check_selection(sel, q, bd, table, lens, 16, keep, 1, 2)
        pg.close()
    # a table row of 65,536 entries: the scratch holds few sequences, the batch goes through it in turns
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 1500, 60).tolist()
    width, hkv, d = 65_536, 2, 64
    n_pages = sum(O.n_pages_of(x, 16) for x in lens)
    table = table_for(lens, 16, width, n_pages, 3)
    pg = make(B, n_q_heads=6, n_kv_heads=hkv, head_dim=d, n_pages=n_pages, max_seqs=60, max_seq_pages=width)
    q, kp = normal((60, 6, d), DT["bf16"], 1), normal((n_pages, hkv, 16, d), DT["bf16"], 2, 0.3)
    bd = torch.zeros((n_pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    sel = torch.full((60, hkv, 11), -1, dtype=torch.int32, device="cuda")
    t, n = i32(table.tolist()), i32(lens)
    pg.page_bounds(kp, t, None, n, bd)
    before = pg.launch_count()
    pg.select_pages(q, bd, t, n, 1, 2, sel)
    assert pg.launch_count() - before > 2
    pg.check()
    check_selection(sel, q, bd, table, lens, 16, 11, 1, 2)
    pg.close()


def test_select_pages_infinite_and_huge_bounds(B):
    """Scores that are infinite or NaN, or so large that an fp32 sum overflows on the way, go to the 64-bit path."""
    for dtype in ("bf16", "f32"):
        lens, page, d, keep = [16 * 300] * 4, 16, 64, 9
        pg, q, kp, vp, table, out, lse = attention_case(B, lens, 3, 1, d, dtype, page, seed=6)
        t, n = i32(table.tolist()), i32(lens)
        bd = torch.zeros((kp.shape[0], 1, 2, d), dtype=DT[dtype], device="cuda")
        pg.page_bounds(kp, t, None, n, bd)
        pages = t.long()
        bd[pages[0, 17], 0, 1, 5] = math.inf
        bd[pages[0, 18], 0, 0, 5] = -math.inf
        q[0, :, 5] = torch.tensor([1.0, -1.0, 2.0], device="cuda")
        bd[pages[1, 40], 0, 0, 3] = -math.inf                      # 0 times it, or a score of -inf: never among the best
        q[1, :, 3] = torch.tensor([-0.5, 0.5, 0.0], device="cuda")
        bd[pages[2, :300], 0] = bd[pages[2, :300], 0] * 1e37       # sums near the largest float
        sel = torch.full((4, 1, keep), -1, dtype=torch.int32, device="cuda")
        pg.select_pages(q, bd, t, n, 0, 1, sel)
        pg.check()
        check_selection(sel, q, bd, table, lens, page, keep, 0, 1)
        pg.close()


# ---------------------------------------------------------------------------------------------- refusals

def test_refusals(B):
    pg, q, kp, vp, table, out, lse = attention_case(B, [20, 30], 4, 2, 64, "bf16", 16)
    t, n = i32(table.tolist()), i32([20, 30])
    sel = torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda")
    bd = torch.zeros((kp.shape[0], 2, 2, 64), dtype=torch.bfloat16, device="cuda")
    for call in (
        lambda: pg.paged_attention(q.float(), kp, vp, t, n, out),                       # type
        lambda: pg.paged_attention(q[:1], kp, vp, t, n, out),                           # batch
        lambda: pg.paged_attention(q, kp[:-1], vp, t, n, out),                          # pool
        lambda: pg.paged_attention(q, kp, vp, t[:, :1], n, out),                        # table width
        lambda: pg.paged_attention(q, kp, vp, t, n.long(), out),
        lambda: pg.paged_attention(q, kp, vp, t, n, out.transpose(0, 1)),
        lambda: pg.paged_attention(q, kp, vp, t, n.cpu(), out),
        lambda: pg.paged_attention(q, kp, vp, t, n, out, lse.double()),
        lambda: pg.paged_attention(q, kp, vp, t, n, out, sel=sel[:, :1]),
        lambda: pg.rope_append(None, q[:, :2], q[:, 2:3], None, torch.zeros(2, dtype=torch.int64, device="cuda"), None, kp, vp),
        lambda: pg.rope_append(None, q[:, :2], q[:, 2:], torch.zeros((2, 2), dtype=torch.int32, device="cuda"),
                               torch.zeros(2, dtype=torch.int64, device="cuda"), None, kp, vp),
        lambda: pg.rope_append(None, q[:, ::2], q[:, 2:], None, torch.zeros(2, dtype=torch.int64, device="cuda"), None, kp, vp),
        lambda: pg.page_store(kp, vp.transpose(2, 3), n, t, kp, vp),
    ):
        with pytest.raises(ValueError):
            call()

    def status(call):
        with pytest.raises(B.MedaError) as e:
            call()
        return e.value.status

    assert status(lambda: pg.select_pages(q, bd, t, n, 2, 2, sel)) == B.MEDA_ERR_INVALID_ARG          # 2 + 2 > 3
    assert status(lambda: pg.select_pages(q, bd, t, n, -1, 2, sel)) == B.MEDA_ERR_INVALID_ARG
    big = i32([1, 1, 1])
    assert status(lambda: pg.paged_attention(q[:1].expand(3, 4, 64).contiguous(), kp, vp, t[:1].expand(3, -1).contiguous(), big,
                                             out[:1].expand(3, 4, 64).contiguous())) == B.MEDA_ERR_SHAPE   # more than max_seqs
    one = i32([0])
    assert status(lambda: pg.page_tables(None, n, i32([0] * kp.shape[0]), one, one, t, i32([0] * 3),
                                         torch.zeros(4, dtype=torch.int64, device="cuda"))) == B.MEDA_ERR_INVALID_ARG
    # misaligned rows and strides
    flat = torch.zeros(4 * 2 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    odd = flat[1:1 + 2 * 2 * 64].view(2, 2, 64)
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    assert status(lambda: pg.rope_append(None, odd, q[:, :2], None, slots, None, kp, vp)) == B.MEDA_ERR_SHAPE
    skew = flat[:2 * 132].as_strided((2, 2, 64), (132, 64, 1))
    assert status(lambda: pg.rope_append(None, skew, q[:, :2], None, slots, None, kp, vp)) == B.MEDA_ERR_SHAPE
    # q_out = q needs dense tokens
    wide = torch.zeros((2, 5, 64), dtype=torch.bfloat16, device="cuda")
    lib = B.load_library()
    assert lib.meda_rope_append(pg._h, wide.data_ptr(), 320, q.data_ptr(), 256, q.data_ptr(), 256, None, 0, slots.data_ptr(), 2,
                                wide.data_ptr(), kp.data_ptr(), vp.data_ptr(), None) == B.MEDA_ERR_INVALID_ARG
    # nothing to do is not an error, whatever the pointers
    assert lib.meda_paged_attention(pg._h, None, None, None, None, None, 1, 0, None, 0, None, None, None) == 0
    assert lib.meda_rope_append(pg._h, None, 0, None, 0, None, 0, None, 0, None, 0, None, None, None, None) == 0
    assert pg.launch_count() == 0
    pg.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vectors_off_their_boundary_are_refused(B, dtype):
    """Every tensor that is read or written as 16-byte vectors, one element into its buffer: refused before any launch."""
    pg, q, kp, vp, table, out, lse = attention_case(B, [20, 30], 4, 2, 64, dtype, 16)
    t, n = i32(table.tolist()), i32([20, 30])
    bd = torch.zeros((kp.shape[0], 2, 2, 64), dtype=kp.dtype, device="cuda")
    sel = torch.zeros((2, 2, 1), dtype=torch.int32, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    k, v = torch.zeros((2, 2, 32, 64), dtype=kp.dtype, device="cuda"), torch.zeros((2, 2, 32, 64), dtype=kp.dtype, device="cuda")
    kn, vn = k[:, :, 0].contiguous(), v[:, :, 0].contiguous()

    def off(x):
        y = torch.zeros(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        assert y.is_contiguous() and y.data_ptr() % 16 != 0
        return y

    calls = [
        (lambda q, bd: pg.select_pages(q, bd, t, n, 0, 1, sel), (q, bd)),
        (lambda q, kp, vp, out: pg.paged_attention(q, kp, vp, t, n, out), (q, kp, vp, out)),
        (lambda k, v, kp, vp, bd: pg.page_store(k, v, n, t, kp, vp, bd), (k, v, kp, vp, bd)),
        (lambda kp, bd: pg.page_bounds(kp, t, None, n, bd), (kp, bd)),
        (lambda q, k, v, out, kp, vp: pg.rope_append(q, k, v, None, slots, out, kp, vp), (q, kn, vn, out, kp, vp)),
    ]
    for call, args in calls:
        for i in range(len(args)):
            with pytest.raises(B.MedaError) as e:
                call(*args[:i], off(args[i]), *args[i + 1:])
            assert e.value.status == B.MEDA_ERR_SHAPE
    assert pg.launch_count() == 0
    pg.close()


# ------------------------------------------------------------------------------------------ a run of them

def decoder_case(keep_pages=0):
    from paper_2502_17599_b200.pipeline import CompressionPass, PagedDecoder
    wl = W.small_variant("paged", window=32, seed=4)
    cps = []
    for s in (4, 9):
        cp = CompressionPass(wl.with_(seed=s), n_streams=2)
        layers = [W.make_layer(wl.with_(seed=s), l, "cuda") for l in range(wl.n_layers)]
        cp.run(*[list(x) for x in zip(*layers)])
        cp.check()
        cps.append(cp)
    dec = PagedDecoder(wl, n_pages=120, max_requests=3, max_rows=400, keep_pages=keep_pages, rope_sections=(24, 20, 20), rope_theta=1e6)
    return wl, cps, dec


def new_token(wl, step, layer, requests):
    q = normal((requests, wl.n_q_heads + 2 * wl.n_kv_heads, wl.head_dim), wl.torch_dtype, 1000 * step + layer)
    hq, hkv = wl.n_q_heads, wl.n_kv_heads
    return q[:, :hq], q[:, hq:hq + hkv], q[:, hq + hkv:]


@pytest.mark.parametrize("keep_pages", [0, 6])
@pytest.mark.parametrize("graph", [False, True])
def test_decoding_over_compressed_caches(B, keep_pages, graph):
    """Two prompts through the compression pass, into pages, then decoding steps in which requests come and go; every layer's
    attention against the oracle on rows kept here.  With `graph` the steps are replays of one captured step."""
    wl, cps, dec = decoder_case(keep_pages)
    L, R, hkv, hq, d = wl.n_layers, 3, wl.n_kv_heads, wl.n_q_heads, wl.head_dim
    rows = {}                                                      # (request, layer) -> (k [hkv][rows][d], v)

    def admit(r, cp):
        dec.admit(r, cp)
        b = cp.budgets.cpu().numpy()
        for l in range(L):
            s = int(b[l, 0])
            rows[r, l] = (P.np64(cp.k_out[l, :, :s]), P.np64(cp.v_out[l, :, :s]))

    out = torch.zeros((L, R, hq, d), dtype=wl.torch_dtype, device="cuda")
    lse = torch.zeros((L, R, hq), device="cuda")
    qkv = torch.zeros((L, R, hq + 2 * hkv, d), dtype=wl.torch_dtype, device="cuda")
    pos = torch.zeros((3, R), dtype=torch.int32, device="cuda")

    def step():
        dec.begin_step()
        for l in range(L):
            dec.attend(l, qkv[l, :, :hq], qkv[l, :, hq:hq + hkv], qkv[l, :, hq + hkv:], pos, out[l], lse[l])

    admit(0, cps[0])
    dec.check()
    captured = None
    if graph:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()                                                 # loads the kernels; its row is taken back below
        side.synchronize()
        dec.release(0)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        rows.clear()
        admit(0, cps[0])
        dec.check()
    live = {0}
    for n in range(22):
        if n == 2:
            admit(2, cps[1])
            live.add(2)
        if n == 15:
            dec.release(0)
            live.discard(0)
        if n == 18:
            admit(1, cps[0])
            live.add(1)
        for l in range(L):
            qkv[l] = torch.cat(new_token(wl, n, l, R), 1)
        pos.copy_(i32([[700 + n, 5, 6 + n], [700 + n, n, 9], [700 + n, 7, 2 * n]]))
        if captured is not None:
            captured.replay()
        else:
            step()
        dec.check()
        p64 = pos.cpu().numpy().astype(np.int64)
        for l in range(L):
            k_rot = O.rope(P.np64(qkv[l, :, hq:hq + hkv]), p64, (24, 20, 20), 0, 0, 1e6)
            q_rot = O.rope(P.np64(qkv[l, :, :hq]), p64, (24, 20, 20), 0, 0, 1e6)
            for r in sorted(live):
                k, v = rows[r, l]
                k = np.concatenate([k, k_rot[r][:, None]], 1)
                v = np.concatenate([v, P.np64(qkv[l, r, hq + hkv:])[:, None]], 1)
                rows[r, l] = (k, v)
                if keep_pages:
                    continue                                       # (selection itself is tested above; here, that all fits together)
                for h in range(hq):
                    g = h // (hq // hkv)
                    want, want_lse, aux = O.attention(q_rot[r, h:h + 1], k[g], v[g])
                    # queries and keys were rounded to bf16 after the rotation, half a step each in every product: a logit
                    # moves by delta, a probability and its normaliser by a factor exp(delta) each
                    delta = 2 * 2.0 ** -8 * 1.01 * aux["mag"][:, None]
                    tol = (attention_tolerance(want, aux, d, k.shape[1], "bf16") + np.expm1(2 * delta) * aux["spread"]) * 1.1
                    assert (np.abs(P.np64(out[l, r, h:h + 1]) - want) <= tol).all(), (n, l, r, h)
    assert dec.lens.view(L, R)[:, 0].eq(0).all()
    for r in live:
        for l in range(L):
            assert int(dec.lens.view(L, R)[l, r]) == rows[r, l][0].shape[1]
    if keep_pages:                                                 # as many pages as there are: the same as without a choice
        l = 0
        seqs = slice(0, R)
        full = torch.zeros_like(out[0])
        sel = torch.zeros((R, hkv, dec.table.shape[1]), dtype=torch.int32, device="cuda")
        dec.pages.select_pages(dec.q_rot, dec.bounds, dec.table[seqs], dec.lens[seqs], 1, 1, sel)
        dec.pages.paged_attention(dec.q_rot, dec.k_pages, dec.v_pages, dec.table[seqs], dec.lens[seqs], full, sel=sel)
        dense = torch.zeros_like(full)
        dec.pages.paged_attention(dec.q_rot, dec.k_pages, dec.v_pages, dec.table[seqs], dec.lens[seqs], dense)
        assert torch.equal(full, dense)
    dec.close()
    for cp in cps:
        cp.close()


def test_a_full_pool_is_reported_and_leaves_the_requests_alone(B):
    wl, cps, dec0 = decoder_case()
    dec0.close()
    from paper_2502_17599_b200.pipeline import PagedDecoder
    total = sum(O.n_pages_of(int(x), 16) for x in cps[0].budgets[:, 0].cpu())
    dec = PagedDecoder(wl, n_pages=total + 1, max_requests=2, max_rows=400)
    dec.admit(0, cps[0])
    dec.check()
    before = dec.table.clone(), dec.lens.clone(), dec.k_pages.clone()
    dec.admit(1, cps[1])
    with pytest.raises(B.MedaError):
        dec.check()
    assert torch.equal(before[1], dec.lens) and torch.equal(before[0], dec.table) and int(dec.active[1]) == 0
    assert torch.equal(before[2][dec.table[dec.table >= 0].long()], dec.k_pages[dec.table[dec.table >= 0].long()])
    dec.close()
    for cp in cps:
        cp.close()


def test_paged_attention_agrees_with_attention_over_the_dense_cache(B):
    wl, cps, dec = decoder_case()
    dec.admit(0, cps[0])
    q = normal((3, wl.n_q_heads, wl.head_dim), wl.torch_dtype, 1)
    for l in range(wl.n_layers):
        dense = torch.zeros((wl.n_q_heads, wl.head_dim), device="cuda")
        cps[0].ctx.decode_attention(l, q[0].contiguous(), cps[0].k_out[l], cps[0].v_out[l], dense, budgets=cps[0].budgets)
        out = torch.zeros_like(q)
        seqs = slice(l * 3, l * 3 + 3)
        dec.pages.paged_attention(q, dec.k_pages, dec.v_pages, dec.table[seqs], dec.lens[seqs], out)
        dec.check()
        # the dense call's fp32 output agrees with fp64 to 1e-4; the paged one is rounded to bf16 on top
        assert ((out[0].float() - dense).abs() <= 2.0 ** -8 * dense.abs() + 2e-4).all()
        assert (out[1:] == 0).all()
    dec.close()
    for cp in cps:
        cp.close()


def test_calls_behind_copies_joins_and_other_kernels_in_a_graph(B):
    """The launches may be set up ahead of the work before them; that must wait all the same, whatever it is: a memset, a copy,
    another stream's kernel, an ordinary kernel, and it must hold inside one captured graph."""
    lens = [700, 33]
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 8, 2, 128, "bf16", 16, seed=14)
    t, n = i32(table.tolist()), i32(lens)
    source, live = torch.stack([n, n - 5, n - 20]), n.clone()
    wants = []
    for i in range(3):
        o = torch.empty_like(out)
        pg.paged_attention(q, kp, vp, t, source[i].contiguous(), o)
        wants.append(o)
    torch.cuda.synchronize()
    pick = torch.zeros(1, dtype=torch.int64, device="cuda")
    big = torch.zeros(32 << 20, device="cuda")
    side = torch.cuda.Stream()
    outs = [torch.empty_like(out) for _ in range(4)]

    def body():
        main = torch.cuda.current_stream()
        live.zero_()
        big.add_(1.0)                                              # something long, so that an early start would read zeros
        live.copy_(source.index_select(0, pick)[0])
        pg.paged_attention(q, kp, vp, t, live, outs[0])
        live.zero_()
        pg.paged_attention(q, kp, vp, t, live, outs[1])
        side.wait_stream(main)
        with torch.cuda.stream(side):
            big.add_(1.0)
            live.copy_(source.index_select(0, pick)[0])
        main.wait_stream(side)
        pg.paged_attention(q, kp, vp, t, live, outs[2])
        outs[3].copy_(outs[2])

    body()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        body()
    for i in (0, 2, 1, 0):
        pick.fill_(i)
        for o in outs:
            o.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], wants[i]) and torch.equal(outs[2], wants[i]) and torch.equal(outs[3], wants[i]) and (outs[1] == 0).all()
        for o in outs:
            o.fill_(math.nan)
        body()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], wants[i]) and torch.equal(outs[2], wants[i]) and (outs[1] == 0).all()
    pg.check()
    pg.close()


def test_two_handles_on_two_streams_and_two_graphs(B):
    """Handles of their own keep calls apart: two graphs that attend over the same pages run side by side."""
    lens = [3000, 17, 900]
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 28, 4, 128, "bf16", 16, seed=4)
    other = make(B, n_q_heads=28, n_kv_heads=4, head_dim=128, page_size=16, n_pages=kp.shape[0], max_seqs=3, max_seq_pages=table.shape[1])
    t, n = i32(table.tolist()), i32(lens)
    q2 = normal(q.shape, q.dtype, 77)
    want = [torch.empty_like(out) for _ in range(2)]
    pg.paged_attention(q, kp, vp, t, n, want[0])
    other.paged_attention(q2, kp, vp, t, n, want[1])
    torch.cuda.synchronize()
    graphs, outs = [], [torch.empty_like(out) for _ in range(2)]
    for h, x, o in ((pg, q, outs[0]), (other, q2, outs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(4):
                h.paged_attention(x, kp, vp, t, n, o)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for o in outs:
            o.fill_(math.nan)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    pg.close()
    other.close()


FIRST_CAPTURE = """
import torch
from paper_2502_17599_b200 import binding as B
pg = B.Pages(n_q_heads=14, n_kv_heads=2, head_dim=128, dtype="{dtype}", page_size=16, n_pages=64, max_seqs=3, max_seq_pages=20)
dt = dict(bf16=torch.bfloat16, f32=torch.float32)["{dtype}"]
torch.manual_seed(1)
rand = lambda *s: torch.randn(s, device="cuda").to(dt)
i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
q, k, v, kn, vn = rand(3, 14, 128), rand(3, 2, 320, 128), rand(3, 2, 320, 128), rand(3, 2, 128), rand(3, 2, 128)
lens, more, none, zero = i32(300, 17, 0), i32(301, 18, 1), i32(0, 0, 0), i32(0)
pos = i32(5, 6, 7).repeat(3, 1)

def buffers():
    z = lambda *s: torch.zeros(s, dtype=dt, device="cuda")
    return dict(kp=z(64, 2, 16, 128), vp=z(64, 2, 16, 128), bd=z(64, 2, 2, 128), table=torch.full((3, 20), -1, dtype=torch.int32, device="cuda"),
                free=torch.arange(64, dtype=torch.int32, device="cuda"), top=i32(0), top2=i32(0), cu=i32(0, 0, 0, 0),
                slots=torch.zeros(3, dtype=torch.int64, device="cuda"), nothing=torch.empty(0, dtype=torch.int64, device="cuda"),
                qr=z(3, 14, 128), sel=torch.zeros((3, 2, 4), dtype=torch.int32, device="cuda"), out=z(3, 14, 128), lse=torch.zeros((3, 14), device="cuda"))

def body(b):
    pg.page_tables(None, lens, b["free"], zero, b["top"], b["table"], b["cu"], b["nothing"])
    pg.page_store(k, v, lens, b["table"], b["kp"], b["vp"], b["bd"])
    pg.page_tables(lens, more, b["free"], b["top"], b["top2"], b["table"], b["cu"], b["slots"])
    pg.rope_append(q, kn, vn, pos, b["slots"], b["qr"], b["kp"], b["vp"])
    pg.page_bounds(b["kp"], b["table"], lens, more, b["bd"])
    pg.select_pages(b["qr"], b["bd"], b["table"], more, 1, 1, b["sel"])
    pg.paged_attention(b["qr"], b["kp"], b["vp"], b["table"], more, b["out"], b["lse"], sel=b["sel"])

captured, eager = buffers(), buffers()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    body(captured)
graph.replay()
pg.check()
body(eager)
pg.check()
for name in captured:
    assert torch.equal(captured[name], eager[name]), name
assert captured["top2"].item() == 19 + 2 + 1 and captured["out"].float().abs().sum() > 0
print("captured first")
"""


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_calls_of_a_process_inside_a_capture(B, dtype):
    """A server may capture its step before it ever ran one: no call may need anything a capture forbids (kernels are loaded then)."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CAPTURE.replace("{dtype}", dtype)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stderr[-2000:]


def test_sequences_may_share_pages_they_only_read(B):
    """Two sequences whose table rows name the same pages, the second with fewer rows of the last one: as with pages of their own."""
    lens = [100, 100, 70]
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 8, 2, 128, "bf16", 16, seed=31)
    own = torch.empty_like(out)
    t = i32(table.tolist())
    kp2, vp2 = kp.clone(), vp.clone()
    for c in range(O.n_pages_of(70, 16)):                            # the third sequence's own copy of the first one's pages
        kp2[int(table[2, c])], vp2[int(table[2, c])] = kp[int(table[0, c])], vp[int(table[0, c])]
    pg.paged_attention(q, kp2, vp2, t, i32(lens), own)
    shared = t.clone()
    shared[2] = t[0]
    pg.paged_attention(q, kp2, vp2, shared, i32(lens), out)
    pg.check()
    assert torch.equal(out, own)
    pg.close()


def test_page_store_of_a_cache_without_room(B):
    """Capacity 0 (an empty tensor has no address): nothing is stored, and a length above it is reported."""
    pg = make(B)
    kp = torch.full((64, 2, 16, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    k = torch.empty((2, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    t = torch.zeros((2, 16), dtype=torch.int32, device="cuda")
    pg.page_store(k, k, i32([0, 0]), t, kp, kp.clone())
    pg.check()
    pg.page_store(k, k, i32([0, 1]), t, kp, kp.clone())
    assert pg.poll_status() == B.MEDA_ERR_WORKSPACE
    assert (kp == 3).all()
    pg.close()


def test_decoder_refuses_more_fixed_pages_than_it_keeps(B):
    from paper_2502_17599_b200.pipeline import PagedDecoder
    wl = W.small_variant("paged", window=32, seed=4)
    for kw in (dict(keep_pages=2), dict(keep_pages=-1), dict(keep_pages=4, n_first=-1)):
        with pytest.raises(ValueError):
            PagedDecoder(wl, n_pages=10, max_requests=1, max_rows=100, **kw)
