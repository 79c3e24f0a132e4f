"""Quantised pages on the device against the oracle: written, read back, appended to, bounded and attended to.

Tolerances.  Codes, steps and lowest values are compared byte for byte: every operation behind them is stated.  Rows read back are low +
step * code, an exact product, one fp32 rounding and one to the type: the oracle's value after the same two roundings, exactly.  Attention: see
coded_tolerance."""
import math

import numpy as np
import pytest
import torch

import parity as P
import test_gpu_pages as T
from oracle import pages_oracle as O

pytestmark = pytest.mark.gpu
DT = T.DT


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def row_bytes(d, bits):
    return d * bits // 8 + 4 * (d // 64)


def empty_pool(n_pages, hkv, page, d, bits, fill=0xff):
    """Bytes of 0xff: whatever no call writes reads back as NaN."""
    return torch.full((n_pages, hkv, page * row_bytes(d, bits)), fill, dtype=torch.uint8, device="cuda")


def rounded(x, dtype):
    """fp64 low + step * code as the device rounds it: to fp32, then to the type."""
    return torch.as_tensor(np.asarray(x, np.float64).astype(np.float32)).to(DT[dtype]).double().numpy()


def rows_of(page, live, page_size, d, bits):
    """What the first `live` rows of a page of every head stand for, fp64 [heads][live][d]."""
    code, step, low = O.unpack_page(page, page_size, d, bits)
    return O.held(code, step, low)[..., :live, :]


def dense(shape, dtype, seed):
    """Rows with a few large dimensions, as keys have them."""
    x = T.normal(shape, torch.float32, seed, 0.4)
    wide = torch.exp(T.normal((shape[-1],), torch.float32, seed + 100))
    return (x * wide).to(DT[dtype])


LENS = [0, 1, 15, 16, 17, 255, 256, 257, 300, 299]


# ------------------------------------------------------------------------------------- store, bounds, read back

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 128), (128, 16), (128, 64), (256, 32), (256, 256)])
def test_store_bounds_and_load(B, bits, dtype, d, page):
    hkv, cap, n = 3, 300, len(LENS)
    width = O.n_pages_of(cap, page)
    n_pages = sum(O.n_pages_of(x, page) for x in LENS) + 4
    table = T.table_for(LENS, page, width, n_pages, d + page)
    pg = T.make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=n, max_seq_pages=width, cache_bits=bits)
    assert pg.page_bytes() == page * row_bytes(d, bits)
    # every other head of a larger cache; rows behind a length are NaN
    base = dense((n, 2 * hkv, cap + 2, d), dtype, 5)
    both = torch.stack([base, base * -1.5])
    k, v = both[0, :, ::2, :cap], both[1, :, ::2, :cap]
    for i, m in enumerate(LENS):
        both[:, i, :, m:] = math.nan
    kp, vp = empty_pool(n_pages, hkv, page, d, bits), empty_pool(n_pages, hkv, page, d, bits)
    bd = torch.full((n_pages, hkv, 2, d), 9.0, dtype=DT[dtype], device="cuda")
    t, lens = T.i32(table.tolist()), T.i32(LENS)
    pg.page_store(k, v, lens, t, kp, vp, bd)
    pg.check()
    want_b, got_b = P.np64(torch.full_like(bd, 9.0)), P.np64(bd)
    held = {}
    for name, src, pool in (("k", k, kp), ("v", v, vp)):
        x, got = P.np64(src).astype(np.float32), pool.cpu().numpy()
        want = np.full_like(got, 0xff)
        held[name] = np.zeros(x.shape)
        for i, m in enumerate(LENS):
            code, step, low = O.quantise(x[i, :, :m], bits)
            held[name][i, :, :m] = rounded(O.held(code, step, low), dtype)
            for c in range(O.n_pages_of(m, page)):
                r = slice(c * page, min(m, c * page + page))
                live = r.stop - r.start
                full = [np.full((hkv, page) + a.shape[2:], 255 if a.dtype == np.uint8 else np.nan, a.dtype) for a in (code, step, low)]
                for a, b in zip(full, (code, step, low)):
                    a[:, :live] = b[:, r]
                full[0] &= (1 << bits) - 1
                page_want = O.pack_page(*full, bits)
                head = d * bits // 8                               # rows behind the length keep their bytes: 0xff, not the oracle's NaN
                page_want[:, live * head:page * head] = 0xff
                page_want[:, page * head + live * 4 * (d // 64):] = 0xff
                want[table[i, c]] = page_want
                if name == "k":
                    lo, hi = O.page_bounds(held["k"][i, :, r].transpose(1, 0, 2))
                    want_b[table[i, c], :, 0], want_b[table[i, c], :, 1] = lo, hi
        np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(got_b, want_b)
    again = torch.full_like(bd, 9.0)
    pg.page_bounds(kp, t, None, lens, again)
    np.testing.assert_array_equal(P.np64(again), want_b)
    part, start = torch.full_like(bd, 9.0), [max(0, m - 3) for m in LENS]
    start[3] = LENS[3]                                             # nothing new
    pg.page_bounds(kp, t, T.i32(start), lens, part)
    pg.check()
    want_part = np.full_like(want_b, 9.0)
    for i, m in enumerate(LENS):
        if start[i] < m:
            for c in range(start[i] // page, O.n_pages_of(m, page)):
                want_part[table[i, c]] = want_b[table[i, c]]
    np.testing.assert_array_equal(P.np64(part), want_part)
    # read back whole, and from a row of each sequence on; heads outside sequences in the second
    back = torch.full((2, n, hkv, cap, d), 5.0, dtype=DT[dtype], device="cuda")
    pg.page_load(kp, vp, t, lens, back[0], back[1])
    pg.check()
    for x, name in ((back[0], "k"), (back[1], "v")):
        for i, m in enumerate(LENS):
            np.testing.assert_array_equal(P.np64(x[i, :, :m]), held[name][i, :, :m])
            assert (x[i, :, m:] == 5).all()
    first = [0, 1, 3, 15, 20, 100, 250, 0, 299, 17]                # none, past the end, mid-page, on a border
    turned = torch.full((2, hkv, n, cap + 1, d), 5.0, dtype=DT[dtype], device="cuda")[:, :, :, :cap]
    three = torch.stack([lens, lens, lens], 1)[:, 1]               # strided lengths
    from3 = torch.stack([T.i32(first)] * 3, 1)[:, 2]
    pg.page_load(kp, vp, t, three, turned[0].transpose(0, 1), turned[1].transpose(0, 1), lens_from=from3)
    pg.check()
    for x, name in ((turned[0], "k"), (turned[1], "v")):
        for i, (a, m) in enumerate(zip(first, LENS)):
            count = max(0, m - a)
            np.testing.assert_array_equal(P.np64(x[:, i, :count]), held[name][i, :, a:a + count])
            assert (x[:, i, count:] == 5).all()
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_groups(B, bits, dtype):
    """Groups of one value, of zeros of either sign, with a NaN, an infinity or a huge element, with ranges below the smallest step."""
    d, page = 128, 16
    pg = T.make(B, n_q_heads=1, n_kv_heads=1, head_dim=d, dtype=dtype, page_size=page, n_pages=1, max_seqs=1, max_seq_pages=1, cache_bits=bits)
    x = torch.randn((1, 1, 12, d), generator=torch.Generator().manual_seed(2)).to(DT[dtype])
    x[0, 0, 0, :64] = -3.25
    x[0, 0, 1] = 0.0
    x[0, 0, 2] = -0.0
    x[0, 0, 3, 5] = math.nan
    x[0, 0, 4, 70] = math.inf
    x[0, 0, 5, 71] = -math.inf
    x[0, 0, 6, 0] = 2.0 ** 126
    big = 2.0 ** 126 * (1 - (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24))
    x[0, 0, 7, 0], x[0, 0, 7, 1] = big, -big
    x[0, 0, 8] = 0.0
    x[0, 0, 8, 9] = 2.0 ** -133                                    # a subnormal of either type
    x[0, 0, 9] = torch.arange(d).to(DT[dtype]) * 2.0 ** -131
    x[0, 0, 10, ::2] = 1.0
    x[0, 0, 10, 1::2] = 1.0 + 2.0 ** -7                            # neighbours in bf16
    x = x.cuda()
    kp, vp = empty_pool(1, 1, page, d, bits), empty_pool(1, 1, page, d, bits)
    back = torch.empty((2, 1, 1, 12, d), dtype=DT[dtype], device="cuda")
    bd = torch.empty((1, 1, 2, d), dtype=DT[dtype], device="cuda")
    pg.page_store(x, x.clone(), T.i32([12]), T.i32([[0]]), kp, vp, bd)
    pg.page_load(kp, vp, T.i32([[0]]), T.i32([12]), back[0], back[1])
    pg.check()
    code, step, low = O.quantise(P.np64(x[0, 0]).astype(np.float32), bits)
    want = rounded(O.held(code, step, low), dtype)
    assert np.isnan(want).sum() == 4 * 64
    np.testing.assert_array_equal(P.np64(back[0, 0, 0]), want)
    np.testing.assert_array_equal(P.np64(back[1, 0, 0]), want)
    np.testing.assert_array_equal(P.np64(bd[0, 0]), np.stack([want.min(0), want.max(0)]))
    pg.close()


@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_store_and_load_skip_and_report(B, bits, dtype):
    hkv, d, page, cap = 2, 64, 16, 40
    table = np.array([[5, 2, 1], [3, 4, 0], [6, 99, 7]], np.int32)   # the third's second page is outside the pool
    pg = T.make(B, n_q_heads=2, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=8, max_seqs=3, max_seq_pages=3, cache_bits=bits)
    k, v = dense((3, hkv, 48, d), dtype, 1), dense((3, hkv, 48, d), dtype, 2)
    shape = (8, hkv, pg.page_bytes()) if bits else (8, hkv, page, d)
    kp, vp = (torch.zeros(shape, dtype=torch.uint8 if bits else DT[dtype], device="cuda") for _ in range(2))
    t = T.i32(table.tolist())
    if bits:
        pg.page_store(k[:, :, :cap], v[:, :, :cap], T.i32([33, 41, 20]), t, kp, vp)      # the second is longer than its source
        assert pg.poll_status() in (B.MEDA_ERR_WORKSPACE, B.MEDA_ERR_INVALID_ARG) and pg.poll_status() == 0
        assert (kp[[0, 3, 4, 7]] == 0).all() and (kp[[1, 2, 5, 6]] != 0).any(-1).all()
        pg.page_store(k, v, T.i32([-1, 49, 0]), t, kp, vp)
        assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
        assert (kp[[0, 3, 4, 7]] == 0).all()
    pg.page_store(k, v, T.i32([48, 48, 16]), t, kp, vp)
    pg.check()
    whole = torch.full((2, 3, hkv, 48, d), 7.0, dtype=DT[dtype], device="cuda")
    pg.page_load(kp, vp, t, T.i32([48, 48, 16]), whole[0], whole[1])
    pg.check()
    if not bits:
        assert torch.equal(whole[0, :2], k[:2]) and torch.equal(whole[1, 2, :, :16], v[2, :, :16]) and (whole[:, 2, :, 16:] == 7).all()

    def load(lens, first=None, capacity=40):
        out = torch.full((2, 3, hkv, capacity, d), 7.0, dtype=DT[dtype], device="cuda")
        pg.page_load(kp, vp, t, T.i32(lens), out[0], out[1], lens_from=None if first is None else T.i32(first))
        return out, pg.poll_status()

    out, status = load([33, 41, 16])                               # the second has more rows than fit
    assert status == B.MEDA_ERR_WORKSPACE and torch.equal(out[:, 0, :, :33], whole[:, 0, :, :33]) and (out[:, 1] == 7).all()
    assert torch.equal(out[:, 2, :, :16], whole[:, 2, :, :16]) and (out[:, 2, :, 16:] == 7).all()
    out, status = load([33, 41, 20], [0, 1, 0])                    # now it fits; the third's second page is outside the pool
    assert status == B.MEDA_ERR_INVALID_ARG and torch.equal(out[:, 1, :, :40], whole[:, 1, :, 1:41])
    assert torch.equal(out[:, 2, :, :16], whole[:, 2, :, :16]) and (out[:, 2, :, 16:] == 7).all()
    out, status = load([-1, 49, 16], [0, 20, 17])                  # no lengths; a start behind the end is no rows
    assert status == B.MEDA_ERR_INVALID_ARG and (out == 7).all()
    out, status = load([48, 48, 16], [48, 49, -1])
    assert status == B.MEDA_ERR_INVALID_ARG and (out == 7).all()
    out, status = load([48, 48, 16], [8, 48, 3])
    assert status == 0 and torch.equal(out[:, 0, :, :40], whole[:, 0, :, 8:]) and (out[:, 1] == 7).all()
    assert torch.equal(out[:, 2, :, :13], whole[:, 2, :, 3:16])
    out, status = load([0, 0, 0], capacity=0)
    assert status == 0
    out, status = load([0, 1, 0], capacity=0)
    assert status == B.MEDA_ERR_WORKSPACE
    pg.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_rows_of_pages_that_are_not_quantised_read_back(B, dtype, d, page):
    hkv, n = 2, len(LENS)
    width = O.n_pages_of(300, page)
    n_pages = sum(O.n_pages_of(x, page) for x in LENS)
    table = T.table_for(LENS, page, width, n_pages, 1)
    pg = T.make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=n, max_seq_pages=width)
    k, v = dense((n, hkv, 300, d), dtype, 1), dense((n, hkv, 300, d), dtype, 2)
    kp, vp = (torch.zeros((n_pages, hkv, page, d), dtype=DT[dtype], device="cuda") for _ in range(2))
    t, lens = T.i32(table.tolist()), T.i32(LENS)
    pg.page_store(k, v, lens, t, kp, vp)
    first = [0, 0, 3, 15, 16, 100, 255, 13, 299, 17]
    out = torch.full((2, n, hkv, 300, d), 7.0, dtype=DT[dtype], device="cuda")
    pg.page_load(kp, vp, t, lens, out[0], out[1], lens_from=T.i32(first))
    pg.check()
    for i, (a, m) in enumerate(zip(first, LENS)):
        count = max(0, m - a)
        assert torch.equal(out[0, i, :, :count], k[i, :, a:a + count]) and torch.equal(out[1, i, :, :count], v[i, :, a:a + count])
        assert (out[:, i, :, count:] == 7).all()
    pg.close()


# ---------------------------------------------------------------------------------------------------- append

APPENDS = [(64, (16, 8, 8), 0), (64, (8, 0, 0), 0), (128, (24, 20, 20), 1), (128, (64, 0, 0), 0), (128, (4, 2, 2), 1), (256, (64, 32, 32), 0), (256, (40, 32, 32), 1)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("d,sections,order", APPENDS)
def test_rope_append(B, bits, dtype, pairing, d, sections, order):
    hq, hkv, page, tokens, n_pages = 6, 2, 16, 37, 9
    theta = 1e6
    pg = T.make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=1, max_seq_pages=1, cache_bits=bits,
                rope_theta=theta, rope_sections=sections, rope_order=order, rope_pairing=pairing)
    qkv = dense((tokens, hq + 2 * hkv, d), dtype, d + bits)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    rng = np.random.default_rng(d)
    pos = rng.integers(-3, 200_000, (3, tokens))
    pos[:, 0], pos[:, 1], pos[:, 2] = 0, 2 ** 31 - 1, -2 ** 31
    slots = rng.permutation(n_pages * page)[:tokens]
    slots[5] = -1
    q_out = torch.full((tokens, hq, d), 7.0, dtype=DT[dtype], device="cuda")
    kp, vp = empty_pool(n_pages, hkv, page, d, bits), empty_pool(n_pages, hkv, page, d, bits)
    pg.rope_append(q, k, v, T.i32(pos.tolist()), torch.tensor(slots, device="cuda"), q_out, kp, vp)
    pg.check()
    turned = {}
    for name, x in (("q", q), ("k", k)):
        y = O.rope_fp32(P.np64(x), pos, sections, order, pairing, theta)
        turned[name] = torch.as_tensor(y).to(DT[dtype]).double().numpy()
    turned["v"] = P.np64(v)
    live = slots >= 0
    np.testing.assert_array_equal(P.np64(q_out)[live], turned["q"][live])
    assert (q_out[5] == 7).all()
    for pool, name in ((kp, "k"), (vp, "v")):
        got = O.unpack_page(pool.cpu().numpy(), page, d, bits)
        want = O.quantise(turned[name].astype(np.float32), bits)
        written = np.zeros((n_pages, page), bool)
        for i, s in enumerate(slots):
            if s >= 0:
                written[s // page, s % page] = True
                for a, b in zip(got, want):
                    np.testing.assert_array_equal(a[s // page, :, s % page], b[i], err_msg=f"token {i}")
        assert np.isnan(got[1].transpose(0, 2, 1, 3)[~written]).all()      # everything else is as it was
        assert (got[0].transpose(0, 2, 1, 3, 4)[~written] == (1 << bits) - 1).all()
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
def test_rope_append_in_place_without_queries_without_rotation_and_bad_slots(B, bits):
    hq, hkv, d, page, n_pages, t = 3, 2, 128, 16, 130, 2000
    pg = T.make(B, n_q_heads=hq * hkv, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_seqs=1, max_seq_pages=1, cache_bits=bits)
    q, k, v = dense((t, hq * hkv, d), "bf16", 1), dense((t, hkv, d), "bf16", 2), dense((t, hkv, d), "bf16", 3)
    slots = torch.tensor(np.random.default_rng(0).permutation(n_pages * page)[:t], device="cuda")
    pos = torch.arange(t, dtype=torch.int32, device="cuda").expand(3, t).contiguous()
    pools = [empty_pool(n_pages, hkv, page, d, bits) for _ in range(6)]
    out = torch.empty_like(q)
    pg.rope_append(q, k, v, pos, slots, out, pools[0], pools[1])
    mine = q.clone()
    pg.rope_append(mine, k, v, pos, slots, mine, pools[2], pools[3])       # in place
    assert torch.equal(mine, out) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    pg.rope_append(None, k, v, pos, slots, None, pools[4], pools[5])       # keys and values alone
    pg.check()
    assert torch.equal(pools[0], pools[4]) and torch.equal(pools[1], pools[5])
    # no positions: the rows are quantised as they are, and a store of them writes the same bytes
    rows = torch.empty((1, hkv, n_pages * page, d), dtype=torch.bfloat16, device="cuda")
    whole = [empty_pool(n_pages, hkv, page, d, bits) for _ in range(4)]
    every = torch.arange(n_pages * page, device="cuda")
    kk, vv = dense((n_pages * page, hkv, d), "bf16", 8), dense((n_pages * page, hkv, d), "bf16", 9)
    pg.rope_append(None, kk, vv, None, every, None, whole[0], whole[1])
    one = T.make(B, n_q_heads=hkv, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_seqs=1, max_seq_pages=n_pages, cache_bits=bits)
    rows.copy_(kk.transpose(0, 1)[None])
    one.page_store(rows, vv.transpose(0, 1)[None].contiguous(), T.i32([n_pages * page]), T.i32([list(range(n_pages))]), whole[2], whole[3])
    one.check()
    assert torch.equal(whole[0], whole[2]) and torch.equal(whole[1], whole[3])
    # slots outside the pool are recorded and skipped
    bad = slots.clone()
    bad[3], bad[1999] = n_pages * page, -2
    fresh = [empty_pool(n_pages, hkv, page, d, bits) for _ in range(2)]
    out5 = torch.full_like(q, 7.0)
    pg.rope_append(q, k, v, pos, bad, out5, *fresh)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[3] = keep[1999] = False
    assert torch.equal(out5[keep], out[keep]) and (out5[~keep] == 7).all()
    head = page * d * bits // 8
    codes = [x[..., :head].view(n_pages, hkv, page, -1).transpose(1, 2).reshape(n_pages * page, hkv, -1) for x in (pools[0], fresh[0])]
    assert torch.equal(codes[0][slots[keep]], codes[1][slots[keep]]) and (codes[1][slots[~keep]] == 0xff).all()
    pg.close()
    one.close()


# ------------------------------------------------------------------------------------------------- attention

def coded_attention(q_heads, k, v):
    """k, v: (codes, step, low) of the rows of one head -> (out, lse, sizes of what is added up)."""
    kr, vr = O.held(*k), O.held(*v)
    g, d = q_heads.shape
    if len(kr) == 0:
        return np.zeros((g, d)), np.full(g, -np.inf), None
    s = q_heads @ kr.T / np.sqrt(d)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    z = e.sum(-1, keepdims=True)
    p = e / z
    part = lambda c, step, low: (O.held(c, step, 0 * low), O.held(0 * c, step, np.abs(low)))
    (kc, kl), (vc, vl) = part(*k), part(*v)
    aux = dict(mag=(np.abs(q_heads) @ (kc + kl).T / np.sqrt(d)).max(-1), codes=p @ vc, lows=p @ vl, top=p.max(-1), range=vc.max(), rows=len(kr))
    return p @ vr, (m + np.log(z))[:, 0], aux


def coded_tolerance(want, aux, d, dtype):
    """Absolute bound on |out - want|.  A logit is the sum of step * (q . codes) and low * (sum of q) over the groups, d + d / 64 products
    accumulated in fp32 (2^-22 per step, which also covers an accumulator that truncates); the sum of q enters in three bf16 parts (2^-24):
    off by at most delta = (d + 32) 2^-22 max_j sum |q| (step code + |low|) / sqrt(d), which moves a probability by exp(delta) and
    its normaliser by as much.  exp2 is off by 2^-22, sums of `rows` terms by rows 2^-22.  All of that is relative to sum p (step code +
    |low|).  The weight p * step of a row's codes enters the product in fp16, 2^-11 relative (two such parts for fp32, 2^-22), and no
    finer than 2^-25 * 2^-6 of the largest step's next power of two (p up to 1 scaled by 2^6).  The result is rounded once."""
    delta = (d + 32) * 2.0 ** -22 * aux["mag"]
    rel = 2 * delta * (1 + delta) + (aux["rows"] + 64) * 2.0 ** -22
    weight = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    floor = aux["rows"] * aux["top"] * 2.0 ** -31 * 2 * aux["range"] * (1 if dtype == "bf16" else 2.0 ** -8)
    return (aux["codes"] + aux["lows"]) * rel[:, None] + weight * 1.01 * aux["codes"] + floor[:, None] + T.HALF_STEP[dtype] * 1.01 * np.abs(want) + 1e-30


def lse_tolerance(lse, aux, d):
    return (d + 32) * 2.0 ** -22 * aux["mag"] + (aux["rows"] + 64) * 2.0 ** -22 + 2.0 ** -21 * np.abs(lse) + 1e-6


def check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype, sel=None, keep=0):
    hq, d = q.shape[1:]
    hkv = kp.shape[1]
    group = hq // hkv
    got, got_lse, qh = P.np64(out), P.np64(lse) if lse is not None else None, P.np64(q)
    for i, m in enumerate(lens):
        c = O.n_pages_of(m, page)
        at = torch.as_tensor(table[i, :c].astype(np.int64), device="cuda")
        k, v = (O.unpack_page(x[at].cpu().numpy(), page, d, bits) for x in (kp, vp))
        for g in range(hkv):
            rows = np.arange(m)
            if sel is not None:
                rows = np.concatenate([np.arange(x * page, min(m, x * page + page)) for x in sel[i, g, :min(keep, c)]]).astype(np.int64) if c else rows
            kg, vg = ([a[:, g].reshape((-1,) + a.shape[3:])[rows] for a in x] for x in (k, v))
            heads = slice(g * group, (g + 1) * group)
            want, want_lse, aux = coded_attention(qh[i, heads], kg, vg)
            if len(rows) == 0:
                assert (got[i, heads] == 0).all() and (got_lse is None or (got_lse[i, heads] == -np.inf).all())
                continue
            tol = coded_tolerance(want, aux, d, dtype)
            assert (np.abs(got[i, heads] - want) <= tol).all(), (i, g, m, float((np.abs(got[i, heads] - want) - tol).max()))
            if got_lse is not None:
                assert (np.abs(got_lse[i, heads] - want_lse) <= lse_tolerance(want_lse, aux, d)).all(), (i, g, m)


def attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=0, q_std=2.0):
    """Pools written by the oracle; what no sequence owns is 0xff: NaN steps and lowest values."""
    width = max(1, max(O.n_pages_of(x, page) for x in lens) + 1)
    n_pages = sum(O.n_pages_of(x, page) for x in lens) + 3
    table = T.table_for(lens, page, width, n_pages, seed)
    pg = T.make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=len(lens), max_seq_pages=width, cache_bits=bits)
    owned = np.zeros((n_pages, page), bool)
    for i, m in enumerate(lens):
        for c in range(O.n_pages_of(m, page)):
            owned[table[i, c], :min(page, m - c * page)] = True
    pools = []
    for s, std, mean in ((1, 0.3, 0.1), (2, 0.5, -0.2)):
        rng = np.random.default_rng(seed + s)
        x = rng.normal(mean, std, (n_pages, hkv, page, d)).astype(np.float32) * rng.uniform(0.2, 4, (hkv, 1, d)).astype(np.float32)
        code, step, low = O.quantise(x, bits)
        dead = np.broadcast_to(~owned[:, None], (n_pages, hkv, page))
        code[dead], step[dead], low[dead] = (1 << bits) - 1, np.nan, np.nan
        pools.append(torch.as_tensor(O.pack_page(code, step, low, bits), device="cuda"))
    q = T.normal((len(lens), hq, d), DT[dtype], seed + 3, 0.0, q_std)
    out = torch.full((len(lens), hq, d), math.nan, dtype=DT[dtype], device="cuda")
    return pg, q, *pools, table, out, torch.full((len(lens), hq), math.nan, device="cuda")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page", [(1, 1, 64, 16), (4, 2, 64, 32), (6, 2, 128, 16), (7, 1, 128, 64), (8, 8, 128, 128), (28, 4, 128, 16),
                                           (8, 1, 64, 256), (9, 1, 64, 16), (16, 1, 128, 16), (24, 2, 128, 32), (2, 2, 256, 16), (10, 2, 256, 32),
                                           (16, 1, 256, 64), (11, 1, 256, 16)])
def test_attention_edges(B, bits, dtype, hq, hkv, d, page):
    lens = T.EDGES
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=hq + d)
    t = T.i32(table.tolist())
    pg.paged_attention(q, kp, vp, t, T.i32(lens), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype)
    # again without lse, strided lengths, another stream: the same bits
    lens3 = torch.stack([T.i32(lens), T.i32([9999] * len(lens))], 1)[:, 0]
    out2 = torch.full_like(out, math.nan)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pg.paged_attention(q, kp, vp, t, lens3, out2, stream=s)
    s.synchronize()
    assert torch.equal(out, out2)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,lens", [
    ("bf16", 7, 1, 128, 16, [5003]), ("bf16", 28, 4, 128, 64, [20001]), ("bf16", 4, 4, 64, 32, [10000, 3, 9000]), ("bf16", 16, 1, 128, 16, [15011]),
    ("f32", 7, 1, 128, 32, [7001]), ("f32", 3, 1, 64, 16, [6000, 1, 0, 12345]), ("bf16", 8, 1, 256, 16, [9001, 100]), ("f32", 12, 1, 256, 16, [4001])])
def test_attention_split_over_many_blocks(B, bits, dtype, hq, hkv, d, page, lens):
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=11)
    t, n = T.i32(table.tolist()), T.i32(lens)
    pg.paged_attention(q, kp, vp, t, n, out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype)
    for _ in range(3):                                             # joined in a fixed order: the same bits every time
        out2, lse2 = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
        pg.paged_attention(q, kp, vp, t, n, out2, lse2)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
def test_attention_many_short_sequences(B, bits):
    lens = np.random.default_rng(0).integers(0, 60, 1500).tolist()
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 4, 2, 64, "bf16", 16, bits, seed=3)
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, 16, bits, "bf16")
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,lens,keep", [(28, 4, 128, 16, [5000, 17, 0, 300], 40), (4, 4, 64, 64, [2000, 64], 7), (16, 1, 256, 32, [3000], 30)])
def test_attention_over_chosen_pages(B, bits, dtype, hq, hkv, d, page, lens, keep):
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=21)
    t, n = T.i32(table.tolist()), T.i32(lens)
    bd = torch.full((kp.shape[0], hkv, 2, d), math.nan, dtype=DT[dtype], device="cuda")
    sel = torch.full((len(lens), hkv, keep), -1, dtype=torch.int32, device="cuda")
    pg.page_bounds(kp, t, None, n, bd)
    pg.select_pages(q, bd, t, n, 1, 2, sel)
    pg.paged_attention(q, kp, vp, t, n, out, lse, sel=sel)
    pg.check()
    T.check_selection(sel, q, bd, table, lens, page, keep, 1, 2)
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype, sel.cpu().numpy(), keep)
    # in another order: the same pages, within the same bound
    pg.paged_attention(q, kp, vp, t, n, out, lse, sel=torch.where(sel[:1] >= 0, sel.flip(-1), sel) if min(lens) >= keep * page else sel)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype, sel.cpu().numpy(), keep)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_scales_far_apart(B, bits, dtype):
    """Rows whose steps differ by 2^40 in one cache, tiny and huge values, a first row that takes all the weight and has tiny values, and logits
    that decide alone: precision is relative to what is added up."""
    lens, hq, hkv, d, page = [400, 700, 90], 4, 2, 128, 16
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=5)
    rng = np.random.default_rng(1)
    n_pages = kp.shape[0]
    x = rng.normal(0, 1, (n_pages, hkv, page, d)) * 2.0 ** rng.integers(-20, 21, (n_pages, hkv, page, 1))
    x[table[1, 0], :, 0] *= 2.0 ** -30
    x[table[2, :6]] *= 2.0 ** 60
    vp.copy_(torch.as_tensor(O.pack_page(*O.quantise(x.astype(np.float32), bits), bits)))
    k = rng.normal(0, 0.3, (n_pages, hkv, page, d))
    k[table[1, 0], :, 0] = P.np64(q[1, ::hq // hkv])               # row 0 of sequence 1 answers its first heads
    k[table[0, 7], :, 3] = 300 * P.np64(q[0, 1::hq // hkv])        # a logit far above all others
    kp.copy_(torch.as_tensor(O.pack_page(*O.quantise(k.astype(np.float32), bits), bits)))
    t = T.i32(table.tolist())
    pg.paged_attention(q, kp, vp, t, T.i32(lens), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_over_groups_that_read_back_as_nan(B, bits, dtype):
    """A key group of NaN makes its head's outputs NaN in its own sequence; a value group its 64 dimensions; a query that is not finite its own
    head's."""
    lens, hq, hkv, d, page = [40, 40, 40], 4, 2, 128, 16
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=6)
    more = page * d * bits // 8
    half = lambda pool: pool[:, :, more:].view(torch.bfloat16).view(-1, hkv, page, 2, d // 64)
    half(kp)[int(table[0, 1]), 1, 3, :, 0] = math.nan              # sequence 0, KV head 1
    half(vp)[int(table[1, 2]), 0, 7, :, 1] = math.nan              # sequence 1, KV head 0, the second 64 dimensions
    q[2, 1, 5] = math.nan
    q[2, 2, 9] = math.inf
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse)
    pg.check()
    nan = out.isnan().cpu()
    want = torch.zeros_like(nan)
    want[0, 2:] = True
    want[1, :2, 64:] = True
    want[2, 1:3] = True
    assert torch.equal(nan, want)
    assert torch.equal(lse.isnan().cpu(), torch.tensor([[0, 0, 1, 1], [0, 0, 0, 0], [0, 1, 1, 0]], dtype=torch.bool))
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_of_every_size(B, bits, dtype):
    """Queries from subnormal to huge: tiny ones weigh all rows alike, and their largest element may be anywhere."""
    lens, hq, hkv, d, page = [100] * 6, 8, 1, 64, 16
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=9)
    scale = torch.tensor([0.0, 2.0 ** -130, 2.0 ** -100, 2.0 ** -14, 1.0, 2.0 ** 5], device="cuda")
    q.copy_((q.double() * scale[:, None, None]).to(q.dtype))
    q[3, :, 0] = 2.0 ** -40                                        # beside elements of 2^-14
    q[4, 0] = 0.0
    q[4, 0, 17] = 3.0
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse)
    pg.check()
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, dtype)
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_huge_logits_and_queries(B, bits, dtype):
    """Logits of up to 10^8 in an order that moves the maximum in every tile (weights in fp16 must not overflow), queries of 2^100 with keys as small,
    and of 2^110, which are refused as NaN."""
    lens, hq, hkv, d, page = [300, 300, 300, 40], 2, 1, 64, 16
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, hq, hkv, d, dtype, page, bits, seed=12)
    k = np.zeros((kp.shape[0], hkv, page, d))
    rows = np.arange(300)
    for i, top in ((0, 1e8), (1, 1e4), (2, 2.0 ** -90)):
        for c in range(O.n_pages_of(300, page)):
            at = rows[c * page:(c + 1) * page]
            k[table[i, c], 0, :len(at), 0] = top * (at + 1) / 300
    k[table[0, 18], 0, 5] = 0.0
    kp.copy_(torch.as_tensor(O.pack_page(*O.quantise(k.astype(np.float32), bits), bits)))
    q.zero_()
    q[0, :, 0], q[1, :, 0], q[2, :, 0], q[3, 0, 3], q[3, 1, 3] = 1.0, 1.0, 2.0 ** 100, 2.0 ** 110, -(2.0 ** 109)
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse)
    pg.check()
    check_attention(out[:3], lse[:3], q[:3], kp, vp, table[:3], lens[:3], page, bits, dtype)
    assert out[3, 0].isnan().all() and lse[3, 0].isnan() and not out[3, 1].isnan().any()       # (keys of 0 there)
    pg.close()


@pytest.mark.parametrize("dtype,bits,hq,d", [("bf16", 4, 1, 256), ("f32", 4, 2, 256), ("bf16", 8, 1, 256), ("bf16", 4, 16, 128), ("f32", 8, 9, 64)])
def test_attention_of_the_largest_batch(B, dtype, bits, hq, d):
    """8,192 sequences of 0 to 40 rows: the prefix sums leave the least shared memory to the rings.  Outputs by a plain form on the device in
    64 bits, to the bound of check_attention, with the keys' and values' sizes as they are."""
    page, n = 16, 8192
    lens = np.random.default_rng(1).integers(0, 41, n)
    n_pages = 700
    pg = T.make(B, n_q_heads=hq, n_kv_heads=1, head_dim=d, dtype=dtype, page_size=page, n_pages=n_pages, max_seqs=n, max_seq_pages=3, cache_bits=bits)
    rng = np.random.default_rng(2)
    pools, held = [], []
    for std in (0.3, 0.5):
        code, step, low = O.quantise(rng.normal(0.1, std, (n_pages, 1, page, d)).astype(np.float32), bits)
        pools.append(torch.as_tensor(O.pack_page(code, step, low, bits), device="cuda"))
        sizes = O.held(code, step, 0 * low) + np.abs(O.held(0 * code, step, low))
        held += [torch.as_tensor(x, device="cuda") for x in (O.held(code, step, low)[:, 0], sizes[:, 0])]
    table = torch.as_tensor(rng.integers(0, n_pages, (n, 3)).astype(np.int32), device="cuda")          # (read only: pages may be shared)
    q = T.normal((n, hq, d), DT[dtype], 3, 0.0, 2.0)
    out, lse = torch.full_like(q, math.nan), torch.full((n, hq), math.nan, device="cuda")
    pg.paged_attention(q, *pools, table, T.i32(lens.tolist()), out, lse)
    pg.check()
    k, k_size, v, v_size = (x[table.long()].flatten(1, 2) for x in held)
    live = torch.arange(48, device="cuda")[None] < torch.as_tensor(lens, device="cuda")[:, None]
    s = torch.where(live[:, None], q.double() @ k.transpose(1, 2) / math.sqrt(d), -math.inf)
    p = torch.where(live.any(1)[:, None, None], torch.softmax(s, -1), 0.0)
    want, mag = p @ v, torch.where(live[:, None], q.double().abs() @ k_size.transpose(1, 2) / math.sqrt(d), 0.0).amax(-1, keepdim=True)
    delta = (d + 32) * 2.0 ** -22 * mag
    tol = (p @ v_size) * (2 * delta * (1 + delta) + 2.0 ** -15 + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * 1.01) + T.HALF_STEP[dtype] * 1.01 * want.abs() + 1e-6
    assert ((out.double() - want).abs() <= tol).all()
    norm = torch.logsumexp(s, -1)
    assert torch.equal(lse.isinf(), norm.isinf())
    assert ((lse.double() - norm).abs() <= delta[..., 0] + 2.0 ** -15 + 2.0 ** -21 * norm.abs())[~norm.isinf()].all()
    pg.close()


def test_bad_pages_and_lengths_are_reported_and_skipped(B):
    page, d, lens, bits = 16, 64, [48, 33], 4
    pg, q, kp, vp, table, out, lse = attention_case(B, lens, 2, 1, d, "bf16", page, bits, seed=8)
    bad = table.copy()
    bad[0, 1], bad[1, 0] = -1, 5000
    pg.paged_attention(q, kp, vp, T.i32(bad.tolist()), T.i32(lens), out, lse)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    sel = np.array([[[0, 2]], [[1, 2]]])
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, "bf16", sel, 2)
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32([-3, 33]), out, lse)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all() and out[1].isfinite().all()
    # chosen pages that are none of the sequence's
    pick = T.i32([[[0, 3]], [[-1, 1]]])
    pg.paged_attention(q, kp, vp, T.i32(table.tolist()), T.i32(lens), out, lse, sel=pick)
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, "bf16", np.array([[[0]], [[1]]]), 1)
    # an append whose slot is good into a page that a bad table does not name is still there
    pg.close()


@pytest.mark.parametrize("bits", [4, 8])
def test_pools_beyond_four_gib(B, bits):
    hkv, d, page = 8, 256, 64
    page_bytes = page * row_bytes(d, bits)
    n_pages = int(4.6e9) // (hkv * page_bytes)
    pg = T.make(B, n_q_heads=16, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_seqs=2, max_seq_pages=20, cache_bits=bits)
    kp, vp = (torch.empty((n_pages, hkv, page_bytes), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert kp.numel() > 2 ** 32
    lens = [70, 1111]
    table = np.full((2, 20), 1 << 30, np.int32)
    table[0, :2] = [n_pages - 1, 5]
    table[1, :18] = n_pages - 2 - 100 * np.arange(18)
    k, v = dense((2, hkv, 1200, d), "bf16", 1), dense((2, hkv, 1200, d), "bf16", 2)
    bd = torch.empty((n_pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    t = T.i32(table.tolist())
    pg.page_store(k, v, T.i32([69, 1111]), t, kp, vp, bd)
    row, val = dense((1, hkv, d), "bf16", 4), dense((1, hkv, d), "bf16", 5)
    pg.rope_append(None, row, val, None, torch.tensor([5 * page + 5], device="cuda"), None, kp, vp)
    k[0, :, 69], v[0, :, 69] = row[0], val[0]
    back = torch.zeros((2, 2, hkv, 1200, d), dtype=torch.bfloat16, device="cuda")
    pg.page_load(kp, vp, t, T.i32(lens), back[0], back[1])
    q, out, lse = T.normal((2, 16, d), torch.bfloat16, 3, 0.0, 0.5), torch.empty((2, 16, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 16), device="cuda")
    pg.paged_attention(q, kp, vp, t, T.i32(lens), out, lse)
    pg.check()
    for x, y in ((k, back[0]), (v, back[1])):
        for i, m in enumerate(lens):
            np.testing.assert_array_equal(P.np64(y[i, :, :m]), rounded(O.held(*O.quantise(P.np64(x[i, :, :m]).astype(np.float32), bits)), "bf16"))
    check_attention(out, lse, q, kp, vp, table, lens, page, bits, "bf16")
    pg.close()


# ------------------------------------------------------------------------------------------------- refusals

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
def test_refusals(B, bits, dtype):
    pg, q, kp, vp, table, out, lse = attention_case(B, [20, 30], 4, 2, 64, dtype, 16, bits)
    t, n = T.i32(table.tolist()), T.i32([20, 30])
    k, v = (torch.zeros((2, 2, 32, 64), dtype=DT[dtype], device="cuda") for _ in range(2))
    kn, slots = k[:, :, 0].contiguous(), torch.zeros(2, dtype=torch.int64, device="cuda")
    bd = torch.zeros((kp.shape[0], 2, 2, 64), dtype=DT[dtype], device="cuda")
    plain = torch.zeros((kp.shape[0], 2, 16, 64), dtype=DT[dtype], device="cuda")
    wide = torch.zeros((2, 2, 32, 128), dtype=DT[dtype], device="cuda")
    for call in (
        lambda: pg.paged_attention(q, plain, plain, t, n, out),                         # pools of rows as they are
        lambda: pg.page_store(k, v, n, t, plain, vp),
        lambda: pg.paged_attention(q, kp.view(torch.int8), vp, t, n, out),
        lambda: pg.paged_attention(q, kp[:-1], vp, t, n, out),
        lambda: pg.paged_attention(q, kp, vp[..., :-16], t, n, out),
        lambda: pg.rope_append(None, kn, kn, None, slots, None, kp.transpose(0, 1), vp),
        lambda: pg.page_bounds(plain, t, None, n, bd),
        lambda: pg.page_load(kp, plain, t, n, k, v),
        lambda: pg.page_load(kp, vp, t, n, k, v[:, :, :16]),
        lambda: pg.page_load(kp, vp, t, n, k, wide[..., :64]),                          # rows that are not dense
        lambda: pg.page_load(kp, vp, t, n, k[:1], v[:1]),
        lambda: pg.page_load(kp, vp, t, n.long(), k, v),
        lambda: pg.page_load(kp, vp, t[:, :1], n, k, v),
        lambda: pg.page_load(kp, vp, t, n, k, v, lens_from=n[:1]),
        lambda: pg.page_load(kp, vp, t, n, k, v, lens_from=torch.stack([n, n], 1)[:, 0]),
        lambda: pg.page_load(kp, vp, t, n, k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1)),      # sequences on top of one another
        lambda: pg.page_load(kp, vp, t, n, k[:, :1].expand(-1, 2, -1, -1), v[:, :1].expand(-1, 2, -1, -1)),
        lambda: pg.page_load(kp, vp, t, n, k.view(-1).as_strided((2, 2, 32, 64), (4096, 1024, 64, 1)), v.view(-1).as_strided((2, 2, 32, 64), (4096, 1024, 64, 1))),
    ):
        with pytest.raises(ValueError):
            call()

    def off(x):                                                    # one byte or element into its buffer
        y = torch.zeros(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        assert y.is_contiguous() and y.data_ptr() % 16 != 0
        return y

    calls = [
        (lambda q, kp, vp, out: pg.paged_attention(q, kp, vp, t, n, out), (q, kp, vp, out)),
        (lambda k, v, kp, vp, bd: pg.page_store(k, v, n, t, kp, vp, bd), (k, v, kp, vp, bd)),
        (lambda kp, vp, k, v: pg.page_load(kp, vp, t, n, k, v), (kp, vp, k, v)),
        (lambda kp, bd: pg.page_bounds(kp, t, None, n, bd), (kp, bd)),
        (lambda q, k, v, out, kp, vp: pg.rope_append(q, k, v, None, slots, out, kp, vp), (q, kn, kn.clone(), out, kp, vp)),
    ]
    for call, args in calls:
        for i in range(len(args)):
            with pytest.raises(B.MedaError) as e:
                call(*args[:i], off(args[i]), *args[i + 1:])
            assert e.value.status == B.MEDA_ERR_SHAPE
    lib = B.load_library()
    load = lambda **kw: lib.meda_page_load(*{**dict(h=pg._h, k=kp.data_ptr(), v=vp.data_ptr(), t=t.data_ptr(), f=None, n=n.data_ptr(), s=1, c=2, ko=k.data_ptr(),
                                                    vo=v.data_ptr(), ss=4096, hs=2048, cap=32, st=None), **kw}.values())
    assert load(c=3) == B.MEDA_ERR_SHAPE and load(c=-1) == B.MEDA_ERR_INVALID_ARG and load(ss=4097) == B.MEDA_ERR_SHAPE and load(hs=2049) == B.MEDA_ERR_SHAPE
    assert load(ko=None) == B.MEDA_ERR_INVALID_ARG and load(t=None) == B.MEDA_ERR_INVALID_ARG and load(cap=-1) == B.MEDA_ERR_INVALID_ARG
    assert load(c=0, k=None, n=None, ko=None) == 0
    assert pg.launch_count() == 0
    pg.close()
    with pytest.raises(ValueError):
        pg.page_load(kp, vp, t, n, k, v)
