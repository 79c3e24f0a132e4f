"""Attention over quantised pages where numbers are far apart or large: logits beyond 2^26, rows that count for nothing beside rows that do, keys and
values next to fp32's end.

Tolerances.  A logit is the sum over the groups of step * (q . codes) and low * (sum of q), d + d / 64 products added up in fp32 (2^-22 for each, which also
covers an accumulator that truncates), and is rounded once more: off by at most delta = (d + 34) 2^-22 sum |q| (step code + |low|) / sqrt(d); that moves a
probability by exp(delta) and its normaliser by as much.  exp2 is off by 2^-22, sums of `rows` terms by rows 2^-22.  The weight p * step of a row's codes
enters its product in fp16, off by 2^-11 of itself for bf16 outputs and by 2^-22 for fp32 ones (two parts), and no finer than 2^-25 where the largest
weight of its head and 64 dimensions is 2^-6 or more (fp32: 1 or more).  The result is rounded once.  All of it is relative to what is added up,
p * step * code and p * |low|: a row without weight is not in it."""
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


def pool(x, bits):
    return torch.as_tensor(O.pack_page(*O.quantise(np.asarray(x).astype(np.float32), bits), bits), device="cuda")


def attend(B, q, k, v, dtype, bits, times=1):
    """k, v [n][rows][d], q [n][hq][d]: every sequence one page of one KV head, all of them `times` over (a batch large enough that a warp goes
    through several tiles of one) -> out, lse [times][n][hq]..."""
    (n, rows, d), hq = k.shape, q.shape[1]
    page = max(16, 1 << (rows - 1).bit_length())
    kp, vp = (pool(np.concatenate([x, np.zeros((n, page - rows, d))], 1)[:, None], bits) for x in (k, v))
    pg = T.make(B, n_q_heads=hq, n_kv_heads=1, head_dim=d, dtype=dtype, page_size=page, n_pages=n, max_seqs=n * times, max_seq_pages=1, cache_bits=bits)
    many = q.repeat(times, 1, 1)
    out, lse = torch.full_like(many, math.nan), torch.full(many.shape[:2], math.nan, device="cuda")
    pg.paged_attention(many, kp, vp, T.i32([[i] for i in range(n)]).repeat(times, 1), T.i32([rows] * (n * times)), out, lse)
    pg.check()
    pg.close()
    return out.view(times, *q.shape), lse.view(times, n, hq)


def parts(v, bits):
    """What rows of values [..., d] read back as, and the sizes of their code and low parts."""
    code, step, low = O.quantise(np.asarray(v).astype(np.float32), bits)
    return O.held(code, step, low), O.held(code, step, 0 * low), O.held(0 * code, step, np.abs(low))


def check(out, lse, q, k, v, bits, dtype):
    """out [times][n][hq][d] against softmax over the rows k, v [n][rows][d], q [n][hq][d]; see the file's head."""
    rows, d = k.shape[1:]
    kr, kc, kl = parts(k, bits)
    vr, vc, vl = parts(v, bits)
    s = np.einsum("nhd,nrd->nhr", q, kr) / math.sqrt(d)
    top = s.max(-1, keepdims=True)
    e = np.exp(s - top)
    z = e.sum(-1, keepdims=True)
    p = e / z
    mag = (np.einsum("nhd,nrd->nhr", np.abs(q), kc + kl) / math.sqrt(d)).max(-1, keepdims=True)
    delta = (d + 34) * 2.0 ** -22 * mag
    rel = 2 * delta * (1 + delta) + (rows + 64) * 2.0 ** -22
    codes, lows = p @ vc, p @ vl
    step = O.quantise(np.asarray(v).astype(np.float32), bits)[1]                    # [n][rows][groups]
    weight = (p[..., None] * step[:, None]).max(2).repeat(64, -1)                   # the largest of each head and group
    fine = (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * 1.01 * codes + rows * (2.0 ** -19 if dtype == "bf16" else 2.0 ** -25) * weight * (1 << bits)
    want = p @ vr
    tol = (codes + lows) * rel + fine + T.HALF_STEP[dtype] * 1.01 * np.abs(want) + 1e-30
    off = np.abs(P.np64(out) - want)
    assert (off <= tol).all(), float((off / tol).max())
    norm = (top + np.log(z))[..., 0]
    assert (np.abs(P.np64(lse) - norm) <= delta[..., 0] + (rows + 64) * 2.0 ** -22 + 2.0 ** -21 * np.abs(norm) + 1e-6).all()


BOTH = [pytest.mark.parametrize("bits", [4, 8]), pytest.mark.parametrize("dtype", ["bf16", "f32"])]


def both(f):
    for m in BOTH:
        f = m(f)
    return f


@both
@pytest.mark.parametrize("order,d,hq", [("rising", 64, 1), ("falling", 64, 1), ("mixed", 64, 1), ("mixed", 64, 16), ("rising", 128, 3), ("mixed", 128, 9),
                                        ("rising", 256, 2), ("mixed", 256, 11)])
def test_logits_far_beyond_the_mantissa(B, dtype, bits, order, d, hq):
    """Logits of 10^6 to 10^30, a dozen in every binade up to 10^11: the row that sets the reference has a weight of 1, whatever the rounding of its logit.
    What rows read back as differs by 2^-9 or more of the largest, so one row decides (or several alike): the output is their values' mean.  Its weight
    is exact (a step is a bf16), the sums are off by 2^-22 of their size for each row and for 64 products beside it, and the result is
    rounded once."""
    rows = 40
    tops = np.concatenate([8e6 * 2.0 ** (np.arange(200) / 12), 8e12 * 10.0 ** np.arange(18)])
    n = len(tops)
    rng = np.random.default_rng(bits)
    ranks = {"rising": np.arange(rows), "falling": np.arange(rows)[::-1], "mixed": rng.permutation(rows)}[order]
    k = np.zeros((n, rows, d))
    k[:, :, 0] = tops[:, None] * (ranks + 1) / rows
    v = rng.normal(0.3, 1, (n, rows, d))
    q = torch.zeros((n, hq, d), dtype=T.DT[dtype], device="cuda")
    q[:, :, 0] = 1.0
    out, lse = attend(B, q, k, v, dtype, bits, 30)
    s = parts(k, bits)[0][:, :, 0] / math.sqrt(d)
    at = s == s.max(1, keepdims=True)
    assert (np.where(at, -np.inf, s).max(1) <= s.max(1) * (1 - 2.0 ** -9)).all()
    p = at / at.sum(1, keepdims=True)
    vr, vc, vl = parts(v, bits)
    want, size = np.einsum("nr,nrd->nd", p, vr), np.einsum("nr,nrd->nd", p, vc + vl)
    tol = size * (rows + 64) * 2.0 ** -22 + T.HALF_STEP[dtype] * 1.01 * np.abs(want)
    off = np.abs(P.np64(out) - want[:, None])
    assert (off <= tol[:, None]).all(), float((off / tol[:, None]).max())
    norm = s.max(1) + np.log(at.sum(1))
    assert (np.abs(P.np64(lse) - norm[:, None]) <= 2.0 ** -21 * norm[:, None]).all()


@both
@pytest.mark.parametrize("d", [64, 128, 256])
def test_huge_values_of_rows_that_count_for_nothing(B, dtype, bits, d):
    """A row with a step of 2^26 to 2^60 times the others' whose logit is 100 below theirs (a weight of 2^-144: nothing), at the front, in the middle, at the
    end; in all groups of 64 dimensions and in one of them.  A third head has that row and nothing else."""
    rows, hq, n = 120, 3, 0
    rng = np.random.default_rng(d + bits)
    ks, vs = [], []
    q = rng.normal(0, 1, (hq, d))
    q[:2, 0], q[2, 0] = 8.0, -8.0
    for where in (0, 15, 33, 63, 64, 119):
        for far in (26, 31, 40, 60):
            for group in (None, 0):
                k, v = rng.normal(0, 0.05, (rows, d)), rng.normal(0.2, 1, (rows, d))
                k[:, 0] = 3.0
                k[where, 0] = 3.0 - 110 * math.sqrt(d) / 8
                v[where, slice(None) if group is None else slice(0, 64)] *= 2.0 ** far
                ks.append(k), vs.append(v)
                n += 1
    k, v = np.stack(ks), np.stack(vs)
    qd = torch.as_tensor(np.broadcast_to(q, (n, hq, d)).copy()).to(T.DT[dtype]).cuda()
    out, lse = attend(B, qd, k, v, dtype, bits, 50)
    s = np.einsum("hd,nrd->nhr", P.np64(qd)[0], parts(k, bits)[0]) / math.sqrt(d)
    assert all((s[i, :2, w] < s[i, :2].max(-1) - 95).all() and s[i, 2].argmax() == w for i, w in enumerate(np.repeat((0, 15, 33, 63, 64, 119), 8)))
    check(out, lse, P.np64(qd), k, v, bits, dtype)


@both
def test_groups_of_very_different_sizes(B, dtype, bits):
    """Values whose second 64 dimensions are 2^-30 of the first ones: each group is as exact as if it were alone."""
    rows, hq, d, n = 50, 3, 128, 4
    rng = np.random.default_rng(bits)
    k, v = rng.normal(0, 0.3, (n, rows, d)), rng.normal(0.2, 1, (n, rows, d))
    v[:2, :, 64:] *= 2.0 ** -30
    v[2:, :, :64] *= 2.0 ** -30
    q = T.normal((n, hq, d), T.DT[dtype], 3)
    out, lse = attend(B, q, k, v, dtype, bits, 50)
    check(out, lse, P.np64(q), k, v, bits, dtype)


@both
@pytest.mark.parametrize("d", [64, 256])
def test_keys_up_to_the_largest_that_are_held(B, dtype, bits, d):
    """Keys of 2^100 to just below 2^126 with queries as small: logits of some 16."""
    sizes = [100, 105, 107, 112, 120, 125.9]
    rows, hq, n = 40, 2, len(sizes)
    rng = np.random.default_rng(d)
    k, v = rng.uniform(-1, 1, (n, rows, d)), rng.normal(0.2, 1, (n, rows, d))
    k[n - 1] = np.abs(k[n - 1])                                    # all of one sign: the largest sums
    big = 2.0 ** np.array(sizes)[:, None, None]
    q = torch.as_tensor(rng.uniform(0.5, 1, (n, hq, d)) * 4 / big).to(T.DT[dtype]).cuda()
    out, lse = attend(B, q, k * big, v, dtype, bits)
    check(out, lse, P.np64(q), k * big, v, bits, dtype)


@both
def test_values_near_the_end_of_fp32(B, dtype, bits):
    """256 rows of 2^117: their sum is within fp32 as long as no weight is above 1, however the rows come (here later logits are above the first ones, by
    less than what would move a reference that may stay behind)."""
    rows, d, n = 256, 64, 3
    rng = np.random.default_rng(1)
    k, v = np.zeros((n, rows, d)), (2 + rng.random((n, rows, d))) * 2.0 ** 116
    k[0, 40:, 0], k[1, 40:, 0], k[2, 40:, 0] = 5.0, 5.5, 7.0
    v[2] *= -1
    q = torch.zeros((n, 1, d), dtype=T.DT[dtype], device="cuda")
    q[:, 0, 0] = 8.0
    out, lse = attend(B, q, k, v, dtype, bits, 1000)
    assert torch.isfinite(out).all()
    check(out, lse, P.np64(q), k, v, bits, dtype)


@both
def test_a_row_that_counts_less_and_less(B, dtype, bits):
    """A row of 2^40 times the others' values that counts when it is met and is left behind by logits that rise: in the end its part of the sum is far above, about,
    or far below the others'.  What came before, between and after is as exact as the largest part lets it be seen."""
    rows, hq, d = 120, 2, 64
    rng = np.random.default_rng(bits)
    ks, vs = [], []
    for where in (0, 20, 50):
        for far in (5, 20, 35, 38, 40, 42, 45, 60, 100, 140):
            k, v = rng.normal(0, 0.01, (rows, d)), rng.normal(0.2, 1, (rows, d))
            k[:, 0] = np.maximum(0, np.arange(rows) - where) / (rows - 1 - where) * far * math.log(2)
            v[where] *= 2.0 ** 40
            ks.append(k), vs.append(v)
    k, v = np.stack(ks), np.stack(vs)
    q = np.zeros((len(k), hq, d))
    q[:, 0, 0], q[:, 1, 0], q[:, :, 1:] = 8.0, 4.0, rng.normal(0, 0.1, (len(k), hq, d - 1))
    q = torch.as_tensor(q).to(T.DT[dtype]).cuda()
    out, lse = attend(B, q, k, v, dtype, bits, 50)
    check(out, lse, P.np64(q), k, v, bits, dtype)
