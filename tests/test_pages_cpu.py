"""Paged caches without a GPU: refused geometries and handles answer before any CUDA call, and the oracle of the paged
operators against brute force and closed forms."""
import ctypes
import math

import numpy as np
import pytest

from oracle import meda_oracle as M
from oracle import pages_oracle as O


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


GOOD = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", page_size=16, n_pages=10, max_seqs=4, max_seq_pages=8)


@pytest.mark.parametrize("status,kw", [
    (-2, dict(n_q_heads=3)), (-2, dict(n_q_heads=34)), (-2, dict(head_dim=96)), (-2, dict(page_size=8)), (-2, dict(page_size=48)),
    (-2, dict(page_size=512)), (-2, dict(n_pages=0)), (-2, dict(max_seqs=0)), (-2, dict(max_seqs=16385)), (-2, dict(max_seq_pages=0)),
    (-2, dict(max_seq_pages=262145)), (-2, dict(max_seqs=16384, max_seq_pages=262144)), (-1, dict(rope_theta=1.0)),
    (-1, dict(rope_theta=math.nan)), (-1, dict(rope_theta=math.inf)), (-2, dict(rope_sections=(40, 0, 0))), (-2, dict(rope_sections=(12, 0, 0))),
    (-2, dict(rope_sections=(0, 0, 0))), (-2, dict(rope_sections=(40, -8, 0))), (-2, dict(rope_sections=(0, 16, 16), rope_order=1)),
    (-1, dict(rope_order=2)), (-1, dict(rope_pairing=-1))])
def test_create_refuses(B, status, kw):
    with pytest.raises(B.MedaError) as e:
        B.Pages(**{**GOOD, **kw})
    assert e.value.status == status


def test_null_handles(B):
    lib = B.load_library()
    one = 256                                                      # never dereferenced
    assert lib.meda_pages_create(None, ctypes.byref(ctypes.c_void_p())) == -1
    assert lib.meda_pages_poll_status(None, None) == -1
    assert lib.meda_pages_workspace_bytes(None) == 0 and lib.meda_pages_launch_count(None) == 0
    lib.meda_pages_destroy(None)
    assert lib.meda_page_tables(None, one, 1, one, 1, 1, one, one, one, one, one, one, 1, None) == -1
    assert lib.meda_page_store(None, one, one, 0, 0, 1, one, 1, 1, one, one, one, one, None) == -1
    assert lib.meda_page_bounds(None, one, one, one, one, 1, 1, one, None) == -1
    assert lib.meda_rope_append(None, one, 0, one, 0, one, 0, one, 0, one, 1, one, one, one, None) == -1
    assert lib.meda_select_pages(None, one, one, one, one, 1, 1, 0, 0, 1, one, None) == -1
    assert lib.meda_paged_attention(None, one, one, one, one, one, 1, 1, None, 0, one, None, None) == -1


def test_binding_refuses_unknown_types(B):
    with pytest.raises(ValueError):
        B.Pages(**{**GOOD, "dtype": "f16"})
    with pytest.raises(ValueError):
        B.Pages(**{**GOOD, "rope_sections": (16, 16)})


def test_oracle_tables_conserve_pages():
    rng = np.random.default_rng(0)
    n, page, width, n_pages = 5, 4, 6, 25
    table, free, top, lens = np.full((n, width), -1), np.arange(n_pages), 0, np.zeros(n, int)
    failed = 0
    for _ in range(300):
        new = rng.integers(0, width * page + 1, n)
        table, free, top, cu, slots, ok = O.page_tables(lens, new, free, top, table, page, 200)
        failed += not ok
        if ok:
            assert cu[-1] == np.maximum(new - lens, 0).sum() and (slots[:cu[-1]] >= 0).all() and (slots[cu[-1]:] == -1).all()
            assert len(set(slots[:cu[-1]].tolist())) == cu[-1]
            lens = new
        held = [table[i, p] for i in range(n) for p in range(O.n_pages_of(lens[i], page))]
        assert sorted(held + free[top:].tolist()) == list(range(n_pages))
    assert 0 < failed < 300


def test_oracle_rope_preserves_norms_and_relative_positions():
    rng = np.random.default_rng(1)
    for order, sections in ((0, (8, 4, 4)), (1, (6, 5, 5))):
        for pairing in (0, 1):
            x = rng.normal(size=(3, 2, 40))
            pos = rng.integers(0, 5000, (3, 3))
            y = O.rope(x, pos, sections, order, pairing, 1e4)
            np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
            np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
            # the same shift on every axis leaves products as they are
            a, b = rng.normal(size=(1, 1, 40)), rng.normal(size=(1, 1, 40))
            at = lambda v, p: O.rope(v, np.array(p)[:, None], sections, order, pairing, 1e4)[0, 0]
            np.testing.assert_allclose(at(a, [5, 9, 2]) @ at(b, [1, 4, 7]), at(a, [105, 109, 102]) @ at(b, [101, 104, 107]))
            # the negative angle is the inverse (and the gradient)
            np.testing.assert_allclose(O.rope(y, -pos, sections, order, pairing, 1e4), x, atol=1e-12)


def test_oracle_score_bounds_every_logit_and_selection_matches_brute_force():
    rng = np.random.default_rng(2)
    k = rng.normal(size=(12, 8, 16))                               # 12 pages of 8 rows
    b = np.stack([O.page_bounds(p) for p in k])
    q = rng.normal(size=(3, 16))
    s = O.page_scores(q, b)
    logits = np.einsum("hd,prd->hpr", q, k)
    assert (s >= logits.max((0, 2)) - 1e-6).all()
    for keep, first, last in ((1, 0, 0), (4, 1, 1), (12, 0, 0), (20, 2, 2), (5, 2, 3)):
        got = O.select_pages(s, keep, first, last)
        forced = [c for c in range(12) if c < first or c >= 12 - last]
        rest = sorted((c for c in range(12) if c not in forced), key=lambda c: (-s[c], c))
        assert got.tolist() == sorted((forced + rest)[:min(keep, 12)])
    tie = np.array([1, 2, 2, np.nan, 2, 0], np.float32)
    assert O.select_pages(tie, 3, 0, 0).tolist() == [1, 2, 3]


def test_oracle_attention_matches_the_dense_decoding_step():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(6, 32)), rng.normal(size=(2, 50, 32)), rng.normal(size=(2, 50, 32))
    want = M.decode_attention(q, k, v)
    for g in range(2):
        out, lse, _ = O.attention(q[3 * g:3 * g + 3], k[g], v[g])
        np.testing.assert_allclose(out, want[3 * g:3 * g + 3])
        np.testing.assert_allclose(lse, np.log(np.exp(q[3 * g:3 * g + 3] @ k[g].T / np.sqrt(32)).sum(-1)))
        # two halves joined by their log-sums
        a, la, _ = O.attention(q[3 * g:3 * g + 3], k[g, :20], v[g, :20])
        b, lb, _ = O.attention(q[3 * g:3 * g + 3], k[g, 20:], v[g, 20:])
        w = np.exp(la - np.logaddexp(la, lb))[:, None]
        np.testing.assert_allclose(w * a + (1 - w) * b, out)
