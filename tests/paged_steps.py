"""Decoding steps of pipeline.PagedDecoder beside a plain copy of what its caches should hold."""
import numpy as np
import torch

import parity as P
import test_gpu_pages as T
from oracle import pages_oracle as O
from paper_2502_17599_b200 import workloads as W

SECTIONS, THETA = (24, 20, 20), 1e6


def workload(**kw):
    return W.small_variant("paged", **{**dict(window=32, seed=4), **kw})


def compressed(wl, **kw):
    from paper_2502_17599_b200.pipeline import CompressionPass
    cp = CompressionPass(wl, n_streams=2, **kw)
    layers = [W.make_layer(wl, l, "cuda") for l in range(wl.n_layers)]
    cp.run(*[list(x) for x in zip(*layers)])
    return cp


def decoder(wl, n_pages, max_requests, max_rows, **kw):
    from paper_2502_17599_b200.pipeline import PagedDecoder
    return PagedDecoder(wl, n_pages=n_pages, max_requests=max_requests, max_rows=max_rows, rope_sections=SECTIONS, rope_theta=THETA, **kw)


class Steps:
    """The decoder, the buffers of a step and, per (request, layer), the rows its cache should hold (keys as they were rotated, in
    64 bits).  What a layer's call left behind for its own use (rotated queries, chosen pages) is copied, so that a captured step can be looked
    at afterwards."""

    def __init__(self, wl, dec):
        L, R, hq, hkv, d = wl.n_layers, dec.max_requests, wl.n_q_heads, wl.n_kv_heads, wl.head_dim
        self.wl, self.dec, self.rows, self.n = wl, dec, {}, 0
        dt = dict(dtype=wl.torch_dtype, device="cuda")
        self.out, self.q_rot = torch.zeros((L, R, hq, d), **dt), torch.zeros((L, R, hq, d), **dt)
        self.lse = torch.zeros((L, R, hq), device="cuda")
        self.qkv = torch.zeros((L, R, hq + 2 * hkv, d), **dt)
        self.pos = torch.zeros((3, R), dtype=torch.int32, device="cuda")
        self.sel = torch.zeros((L,) + tuple(dec.sel.shape), dtype=torch.int32, device="cuda") if dec.keep_pages else None

    def admit(self, r, cp):
        self.dec.admit(r, cp)
        b = cp.budgets.cpu().numpy()
        for l in range(self.wl.n_layers):
            s = int(b[l, 0])
            self.rows[r, l] = (P.np64(cp.k_out[l, :, :s]), P.np64(cp.v_out[l, :, :s]))

    def release(self, r):
        self.dec.release(r)
        for l in range(self.wl.n_layers):
            del self.rows[r, l]

    def body(self):
        hq, hkv = self.wl.n_q_heads, self.wl.n_kv_heads
        self.dec.begin_step()
        for l in range(self.wl.n_layers):
            x = self.qkv[l]
            self.dec.attend(l, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], self.pos, self.out[l], self.lse[l])
            self.q_rot[l].copy_(self.dec.q_rot)
            if self.sel is not None:
                self.sel[l].copy_(self.dec.sel)

    def step(self, grown, run=None):
        """One step (`run` replays a captured body) in which the requests `grown` are expected to get a row."""
        hq, hkv, R = self.wl.n_q_heads, self.wl.n_kv_heads, self.dec.max_requests
        for l in range(self.wl.n_layers):
            self.qkv[l] = T.normal(tuple(self.qkv[l].shape), self.wl.torch_dtype, 1000 * self.n + l)
        self.pos.copy_(T.i32([[700 + self.n + r, 5 + r, 6 + self.n] for r in range(R)]).T)
        (run or self.body)()
        p64 = self.pos.cpu().numpy().astype(np.int64)
        for l in range(self.wl.n_layers):
            turned = O.rope(P.np64(self.qkv[l, :, hq:hq + hkv]), p64, SECTIONS, 0, 0, THETA)
            for r in grown:
                k, v = self.rows[r, l]
                self.rows[r, l] = (np.concatenate([k, turned[r][:, None]], 1), np.concatenate([v, P.np64(self.qkv[l, r, hq + hkv:])[:, None]], 1))
        self.n += 1

    def pages(self, r, l):
        """(sequence, rows, its pages as an index)."""
        seq, rows = l * self.dec.max_requests + r, self.rows[r, l][0].shape[1]
        return seq, rows, self.dec.table[seq, :O.n_pages_of(rows, self.dec.pages.cfg.page_size)].long()

    def check_caches(self, requests):
        """Lengths, and the pools' rows: values exactly, keys to half a step of the rotated ones."""
        assert self.dec.lens.view(self.wl.n_layers, -1).cpu()[:, [r for r in range(self.dec.max_requests) if (r, 0) not in self.rows]].eq(0).all()
        for r in requests:
            for l in range(self.wl.n_layers):
                seq, rows, pages = self.pages(r, l)
                assert int(self.dec.lens[seq]) == rows
                k, v = (P.np64(x[pages].transpose(0, 1).reshape(self.wl.n_kv_heads, -1, self.wl.head_dim)[:, :rows]) for x in (self.dec.k_pages, self.dec.v_pages))
                np.testing.assert_array_equal(v, self.rows[r, l][1])
                want = self.rows[r, l][0]
                # the rotation's own error (see test_gpu_pages): 2^-20 of |a| + |b|, each below the largest element
                assert (np.abs(k - want) <= 2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -19 * np.abs(want).max()).all()

    def check_outputs(self, requests):
        """Attention over what the pools hold, with the rotated queries as they were used."""
        page = self.dec.pages.cfg.page_size
        for l in range(self.wl.n_layers):
            at = [l * self.dec.max_requests + r for r in requests]
            lens = [self.rows[r, l][0].shape[1] for r in requests]
            table = self.dec.table[at].cpu().numpy()
            sel = self.sel[l, requests].cpu().numpy() if self.sel is not None else None
            T.check_attention(self.out[l, requests], self.lse[l, requests], self.q_rot[l, requests], self.dec.k_pages, self.dec.v_pages, table, lens, page,
                              self.wl.dtype, sel, self.dec.keep_pages)

    def check_choice(self, requests):
        """Key bounds of every page in use from the pool's own rows, and the pages chosen by them.  Returns how many choices left a page out."""
        page, left_out = self.dec.pages.cfg.page_size, 0
        group = self.wl.n_q_heads // self.wl.n_kv_heads
        for l in range(self.wl.n_layers):
            for r in requests:
                _, rows, pages = self.pages(r, l)
                k, bounds = P.np64(self.dec.k_pages[pages]), P.np64(self.dec.bounds[pages])
                for c in range(len(pages)):
                    lo, hi = O.page_bounds(k[c, :, :min(page, rows - c * page)].transpose(1, 0, 2))
                    np.testing.assert_array_equal(bounds[c, :, 0], lo)
                    np.testing.assert_array_equal(bounds[c, :, 1], hi)
                q, sel = P.np64(self.q_rot[l, r]), self.sel[l, r].cpu().numpy()
                for g in range(self.wl.n_kv_heads):
                    want = O.select_pages(O.page_scores(q[g * group:(g + 1) * group], bounds[:, g]), self.dec.keep_pages, self.dec.n_first, self.dec.n_last)
                    np.testing.assert_array_equal(sel[g, :len(want)], want)
                    left_out += len(want) < len(pages)
        return left_out
