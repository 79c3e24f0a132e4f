"""Decoding over quantised caches as a run of calls: PagedDecoder with cache_bits, captured steps, handles side by side, and what
quantising costs against the caches as they were."""
import math

import numpy as np
import pytest
import torch

import paged_steps as S
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


class Steps(S.Steps):
    """Rows beside the decoder as it should hold them: what their codes stand for, rounded to the type."""

    def held(self, x):
        bits = self.dec.pages.cache_bits
        return Q.rounded(O.held(*O.quantise(np.asarray(x, np.float32), bits)), self.wl.dtype)

    def admit(self, r, cp):
        super().admit(r, cp)
        for l in range(self.wl.n_layers):
            self.rows[r, l] = tuple(self.held(x) for x in self.rows[r, l])

    def step(self, grown, run=None):
        old = {key: value for key, value in self.rows.items()}
        super().step(grown, run)
        hq, hkv = self.wl.n_q_heads, self.wl.n_kv_heads
        p64 = self.pos.cpu().numpy().astype(np.int64)
        for l in range(self.wl.n_layers):
            x = self.qkv[l]
            k = O.rope_fp32(P.np64(x[:, hq:hq + hkv]), p64, S.SECTIONS, 0, 0, S.THETA)
            k = torch.as_tensor(k).to(self.wl.torch_dtype).double().numpy()
            for r in grown:
                a, b = old[r, l]
                self.rows[r, l] = (np.concatenate([a, self.held(k[r])[:, None]], 1), np.concatenate([b, self.held(P.np64(x[r, hq + hkv:]))[:, None]], 1))

    def check_caches(self, requests):
        """The rows of every layer through read(), exactly."""
        wl = self.wl
        for r in requests:
            rows = max(self.rows[r, l][0].shape[1] for l in range(wl.n_layers))
            k, v = (torch.full((wl.n_layers, wl.n_kv_heads, rows + 1, wl.head_dim), 5.0, dtype=wl.torch_dtype, device="cuda") for _ in range(2))
            count = self.dec.read(r, k, v).tolist()
            for l in range(wl.n_layers):
                n = self.rows[r, l][0].shape[1]
                assert count[l] == n == int(self.dec.lens[l * self.dec.max_requests + r])
                np.testing.assert_array_equal(P.np64(k[l, :, :n]), self.rows[r, l][0])
                np.testing.assert_array_equal(P.np64(v[l, :, :n]), self.rows[r, l][1])
                assert (k[l, :, n:] == 5).all() and (v[l, :, n:] == 5).all()

    def check_outputs(self, requests):
        dec = self.dec
        for l in range(self.wl.n_layers):
            at = [l * dec.max_requests + r for r in requests]
            sel = self.sel[l, requests].cpu().numpy() if self.sel is not None else None
            Q.check_attention(self.out[l, requests], self.lse[l, requests], self.q_rot[l, requests], dec.k_pages, dec.v_pages, dec.table[at].cpu().numpy(),
                              [self.rows[r, l][0].shape[1] for r in requests], dec.pages.cfg.page_size, dec.pages.cache_bits, self.wl.dtype, sel, dec.keep_pages)

    def check_choice(self, requests):
        page, group = self.dec.pages.cfg.page_size, self.wl.n_q_heads // self.wl.n_kv_heads
        for l in range(self.wl.n_layers):
            for r in requests:
                _, rows, pages = self.pages(r, l)
                bounds, q, sel = P.np64(self.dec.bounds[pages]), P.np64(self.q_rot[l, r]), self.sel[l, r].cpu().numpy()
                for c in range(len(pages)):
                    lo, hi = O.page_bounds(self.rows[r, l][0][:, c * page:min(rows, c * page + page)].transpose(1, 0, 2))
                    np.testing.assert_array_equal(bounds[c, :, 0], lo)
                    np.testing.assert_array_equal(bounds[c, :, 1], hi)
                for g in range(self.wl.n_kv_heads):
                    want = O.select_pages(O.page_scores(q[g * group:(g + 1) * group], bounds[:, g]), self.dec.keep_pages, self.dec.n_first, self.dec.n_last)
                    np.testing.assert_array_equal(sel[g, :len(want)], want)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("keep_pages", [0, 6])
@pytest.mark.parametrize("graph", [False, True])
def test_decoding_over_quantised_caches(B, bits, keep_pages, graph):
    """Two prompts through the compression pass, into quantised pages, then steps in which requests come and go; with `graph` the
    steps are replays of one captured step."""
    wl = S.workload()
    cps = [S.compressed(wl.with_(seed=s)) for s in (4, 9)]
    dec = S.decoder(wl, 120, 3, 400, keep_pages=keep_pages, cache_bits=bits)
    st = Steps(wl, dec)
    st.admit(0, cps[0])
    st.admit(2, cps[1])
    dec.check()
    run = None
    if graph:
        st.body()                                                  # (a step of nothing: its rows are given back below)
        dec.release(0), dec.release(2)
        st.admit(0, cps[0])
        st.admit(2, cps[1])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.body()
        run = g.replay
    for n in range(4):
        st.step([0, 2], run)
        dec.check()
        st.check_caches([0, 2])
        st.check_outputs([0, 2])
        if keep_pages:
            st.check_choice([0, 2])
    st.release(0)
    st.admit(1, cps[0])
    for n in range(18):                                            # over a page's border
        st.step([1, 2], run)
    dec.check()
    st.check_caches([1, 2])
    st.check_outputs([1, 2])
    dec.close()
    for cp in cps:
        cp.close()


@pytest.mark.parametrize("bits", [0, 4, 8])
def test_read_gives_rows_from_anywhere_and_refuses(B, bits):
    wl = S.workload()
    cp = S.compressed(wl)
    dec = S.decoder(wl, 60, 2, 400, cache_bits=bits)
    dec.admit(1, cp)
    dec.check()
    L, hkv, d, b = wl.n_layers, wl.n_kv_heads, wl.head_dim, cp.budgets[:, 0].tolist()
    whole = torch.zeros((2, L, hkv, max(b), d), dtype=wl.torch_dtype, device="cuda")
    assert dec.read(1, whole[0], whole[1]).tolist() == b
    if not bits:
        for l in range(L):
            assert torch.equal(whole[0, l, :, :b[l]], cp.k_out[l, :, :b[l]]) and torch.equal(whole[1, l, :, :b[l]], cp.v_out[l, :, :b[l]])
    first = T.i32([max(0, x - 5 - l) for l, x in enumerate(b)])
    tail = torch.full((2, L, hkv, 5 + L, d), 5.0, dtype=wl.torch_dtype, device="cuda")
    count = dec.read(1, tail[0], tail[1], first).tolist()
    dec.check()
    for l in range(L):
        assert count[l] == min(b[l], 5 + l)
        assert torch.equal(tail[:, l, :, :count[l]], whole[:, l, :, b[l] - count[l]:b[l]]) and (tail[:, l, :, count[l]:] == 5).all()
    assert dec.read(0, tail[0], tail[1]).tolist() == [0] * L       # nothing admitted there
    dec.check()
    for call in (lambda: dec.read(1, tail[0, :1], tail[1, :1]), lambda: dec.read(1, tail[0, 0], tail[1, 0]), lambda: dec.read(1, tail[0].double(), tail[1])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(IndexError):
        dec.read(2, tail[0], tail[1])
    dec.read(1, tail[0, :, :, :2], tail[1, :, :, :2])              # more rows than fit
    with pytest.raises(B.MedaError) as e:
        dec.check()
    assert e.value.status == B.MEDA_ERR_WORKSPACE
    dec.close()
    cp.close()


def test_read_of_the_only_request(B):
    """The numbers of rows are the caller's own: a release later on does not change them.  Where reading begins may be a column."""
    wl = S.workload()
    cp = S.compressed(wl)
    dec = S.decoder(wl, 60, 1, 400, cache_bits=4)
    dec.admit(0, cp)
    b = cp.budgets[:, 0].tolist()
    whole = torch.zeros((2, wl.n_layers, wl.n_kv_heads, max(b), wl.head_dim), dtype=wl.torch_dtype, device="cuda")
    count = dec.read(0, whole[0], whole[1])
    tail = torch.full_like(whole, 5.0)
    first = T.i32([[x - 3, 0] for x in b])[:, 0]
    assert dec.read(0, tail[0], tail[1], first).tolist() == [3] * wl.n_layers
    dec.check()
    for l in range(wl.n_layers):
        assert torch.equal(tail[:, l, :, :3], whole[:, l, :, b[l] - 3:b[l]]) and (tail[:, l, :, 3:] == 5).all()
    dec.release(0)
    assert count.tolist() == b
    dec.close()
    cp.close()


@pytest.mark.parametrize("bits", [4, 8])
def test_two_handles_on_two_streams_and_two_graphs(B, bits):
    lens = [3000, 17, 900]
    pg, q, kp, vp, table, out, lse = Q.attention_case(B, lens, 28, 4, 128, "bf16", 16, bits, seed=4)
    other = T.make(B, n_q_heads=28, n_kv_heads=4, head_dim=128, page_size=16, n_pages=kp.shape[0], max_seqs=3, max_seq_pages=table.shape[1], cache_bits=bits)
    t, n = T.i32(table.tolist()), T.i32(lens)
    q2 = T.normal(q.shape, q.dtype, 77)
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
bits = {bits}
pg = B.Pages(n_q_heads=14, n_kv_heads=2, head_dim=128, dtype="{dtype}", page_size=16, n_pages=64, max_seqs=3, max_seq_pages=20, cache_bits=bits)
dt = dict(bf16=torch.bfloat16, f32=torch.float32)["{dtype}"]
torch.manual_seed(1)
rand = lambda *s: torch.randn(s, device="cuda").to(dt)
i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
q, k, v, kn, vn = rand(3, 14, 128), rand(3, 2, 320, 128), rand(3, 2, 320, 128), rand(3, 2, 128), rand(3, 2, 128)
lens, more, zero = i32(300, 17, 0), i32(301, 18, 1), i32(0)
pos = i32(5, 6, 7).repeat(3, 1)

def buffers():
    z = lambda *s: torch.zeros(s, dtype=dt, device="cuda")
    b = lambda: torch.zeros((64, 2, pg.page_bytes()), dtype=torch.uint8, device="cuda")
    return dict(kp=b(), vp=b(), bd=z(64, 2, 2, 128), table=torch.full((3, 20), -1, dtype=torch.int32, device="cuda"),
                free=torch.arange(64, dtype=torch.int32, device="cuda"), top=i32(0), top2=i32(0), cu=i32(0, 0, 0, 0),
                slots=torch.zeros(3, dtype=torch.int64, device="cuda"), nothing=torch.empty(0, dtype=torch.int64, device="cuda"),
                qr=z(3, 14, 128), sel=torch.zeros((3, 2, 4), dtype=torch.int32, device="cuda"), out=z(3, 14, 128), lse=torch.zeros((3, 14), device="cuda"),
                kb=z(3, 2, 320, 128), vb=z(3, 2, 320, 128))

def body(b):
    pg.page_tables(None, lens, b["free"], zero, b["top"], b["table"], b["cu"], b["nothing"])
    pg.page_store(k, v, lens, b["table"], b["kp"], b["vp"], b["bd"])
    pg.page_tables(lens, more, b["free"], b["top"], b["top2"], b["table"], b["cu"], b["slots"])
    pg.rope_append(q, kn, vn, pos, b["slots"], b["qr"], b["kp"], b["vp"])
    pg.page_bounds(b["kp"], b["table"], lens, more, b["bd"])
    pg.select_pages(b["qr"], b["bd"], b["table"], more, 1, 1, b["sel"])
    pg.paged_attention(b["qr"], b["kp"], b["vp"], b["table"], more, b["out"], b["lse"], sel=b["sel"])
    pg.page_load(b["kp"], b["vp"], b["table"], more, b["kb"], b["vb"])

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
assert captured["top2"].item() == 19 + 2 + 1 and captured["out"].float().abs().sum() > 0 and captured["kb"].float().abs().sum() > 0
print("captured first")
"""


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
def test_first_calls_of_a_process_inside_a_capture(B, dtype, bits):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = FIRST_CAPTURE.replace("{dtype}", dtype).replace("{bits}", str(bits))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stderr[-2000:]


def test_quantised_attention_stays_near_the_caches_own(B):
    """The same rows in bf16, 8 and 4 bits.  With x the caches' elements, a key is off by half a step in every dimension, which moves a logit
    by at most delta = |q|_1 step / 2 / sqrt(d), a probability and its normaliser by exp(delta) each, and a value is off by half a step:
    |out - out_bf16| <= (exp(2 delta) - 1) max |v| + step_v / 2, and the roundings."""
    hq, hkv, d, page, m = 28, 4, 128, 16, 2000
    n_pages = m // page
    k, v = T.normal((1, hkv, m, d), torch.bfloat16, 1, 0.0, 0.2), T.normal((1, hkv, m, d), torch.bfloat16, 2, 0.3)
    q, t, n = T.normal((1, hq, d), torch.bfloat16, 3), T.i32([list(range(n_pages))]), T.i32([m])
    outs = {}
    for bits in (0, 8, 4):
        pg = T.make(B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, n_pages=n_pages, max_seqs=1, max_seq_pages=n_pages, cache_bits=bits)
        shape = (n_pages, hkv, pg.page_bytes()) if bits else (n_pages, hkv, page, d)
        kp, vp = (torch.zeros(shape, dtype=torch.uint8 if bits else torch.bfloat16, device="cuda") for _ in range(2))
        outs[bits] = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda")
        pg.page_store(k, v, n, t, kp, vp)
        pg.paged_attention(q, kp, vp, t, n, outs[bits])
        pg.check()
        pg.close()
    for bits in (8, 4):
        step_k, step_v = (float(O.quantise(P.np64(x).astype(np.float32), bits)[1].max()) for x in (k, v))
        delta = P.np64(q).__abs__().sum(-1)[0] * step_k / 2 / math.sqrt(d)
        bound = (np.exp(2 * delta) - 1)[:, None] * float(v.abs().max()) + step_v / 2 + 2 ** -6 * np.abs(P.np64(outs[0][0])) + 1e-4
        off = np.abs(P.np64(outs[bits][0]) - P.np64(outs[0][0]))
        assert (off <= bound).all()
        assert off.max() > 0
