"""Calls on quantised pages that the documentation allows, or has to refuse, beside those of test_gpu_quantised.py."""
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
