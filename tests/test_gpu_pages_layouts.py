"""Layouts whose strides differ only where an axis has one element."""
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


@pytest.mark.parametrize("n,hkv,cap", [(1, 2, 40), (1, 1, 40), (2, 1, 40), (1, 2, 1), (3, 1, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_and_values_of_one_sequence_head_or_row(B, n, hkv, cap, dtype):
    pg = T.make(B, n_q_heads=2, n_kv_heads=hkv, dtype=dtype, n_pages=16, max_seqs=n, max_seq_pages=3)
    k = T.normal((n, hkv, cap, 64), T.DT[dtype], 1)
    v = T.normal((n, hkv, cap, 64), T.DT[dtype], 2)
    odd = [s if size > 1 else 3 for s, size in zip(v.stride(), v.shape)]        # strides that no step is ever taken along
    v2 = v.as_strided(v.shape, odd)
    assert torch.equal(v, v2) and v2.stride() != k.stride()
    lens, table = T.i32([cap] * n), T.i32([[5 * i, 5 * i + 1, 5 * i + 2] for i in range(n)])
    pools = [torch.zeros((16, hkv, 16, 64), dtype=k.dtype, device="cuda") for _ in range(4)]
    pg.page_store(k, v, lens, table, *pools[:2])
    pg.page_store(k, v2, lens, table, *pools[2:])
    pg.check()
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
    for i in range(n):
        assert torch.equal(pools[3][5 * i:5 * i + 3].transpose(0, 1).reshape(hkv, 48, 64)[:, :cap], v[i])
    for t in (v[:, :, :, :63], v[0], v[:, :, :0], v.transpose(2, 3)):
        with pytest.raises(ValueError):
            pg.page_store(k, t, lens, table, *pools[:2])
    if n > 1:
        with pytest.raises(ValueError):                            # there the strides count
            pg.page_store(k, torch.stack([v, v], 1)[:, 0], lens, table, *pools[:2])
    pg.close()


def test_bounds_of_one_sequence_with_lengths_of_different_strides(B):
    pg = T.make(B, max_seqs=2, max_seq_pages=3)
    k = T.normal((64, 2, 16, 64), torch.bfloat16, 1)
    table, bounds = T.i32([[5, 6, 7]]), [torch.zeros((64, 2, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens = T.i32([[40, 0, 0]])[:, 0].as_strided((1,), (3,))
    pg.page_bounds(k, table, T.i32([17]), T.i32([40]), bounds[0])
    pg.page_bounds(k, table, T.i32([17]), lens, bounds[1])
    pg.check()
    assert torch.equal(bounds[0], bounds[1]) and torch.equal(bounds[0][6, :, 0], k[6].amin(1)) and (bounds[0][5] == 0).all()
    with pytest.raises(ValueError):                                # there the strides count
        pg.page_bounds(k, T.i32([[5, 6, 7], [8, 9, 10]]), T.i32([1, 2]), T.i32([[3, 0], [4, 0]])[:, 0], bounds[1])
    pg.close()


def test_the_largest_number_of_tokens(B):
    """2^31 - 1 of them, nearly all padding: keys and values are one row each that every token shows (token stride 0)."""
    pg, t = T.make(B), 2 ** 31 - 1
    k, v = T.normal((1, 2, 64), torch.bfloat16, 1), T.normal((1, 2, 64), torch.bfloat16, 2)
    slots = torch.full((t,), -1, dtype=torch.int64, device="cuda")
    slots[0], slots[t // 2], slots[-1] = 5, 70, 1023
    kp, vp = (torch.zeros((64, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pg.rope_append(None, k.expand(t, 2, 64), v.expand(t, 2, 64), None, slots, None, kp, vp)
    pg.check()
    for pool, row in ((kp, k), (vp, v)):
        cells = pool.transpose(1, 2).reshape(-1, 2, 64)
        assert torch.equal(cells[[5, 70, 1023]], row.expand(3, 2, 64)) and (cells != 0).any(-1).any(-1).sum() == 3
    pg.close()
