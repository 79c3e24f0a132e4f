"""Slot maps of 2^31 - 1 entries: counters of the kernel's loops end at most one stride behind the last entry, past 2^31."""
import pytest
import torch

import test_gpu_pages as T

pytestmark = pytest.mark.gpu

SLOTS = 2 ** 31 - 1


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def chunks(n, size=1 << 27):
    return [(a, min(n, a + size)) for a in range(0, n, size)]


@pytest.mark.parametrize("lens", [[40, 20], [0, 65]])
def test_refused_changes(B, lens):
    """A pool without pages, or a length out of range: every slot is -1."""
    pg = T.make(B, page_size=16, n_pages=4, max_seqs=2, max_seq_pages=4)
    slots = torch.zeros(SLOTS, dtype=torch.int64, device="cuda")
    table, free, top, cu = T.i32([[3] * 4] * 2), T.i32([0, 1, 2, 3]), T.i32([0]), T.i32([-5, -5, -5])
    pg.page_tables(None, T.i32(lens), free, T.i32([0]), top, table, cu, slots)
    assert pg.poll_status() == (B.MEDA_ERR_WORKSPACE if lens[0] else B.MEDA_ERR_INVALID_ARG)
    assert all((slots[a:b] == -1).all() for a, b in chunks(SLOTS))
    assert (table == 3).all() and cu.tolist() == [0, 0, 0] and top.tolist() == [0]
    pg.close()


@pytest.mark.parametrize("rows", [SLOTS, SLOTS - 100, 1000])
def test_as_many_new_rows(B, rows):
    """8,192 sequences of 1,024 pages of 256 rows, or next to none, in a map of 2^31 - 1 slots."""
    n, width, page = 8192, 1024, 256
    pg = T.make(B, page_size=page, n_pages=n * width, max_seqs=n, max_seq_pages=width)
    free = torch.randperm(n * width, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.int32)
    lens = (rows - torch.arange(n, device="cuda") * width * page).clamp(0, width * page).to(torch.int32)
    table, top, cu = torch.full((n, width), -1, dtype=torch.int32, device="cuda"), T.i32([-5]), torch.full((n + 1,), -5, dtype=torch.int32, device="cuda")
    slots = torch.zeros(SLOTS, dtype=torch.int64, device="cuda")
    pg.page_tables(None, lens, free, T.i32([0]), top, table, cu, slots)
    pg.check()
    pages = -(-rows // page)
    assert top.tolist() == [pages] and int(cu[-1]) == rows and torch.equal(cu[1:] - cu[:-1], lens)
    flat = table.view(-1)                                          # (only the last sequence is not full)
    assert torch.equal(flat[:pages], free[:pages]) and (flat[pages:] == -1).all()
    for a, b in chunks(rows):
        t = torch.arange(a, b, device="cuda")
        assert torch.equal(slots[a:b], flat[t // page].long() * page + t % page)
    assert all((slots[rows + a:rows + b] == -1).all() for a, b in chunks(SLOTS - rows))
    pg.close()
