"""Paged calls and status polls on a stream of their own."""
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


def test_a_poll_waits_for_its_own_stream_only(B):
    """The default stream is busy for about a second; a poll of another stream returns meanwhile, with that stream's error, which it
    clears."""
    pg = T.make(B)
    q, pool = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((64, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    table, lens, out = torch.zeros((1, 16), dtype=torch.int32, device="cuda"), T.i32([-1]), torch.empty_like(q)
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    pg.paged_attention(q, pool, pool, table, lens, out)            # loads the kernels
    assert pg.poll_status() == B.MEDA_ERR_INVALID_ARG
    torch.cuda.synchronize()
    torch.cuda._sleep(2_000_000_000)
    done.record()
    for _ in range(3):
        pg.paged_attention(q, pool, pool, table, lens, out, stream=side)
        assert pg.poll_status(side) == B.MEDA_ERR_INVALID_ARG
        assert pg.poll_status(side) == 0
    assert not done.query()
    torch.cuda.synchronize()
    pg.close()
