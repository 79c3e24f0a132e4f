"""Decoding steps that cannot give every request a row: a request at its last row, a pool without a page left."""
import math

import pytest
import torch

import paged_steps as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def longest(cp):
    return int(cp.budgets[:, 0].max())


@pytest.mark.parametrize("keep_pages", [0, 6])
@pytest.mark.parametrize("graph", [False, True])
def test_a_request_at_its_limit_does_not_hold_up_the_others(B, keep_pages, graph):
    """Request 0 reaches max_rows in its longest layer: from then on it gets no row in any layer, its outputs are NaN and check() names
    it, while request 1 goes on as if it were alone."""
    wl = S.workload()
    cps = [S.compressed(wl), S.compressed(wl.with_(seed=9, rho=0.1))]
    most = longest(cps[0])
    dec = S.decoder(wl, 120, 3, most + 5, keep_pages=keep_pages)
    room = dec.table.shape[1] * 16 - most                          # steps until request 0 is full: its last page may be filled
    assert room >= 5
    assert longest(cps[1]) + room + 4 < dec.table.shape[1] * 16
    st = S.Steps(wl, dec)
    st.admit(0, cps[0])
    st.admit(2, cps[1])
    run = None
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            st.step([0, 2])                                        # loads the kernels
        side.synchronize()
        room -= 1
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            st.body()
        run = captured.replay
    for n in range(room + 3):
        grown = [0, 2] if n < room else [2]
        before = dec.table.clone()
        st.step(grown, run)
        assert dec.advanced.tolist() == [int(r in grown) for r in range(3)]
        st.check_caches([0, 2])
        st.check_outputs(grown)
        if keep_pages:
            st.check_choice(grown)
        if n < room:
            dec.check()
        else:
            assert st.out[:, 0].isnan().all() and st.lse[:, 0].isnan().all()
            assert torch.equal(before.view(wl.n_layers, 3, -1)[:, 0], dec.table.view(wl.n_layers, 3, -1)[:, 0])
            with pytest.raises(B.MedaError) as e:
                dec.check()
            assert "[0]" in str(e.value)
            dec.check()                                            # reported once
    st.release(0)
    st.step([2], run)
    dec.check()
    st.check_caches([2])
    st.check_outputs([2])
    st.admit(0, cps[1])                                            # its number is free for a new request
    st.step([0, 2], run)
    dec.check()
    st.check_caches([0, 2])
    st.check_outputs([0, 2])
    dec.close()
    for cp in cps:
        cp.close()


def test_a_step_the_pool_cannot_serve_is_seen_in_its_outputs(B):
    """No page is left for one of the requests: nobody gets a row, every active request's outputs are NaN (not those of an earlier
    query), and after one of them has left the step can be taken again."""
    wl = S.workload()
    cp = S.compressed(wl)
    rows = cp.budgets[:, 0].tolist()
    used = lambda n: 2 * sum(-(-(x + n) // 16) for x in rows)      # pages of both requests after n steps
    dec = S.decoder(wl, used(1), 2, 400)
    st = S.Steps(wl, dec)
    st.admit(0, cp)
    st.admit(1, cp)
    served = max(n for n in range(17) if used(n) == used(1))       # steps until some layer needs another page
    for n in range(served):
        st.step([0, 1])
        dec.check()
        st.check_outputs([0, 1])
    for again in range(2):
        st.step([])
        assert dec.advanced.tolist() == [0, 0]
        assert st.out.isnan().all() and st.lse.isnan().all()
        with pytest.raises(B.MedaError) as e:
            dec.check()
        assert e.value.status == B.MEDA_ERR_WORKSPACE and "[0, 1]" in str(e.value)
        st.check_caches([0, 1])
    st.release(1)
    st.step([0])
    dec.check()
    assert dec.advanced.tolist() == [1, 0]
    st.check_caches([0])
    st.check_outputs([0])
    dec.close()
    cp.close()
