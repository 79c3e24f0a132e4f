"""What PagedDecoder.admit and release do with requests and caches that do not fit, and between the layers of a step."""
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


def state(dec):
    names = ("table", "lens", "free_pages", "free_top", "active", "slots", "k_pages", "v_pages")
    return {x: getattr(dec, x).clone() for x in names}


def same(dec, before):
    return all(torch.equal(getattr(dec, x), y) for x, y in before.items() if x not in ("k_pages", "v_pages")) and all(
        torch.equal(getattr(dec, x).view(torch.int16), before[x].view(torch.int16)) for x in ("k_pages", "v_pages"))


@pytest.mark.parametrize("request_", [-1, -3, 3, 4])
def test_requests_out_of_range_are_refused(B, request_):
    wl = S.workload()
    cp = S.compressed(wl)
    dec = S.decoder(wl, 120, 3, 400)
    dec.admit(2, cp)
    before = state(dec)
    for call in (lambda: dec.admit(request_, cp), lambda: dec.release(request_)):
        with pytest.raises(IndexError):
            call()
    assert same(dec, before)
    dec.check()
    dec.close()
    cp.close()


def test_caches_of_another_shape_are_refused_and_change_nothing(B):
    """The request keeps what it held, and nothing is taken from the pool."""
    wl = S.workload()
    cp = S.compressed(wl)
    dec = S.decoder(wl, 120, 2, 400)
    dec.admit(0, cp)
    before = state(dec)
    for kw in (dict(n_layers=1), dict(n_layers=4), dict(n_kv_heads=3), dict(n_kv_heads=1), dict(head_dim=64), dict(dtype="f32")):
        other = S.compressed(wl.with_(**kw))
        for r in (0, 1):
            with pytest.raises(ValueError):
                dec.admit(r, other)
        assert same(dec, before), kw
        other.close()
    dec.check()
    dec.close()
    cp.close()


def test_a_compression_that_ran_out_of_rows_is_not_admitted(B):
    """Its budgets name rows that its buffers do not have: the request stays empty, and check() says so."""
    wl = S.workload()
    good, short = S.compressed(wl), S.compressed(wl, row_capacity=20)
    with pytest.raises(B.MedaError):
        short.check()
    assert int(short.budgets[:, 0].max()) > 20
    dec = S.decoder(wl, 120, 2, 400)
    dec.admit(0, good)
    dec.check()
    before = state(dec)
    dec.admit(1, short)
    with pytest.raises(B.MedaError) as e:
        dec.check()
    assert e.value.status == B.MEDA_ERR_WORKSPACE
    assert same(dec, before)
    dec.check()
    dec.close()
    good.close()
    short.close()


@pytest.mark.parametrize("keep_pages", [0, 6])
def test_leaving_between_the_layers_of_a_step(B, keep_pages):
    """A request is released after a step has begun and its pages go to another: the layers still to come write nothing of the one
    that left."""
    wl = S.workload()
    cp = S.compressed(wl)
    dec = S.decoder(wl, 120, 3, 400, keep_pages=keep_pages)
    st = S.Steps(wl, dec)
    st.admit(0, cp)
    st.admit(2, cp)
    hq, hkv = wl.n_q_heads, wl.n_kv_heads
    st.step([0, 2])
    dec.begin_step()
    st.release(0)
    st.admit(1, cp)                                                # takes over the pages just given back
    x = torch.full_like(st.qkv[0], 7.0)
    at = dec.slots[:, 2].clone()
    for l in range(wl.n_layers):
        dec.attend(l, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], st.pos, st.out[l], st.lse[l])
    dec.check()
    st.check_caches([1])
    assert torch.equal(at, dec.slots[:, 2]) and (at >= 0).all()    # the request that stayed got its rows
    for l in range(wl.n_layers):
        assert (dec.v_pages[at[l] // 16, :, at[l] % 16] == 7.0).all()
    # a request that is replaced is one that left
    dec.begin_step()
    st.admit(1, cp)
    for l in range(wl.n_layers):
        dec.attend(l, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], st.pos, st.out[l], st.lse[l])
    dec.check()
    st.check_caches([1])
    dec.close()
    cp.close()
