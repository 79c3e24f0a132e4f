"""Quantised pages without a GPU: refused handles, and the oracle of the format against its definition and brute force."""
import ctypes

import numpy as np
import pytest

from oracle import pages_oracle as O
from test_pages_cpu import GOOD


@pytest.fixture(scope="module")
def B():
    from paper_2502_17599_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("bits", [1, 2, 3, 5, 6, 7, 9, 16, -4])
def test_create_refuses_other_widths(B, bits):
    with pytest.raises(ValueError):
        B.Pages(**GOOD, cache_bits=bits)
    config = B.meda_pages_config(4, 2, 64, 0, 16, 10, 4, 8, 1e4, (ctypes.c_int32 * 3)(32, 0, 0), 0, 0)
    handle = ctypes.c_void_p(7)
    assert B.load_library().meda_pages_create_quantised(ctypes.byref(config), bits, ctypes.byref(handle)) == B.MEDA_ERR_INVALID_ARG
    assert handle.value is None


@pytest.mark.parametrize("status,kw", [(-2, dict(n_q_heads=3)), (-2, dict(head_dim=96)), (-2, dict(page_size=8)), (-2, dict(n_pages=0)),
                                       (-1, dict(rope_theta=1.0)), (-1, dict(rope_pairing=2))])
@pytest.mark.parametrize("bits", [4, 8])
def test_create_refuses_what_other_handles_refuse(B, status, kw, bits):
    with pytest.raises(B.MedaError) as e:
        B.Pages(**{**GOOD, **kw}, cache_bits=bits)
    assert e.value.status == status


@pytest.mark.parametrize("bits", [4, 8])
def test_pools_of_256_gib_are_refused(B, bits):
    geometry = dict(n_q_heads=16, n_kv_heads=8, head_dim=256, dtype="bf16", page_size=256, max_seqs=1, max_seq_pages=1)
    n_pages = -(-2 ** 38 // (8 * 256 * (256 * bits // 8 + 16)))
    with pytest.raises(B.MedaError) as e:
        B.Pages(**geometry, n_pages=n_pages, cache_bits=bits)
    assert e.value.status == B.MEDA_ERR_SHAPE
    try:
        B.Pages(**geometry, n_pages=n_pages - 1, cache_bits=bits).close()
    except B.MedaError as e:                                       # (without a GPU, but past the shapes)
        assert e.status == B.MEDA_ERR_CUDA


def test_null_handles(B):
    lib = B.load_library()
    one = 256                                                      # never dereferenced
    assert lib.meda_pages_create_quantised(None, 4, ctypes.byref(ctypes.c_void_p())) == B.MEDA_ERR_INVALID_ARG
    assert lib.meda_pages_page_bytes(None) == 0
    assert lib.meda_page_load(None, one, one, one, None, one, 1, 1, one, one, 0, 0, 1, None) == B.MEDA_ERR_INVALID_ARG


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1.0, 1e20])
def test_a_row_reads_back_to_half_a_step(bits, scale):
    rng = np.random.default_rng(bits)
    x = (rng.normal(0.5, 1, (200, 128)) * rng.uniform(0.1, 30, (1, 128)) * scale).astype(np.float32)
    code, step, low = O.quantise(x, bits)
    assert code.max() == (1 << bits) - 1 and code.min() == 0
    g = x.reshape(200, 2, 64)
    assert (low <= g.min(-1)).all() and (low.astype(np.float64) + step.astype(np.float64) * ((1 << bits) - 1) * (1 + 2.0 ** -22) >= g.max(-1)).all()
    # half a step, and the fp32 roundings of the difference, the reciprocal and the product (2^-24 each) of a code of at most 2^bits - 1
    err = np.abs(O.held(code, step, low) - x).reshape(200, 2, 64)
    assert (err <= step[..., None].astype(np.float64) * (0.5 + 4 * 2.0 ** -24 * (1 << bits))).all()
    # the step is no larger than it has to be: rounded up to eight bits, of a range that grew by the rounding of its lower end
    spread = g.max(-1).astype(np.float64) - low
    assert (step <= spread / ((1 << bits) - 1) * (1 + 2.0 ** -7) * (1 + 2.0 ** -22)).all()


def test_special_groups():
    x = np.zeros((9, 64), np.float32)
    x[1] = -3.25                                                   # one value
    x[2, 5] = np.nan
    x[3, 7] = np.inf
    x[4, 9] = -np.inf
    x[5, 0] = 2.0 ** 126                                           # the first that counts as too large
    x[6, :2] = np.nextafter(np.float32(2.0 ** 126), np.float32(0)), -np.nextafter(np.float32(2.0 ** 126), np.float32(0))
    x[7, 3] = 2.0 ** -149                                          # a range below the smallest step
    x[8] = np.float32(-0.0)
    for bits in (4, 8):
        code, step, low = O.quantise(x, bits)
        back = O.held(code, step, low)
        assert (back[[0, 8]] == 0).all() and (back[1] == -3.25).all() and np.isnan(back[2:6]).all()
        assert np.isfinite(back[6]).all() and (np.abs(back[6] - x[6]) <= step[6] * 0.5001).all()
        assert step[7] == 2.0 ** -126 and (np.abs(back[7] - x[7]) <= 2.0 ** -127).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_pack_and_unpack(bits, d):
    rng = np.random.default_rng(d + bits)
    code = rng.integers(0, 1 << bits, (2, 5, d // 64, 64)).astype(np.uint8)
    step, low = (O._bf16(rng.normal(size=(2, 5, d // 64)).astype(np.float32), False) for _ in range(2))
    page = O.pack_page(code, step, low, bits)
    assert page.shape == (2, 5 * (d * bits // 8 + 4 * (d // 64)))
    for a, b in zip(O.unpack_page(page, 5, d, bits), (code, step, low)):
        np.testing.assert_array_equal(a, b)
    # one code of one row: units of eight dimensions, those of all groups side by side
    one = np.zeros_like(code)
    one[0, 3, d // 64 - 1, 17] = 1
    at = O.pack_page(one, step, low, bits)[0].nonzero()[0][0]
    unit = 2 * (d // 64) + d // 64 - 1                             # dimension 17: unit 2 of the last group, element 1
    assert at == 3 * d * bits // 8 + (unit * 8 + 1) * bits // 8


def test_the_rotation_in_fp32_is_the_rotation():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(7, 2, 128)).astype(np.float32)
    pos = rng.integers(-5, 2 ** 31 - 1, (3, 7))
    for order, sections in ((0, (24, 20, 20)), (1, (24, 20, 20)), (0, (16, 8, 8))):
        for pairing in (0, 1):
            # far positions: the fixed-point frequency is off by 2^-53 of itself, the position below 2^31
            want = O.rope(x.astype(np.float64), pos, sections, order, pairing, 1e6)
            got = O.rope_fp32(x, pos, sections, order, pairing, 1e6)
            assert np.abs(got - want).max() <= 2.0 ** 31 * 2.0 ** -51 * 8 + 3 * 2.0 ** -24 * 8
            near = pos % 1000
            want = O.rope(x.astype(np.float64), near, sections, order, pairing, 1e6)
            assert np.abs(O.rope_fp32(x, near, sections, order, pairing, 1e6) - want).max() <= 4 * 2.0 ** -24 * 8
