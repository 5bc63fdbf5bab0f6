"""The 8-bit KV cache without a GPU: the reference's rounding pinned by hand and by its bounds, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests import fp8_cache_ref as ref


def test_codes_stand_for_torchs_numbers():
    got = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, ref.VALUES, equal_nan=True)


def row(*x):
    return np.array(list(x) + [0.0] * (128 - len(x)))


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (224.0, -1), (225.0, 0), (1.75, -8), (1.7578125, -7), (0.0, -110), (2.0 ** -130, -110),
                                   (448 * 2.0 ** -110, -110), (450 * 2.0 ** -110, -109), (3.3895313892515355e38, 120)])
def test_exponent_by_hand(top, e):
    codes, got = ref.quantize(row(top, -top / 2))
    assert int(got) == e and (top < 1e-30 or abs(ref.VALUES[codes[0]]) >= 224)


def test_rounding_by_hand():
    # unit 2^-3 around 1 .. 2 (with 448 in the row the exponent is 0): ties go to the even mantissa
    codes, e = ref.quantize(row(448.0, 1.0625, 1.1875, -1.0625, 1.07, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, -2.0 ** -11, 464.0 - 16))
    assert int(e) == 0
    assert ref.VALUES[codes[:10]].tolist() == [448.0, 1.0, 1.25, -1.0, 1.125, 0.0, 2.0 ** -8, 2.0 ** -9, 0.0, 448.0]
    assert codes[8] == 0x80                                                       # a negative number that rounds to nothing
    codes, e = ref.quantize(row(3.3895313892515355e38, -np.inf, -1.9 * 2.0 ** 127))
    assert int(e) == 120 and ref.VALUES[codes[:3]].tolist() == [240.0, -240.0, -240.0]
    codes, e = ref.quantize(row(np.inf, -np.inf, np.nan, 3.0))
    assert int(e) == -7 and codes[:3].tolist() == [0x7E, 0xFE, 0x7F] and ref.VALUES[codes[3]] * 2.0 ** -7 == 3.0


def test_bound_of_the_rounding():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 128)) * np.exp2(rng.integers(-100, 100, (200, 1)).astype(float))
    codes, e = ref.quantize(x)
    unit = np.exp2(e[:, None].astype(float))
    err = np.abs(ref.VALUES[codes] * unit - x)
    assert (err <= np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -10)).all()
    assert (np.abs(x).max(1) > 224 * unit[:, 0]).all()


def test_refusals():
    lib = B.load_library()
    buf = ctypes.create_string_buffer(8192)
    base = (ctypes.addressof(buf) + 255) // 256 * 256
    p, odd = ctypes.c_void_p(base), ctypes.c_void_p(base + 8)
    shape = B.make_shape(2, 1, 4, 2, 3, 1, 1)
    call = lambda s, a: lib.marl_kv_append_fp8(ctypes.byref(s), *a, None, None)
    for k in range(7):                                                            # k_new, v_new, k_pages, v_pages, exponents, table, lens
        assert call(shape, [p] * k + [None] + [p] * (6 - k)) == -1
        if k < 5:
            assert call(shape, [p] * k + [odd] + [p] * (6 - k)) == -1
    assert call(B.make_shape(2, 1, 4, 2, 3, 1, 0), [p] * 7) == -1 and call(B.make_shape(0, 1, 4, 2, 3, 1, 1), [None] * 7) == 0
    assert call(B.make_shape(2, 1, 4, 2, 3, 1, 1, head_dim=64), [p] * 7) == -2 and call(B.make_shape(-2, 1, 4, 2, 3, 1, 1), [p] * 7) == -1
    pshape = B.make_prefill_shape(5, 1, 4, 2, 3, 2)
    call = lambda s, a: lib.marl_kv_write_prompt_fp8(ctypes.byref(s), *a, None, None)
    for k in range(8):                                                            # ..., exponents, table, q_start, q_pos0
        assert call(pshape, [p] * k + [None] + [p] * (7 - k)) == -1
        if k < 5:
            assert call(pshape, [p] * k + [odd] + [p] * (7 - k)) == -1
    assert call(B.make_prefill_shape(0, 1, 4, 2, 3, 2), [None] * 8) == 0 and call(B.make_prefill_shape(5, 1, 4, 2, 3, 2, page_size=32), [p] * 8) == -2
    read = lambda Hkv=2, pages=3, out=4, n=2, a=(p,) * 7: lib.marl_kv_read_pages_fp8(Hkv, pages, *a[:3], out, *a[3:], n, None, None)
    for k in range(7):                                                            # codes, codes, exponents, k_pages, v_pages, src, dst
        assert read(a=[p] * k + [None] + [p] * (6 - k)) == -1
        if k < 5:
            assert read(a=[p] * k + [odd] + [p] * (6 - k)) == -1
    assert read(Hkv=0) == read(pages=0) == read(out=0) == read(n=-1) == -1 and read(Hkv=4, n=1 << 29) == -2 and read(n=0, a=[None] * 7) == 0


def test_binding_refuses_other_tensors():
    shape = B.make_shape(2, 1, 4, 2, 3, 1, 1)
    k, v, ex = B.alloc_kv_fp8(3, 2, "cpu")
    new, i32 = torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        B.marl_kv_append_fp8(shape, new, new, k, v, ex, i32, i32[:, 0])
    for a in ((k.view(torch.uint8), v, ex), (k, v[:2], ex), (k, v, ex.float())):
        with pytest.raises(ValueError):
            B._require_fp8_cache(3, 2, *a)
