"""Calls of more workgroups than one launch can hold are refused before any launch: by their sizes alone, on pointers that nobody follows."""
import ctypes

import pytest

from paper_2602_09578_amd import binding as B
from tests.test_norm_rope_host import shape as norm_shape

UNSUPPORTED = -2
LAUNCH = 1 << 24          # workgroups of 256 threads: 2^32 threads


@pytest.fixture
def p():
    buf = ctypes.create_string_buffer(4096 + 256)
    yield ctypes.c_void_p((ctypes.addressof(buf) + 255) // 256 * 256)


@pytest.mark.parametrize("Hkv,n", [(1, LAUNCH), (8, LAUNCH // 8), (3, LAUNCH // 3 + 1)])
def test_pages_read_back(p, Hkv, n):
    assert B.load_library().marl_kv_read_pages_fp8(Hkv, 3, p, p, p, 4, p, p, p, p, n, None, None) == UNSUPPORTED


def test_append(p):
    s = B.make_shape(LAUNCH, 1, 1, 1, 3, 1, 1)
    assert B.load_library().marl_kv_append_fp8(ctypes.byref(s), *[p] * 7, None, None) == UNSUPPORTED


@pytest.mark.parametrize("NS,Hq,Hkv", [(LAUNCH, 8, 8), (LAUNCH // 2, 16, 1), (4 * LAUNCH, 1, 1), (((1 << 27) - 1032) // 11 + 1, 11, 1)])
def test_attention(p, NS, Hq, Hkv):
    s = B.make_shape(NS, 1, Hq, Hkv, 3, 1, 1)
    assert B.load_library().marl_decode_attn_fp8(ctypes.byref(s), p, 1 << 50, *[p] * 9, 0.1, p, None) == UNSUPPORTED


# a wave takes up to four groups of 512 / head_dim heads of a token, a workgroup has four waves
@pytest.mark.parametrize("T,Hq,Hkv,D", [(4 * LAUNCH, 1, 1, 64), (4 * LAUNCH - 3, 4, 8, 128), (2 * LAUNCH, 28, 4, 64), (2 * LAUNCH, 17, 15, 128)])
def test_norm(p, T, Hq, Hkv, D):
    s = norm_shape(num_tokens=T, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, rotary_dim=64, q_stride=0, k_stride=0, q_out_stride=Hq * D, k_out_stride=Hkv * D)
    per_token = -(-(-(-Hq * D // 512) + -(-Hkv * D // 512)) // 4)
    assert T * per_token > 4 * (LAUNCH - 1)
    assert B.load_library().marl_qk_norm_rope(ctypes.byref(s), *[p] * 8, None, None) == UNSUPPORTED


# (128 threads a workgroup)
@pytest.mark.parametrize("NG,Hkv", [(LAUNCH, 2), (2 * LAUNCH, 1)])
def test_prompt(p, NG, Hkv):
    s = B.make_prefill_shape(5, NG, Hkv, Hkv, 3, 1)
    lib = B.load_library()
    assert lib.marl_kv_write_prompt_fp8(ctypes.byref(s), *[p] * 8, None, None) == UNSUPPORTED
    assert lib.marl_kv_write_prompt(ctypes.byref(s), *[p] * 7, None, None) == UNSUPPORTED
