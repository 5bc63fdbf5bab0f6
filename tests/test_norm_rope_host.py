"""Norm of query / key heads with the rotation: the reference against its own differences, and what is refused, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests import norm_rope_ref as ref


@pytest.mark.parametrize("D,rot,adjacent", [(64, 64, False), (64, 32, True), (128, 0, False)])
def test_reference_gradient_equals_differences(D, rot, adjacent):
    rng = np.random.default_rng(5)
    T, H, eps = 3, 2, 1e-6
    x, dz, v = (rng.standard_normal((T, H, D)) for _ in range(3))
    w, vw = 1 + 0.3 * rng.standard_normal(D), rng.standard_normal(D)
    M = ref.rotation(ref.table(50, rot).astype(np.float64), rng.integers(0, 50, T), D, adjacent)
    dx, dw, _, _ = ref.backward(dz, x, w, M, eps)
    f = lambda h: (dz * ref.forward(x + h * v, w + h * vw, M, eps)[0]).sum()
    h = 1e-5
    # central differences: h^2 / 6 of the third derivative (order 1e3 here) and rounding 1e-16 / h of the value (order 10)
    assert abs((f(h) - f(-h)) / (2 * h) - ((dx * v).sum() + (dw * vw).sum())) < 1e-6


def test_reference_by_hand():
    x = np.zeros((1, 1, 64))
    x[0, 0, 0], x[0, 0, 1] = 3.0, 4.0                       # mean square 25 / 64, so r = 8 / 5
    M = ref.rotation(np.array([[0.0] * 8 + [1.0] * 8]), np.array([0]), 64, True)    # a quarter turn of the first 8 pairs
    z, _ = ref.forward(x, np.ones(64), M, 0.0)
    assert np.allclose(z[0, 0, :2], [-6.4, 4.8]) and np.count_nonzero(z) == 2


def shape(**kw):
    d = dict(num_tokens=4, num_q_heads=2, num_kv_heads=1, head_dim=128, rotary_dim=128, max_positions=8, dtype=0, adjacent_pairs=0,
             eps=1e-6, reserved=0, q_stride=256, k_stride=128, q_out_stride=256, k_out_stride=128, dq_stride=256, dk_stride=128)
    d.update(kw)
    return B.NormRopeShape(*[d[n] for n, _ in B.NormRopeShape._fields_])


BAD_SHAPES = [(dict(num_tokens=-1), -1), (dict(num_q_heads=0), -1), (dict(num_kv_heads=0), -1), (dict(rotary_dim=-16), -1),
              (dict(rotary_dim=144), -1), (dict(max_positions=0), -1), (dict(eps=float("nan")), -1), (dict(eps=-1.0), -1),
              (dict(head_dim=96, rotary_dim=96), -2), (dict(rotary_dim=24), -2), (dict(dtype=2), -2), (dict(adjacent_pairs=2), -2),
              (dict(num_tokens=1 << 30), -2)]


@pytest.mark.parametrize("kw,status", BAD_SHAPES)
def test_bad_shapes_are_refused(kw, status):
    lib = B.load_library()
    buf = ctypes.create_string_buffer(4096 + 256)
    p = ctypes.c_void_p((ctypes.addressof(buf) + 255) // 256 * 256)
    n = ctypes.c_size_t(0)
    s = shape(**kw)
    assert lib.marl_qk_norm_rope_workspace_bytes(ctypes.byref(s), ctypes.byref(n)) == status
    assert lib.marl_qk_norm_rope(ctypes.byref(s), *[p] * 8, None, None) == status
    assert lib.marl_qk_norm_rope_backward(ctypes.byref(s), p, 1 << 20, *[p] * 12, None, None) == status


def test_bad_arguments_are_refused():
    lib = B.load_library()
    buf = ctypes.create_string_buffer(4096 + 256)
    base = (ctypes.addressof(buf) + 255) // 256 * 256
    good = [ctypes.c_void_p(base)] * 8       # q, k, q_weight, k_weight, cos_sin, positions, q_out, k_out
    call = lambda s, a: lib.marl_qk_norm_rope(ctypes.byref(s), *a, None, None)
    for k in range(8):
        for p in (None, ctypes.c_void_p(base + 4)):
            if (p is None and k in (2, 3)) or (p is not None and k == 5):
                continue                     # a weight may be missing, positions are read one by one
            assert call(shape(), good[:k] + [p] + good[k + 1:]) == -1, k
    assert call(shape(q_stride=260), good) == -1 and call(shape(k_stride=-128), good) == -1
    assert call(shape(q_out_stride=128), good) == -1 and call(shape(k_out_stride=0), good) == -1
    assert call(shape(num_tokens=0), [None] * 8) == 0
    back = [ctypes.c_void_p(base)] * 12      # dq_out, dk_out, q, k, q_weight, k_weight, cos_sin, positions, dq, dk, dq_weight, dk_weight
    call = lambda s, ws, n, a: lib.marl_qk_norm_rope_backward(ctypes.byref(s), ws, n, *a, None, None)
    p = ctypes.c_void_p(base)
    assert call(shape(), None, 1 << 30, back) == -1 and call(shape(), ctypes.c_void_p(base + 8), 1 << 30, back) == -1
    assert call(shape(), p, 1024 * 2 * 128 * 4 - 1, back) == -3
    for k in (0, 1, 2, 3, 6, 7, 8, 9):
        assert call(shape(), p, 1 << 30, back[:k] + [None] + back[k + 1:]) == -1, k
    assert call(shape(dq_stride=128), p, 1 << 30, back) == -1
    assert call(shape(), p, 1 << 30, back[:10] + [ctypes.c_void_p(base + 2)] + back[11:]) == -1
    assert lib.marl_qk_norm_rope(None, *good, None, None) == -1


def test_binding_refuses_host_and_wrong_tensors():
    q, k = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(4, 1, 128, dtype=torch.bfloat16)
    w, cs, pos = torch.ones(128, dtype=torch.bfloat16), torch.zeros(8, 128), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        B.marl_qk_norm_rope(q, k, w, w, cs, pos, 1e-6, q, k)
    with pytest.raises(ValueError, match="bf16 or float32"):
        B.marl_qk_norm_rope(q.half(), k.half(), w, w, cs, pos, 1e-6, q, k)
    assert B.marl_qk_norm_rope_workspace_bytes(10, 8, 2, 128) == 1024 * 2 * 128 * 4
