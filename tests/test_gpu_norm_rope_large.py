"""Norm of query / key heads with the rotation in calls that fill the GPU: four steps a wave, results past the caches.  Every element against the
formulas in 64 bits (tests/norm_rope_ref.py has them too, for small sizes).

Tolerances as in tests/test_gpu_norm_rope.py.  A sum of dw is deeper here: a lane adds four heads of each of its units (4096 waves, or as many as there are),
then come at most 3 + 4 additions in the workgroup and 4 + 3 + 32 over 1024 workgroups; dy and n have 24 roundings more between them."""
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests.test_gpu_norm_rope import EPS, EPS32, make

pytestmark = pytest.mark.gpu


def turn(y, c, s, adjacent, back=False):
    """The rotation (back: its transpose) of the first 2 h channels of y [T, H, D] by c, s [T, h]."""
    h = c.shape[1]
    c, s = c[:, None], -s[:, None] if back else s[:, None]
    a, b = (y[..., 0: 2 * h: 2], y[..., 1: 2 * h: 2]) if adjacent else (y[..., :h], y[..., h: 2 * h])
    z = y.clone()
    za, zb = a * c - b * s, b * c + a * s
    if adjacent:
        z[..., 0: 2 * h: 2], z[..., 1: 2 * h: 2] = za, zb
    else:
        z[..., :h], z[..., h: 2 * h] = za, zb
    return z


def turn_abs(y, c, s, adjacent):
    """Sums of the magnitudes that a turn adds up."""
    h = c.shape[1]
    c, s = c[:, None].abs(), s[:, None].abs()
    m = y.abs()
    a, b = (m[..., 0: 2 * h: 2], m[..., 1: 2 * h: 2]) if adjacent else (m[..., :h], m[..., h: 2 * h])
    z = m.clone()
    za, zb = a * c + b * s, b * c + a * s
    if adjacent:
        z[..., 0: 2 * h: 2], z[..., 1: 2 * h: 2] = za, zb
    else:
        z[..., :h], z[..., h: 2 * h] = za, zb
    return z


def close(got, want, magnitude, units, dtype):
    allowed = units * EPS32 * magnitude + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0) + 1e-37
    worst = float(((got.double() - want).abs() / allowed).max())
    assert worst <= 1.0, f"{worst} of the tolerance"


BF, F32 = torch.bfloat16, torch.float32
# T, Hq, Hkv, D, rot, adjacent, dtype, results past the caches (bf16 of more than 32 MB).  A wave has four steps of 512 / D heads; where the queries' steps are
# no multiple of four (5, 7, 3, 2, 1, 6 of them here) one of its steps is the first of the keys'.
CASES = [(4500, 28, 4, 128, 128, False, BF, True), (4097, 20, 12, 128, 64, True, BF, True), (8200, 8, 8, 128, 128, False, BF, True),
         (8193, 12, 3, 128, 32, False, BF, False), (9000, 4, 4, 64, 64, False, BF, False), (8500, 13, 5, 64, 32, True, BF, False),
         (33000, 8, 2, 64, 64, False, BF, True), (8200, 5, 3, 256, 256, False, BF, True), (4200, 12, 4, 256, 64, True, BF, True),
         (8200, 2, 1, 256, 112, False, BF, False), (4500, 28, 4, 128, 128, False, F32, False), (8300, 7, 9, 128, 96, True, F32, False),
         (8200, 3, 2, 256, 0, False, F32, False), (9001, 16, 1, 64, 48, False, F32, False)]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,adjacent,dtype,past", CASES)
def test_large_calls(T, Hq, Hkv, D, rot, adjacent, dtype, past):
    print("case: norm rope, large", T, Hq, Hkv, D, rot, adjacent, dtype, flush=True)
    steps = -(-Hq * D // 512) + -(-Hkv * D // 512)
    assert T * -(-steps // 4) >= 8192 and past == (dtype == BF and T * (Hq + Hkv) * D * 2 > 32 << 20)
    d = make(T, Hq, Hkv, D, rot, dtype, T + D)
    angle = d["cos_sin"][d["positions"].long()].double()
    c, s = angle[:, : rot // 2], angle[:, rot // 2:]
    q_out, k_out = torch.empty(T, Hq, D, dtype=dtype, device="cuda"), torch.empty(T, Hkv, D, dtype=dtype, device="cuda")
    args = d["q_weight"], d["k_weight"], d["cos_sin"], d["positions"], EPS
    B.marl_qk_norm_rope(d["q"], d["k"], *args, q_out, k_out, adjacent)
    ws = B.alloc_workspace(B.marl_qk_norm_rope_workspace_bytes(T, Hq, Hkv, D), "cuda")
    ws.fill_(0xFF)
    dq, dk = torch.empty_like(q_out), torch.empty_like(k_out)
    dqw, dkw = (torch.full((D,), float("nan"), device="cuda") for _ in range(2))
    B.marl_qk_norm_rope_backward(d["dq_out"], d["dk_out"], d["q"], d["k"], *args, dq, dk, dqw, dkw, ws, adjacent)
    units = T * -(-steps // (2 if dtype == F32 else 4))
    depth = 4 * -(-units // min(4096, units)) + 7 + 39 + 24
    for n, z, dx, dw in (("q", q_out, dq, dqw), ("k", k_out, dk, dkw)):
        x, w, dz = d[n].double(), d[n + "_weight"].double(), d["d" + n + "_out"].double()
        r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        y = x * r * w
        close(z, turn(y, c, s, adjacent), turn_abs(y, c, s, adjacent), 24, dtype)
        del y
        norm, dy, dy_abs = x * r, turn(dz, c, s, adjacent, back=True), turn_abs(dz, c, s, adjacent)
        g, g_abs = dy * w, dy_abs * w.abs()
        want = r * (g - norm * (g * norm).mean(-1, keepdim=True))
        magnitude = r * (g_abs + norm.abs() * (g_abs * norm.abs()).mean(-1, keepdim=True))
        close(dx, want, magnitude, 48, dtype)
        close(dw, (dy * norm).sum((0, 1)), (dy_abs * norm.abs()).sum((0, 1)), depth, F32)
    again = [torch.empty_like(t) for t in (q_out, k_out)]
    B.marl_qk_norm_rope(d["q"], d["k"], *args, *again, adjacent)
    dqw2 = torch.empty_like(dqw)
    B.marl_qk_norm_rope_backward(d["dq_out"], d["dk_out"], d["q"], d["k"], *args, dq.zero_(), dk.zero_(), dqw2, None, ws, adjacent)
    assert torch.equal(again[0], q_out) and torch.equal(again[1], k_out) and torch.equal(dqw2, dqw)
