"""The 8-bit rollout example: its operators together, as a program uses them.

Tolerances: of the attention those of tests/test_gpu_attn_fp8.py (a weight rounded to bf16, 2^-8, and 2^-12 for its score, times the
weighted mean of the values' magnitudes; a bf16 result once more 2^-8 of its value); of the gradient those of tests/test_gpu_norm_rope.py
(48 units of 2^-24 of the magnitudes for dx, 128 for dw, and 2^-8 of the value for a bf16 result)."""
import numpy as np
import pytest
import torch

from examples import rollout_8bit as E
from oracle import reference as ref
from paper_2602_09578_amd import inputs as I
from tests import fp8_cache_ref as fp8
from tests import norm_rope_ref
from tests.helpers import to_bf16_bits

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -24
f64 = lambda t: t.detach().double().cpu().numpy()


@pytest.mark.parametrize("prompts,samples,tokens,steps", [(3, 5, 90, 21), (2, 16, 700, 33), (1, 1, 1, 2)])
def test_rollout(prompts, samples, tokens, steps):
    print("case: 8-bit rollout", prompts, samples, tokens, steps, flush=True)
    r = E.run(prompts, samples, tokens, steps, seed=steps)
    d = r.decoder
    NS = prompts * samples
    assert bool((d.suffix_lens == steps).all())
    assert torch.equal(d.positions.cpu(), torch.tensor(r.lens, dtype=torch.int32).repeat_interleave(samples) + steps)
    kc, vc, ex = (t.cpu() for t in (r.cache[0].view(torch.uint8), r.cache[1].view(torch.uint8), r.cache[2]))
    k, v = fp8.keys(kc.numpy(), ex.numpy()), fp8.values(vc.numpy(), ex.numpy())
    # the last step's attention over what the cache holds
    args = lambda values: ref.decode_attn(I.bf16_bits(d.q.cpu()), to_bf16_bits(k), to_bf16_bits(values), d.tables[0].cpu().numpy(), d.tables[1].cpu().numpy(),
                                          d.prefix_lens.cpu().numpy(), d.suffix_lens.cpu().numpy(), d.group_of_seq.cpu().numpy(), E.SCALE, E.HQ, E.HKV)
    want, magnitude, got = args(v), args(np.abs(v)), f64(d.out)
    assert got.shape == (NS, E.HQ, E.D)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -12) * magnitude + 2.0 ** -8 * np.abs(want)).all()
    # the key that the last step wrote
    last = steps - 1
    page, slot = d.tables[1].cpu().numpy()[:, last // 16], last % 16
    codes, e = fp8.quantize(f64(d.k))
    assert np.array_equal(kc.numpy()[page, :, slot], codes) and np.array_equal(ex.numpy()[page, :, 0, slot], e)
    assert np.isfinite(f64(r.out)).all()


def test_train_step():
    print("case: 8-bit rollout, gradient", flush=True)
    T = 150
    layer = E.Layer("cuda", 64, seed=5)
    g = torch.Generator().manual_seed(6)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    x, positions, dq, dk = rnd(T, E.HIDDEN), (torch.arange(T, dtype=torch.int32) % 64).cuda(), rnd(T, E.HQ, E.D), rnd(T, E.HKV, E.D)
    r = E.train_step(layer, x, positions, dq, dk)
    M = norm_rope_ref.rotation(f64(layer.cos_sin), positions.cpu().numpy(), E.D, False)
    at = 0
    for dz, weight, dw in ((dq, layer.q_weight, r.q_weight), (dk, layer.k_weight, r.k_weight)):
        n = dz.shape[1] * E.D
        xs, dx = (f64(t[:, at: at + n]).reshape(T, -1, E.D) for t in (r.qkv, r.dqkv))
        want, want_w, mag, mag_w = norm_rope_ref.backward(f64(dz), xs, f64(weight), M, E.EPS)
        assert (np.abs(dx - want) <= 48 * EPS32 * mag + 2.0 ** -8 * np.abs(want)).all()
        assert (np.abs(f64(dw) - want_w) <= 128 * EPS32 * mag_w + 2.0 ** -8 * np.abs(want_w)).all()
        at += n
    assert not bool(r.dqkv[:, at:].any())
