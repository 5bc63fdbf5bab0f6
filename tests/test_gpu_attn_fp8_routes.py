"""Decode attention over an 8-bit cache: which kernels a call takes, and its results where those are the general ones with default chunks.

The tolerance is that of tests/test_gpu_attn_fp8.py."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from paper_2602_09578_amd import inputs as I
from tests import fp8_cache_ref as fp8
from tests.test_gpu_attn import custom_inputs
from tests.test_gpu_attn_fp8 import PARTS, Cache, check

pytestmark = pytest.mark.gpu
GENERAL = {"plan", "suffix", "merge"}


def widen(inp, prefix_pages, suffix_pages):
    """The same call in table rows of so many pages."""
    def wide(t, pages):
        assert pages >= t.shape[1]
        w = torch.full((t.shape[0], pages), -1, dtype=torch.int32)
        w[:, : t.shape[1]] = t
        return w
    return I.AttnInputs(**{**inp.__dict__, "prefix_block_table": wide(inp.prefix_block_table, prefix_pages),
                           "suffix_block_table": wide(inp.suffix_block_table, suffix_pages)})


@pytest.mark.parametrize("seqs,Hkv,prefix_pages,suffix_pages,stages", [
    (1, 1, 4, (1 << 16) - 5, PARTS), (1, 1, 4, (1 << 16) - 4, GENERAL), (1, 1, 1 << 16, 250, GENERAL), (2, 1, 1 << 15, 1 << 15, GENERAL), (1, 1, 1 << 15, 1 << 14, PARTS)])
def test_rows_of_a_million_tokens(seqs, Hkv, prefix_pages, suffix_pages, stages):
    """One or two pairs in rows for 2^20 tokens go to the general kernels, rows for fewer to the small call's."""
    print("case: fp8 attention, wide rows", seqs, prefix_pages, suffix_pages, flush=True)
    c, _ = check(widen(custom_inputs([50], [4000, 33][:seqs], [0] * seqs, 4, Hkv, seed=5), prefix_pages, suffix_pages))
    assert c.stages() == stages


DEFAULTS = [  # prompts' lengths, samples, Hq, Hkv, pages of the tables, the shape's default chunks, rows of a prefix block
    ("wide blocks, own chunks of 256", [1500, 909], 20, 28, 4, 1024, 128, (256, 512), 256),
    ("wide blocks, prefix chunks of 256", [2001, 600], 40, 16, 4, 420, 200, (512, 256), 256),
    ("narrow blocks, both of 256", [1400, 0, 700, 4100], 16, 8, 8, 257, 32, (256, 256), 128),
    ("narrow blocks, one prompt", [900], 70, 6, 6, 600, 20, (256, 256), 128),
]


@pytest.mark.parametrize("case", DEFAULTS, ids=[c[0] for c in DEFAULTS])
def test_default_chunks_of_256_become_512(case):
    """General calls with default chunks, in a workspace of the size that the shape has: the results, and the bits of a call that names chunks of 512."""
    name, prompts, samples, Hq, Hkv, prefix_pages, suffix_pages, chunks, block = case
    print("case: fp8 attention, default chunks,", name, flush=True)
    rng = np.random.default_rng(samples)
    gos = rng.permutation(np.repeat(np.arange(len(prompts)), samples))
    slens = rng.choice([0, 1, 64, 127, 128, 129, 200, 256, 257, 320], size=len(gos))
    slens[:4] = [320, 300, 0, 257]
    inp = widen(custom_inputs(prompts, slens, gos, Hq, Hkv, seed=samples), prefix_pages, suffix_pages)
    c, got = check(inp)
    assert c.stages() == GENERAL
    call = B.prepare_attn(c.dev, B.MARL_OUT_F32)
    L = B.marl_attn_plan_layout_for(call.shape)
    assert (L.suffix_chunk_tokens, L.prefix_chunk_tokens, L.rows_per_qblock) == (*chunks, block)
    assert call.workspace.numel() == B.marl_workspace_bytes(call.shape) == L.total_bytes
    named, _ = c.run(suffix_chunk_tokens=512, prefix_chunk_tokens=max(512, chunks[1]))
    assert np.array_equal(got, named)
    # the bf16 call on the same values: weights are rounded alike, only the sums' order differs
    dev = c.bf16.to("cuda")
    other = B.prepare_attn(dev, B.MARL_OUT_F32)
    B.run_attn(dev, other)
    torch.cuda.synchronize()
    assert (np.abs(got - other.out.cpu().numpy()) <= 2 * (2.0 ** -8 + 2.0 ** -12) * c.magnitude()).all()


@pytest.mark.parametrize("prompt,samples,Hq,Hkv", [(20001, 3, 4, 1), (40000, 3, 14, 2), (16200, 20, 4, 1), (36999, 40, 4, 2), (20500, 100, 4, 2)])
def test_prefix_items_of_more_than_256_steps(prompt, samples, Hq, Hkv):
    """Named prefix chunks of 65536 tokens: the list of an item's blocks, which holds 256 steps, is filled again while it runs; one to eight row tiles, and blocks of 256 rows."""
    print("case: fp8 attention, long prefix items", prompt, samples, flush=True)
    rng = np.random.default_rng(samples)
    inp = custom_inputs([prompt, 16140], rng.integers(0, 140, samples + 2), [0] * samples + [1, 1], Hq, Hkv, seed=prompt)
    check(inp, suffix_chunk_tokens=512, prefix_chunk_tokens=65536)


@pytest.mark.parametrize("prefix_chunk", [96, 8192])
def test_large_values_under_large_weights(prefix_chunk):
    """Values just below 2^100, where results are finite by the header: a prefix whose scores rise by 4.9 after its first tokens, so that weights reach 30 and lanes' sums
    240 of the 256 that they may have before the reference maximum moves."""
    print("case: fp8 attention, large values", prefix_chunk, flush=True)
    inp = custom_inputs([6000, 700], [0, 50, 3, 129], [0, 0, 1, 1], 14, 2, seed=8, poison=False)
    inp.q[:] = 0.0
    inp.q[:, :, 0] = 1.0
    inp.scale = 4.9 / 1.4426950408889634
    for g, n in ((0, 6000), (1, 700)):
        pages = inp.prefix_block_table[g, : -(-n // 16)].long()
        inp.k_pages[pages] = 1.0
        inp.k_pages[pages[:6]] = 0.0
    c = Cache(inp, spread=False)
    c.ex[:, :, 1, :] = 91
    v = c.v.view(torch.uint8)
    v |= 0x70                                              # codes of 128 to 448
    v &= 0x7f
    v[v == 0x7f] = 0x7e
    c.bf16.v_pages = torch.from_numpy(fp8.values(v.cpu().numpy(), c.ex.cpu().numpy()).astype(np.float32)).to(torch.bfloat16)
    for chunks in ({}, dict(suffix_chunk_tokens=64, prefix_chunk_tokens=prefix_chunk)):
        got, _ = c.run(**chunks)
        assert np.isfinite(got).all() and np.abs(got).max() > 2.0 ** 97
        assert (np.abs(got - c.want()) <= (2.0 ** -8 + 2.0 ** -12) * c.magnitude()).all()
