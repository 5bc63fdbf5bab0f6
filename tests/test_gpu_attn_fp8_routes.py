"""Decode attention over an 8-bit cache: which kernels a call takes, and its results where those are the general ones with default chunks.

The tolerance is that of tests/test_gpu_attn_fp8.py."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from paper_2602_09578_amd import inputs as I
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
