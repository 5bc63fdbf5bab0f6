"""The prompt scatter into an 8-bit cache on each way that its launch has, bit for bit against the cache's definition."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests import fp8_cache_ref as ref
from tests.test_gpu_fp8_cache import f64, on_gpu, poisoned, rows, same

pytestmark = pytest.mark.gpu


def way(NT, NG, Hkv, cols):
    """The launch's rule, to know that a case takes the way that it is here for; and the workgroups of a (group, KV head)."""
    every, places, mean = min(cols, NT // 16 + 2), NT // 16 + 2 * NG, -(-NT // (16 * NG))
    few_empty = NG * every * Hkv <= 2048 or NG * every <= (4 if places * Hkv >= 8192 else 2) * places
    taken = every if few_empty else min(every, 2 * mean + 2)
    if not few_empty and -(-every // taken) * 8800 > places * Hkv * 3 and NG <= 1024:
        return "places", 0
    taken = min(taken, ((1 << 25) - 1) // (NG * Hkv))
    return ("columns" if taken == every else "rounds"), taken


def check(Hkv, chunks, ctx, want_way, cols=None, start=None, bad_pages=(), flag=0):
    chunks, ctx = np.asarray(chunks), np.asarray(ctx)
    NG, NT = len(chunks), int(chunks.sum())
    start = np.concatenate([[0], np.cumsum(chunks)]) if start is None else np.asarray(start)
    n = np.diff(start)
    cols = cols or int((-(-(chunks + ctx) // 16)).max())
    rng = np.random.default_rng(NG)
    # pages for the columns that a chunk touches, of the consistent groups
    groups = np.nonzero(n > 0)[0]
    columns = [(g, c) for g in groups for c in range(ctx[g] // 16, (ctx[g] + n[g] - 1) // 16 + 1)]
    pages = len(columns) + 5
    table = np.full((NG, cols), -1, np.int32)
    for (g, c), page in zip(columns, rng.permutation(pages)):
        table[g, c] = page
    for g, c in bad_pages:
        table[g, c] = pages
    host = [t.numpy().copy() for t in poisoned(pages, Hkv, NG)]
    dev = on_gpu(*(torch.from_numpy(h.copy()) for h in host))
    kn, vn = rows((NT, Hkv), 31), rows((NT, Hkv), 32)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    shape = B.make_prefill_shape(NT, NG, Hkv, Hkv, pages, cols)
    assert way(NT, NG, Hkv, cols)[0] == want_way
    B.marl_kv_write_prompt_fp8(shape, kn.cuda(), vn.cuda(), *dev, cuda(table), cuda(start), cuda(ctx), flags)
    (kc, ke), (vc, ve) = ref.quantize(f64(kn)), ref.quantize(f64(vn))
    token = np.concatenate([start[g] + np.arange(n[g]) for g in groups])
    pos = np.concatenate([ctx[g] + np.arange(n[g]) for g in groups])
    page = table[np.repeat(groups, n[groups]), pos // 16]
    keep = page < pages
    token, page, slot = token[keep], page[keep][:, None], (pos % 16)[keep][:, None]
    heads = np.arange(Hkv)[None]
    host[0][page, heads, slot], host[2][page, heads, 0, slot] = kc[token], ke[token]
    host[1][page, heads, :, slot], host[2][page, heads, 1, slot] = vc[token], ve[token]
    torch.cuda.synchronize()
    same(dev, host)
    assert int(flags) == flag


CASES = [
    # by places: up to the groups that a wave sees at once, one more, and the most that it is done for
    ("one long chunk among single tokens", 8, [900] + [1] * 31, [0] * 32, "places"),
    ("few columns of wide tables", 8, [18, 2, 34, 1, 14, 3, 16], [15, 15, 31, 4000, 2, 14, 16], "columns"),
    ("64 groups", 4, [2000] + [1] * 63, [3] + [900] * 63, "places"),
    ("65 groups", 4, [1] * 64 + [2000], [900] * 64 + [15], "places"),
    ("1024 groups", 2, [1] * 500 + [1500] + [2, 17, 0] * 174 + [18], [95] * 1024, "places"),
    # a chunk's workgroups go round
    ("1025 groups", 2, [1] * 500 + [1500] + [2, 17, 0] * 174 + [18] * 2, [95] * 1025, "rounds"),
    ("a chunk of more than twice the mean", 4, [700] * 30 + [1500], [300] * 31, "rounds"),
    ("every column", 4, [700] * 30 + [650], [300] * 31, "columns"),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_ways(case):
    print("case: fp8 prompt,", case[0], flush=True)
    check(*case[1:])


@pytest.mark.parametrize("groups,Hkv", [(40, 2), (80, 2)])
def test_groups_that_share_rows(groups, Hkv):
    """By places, where several groups have the same rows: every consistent one has its pages written, one after the other by the same workgroups."""
    print("case: fp8 prompt, shared rows", groups, flush=True)
    start = np.zeros(groups + 1, int)
    start[1:groups:2] = 21
    check(Hkv, [21] * groups, [979] * groups, "places", start=start, flag=B.FLAG_BAD_GROUP)


@pytest.mark.parametrize("groups", [32, 100])
def test_pages_that_are_none(groups):
    """By places: pages that do not exist among those that do, in the middle and at the end of chunks."""
    print("case: fp8 prompt, bad pages", groups, flush=True)
    check(8, [900] + [33] * (groups - 1), [0] + [2000] * (groups - 1), "places",
          bad_pages=[(0, 3), (0, 4), (0, 56), (5, 125), (9, 127), (groups - 1, 126)], flag=B.FLAG_BAD_PAGE)


def test_more_columns_than_a_launch_has_workgroups():
    """Half a million groups of eight columns, eight KV heads: one column too many for a launch, so a chunk of eight goes round."""
    print("case: fp8 prompt, 2^19 groups", flush=True)
    NG = 1 << 19
    chunks, ctx = np.zeros(NG, int), np.zeros(NG, int)
    chunks[[7, 8, 300000, NG - 1]], ctx[[7, 300000, NG - 1]] = [120, 1, 40, 128], [3, 80, 0]
    assert way(int(chunks.sum()), NG, 8, 8)[1] == 7
    check(8, chunks, ctx, "rounds")
