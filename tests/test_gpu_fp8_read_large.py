"""Pages of an 8-bit cache read back in calls of more than 32 MB, whose results are stored past the caches."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests import fp8_cache_ref as ref
from tests.test_gpu_fp8_cache import f64, on_gpu, poisoned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,Hkv", [(4100, 1), (1500, 3)])
def test_read_many_pages(n, Hkv):
    print("case: fp8 read, many pages", n, Hkv, flush=True)
    assert n * Hkv * 8192 > 32 << 20
    rng = np.random.default_rng(n)
    pages, out_pages = n // 3, n + 5                        # (a source may serve several pages)
    k, v, _ = poisoned(pages, Hkv, n)
    ex = rng.integers(-110, 119, (pages, Hkv, 2, 16)).astype(np.int8)
    src, dst = rng.integers(0, pages, n).astype(np.int32), rng.permutation(out_pages)[:n].astype(np.int32)
    src[[7, n - 1]], dst[1234] = (-1, pages), out_pages
    good = (src >= 0) & (src < pages) & (dst < out_pages)
    want = np.full((out_pages, Hkv, 16, 128), 5.0), np.full((out_pages, Hkv, 128, 16), 5.0)
    want[0][dst[good]] = ref.keys(k.numpy(), ex)[src[good]]
    want[1][dst[good]] = ref.values(v.numpy(), ex)[src[good]]
    out = [torch.full(w.shape, 5.0, dtype=torch.bfloat16, device="cuda") for w in want]
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.marl_kv_read_pages_fp8(*on_gpu(k, v, torch.from_numpy(ex)), torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(), *out, flags)
    torch.cuda.synchronize()
    assert all(np.array_equal(f64(o), w, equal_nan=True) for o, w in zip(out, want)) and int(flags) == B.FLAG_BAD_PAGE
