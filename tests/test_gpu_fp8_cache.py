"""The 8-bit KV cache on the GPU, bit for bit against its definition: appended tokens, prompts, pages read back."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from tests import fp8_cache_ref as ref

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(shape, seed):
    """bf16 rows [.., 128] of many magnitudes, with what can go wrong among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, 128, generator=g) * torch.exp2(torch.randint(-12, 12, (*shape, 1), generator=g).float())
    flat = x.view(-1, 128)
    for k in range(min(len(flat), 400)):
        r = flat[(7 * k) % len(flat)]
        kind = k % 16
        if kind == 0: r.zero_()
        if kind == 1: r[5], r[9] = float("inf"), -float("inf")
        if kind == 2: r[0] = float("nan")
        if kind == 3: r[:] = float("inf")
        if kind == 4: r[:] = 3.3895e38
        if kind == 5: r *= 2.0 ** -118                     # below the smallest exponent
        if kind == 6: r *= 2.0 ** -30 * (1.0 - 2.0 * (torch.arange(128) % 2))
        if kind == 7: r[100] = 1e20                        # everything else rounds to nothing
        if kind == 8: r[:] = torch.arange(128) * 7 / 4.0   # ties
        if kind == 9: r[:] = 1.75 * 2.0 ** (k % 200 - 100)       # a power of two below and above the largest code
        if kind == 10: r[:] = -1.7578125 * 2.0 ** (k % 200 - 100)
        if kind == 11: r[3] = -0.0
        if kind == 12: r[:] = float("nan")
        if kind == 13: r[:] = 1e-40                        # subnormal bf16 numbers
    return x.to(torch.bfloat16)


def poisoned(pages, Hkv, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randint(0, 256, s, generator=g, dtype=torch.int16).to(torch.uint8)
    return r(pages, Hkv, 16, 128), r(pages, Hkv, 128, 16), r(pages, Hkv, 2, 16).view(torch.int8)


def on_gpu(k, v, ex):
    return k.cuda().view(B.FP8), v.cuda().view(B.FP8), ex.cuda()


def same(dev, host):
    for d, h in zip(dev, host):
        assert np.array_equal(d.view(torch.uint8).cpu().numpy(), h.view(np.uint8))


@pytest.mark.parametrize("NS,Hkv", [(1, 1), (5, 3), (64, 8), (40, 9), (33, 17), (300, 4)])
def test_append(NS, Hkv):
    print("case: fp8 append", NS, Hkv, flush=True)
    rng = np.random.default_rng(NS + Hkv)
    cols = 3
    pages = NS * cols + 2
    host = [t.numpy().copy() for t in poisoned(pages, Hkv, NS)]
    dev = on_gpu(*(torch.from_numpy(h.copy()) for h in host))
    table = rng.permutation(pages)[: NS * cols].reshape(NS, cols).astype(np.int32)
    lens = rng.integers(0, cols * 16 - 4, NS).astype(np.int32)
    want_flags = 0
    if NS > 3:
        lens[1], lens[2] = cols * 16, -3                    # full; no length
        table[3, lens[3] // 16] = pages
        want_flags = B.FLAG_LEN_CLAMPED | B.FLAG_BAD_PAGE
    shape = B.make_shape(NS, 1, Hkv, Hkv, pages, 1, cols)
    lens_dev, table_dev, flags = torch.from_numpy(lens).cuda(), torch.from_numpy(table).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    for step in range(3):
        kn, vn = rows((NS, Hkv), 10 * step + 1), rows((NS, Hkv), 10 * step + 2)
        B.marl_kv_append_fp8(shape, kn.cuda(), vn.cuda(), *dev, table_dev, lens_dev, flags)
        for s in range(NS):
            if 0 <= lens[s] < cols * 16 and table[s, lens[s] // 16] < pages:
                ref.store(*host, table[s, lens[s] // 16], lens[s] % 16, f64(kn[s]), f64(vn[s]))
                lens[s] += 1
    torch.cuda.synchronize()
    same(dev, host)
    assert np.array_equal(lens_dev.cpu().numpy(), lens) and int(flags) == want_flags


@pytest.mark.parametrize("Hkv,chunks,ctx", [
    (1, [1], [0]), (2, [16], [0]), (2, [33, 1, 15], [0, 5, 17]), (8, [20, 16, 64, 3], [3, 16, 0, 13]), (3, [100, 7], [1, 250]),
    (4, [5] * 70, [11] * 70), (1, [900] + [1] * 31, [0] * 32), (2, [0, 40, 0], [4, 0, 0])])
def test_prompt(Hkv, chunks, ctx):
    print("case: fp8 prompt", Hkv, chunks[:4], flush=True)
    rng = np.random.default_rng(len(chunks))
    chunks, ctx = np.array(chunks), np.array(ctx)
    cols = int((-(-(chunks + ctx) // 16)).max())
    NG, NT = len(chunks), int(chunks.sum())
    pages = NG * cols + 3
    host = [t.numpy().copy() for t in poisoned(pages, Hkv, NT)]
    dev = on_gpu(*(torch.from_numpy(h.copy()) for h in host))
    table = rng.permutation(pages)[: NG * cols].reshape(NG, cols).astype(np.int32)
    kn, vn = rows((NT, Hkv), 3), rows((NT, Hkv), 4)
    start = np.concatenate([[0], np.cumsum(chunks)]).astype(np.int32)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = B.make_prefill_shape(NT, NG, Hkv, Hkv, pages, cols)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    B.marl_kv_write_prompt_fp8(shape, kn.cuda(), vn.cuda(), *dev, cuda(table), cuda(start), cuda(ctx), flags)
    kf, vf = f64(kn), f64(vn)
    for g in range(NG):
        for t in range(chunks[g]):
            pos = ctx[g] + t
            ref.store(*host, table[g, pos // 16], pos % 16, kf[start[g] + t], vf[start[g] + t])
    torch.cuda.synchronize()
    same(dev, host)
    assert int(flags) == 0


def test_prompt_skips_and_flags():
    """A group past its row, one with a bad start, a page that is none: the others are written whole."""
    Hkv, pages, cols = 2, 8, 2
    host = [t.numpy().copy() for t in poisoned(pages, Hkv, 5)]
    dev = on_gpu(*(torch.from_numpy(h.copy()) for h in host))
    kn, vn = rows((60, Hkv), 8), rows((60, Hkv), 9)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, 1], [2, -4], [3, 4], [5, 6]], dtype=torch.int32, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = B.make_prefill_shape(60, 4, Hkv, Hkv, pages, cols)
    B.marl_kv_write_prompt_fp8(shape, kn.cuda(), vn.cuda(), *dev, table, i32(0, 20, 40, 48, 60), i32(16, 0, -1, 3), flags)
    kf, vf = f64(kn), f64(vn)
    for first, n, pos0, row in ((0, 16, 16, (0, 1)), (20, 16, 0, (2,)), (48, 12, 3, (5, 6))):
        for t in range(n):
            pos = pos0 + t
            ref.store(*host, row[pos // 16], pos % 16, kf[first + t], vf[first + t])
    torch.cuda.synchronize()
    same(dev, host)
    assert int(flags) == B.FLAG_LEN_CLAMPED | B.FLAG_BAD_GROUP | B.FLAG_BAD_PAGE


@pytest.mark.parametrize("n,Hkv", [(1, 1), (7, 3), (40, 8)])
def test_read_pages(n, Hkv):
    """Every code under many exponents; pages that are none are left alone and flagged."""
    print("case: fp8 read", n, Hkv, flush=True)
    rng = np.random.default_rng(n)
    pages, out_pages = n + 4, n + 6
    k, v, ex = poisoned(pages, Hkv, n)
    k[0, 0], v[0, 0] = torch.arange(2048).view(16, 128).to(torch.uint8), torch.arange(2048).view(128, 16).to(torch.uint8)
    ex = torch.from_numpy(rng.integers(-110, 119, ex.shape).astype(np.int8))   # (448 * 2^119: bf16's largest is just above)
    src, dst = rng.permutation(pages)[:n].astype(np.int32), rng.permutation(out_pages)[:n].astype(np.int32)
    src[0], flags = 0, torch.zeros(1, dtype=torch.int32, device="cuda")
    want_k, want_v = np.full((out_pages, Hkv, 16, 128), 5.0), np.full((out_pages, Hkv, 128, 16), 5.0)
    if n > 5:
        src[3], dst[4] = pages, -1
    for s, d in zip(src, dst):
        if s < pages and d >= 0:
            want_k[d] = ref.keys(k.numpy()[s:s + 1], ex.numpy()[s:s + 1])
            want_v[d] = ref.values(v.numpy()[s:s + 1], ex.numpy()[s:s + 1])
    ko = torch.full((out_pages, Hkv, 16, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    vo = torch.full((out_pages, Hkv, 128, 16), 5.0, dtype=torch.bfloat16, device="cuda")
    B.marl_kv_read_pages_fp8(*on_gpu(k, v, ex), torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(), ko, vo, flags)
    torch.cuda.synchronize()
    assert np.array_equal(f64(ko), want_k, equal_nan=True) and np.array_equal(f64(vo), want_v, equal_nan=True)
    assert int(flags) == (B.FLAG_BAD_PAGE if n > 5 else 0)


def test_what_is_read_back_is_stored_as_it_is():
    """A stored row is a row of bf16 numbers that has an 8-bit form without any rounding: its own, or that of twice the codes where its
    largest code is 224."""
    Hkv, NT = 2, 160
    k = rows((NT, Hkv), 21).cuda()
    k = torch.where(torch.isfinite(k.float()), k, torch.ones_like(k))
    v = k.flip(0).contiguous()
    shape = B.make_prefill_shape(NT, 1, Hkv, Hkv, 10, 10)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    table = torch.arange(10, dtype=torch.int32, device="cuda").view(1, 10)
    read = []
    for _ in range(2):
        cache = B.alloc_kv_fp8(10, Hkv, "cuda")
        B.marl_kv_write_prompt_fp8(shape, k, v, *cache, table, i32(0, NT), i32(0))
        ko = torch.empty(10, Hkv, 16, 128, dtype=torch.bfloat16, device="cuda")
        vo = torch.empty(10, Hkv, 128, 16, dtype=torch.bfloat16, device="cuda")
        B.marl_kv_read_pages_fp8(*cache, table[0], table[0], ko, vo)
        k = ko.transpose(1, 2).reshape(NT, Hkv, 128).contiguous()
        v = vo.permute(0, 3, 1, 2).reshape(NT, Hkv, 128).contiguous()
        read.append((ko, vo))
    torch.cuda.synchronize()
    assert torch.equal(read[0][0], read[1][0]) and torch.equal(read[0][1], read[1][1])
