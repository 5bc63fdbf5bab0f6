"""Decode attention over an 8-bit cache against the float64 oracle on the values that the codes stand for, by every kernel route.

Tolerance, element by element, from the operation: a weight is rounded to bf16 before it multiplies its value (to nearest of 8 significant bits: up to 2^-8 of it),
and has the float32 error of its score, at most 128 * 2^-24 of the sum of |q k| scale (about 10 here, 80 with scale 1: 2^-13 and 2^-10 of the weight at
most); so the error is at most (2^-8 + 2^-12) (scale 1: 2^-8 + 2^-10) of the weighted mean of the values' magnitudes, which the oracle gives for the magnitudes as values.
A bf16 output is rounded once more, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from paper_2602_09578_amd import binding as B
from paper_2602_09578_amd import inputs as I
from oracle import reference as ref
from tests import fp8_cache_ref as fp8
from tests.gpu_common import oracle_attn
from tests.helpers import to_bf16_bits
from tests.test_gpu_attn import custom_inputs

pytestmark = pytest.mark.gpu


class Cache:
    """A bf16 problem with its pages quantised: codes and exponents on the GPU, the values they stand for as a bf16 problem again."""

    def __init__(self, inp, seed=0, spread=True):
        rng = np.random.default_rng(seed)
        k, v = inp.k_pages.float().numpy().astype(np.float64), inp.v_pages.float().numpy().astype(np.float64)
        if spread:   # tokens of many magnitudes; keys of at most twice theirs, so that scores stay in range
            k = k * np.exp2(rng.integers(-6, 2, k.shape[:3]))[..., None]
            v = v * np.exp2(rng.integers(-9, 10, (v.shape[0], v.shape[1], v.shape[3])))[:, :, None, :]
        kc, ke = fp8.quantize(k)
        vc, ve = fp8.quantize(v.transpose(0, 1, 3, 2))
        vc = np.ascontiguousarray(vc.transpose(0, 1, 3, 2))
        ex = np.ascontiguousarray(np.stack([ke, ve], 2))
        unused = np.isnan(k).any(-1)                                 # rows that no token owns: any exponent
        ex = np.where(np.stack([unused, unused], 2), rng.integers(-128, 128, ex.shape), ex).astype(np.int8)
        self.bf16 = I.AttnInputs(**{**inp.__dict__, "k_pages": self._bf16(fp8.keys(kc, ex), unused[..., None]),
                                    "v_pages": self._bf16(fp8.values(vc, ex), unused[:, :, None, :])})
        self.dev = inp.to("cuda")
        self.k, self.v, self.ex = torch.from_numpy(kc).cuda().view(B.FP8), torch.from_numpy(vc).cuda().view(B.FP8), torch.from_numpy(ex).cuda()

    @staticmethod
    def _bf16(x, unused):
        x = np.where(unused, np.nan, x)
        t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
        assert torch.equal(torch.nan_to_num(t.double()), torch.nan_to_num(torch.from_numpy(x)))   # (a stored value is a bf16 number)
        return t

    def want(self):
        return oracle_attn(self.bf16)

    def magnitude(self):
        return oracle_attn(I.AttnInputs(**{**self.bf16.__dict__, "v_pages": self.bf16.v_pages.abs()}))

    def run(self, out_dtype=B.MARL_OUT_F32, flags=0, **chunks):
        d = self.dev
        call = B.prepare_attn(d, out_dtype, **chunks)
        call.workspace.fill_(0xFF)
        call.out.fill_(float("nan"))
        B.marl_decode_attn_fp8(call.shape, call.workspace, d.q, self.k, self.v, self.ex, d.prefix_block_table, d.suffix_block_table,
                               d.prefix_lens, d.suffix_lens, d.group_of_seq, d.scale, call.out)
        torch.cuda.synchronize()
        assert B.marl_attn_read_flags(call.workspace) == flags
        return call.out.float().cpu().numpy().astype(np.float64), call

    def stages(self, **chunks):
        d = self.dev
        call = B.prepare_attn(d, B.MARL_OUT_F32, **chunks)
        B.marl_profile_begin(1)
        B.marl_decode_attn_fp8(call.shape, call.workspace, d.q, self.k, self.v, self.ex, d.prefix_block_table, d.suffix_block_table,
                               d.prefix_lens, d.suffix_lens, d.group_of_seq, d.scale, call.out)
        ms, n, _ = B.marl_profile_end()
        assert n == 1
        return {k for k in ("plan", "prefix", "suffix", "merge") if ms[k] > 0}


def check(inp, seed=0, weight=2.0 ** -8 + 2.0 ** -12, **chunks):
    c = Cache(inp, seed)
    want, magnitude = c.want(), c.magnitude()
    got, _ = c.run(**chunks)
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / (weight * magnitude + 1e-30)).max()
    assert worst <= 1.0, f"{worst} of the tolerance"
    again, _ = c.run(**chunks)
    assert np.array_equal(got, again)
    return c, got


RAGGED = ([0, 1, 16, 17, 31, 33, 300], [0, 5, 16, 31, 32, 33, 0, 64, 65, 1, 100, 0], [0, 1, 2, 3, 4, 5, 6, 6, 5, 2, 1, 5])
STEPS = ([47, 48, 49, 63, 64, 65, 127, 128, 129], [63, 64, 65, 127, 128, 129, 255, 256, 257, 47, 48, 49], [0, 1, 2, 3, 4, 5, 6, 7, 8, 0, 1, 2])
SMALL, PARTS = {"prefix"}, {"prefix", "merge"}
CASES = [
    ("ragged, one row per head", *RAGGED, 4, 4, SMALL),
    ("ragged, sixteen rows", *RAGGED, 16, 1, SMALL),
    ("around steps", *STEPS, 14, 2, SMALL),
    ("one token", [0], [1], [0], 7, 1, SMALL),
    ("no tokens at all", [0], [0, 0], [0, 0], 8, 2, SMALL),
    ("no tokens of their own", [40, 70], [0, 0, 0], [0, 1, 1], 28, 4, SMALL),
    ("parts without a step", [0, 6000], [1, 0, 40, 129], [0, 0, 1, 1], 12, 4, PARTS),
    ("one sequence, parts of eight heads", [100], [2300], [0], 16, 8, PARTS),
    ("nine sequences, five heads, parts", [600], [500 - s for s in range(9)], [0] * 9, 5, 5, PARTS),
    ("long rows", [16] * 2, [24000] + [9 + s for s in range(63)], [s % 2 for s in range(64)], 1, 1, PARTS),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_small_calls(case):
    name, pl, sl, gos, Hq, Hkv, stages = case
    print("case: fp8 attention, small call:", name, flush=True)
    c, _ = check(custom_inputs(pl, sl, gos, Hq, Hkv, seed=len(name)))
    assert c.stages() == stages


GENERAL = [dict(suffix_chunk_tokens=8192, prefix_chunk_tokens=8192), dict(suffix_chunk_tokens=64, prefix_chunk_tokens=96), dict(suffix_chunk_tokens=32, prefix_chunk_tokens=32)]


@pytest.mark.parametrize("chunks", GENERAL, ids=lambda c: str(c["suffix_chunk_tokens"]))
@pytest.mark.parametrize("lens", [RAGGED, STEPS], ids=["ragged", "steps"])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (16, 1), (28, 4), (9, 3)])
def test_items(lens, Hq, Hkv, chunks):
    """Prefix and suffix items of one queue: chunks that are less than a step, whole steps and ragged."""
    print("case: fp8 attention, items", Hq, Hkv, chunks, flush=True)
    c, _ = check(custom_inputs(*lens, Hq, Hkv, seed=Hq), **chunks)
    assert "plan" in c.stages(**chunks)


@pytest.mark.parametrize("samples,Hq,Hkv", [(5, 28, 4), (24, 28, 4), (40, 14, 2), (3, 16, 1)])
def test_kinds_of_items(samples, Hq, Hkv):
    """Long and short suffix items beside prefix items, in blocks of 128 and of 256 rows."""
    print("case: fp8 attention, kinds of items", samples, flush=True)
    rng = np.random.default_rng(samples)
    gos = rng.permutation(np.repeat(np.arange(4), samples))
    slens = rng.choice([0, 1, 63, 64, 127, 128, 129, 160, 161, 511, 512, 513, 600, 1100], size=len(gos))
    slens[:3] = [1100, 0, 640]
    inp = custom_inputs([0, 65, 97, 1029], slens, gos, Hq, Hkv, seed=samples)
    for chunks in (dict(suffix_chunk_tokens=512, prefix_chunk_tokens=96), dict(suffix_chunk_tokens=64, prefix_chunk_tokens=32),
                   dict(suffix_chunk_tokens=256, prefix_chunk_tokens=512)):
        check(inp, **chunks)


@pytest.mark.parametrize("seqs,Hkv,samples", [(769, 8, 19), (1600, 4, 40), (1700, 4, 5)])
def test_many_pairs(seqs, Hkv, samples):
    """More than 6144 (sequence, KV head) pairs, narrow and wide blocks: still one queue."""
    print("case: fp8 attention, many pairs", seqs, Hkv, flush=True)
    rng = np.random.default_rng(seqs)
    groups = -(-seqs // samples)
    slens = rng.integers(0, 90, seqs)
    slens[rng.permutation(seqs)[:60]] = rng.integers(129, 700, 60)
    c, _ = check(custom_inputs(rng.integers(0, 150, groups), slens, rng.permutation(np.arange(seqs) % groups), 7 * Hkv, Hkv, seed=seqs), suffix_chunk_tokens=512)
    assert c.stages(suffix_chunk_tokens=512) == {"plan", "suffix", "merge"}


@pytest.mark.parametrize("members,alone,Hq,Hkv", [(150, 12, 4, 4), (70, 0, 14, 2), (80, 0, 4, 2), (69, 2, 28, 4)])
def test_a_row_does_not_depend_on_its_place(members, alone, Hq, Hkv):
    """Samples of one prompt in another order, in groups larger than the plan puts in order (64): the same bits for each, in blocks of 128 and of 256 rows
    and in what is left after them."""
    print("case: fp8 attention, order of rows", members, Hq, flush=True)
    rng = np.random.default_rng(members)
    slens = rng.integers(0, 150, members + alone)
    gos = np.concatenate([np.zeros(members, int), 1 + np.arange(alone)])
    c = Cache(custom_inputs([777] + [40] * alone, slens, gos, Hq, Hkv, seed=members))
    chunks = dict(suffix_chunk_tokens=256, prefix_chunk_tokens=256)
    got, _ = c.run(**chunks)
    order = torch.from_numpy(rng.permutation(members + alone))
    d = c.dev
    c.dev = I.AttnInputs(**{**d.__dict__, **{k: getattr(d, k)[order.cuda()].contiguous() for k in ("q", "suffix_block_table", "suffix_lens", "group_of_seq")}})
    again, _ = c.run(**chunks)
    assert np.array_equal(again, got[order.numpy()])


@pytest.mark.parametrize("seqs,samples,prefix,chunk,Hq", [
    (160, 160, [0], 32, 8),                                  # no prefix at all
    (160, 4, list(range(1, 128, 3))[:40], 32, 8),            # up to four chunks a group
    (200, 2, [128] * 100, 32, 4),                            # more prefix items than any two rounds of workgroups
    (160, 80, [100, 33], 64, 8),                             # blocks of 256 query rows
    (131, 131, [40], 64, 8)])
def test_few_long_items_among_many(seqs, samples, prefix, chunk, Hq):
    """Three suffix items that would end long after all others (4 KV heads, so 640 items and more): the kinds of items are drawn apart.
    (131 sequences: 524 items.)"""
    print("case: fp8 attention, few long items", seqs, len(prefix), flush=True)
    rng = np.random.default_rng(seqs + len(prefix))
    slens = rng.integers(129, 200, seqs)
    slens[rng.permutation(seqs)[:3]] = [6000, 5003, 4100]
    gos = rng.permutation(np.arange(seqs) // samples)
    check(custom_inputs(prefix, slens, gos, Hq, 4, seed=seqs), suffix_chunk_tokens=8192, prefix_chunk_tokens=chunk)


@pytest.mark.parametrize("name,pdiv,ldiv", [("tiny", 1, 1), ("qwen7b", 16, 4), ("skew", 8, 8), ("prefix", 16, 4), ("long32b", 8, 8)])
def test_scaled_workloads(name, pdiv, ldiv):
    print("case: fp8 attention", name, flush=True)
    c, f32 = check(I.build_attn_inputs(I.WORKLOADS[name].scaled(pdiv, ldiv)))
    bf16, _ = c.run(B.MARL_OUT_BF16)
    assert np.all(np.abs(bf16 - f32) <= np.abs(f32) * 2.0 ** -8 + 1e-30)   # one rounding apart


@pytest.mark.parametrize("scale", [-0.11, 0.0, 1.0])
@pytest.mark.parametrize("chunks", [{}, GENERAL[1]], ids=["small", "items"])
def test_scales(scale, chunks):
    print("case: fp8 attention, scale", scale, flush=True)
    check(custom_inputs([90, 40], [33, 7, 129, 64], [0, 0, 1, 1], 28, 4, seed=21, scale=scale),
          weight=2.0 ** -8 + 2.0 ** -10 if scale == 1.0 else 2.0 ** -8 + 2.0 ** -12, **chunks)


@pytest.mark.parametrize("chunks", [{}, GENERAL[1]], ids=["small", "items"])
def test_extreme_magnitudes(chunks):
    """Values of the largest and the smallest exponents beside each other, infinitely far apart for a bf16 weight."""
    inp = custom_inputs([70], [40, 3], [0, 0], 8, 2, seed=6, poison=False)
    for e in (-108, 100):
        c = Cache(inp, spread=False)
        c.ex[:, :, 1, :] = e
        c.bf16.v_pages = torch.from_numpy(fp8.values(c.v.view(torch.uint8).cpu().numpy(), c.ex.cpu().numpy()).astype(np.float32)).to(torch.bfloat16)
        got, _ = c.run(**chunks)
        assert (np.abs(got - c.want()) <= (2.0 ** -8 + 2.0 ** -12) * c.magnitude()).all()


def test_no_group_and_bad_contents():
    """Group ids, lengths and pages out of range are clamped and flagged as by the bf16 call."""
    print("case: fp8 attention, bad contents", flush=True)
    inp = custom_inputs([40, 100], [33, 70, 5, 200], [0, 1, 1, 0], 8, 2, seed=3, poison=False)
    for chunks in ({}, GENERAL[1]):
        for change, flag in (("group", B.FLAG_BAD_GROUP), ("length", B.FLAG_LEN_CLAMPED), ("page", B.FLAG_BAD_PAGE)):
            c = Cache(inp)
            want = c.want()
            rows = slice(None)
            if change == "group":
                c.dev.group_of_seq[2] = 9
                rows = [0, 1, 3]
            elif change == "length":
                c.dev.suffix_lens[1] = -4
                rows = [0, 2, 3]
            else:
                c.dev.suffix_block_table[3, 1] = inp.num_pages
                rows = [0, 1, 2]
            got, _ = c.run(flags=flag, **chunks)
            assert np.isfinite(got).all()
            assert (np.abs(got - want)[rows] <= (2.0 ** -8 + 2.0 ** -12) * c.magnitude()[rows]).all()


def test_against_the_bf16_call():
    """The same values in both caches: only the order of the sums differs, weights are rounded alike."""
    c = Cache(I.build_attn_inputs(I.WORKLOADS["qwen7b"].scaled(16, 4)))
    dev = c.bf16.to("cuda")
    call = B.prepare_attn(dev, B.MARL_OUT_F32)
    B.run_attn(dev, call)
    torch.cuda.synchronize()
    got, _ = c.run()
    assert (np.abs(got - call.out.cpu().numpy()) <= 2 * (2.0 ** -8 + 2.0 ** -12) * c.magnitude()).all()


def test_pages_past_four_gigabytes():
    """Codes at offsets that do not fit 32 bits."""
    print("case: fp8 attention, far pages", flush=True)
    Hkv, pages = 8, (1 << 32) // (8 * 2048) + 40
    inp = custom_inputs([70, 3], [40, 300, 1], [0, 1, 1], 16, Hkv, seed=9)
    near = Cache(inp)
    want, _ = near.run()
    far = torch.zeros(pages, Hkv, 16, 128, dtype=torch.uint8, device="cuda"), torch.zeros(pages, Hkv, 128, 16, dtype=torch.uint8, device="cuda")
    ex = torch.zeros(pages, Hkv, 2, 16, dtype=torch.int8, device="cuda")
    n = inp.num_pages
    far[0][-n:], far[1][-n:], ex[-n:] = near.k.view(torch.uint8), near.v.view(torch.uint8), near.ex
    d = near.dev
    move = lambda t: torch.where(t >= 0, t + (pages - n), t).int()
    shape = B.make_shape(3, 2, 16, Hkv, pages, d.prefix_block_table.shape[1], d.suffix_block_table.shape[1], B.MARL_OUT_F32)
    for chunks in ((0, 0), (64, 96)):
        shape.suffix_chunk_tokens, shape.prefix_chunk_tokens = chunks
        ws, out = B.alloc_workspace(B.marl_workspace_bytes(shape), "cuda"), torch.empty(3, 16, 128, device="cuda")
        B.marl_decode_attn_fp8(shape, ws, d.q, far[0].view(B.FP8), far[1].view(B.FP8), ex, move(d.prefix_block_table), move(d.suffix_block_table),
                               d.prefix_lens, d.suffix_lens, d.group_of_seq, d.scale, out)
        torch.cuda.synchronize()
        if chunks == (0, 0):
            assert np.array_equal(out.cpu().numpy(), want)
        else:
            near_general, _ = near.run(suffix_chunk_tokens=64, prefix_chunk_tokens=96)
            assert np.array_equal(out.cpu().numpy(), near_general)


def test_a_captured_step_replays():
    """Norm and rotation, append and attention of a decode step in a graph, replayed with other inputs and eager work in between."""
    print("case: fp8 attention, graph", flush=True)
    NS, Hq, Hkv, pages = 12, 8, 2, 60
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()
    cache = B.alloc_kv_fp8(pages, Hkv, "cuda")
    qkv, w = rnd(NS, (Hq + 2 * Hkv) * 128), rnd(128)
    ptab, stab = i32(torch.arange(12).view(3, 4)), i32(12 + torch.arange(48).view(12, 4))
    plens, lens, pos, gos = i32([64, 33, 0]), i32([0] * 12), i32([0] * 12), i32([s % 3 for s in range(12)])
    cs = torch.cat([torch.cos(torch.arange(512)[:, None] * 0.1 ** (torch.arange(64) / 16)), torch.sin(torch.arange(512)[:, None] * 0.1 ** (torch.arange(64) / 16))], 1).float().cuda()
    pshape = B.make_prefill_shape(97, 3, Hq, Hkv, pages, 4)
    B.marl_kv_write_prompt_fp8(pshape, rnd(97, Hkv, 128), rnd(97, Hkv, 128), *cache, ptab, i32([0, 64, 97, 97]), i32([0, 0, 0]))
    shape = B.make_shape(NS, 3, Hq, Hkv, pages, 4, 4, B.MARL_OUT_F32)
    ws = B.alloc_workspace(B.marl_workspace_bytes(shape), "cuda")
    q, k = qkv[:, : Hq * 128].view(NS, Hq, 128), qkv[:, Hq * 128: (Hq + Hkv) * 128].view(NS, Hkv, 128)
    q_out, k_out, v, out = torch.empty(NS, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(NS, Hkv, 128, dtype=torch.bfloat16, device="cuda"), \
        torch.empty(NS, Hkv, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(NS, Hq, 128, device="cuda")

    def step():
        v.copy_(qkv[:, (Hq + Hkv) * 128:].view(NS, Hkv, 128))
        B.marl_qk_norm_rope(q, k, w, w, cs, pos, 1e-6, q_out, k_out)
        B.marl_kv_append_fp8(shape, k_out, v, *cache, stab, lens)
        B.marl_decode_attn_fp8(shape, ws, q_out, *cache, ptab, stab, plens, lens, gos, 0.09, out)
        pos.add_(1)

    start = [t.clone() for t in (*cache, lens, pos)]
    restore = lambda: [d.copy_(s) if d.dtype != B.FP8 else d.view(torch.uint8).copy_(s.view(torch.uint8)) for d, s in zip((*cache, lens, pos), start)]
    inputs = [rnd(NS, (Hq + 2 * Hkv) * 128) for _ in range(5)]
    eager = []
    for x in inputs:
        qkv.copy_(x)
        step()
        eager.append(out.clone())
    final = [t.clone() for t in (*cache, lens, pos)]
    restore()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    restore()
    for x, want in zip(inputs, eager):
        qkv.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        (qkv.float() @ qkv.float().t()).sum().item()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((*cache, lens, pos), final))


def test_bad_arguments_are_refused():
    c = Cache(custom_inputs([20], [5, 6], [0, 0], 8, 2, seed=1, poison=False))
    d = c.dev
    call = B.prepare_attn(d, B.MARL_OUT_F32)
    right = [d.q, c.k, c.v, c.ex, d.prefix_block_table, d.suffix_block_table, d.prefix_lens, d.suffix_lens, d.group_of_seq, d.scale, call.out]
    for k, w in ((0, d.q.float()), (1, d.k_pages), (1, c.k.view(torch.uint8)), (2, c.v[:-1]), (3, c.ex.int()), (3, c.ex[:, :, :1]), (4, d.prefix_block_table.long()),
                 (7, d.suffix_lens.cpu()), (10, call.out.half()), (3, None), (1, None)):
        bad = list(right)
        bad[k] = w
        with pytest.raises((ValueError, AttributeError, B.MarlError)):
            B.marl_decode_attn_fp8(call.shape, call.workspace, *bad)
    with pytest.raises(B.MarlError):
        B.marl_decode_attn_fp8(call.shape, call.workspace, *right[:9], float("nan"), call.out)
    with pytest.raises(B.MarlError):
        B.marl_decode_attn_fp8(call.shape, call.workspace[:256], *right)
