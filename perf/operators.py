"""The operators of an 8-bit KV cache and of what feeds it, as calls whose speed is watched.

A rollout engine that keeps its cache in 8 bits holds twice the samples and reads half the bytes.  Around it stand
  * the norm of every query and key head with the position rotation in the same pass, and its gradient,
  * writing new keys and values in 8 bits (a decode step's tokens, a prompt's tokens) and reading pages back in bf16,
  * decode attention over such a cache, with prompts shared by groups of samples.

`listed()` names the fixed cases, `draw()` gives more of the same ranges.  Where `own` is false a pass is computed from
elementary torch operations in 32 bits, rounded once at the end; where it is true by this library's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
LENS_SEED = 2048       # lengths belong to the case (its work is fixed); values and page placement to the seed
MAX_POS = 32768        # positions of the rotation's table
E4M3_MAX = 448.0
MIN_EXPONENT = -110    # smallest scale of a stored row: every stored value is then a normal bf16 number
EPS = 1e-6


# ---- the cases ---------------------------------------------------------------------------------
def listed():
    return [
        # Queries and keys of one decode step of 64 samples (4 prompts x 16): the launch is the cost.
        dict(name="norm_decode", op="norm", tokens=64, Hq=64, Hkv=8, D=128, rot=128, pairs="halves", dtype="bf16", positions="random"),
        # Those of a batch of prompts, as slices of the fused projection's output: bound by its bytes.
        dict(name="norm_prompts", op="norm", tokens=65543, Hq=28, Hkv=4, D=128, rot=128, pairs="halves", dtype="bf16", positions="runs"),
        # A training step's backward pass through them: a small float32 check run with part of each head rotated ...
        dict(name="grad_small", op="grad", tokens=333, Hq=8, Hkv=2, D=128, rot=64, pairs="adjacent", dtype="f32", positions="runs"),
        # ... and a batch of sequences in bf16.
        dict(name="grad_batch", op="grad", tokens=32771, Hq=28, Hkv=4, D=128, rot=128, pairs="halves", dtype="bf16", positions="runs"),
        # The new token of 64 samples goes into the cache.
        dict(name="append_rollout", op="append", seqs=64, Hkv=8, cols=4),
        # The prompts of one agent go into the cache, whole and ragged.
        dict(name="write_prompts", op="prompt", Hkv=4, prompts=64, chunk="uniform:512:2048", context="const:0"),
        # One short prompt's pages in bf16 again, for a further chunk of it ...
        dict(name="read_prompt", op="read", Hkv=4, pages=19),
        # ... and those of six long contexts.
        dict(name="read_contexts", op="read", Hkv=8, pages=3001),
        # One decode step of a handful of samples: two agents, two prompts each, four samples per prompt.
        dict(name="attn_few", op="attn", Hq=8, Hkv=2, agents="2x4 const:256 uniform:1:128; 2x4 const:256 uniform:1:128"),
        # The ordinary decode step: 512 samples of 64 prompts, responses with medians of 256 to 2048 tokens and a long tail.
        dict(name="attn_batch", op="attn", Hq=28, Hkv=4,
             agents="; ".join(f"16x8 uniform:512:2048 lognormal:{m}:0.8:8192" for m in (256, 512, 1024, 2048))),
        # The first steps after a long prompt was expanded into 32 samples: nearly all of the work is the shared prefix.
        dict(name="attn_group_sampling", op="attn", Hq=28, Hkv=4, agents="16x32 const:4096 uniform:0:64"),
        # Long contexts on a larger model's heads: 8192-token prompts, 8k to 24k generated tokens.
        dict(name="attn_long", op="attn", Hq=64, Hkv=8, agents="32x4 const:8192 uniform:8192:24576"),
    ]


HEADS = [(8, 2), (28, 4), (28, 4), (64, 8), (64, 8), (32, 8), (16, 1), (4, 4)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "grad", "append", "prompt", "read", "attn", "attn", "attn"])
    Hq, Hkv = rng.choice(HEADS)
    if op in ("norm", "grad"):
        D = rng.choice([64, 128, 128, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = {"norm": 65543, "grad": 32771}[op] * 32 * 128 * 2 // ((Hq + Hkv) * D * (4 if dtype == "f32" else 2))
        return dict(op=op, tokens=_log_int(rng, 1, most), Hq=Hq, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, 0]),
                    pairs=rng.choice(["halves", "halves", "adjacent"]), dtype=dtype, positions=rng.choice(["runs", "random"]))
    if op == "append":
        return dict(op=op, seqs=_log_int(rng, 1, 4096), Hkv=Hkv, cols=rng.randint(1, 6))
    if op == "prompt":
        hi = _log_int(rng, 1, 4096)
        prompts = max(1, min(_log_int(rng, 1, 64), 320000 // (hi * Hkv)))
        ctx = rng.choice([0, 0, _log_int(rng, 1, 4096)])
        return dict(op=op, Hkv=Hkv, prompts=prompts, chunk=f"uniform:{max(1, hi // 4)}:{hi}",
                    context=f"uniform:0:{ctx}" if ctx else "const:0")
    if op == "read":
        return dict(op=op, Hkv=Hkv, pages=_log_int(rng, 1, 24008 // Hkv))
    agents, room = [], 128 * 32768 * 8 / 2   # padded (sequence, token, KV head) triples of the plain form
    G, hi, top = _log_int(rng, 1, 32), _log_int(rng, 16, 8192), _log_int(rng, 8, 16384)
    for _ in range(rng.randint(1, 3)):
        plen = rng.choice([f"const:{hi}", f"uniform:{hi // 4}:{hi}", f"uniform:0:{hi}"])
        glen = rng.choice([f"uniform:{top // 8}:{top}", f"uniform:0:{top}", f"lognormal:{max(1, top // 4)}:0.8:{top}"])
        prompts = max(1, min(_log_int(rng, 1, 64), int(room / 3 / (G * (hi + top + 32) * Hkv))))
        agents.append(f"{prompts}x{G} {plen} {glen}")
    return dict(op=op, Hq=Hq, Hkv=Hkv, agents="; ".join(agents))


# ---- lengths and pages -------------------------------------------------------------------------
def _lens(text, rng, n):
    kind, *v = text.split(":")
    if kind == "const":
        return np.full(n, int(v[0]), dtype=np.int64)
    if kind == "uniform":
        return rng.integers(int(v[0]), int(v[1]) + 1, size=n, dtype=np.int64)
    z = np.rint(np.exp(math.log(float(v[0])) + float(v[1]) * rng.standard_normal(n))).astype(np.int64)
    return np.clip(z, 1, int(v[2]))


def _attn_lens(case):
    rng = np.random.default_rng(LENS_SEED)
    P, S, group = [], [], []
    for part in case["agents"].split("; "):
        count, plen, glen = part.split()
        prompts, G = (int(x) for x in count.split("x"))
        first = sum(map(len, P))
        P.append(_lens(plen, rng, prompts))
        S.append(_lens(glen, rng, prompts * G))
        group.append(np.repeat(np.arange(first, first + prompts), G))
    return np.concatenate(P), np.concatenate(S), np.concatenate(group)


def _prompt_lens(case):
    rng = np.random.default_rng(LENS_SEED)
    n = case["prompts"]
    return _lens(case["chunk"], rng, n), _lens(case["context"], rng, n)


def _append_lens(case):
    return np.random.default_rng(LENS_SEED).integers(0, case["cols"] * PAGE, size=case["seqs"])


def _table(pages, cols, ids):
    """Block table whose row r names the next pages[r] of `ids`; -1 elsewhere."""
    table = np.full((len(pages), max(1, cols)), -1, dtype=np.int32)
    inside = np.arange(table.shape[1])[None, :] < pages[:, None]
    table[inside] = ids[: int(pages.sum())]
    return table


def _cuda(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


# ---- values in 8 bits --------------------------------------------------------------------------
def _pow2(e):
    """2^e in 32 bits, from its bits (e an integer tensor)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantize(x):
    """Rows of 128 numbers as e4m3 codes and an exponent: the smallest power of two under which the row's largest finite
    magnitude is at most 448."""
    x = x.float()
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    mantissa, exponent = torch.frexp(top)
    e = exponent.int() - 9 + (mantissa > 0.875).int()
    e = torch.where(top > 0, e, torch.full_like(e, MIN_EXPONENT)).clamp(min=MIN_EXPONENT)
    codes = (x * _pow2(-e)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return codes, e.to(torch.int8)


def _cache(pages, Hkv, gen, filled):
    """k_pages, v_pages, exponents of a cache: rows of normal numbers whose spread differs from token to token, or zeros."""
    k = torch.zeros(pages, Hkv, PAGE, 128, dtype=torch.uint8, device="cuda")
    v = torch.zeros(pages, Hkv, 128, PAGE, dtype=torch.uint8, device="cuda")
    ex = torch.zeros(pages, Hkv, 2, PAGE, dtype=torch.int8, device="cuda")
    step = max(1, (1 << 26) // (Hkv * PAGE * 128))
    for a in range(0, pages if filled else 0, step):
        n = min(step, pages - a)
        for which in (0, 1):
            spread = torch.exp(0.5 * torch.randn(n, Hkv, PAGE, 1, generator=gen, device="cuda"))
            x = torch.randn(n, Hkv, PAGE, 128, generator=gen, device="cuda").mul_(spread)
            codes, e = _quantize(x.to(torch.bfloat16))
            codes = codes.view(torch.uint8)
            ex[a:a + n, :, which] = e
            if which == 0:
                k[a:a + n] = codes
            else:
                v[a:a + n] = codes.transpose(2, 3)
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ex


# ---- inputs ------------------------------------------------------------------------------------
def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _norm_state(case, gen):
    T, Hq, Hkv, D, rot = (case[n] for n in ("tokens", "Hq", "Hkv", "D", "rot"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    fused = _randn((T, (Hq + 2 * Hkv) * D), dt, gen).mul_(torch.exp(torch.randn(T, 1, generator=gen, device="cuda")).to(dt))
    s = dict(case=case, q=fused[:, : Hq * D].view(T, Hq, D), k=fused[:, Hq * D: (Hq + Hkv) * D].view(T, Hkv, D))
    for n in ("q_weight", "k_weight"):
        s[n] = (1.0 + 0.25 * torch.randn(D, generator=gen, device="cuda")).to(dt)
    half = rot // 2
    angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * \
        torch.pow(torch.tensor(10000.0, device="cuda", dtype=torch.float64), -torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))
    s["cos_sin"] = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float().contiguous()      # [MAX_POS, rot]
    if case["positions"] == "random":
        s["positions"] = torch.randint(0, MAX_POS, (T,), generator=gen, device="cuda", dtype=torch.int32)
    else:   # whole sequences one after the other
        s["positions"] = (torch.arange(T, device="cuda") % 1531).int()
    names = ("dq", "dk") if case["op"] == "grad" else ("q_out", "k_out")
    s[names[0]] = torch.empty(T, Hq, D, dtype=dt, device="cuda")
    s[names[1]] = torch.empty(T, Hkv, D, dtype=dt, device="cuda")
    if case["op"] == "grad":
        s["dq_out"], s["dk_out"] = _randn((T, Hq, D), dt, gen), _randn((T, Hkv, D), dt, gen)
        s["dq_weight"], s["dk_weight"] = (torch.empty(D, dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _attn_state(case, gen, rng):
    P, S, group = _attn_lens(case)
    npp, nsp = -(-P // PAGE), -(-S // PAGE)
    used = int(npp.sum() + nsp.sum())
    pages = max(1, used + used // 20 + 1)
    ids = rng.permutation(pages).astype(np.int32)
    ptab = _table(npp, int(npp.max()), ids)
    stab = _table(nsp, int(nsp.max()), ids[int(npp.sum()):])
    k, v, ex = _cache(pages, case["Hkv"], gen, True)
    # what no token owns may hold anything: here the code that stands for no number
    held = np.zeros(pages, dtype=np.int64)
    for tab, n, lens in ((ptab, npp, P), (stab, nsp, S)):
        inside = np.arange(tab.shape[1])[None, :] < n[:, None]
        held[tab[inside]] = np.clip(lens[:, None] - np.arange(tab.shape[1])[None, :] * PAGE, 0, PAGE)[inside]
    empty = torch.arange(PAGE, device="cuda")[None, :] >= _cuda(held, np.int64)[:, None]
    k.view(torch.uint8).masked_fill_(empty[:, None, :, None], 0x7F)
    v.view(torch.uint8).masked_fill_(empty[:, None, None, :], 0x7F)
    q = _randn((len(S), case["Hq"], 128), torch.bfloat16, gen)
    return dict(case=case, q=q, k_pages=k, v_pages=v, exponents=ex, prefix_table=_cuda(ptab), suffix_table=_cuda(stab),
                prefix_lens=_cuda(P), suffix_lens=_cuda(S), group_of_seq=_cuda(group), scale=1.0 / math.sqrt(128),
                out=torch.empty_like(q))


def prepare(case, seed):
    op = case["op"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    if op in ("norm", "grad"):
        return _norm_state(case, gen)
    if op == "attn":
        return _attn_state(case, gen, rng)
    Hkv = case["Hkv"]
    if op == "read":
        n = case["pages"]
        pages = n + n // 8 + 1
        k, v, ex = _cache(pages, Hkv, gen, True)
        return dict(case=case, k_pages=k, v_pages=v, exponents=ex, src=_cuda(rng.permutation(pages)[:n]), dst=_cuda(rng.permutation(n)),
                    k_out=torch.zeros(n, Hkv, PAGE, 128, dtype=torch.bfloat16, device="cuda"),
                    v_out=torch.zeros(n, Hkv, 128, PAGE, dtype=torch.bfloat16, device="cuda"))
    if op == "append":
        n, cols = case["seqs"], case["cols"]
        lens = _append_lens(case)
        held = lens // PAGE + 1
        pages = int(held.sum()) + 3
        table = _table(held, cols, rng.permutation(pages).astype(np.int32))
        s = dict(case=case, lens=_cuda(lens), lens_now=_cuda(lens), table=_cuda(table))
    else:
        chunk, ctx = _prompt_lens(case)
        held = -(-(chunk + ctx) // PAGE)
        pages, n = int(held.sum()) + 3, int(chunk.sum())
        s = dict(case=case, table=_cuda(_table(held, int(held.max()), rng.permutation(pages).astype(np.int32))),
                 q_start=_cuda(np.concatenate([[0], np.cumsum(chunk)])), q_pos0=_cuda(ctx))
    k, v, ex = _cache(pages, Hkv, gen, False)
    spread = lambda: torch.exp(0.5 * torch.randn(n, Hkv, 1, generator=gen, device="cuda"))  # noqa: E731
    s.update(k_pages=k, v_pages=v, exponents=ex, pages=pages,
             k_new=(torch.randn(n, Hkv, 128, generator=gen, device="cuda") * spread()).to(torch.bfloat16),
             v_new=(torch.randn(n, Hkv, 128, generator=gen, device="cuda") * spread()).to(torch.bfloat16))
    return s


# ---- one pass, plain ---------------------------------------------------------------------------
def _angles(s):
    case = s["case"]
    cs = s["cos_sin"][s["positions"].long()][:, None, :]
    return cs[..., : case["rot"] // 2], cs[..., case["rot"] // 2:]


def _split(y, case):
    """The two members of every pair, and what is not rotated."""
    rot = case["rot"]
    if case["pairs"] == "halves":
        return y[..., : rot // 2], y[..., rot // 2: rot], y[..., rot:]
    return y[..., 0:rot:2], y[..., 1:rot:2], y[..., rot:]


def _join(a, b, rest, case):
    if case["pairs"] == "halves":
        return torch.cat([a, b, rest], -1)
    return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)


def _plain_norm(s, x, weight):
    x32 = x.float()
    y = x32 * torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS) * weight.float()
    c, sn = _angles(s)
    a, b, rest = _split(y, s["case"])
    return _join(a * c - b * sn, b * c + a * sn, rest, s["case"]).to(x.dtype)


def _plain_grad(s, dz, x, weight):
    x32, dz = x.float(), dz.float()
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS)
    n = x32 * r
    c, sn = _angles(s)
    a, b, rest = _split(dz, s["case"])
    dy = _join(a * c + b * sn, b * c - a * sn, rest, s["case"])
    g = dy * weight.float()
    dx = r * (g - n * (g * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (dy * n).sum((0, 1))


def _plain_store(s, page, slot):
    """Keys and values of the new tokens at (page, slot), quantised."""
    for pages, new, which in ((s["k_pages"], s["k_new"], 0), (s["v_pages"], s["v_new"], 1)):
        codes, e = _quantize(new)
        if which == 0:
            pages.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
        else:
            pages.view(torch.uint8)[page, :, :, slot] = codes.view(torch.uint8)
        s["exponents"][page, :, which, slot] = e


def _plain_attn(s):
    Hq, Hkv = s["case"]["Hq"], s["case"]["Hkv"]
    NS, R = s["q"].shape[0], Hq // Hkv
    group = s["group_of_seq"].long()
    pages = torch.cat([s["prefix_table"][group], s["suffix_table"]], 1).long().clamp(min=0)        # [NS, n]
    at = lambda cols: torch.arange(cols * PAGE, device="cuda")[None, :]  # noqa: E731
    valid = torch.cat([at(s["prefix_table"].shape[1]) < s["prefix_lens"][group][:, None],
                       at(s["suffix_table"].shape[1]) < s["suffix_lens"][:, None]], 1)             # [NS, n * 16]
    scales = _pow2(s["exponents"][pages])                                                          # [NS, n, Hkv, 2, 16]
    K = s["k_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float().mul_(scales[:, :, :, 0, :, None])
    K = K.permute(0, 2, 1, 3, 4).reshape(NS, Hkv, -1, 128)
    x = torch.matmul(s["q"].float().view(NS, Hkv, R, 128), K.transpose(2, 3)).mul_(s["scale"])
    del K
    x = x.masked_fill_(~valid[:, None, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))))
    total = p.sum(-1, keepdim=True)
    V = s["v_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float().mul_(scales[:, :, :, 1, None, :])
    V = V.permute(0, 2, 1, 4, 3).reshape(NS, Hkv, -1, 128)
    V = V.masked_fill_(~valid[:, None, :, None], 0.0)
    out = torch.matmul(p, V) / torch.where(total > 0, total, torch.ones_like(total))               # (no token: zeros)
    return out.view(NS, Hq, 128).to(torch.bfloat16)


def _plain(s):
    op = s["case"]["op"]
    if op == "norm":
        return dict(q=_plain_norm(s, s["q"], s["q_weight"]), k=_plain_norm(s, s["k"], s["k_weight"]))
    if op == "grad":
        dq, dqw = _plain_grad(s, s["dq_out"], s["q"], s["q_weight"])
        dk, dkw = _plain_grad(s, s["dk_out"], s["k"], s["k_weight"])
        return dict(dq=dq, dk=dk, dq_weight=dqw, dk_weight=dkw)
    if op == "attn":
        return dict(out=_plain_attn(s))
    if op == "read":
        src, dst = s["src"].long(), s["dst"].long()
        scales = _pow2(s["exponents"][src])
        s["k_out"][dst] = (s["k_pages"].view(torch.uint8)[src].view(torch.float8_e4m3fn).float() * scales[:, :, 0, :, None]).to(torch.bfloat16)
        s["v_out"][dst] = (s["v_pages"].view(torch.uint8)[src].view(torch.float8_e4m3fn).float() * scales[:, :, 1, None, :]).to(torch.bfloat16)
        return dict(k=s["k_out"], v=s["v_out"])
    if op == "append":
        s["lens"].copy_(s["lens_now"])
        pos = s["lens"].long()
        page = s["table"].gather(1, (pos // PAGE)[:, None])[:, 0].long()
        _plain_store(s, page, pos % PAGE)
        s["lens"].add_(1)
        return dict(k=s["k_pages"], v=s["v_pages"], exponents=s["exponents"], lens=s["lens"])
    start = s["q_start"].long()
    t = torch.arange(s["k_new"].shape[0], device="cuda")
    g = torch.searchsorted(start[1:], t, right=True)
    pos = t - start[g] + s["q_pos0"].long()[g]
    _plain_store(s, s["table"][g, pos // PAGE].long(), pos % PAGE)
    return dict(k=s["k_pages"], v=s["v_pages"], exponents=s["exponents"])


# ---- one pass, by the library ------------------------------------------------------------------
def _kept(s, B):
    """Shape descriptor and workspace, which a program makes once for its batch."""
    case, op = s["case"], s["case"]["op"]
    if op == "attn":
        shape = B.make_shape(s["q"].shape[0], s["prefix_lens"].shape[0], case["Hq"], case["Hkv"], s["k_pages"].shape[0],
                             s["prefix_table"].shape[1], s["suffix_table"].shape[1])
        return shape, B.alloc_workspace(B.marl_workspace_bytes(shape), "cuda")
    if op == "grad":
        return None, B.alloc_workspace(B.marl_qk_norm_rope_workspace_bytes(case["tokens"], case["Hq"], case["Hkv"], case["D"]), "cuda")
    if op == "append":
        return B.make_shape(case["seqs"], 1, case["Hkv"], case["Hkv"], s["pages"], 1, case["cols"]), None
    if op == "prompt":
        return B.make_prefill_shape(s["k_new"].shape[0], case["prompts"], case["Hkv"], case["Hkv"], s["pages"], s["table"].shape[1]), None
    return None, None


def _library(s):
    from paper_2602_09578_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if "kept" not in s:
        s["kept"] = _kept(s, B)
    shape, ws = s["kept"]
    if op == "norm":
        B.marl_qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos_sin"], s["positions"], EPS, s["q_out"], s["k_out"],
                            adjacent_pairs=case["pairs"] == "adjacent")
        return dict(q=s["q_out"], k=s["k_out"])
    if op == "grad":
        B.marl_qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos_sin"], s["positions"],
                                     EPS, s["dq"], s["dk"], s["dq_weight"], s["dk_weight"], ws, adjacent_pairs=case["pairs"] == "adjacent")
        return dict(dq=s["dq"], dk=s["dk"], dq_weight=s["dq_weight"], dk_weight=s["dk_weight"])
    if op == "attn":
        return dict(out=B.marl_decode_attn_fp8(shape, ws, s["q"], s["k_pages"], s["v_pages"], s["exponents"], s["prefix_table"],
                                               s["suffix_table"], s["prefix_lens"], s["suffix_lens"], s["group_of_seq"], s["scale"], s["out"]))
    if op == "read":
        B.marl_kv_read_pages_fp8(s["k_pages"], s["v_pages"], s["exponents"], s["src"], s["dst"], s["k_out"], s["v_out"])
        return dict(k=s["k_out"], v=s["v_out"])
    if op == "append":
        s["lens"].copy_(s["lens_now"])
        B.marl_kv_append_fp8(shape, s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["exponents"], s["table"], s["lens"])
        return dict(k=s["k_pages"], v=s["v_pages"], exponents=s["exponents"], lens=s["lens"])
    B.marl_kv_write_prompt_fp8(shape, s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["exponents"], s["table"], s["q_start"], s["q_pos0"])
    return dict(k=s["k_pages"], v=s["v_pages"], exponents=s["exponents"])


def run(state):
    return _library(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------
def work(case):
    op, Hkv = case["op"], case["Hkv"]
    if op in ("norm", "grad"):
        T, D, size = case["tokens"], case["D"], 4 if case["dtype"] == "f32" else 2
        n = T * (case["Hq"] + Hkv) * D
        angles = 4 * case["rot"] * min(T, 1531 if case["positions"] == "runs" else MAX_POS)
        return dict(bytes=n * size * (3 if op == "grad" else 2) + angles + 4 * T + D * (2 * size + (8 if op == "grad" else 0)),
                    flops=n * (16 if op == "grad" else 7))
    token = 2 * 128 + 2            # a token's key and value of one KV head: codes and exponents
    if op == "read":
        n = case["pages"] * Hkv * PAGE
        return dict(bytes=n * (token + 2 * 128 * 2) + 8 * case["pages"], flops=0)
    if op == "append":
        n = case["seqs"]
        return dict(bytes=n * Hkv * (2 * 128 * 2 + token) + 12 * n, flops=4 * n * Hkv * 128)
    if op == "prompt":
        n = int(_prompt_lens(case)[0].sum())
        return dict(bytes=n * Hkv * (2 * 128 * 2 + token) + 4 * (n // PAGE), flops=4 * n * Hkv * 128)
    P, S, group = _attn_lens(case)
    pairs = int(S.sum() + P[group].sum())
    return dict(bytes=int(P.sum() + S.sum()) * Hkv * token + len(S) * case["Hq"] * 128 * 4, flops=4 * 128 * case["Hq"] * pairs)


# ---- the same in 64 bits -----------------------------------------------------------------------
def _e4m3_values():
    """The number that each of the 256 codes stands for: sign, 4 bits of exponent (bias 7), 3 of mantissa."""
    def value(c):
        e, m = (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            return math.nan
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        return -v if c & 128 else v
    return torch.tensor([value(c) for c in range(256)], dtype=torch.float64, device="cuda")


def _nearest_e4m3(x):
    """Rows in units of 2^e and e, by the definition: nearest of the values that e4m3 has, ties to the even mantissa."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e))
    e = torch.where(top > 0, e, torch.full_like(e, MIN_EXPONENT)).clamp(min=MIN_EXPONENT)
    y = x * torch.exp2(-e)
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit, e[..., 0]


def _exact_store(s, where):
    """`where`: (token, page, slot) triples.  The codes' values after the new tokens are in."""
    k, v = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("k_pages", "v_pages"))
    t, page, slot = (torch.from_numpy(np.ascontiguousarray(w)).cuda() for w in where)
    k[page, :, slot, :] = _nearest_e4m3(s["k_new"])[0][t]
    v[page, :, :, slot] = _nearest_e4m3(s["v_new"])[0][t]
    return k, v


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op in ("norm", "grad"):
        D, rot = case["D"], case["rot"]
        d = torch.arange(D, device="cuda")
        if case["pairs"] == "halves":
            partner = torch.where(d < rot // 2, d + rot // 2, d - rot // 2)
            index, first = d % max(rot // 2, 1), d < rot // 2
        else:
            partner, index, first = d ^ 1, d // 2, d % 2 == 0
        turned = d < rot
        partner = torch.where(turned, partner, d)
        table = s["cos_sin"].double()[s["positions"].long()]
        cos, sin = torch.ones(case["tokens"], D, dtype=torch.float64, device="cuda"), torch.zeros(case["tokens"], D, dtype=torch.float64, device="cuda")
        cos[:, turned] = table[:, index[turned]]
        sin[:, turned] = table[:, rot // 2 + index[turned]]
        sin = torch.where(first, -sin, sin)[:, None, :]            # z_d = y_d cos_d + y_partner sin_d
        cos = cos[:, None, :]
        result = {}
        for n in ("q", "k"):
            x, w = s[n].double(), s[n + "_weight"].double()
            r = 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS)
            if op == "norm":
                y = x * r * w
                result[n] = y * cos + y[..., partner] * sin
            else:
                dz = s["d" + n + "_out"].double()
                dy = dz * cos + (dz * sin)[..., partner]
                gx = dy * w
                result["d" + n] = r * gx - x * r ** 3 * (gx * x).sum(-1, keepdim=True) / D
                result["d" + n + "_weight"] = (dy * x * r).sum((0, 1))
        return result
    if op == "read":
        values = _e4m3_values()
        k, v = torch.empty(s["k_out"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["v_out"].shape, dtype=torch.float64, device="cuda")
        src, dst = s["src"].long(), s["dst"].long()
        two = torch.exp2(s["exponents"].double())[src]
        k[dst] = values[s["k_pages"].view(torch.uint8)[src].long()] * two[:, :, 0, :, None]
        v[dst] = values[s["v_pages"].view(torch.uint8)[src].long()] * two[:, :, 1, None, :]
        return dict(k=k, v=v)
    if op == "append":
        pos, table = _append_lens(case), s["table"].cpu().numpy()
        n = np.arange(case["seqs"])
        k, v = _exact_store(s, (n, table[n, pos // PAGE].astype(np.int64), pos % PAGE))
        return dict(k=k, v=v, exponents=None, lens=None)
    if op == "prompt":
        chunk, ctx = _prompt_lens(case)
        table = s["table"].cpu().numpy()
        g = np.repeat(np.arange(len(chunk)), chunk)
        pos = np.concatenate([np.arange(c, c + n) for n, c in zip(chunk, ctx)])
        k, v = _exact_store(s, (np.arange(len(pos)), table[g, pos // PAGE].astype(np.int64), pos % PAGE))
        return dict(k=k, v=v, exponents=None)
    values = _e4m3_values()
    P, S, group = _attn_lens(case)
    Hkv, R = case["Hkv"], case["Hq"] // case["Hkv"]

    def tokens(row, n):
        ids = row[: -(-n // PAGE)].long()
        two = torch.exp2(s["exponents"][ids].double())
        k = values[s["k_pages"].view(torch.uint8)[ids].long()] * two[:, :, 0, :, None]
        v = values[s["v_pages"].view(torch.uint8)[ids].long()] * two[:, :, 1, None, :]
        return (k.permute(1, 0, 2, 3).reshape(Hkv, -1, 128)[:, :n], v.permute(1, 0, 3, 2).reshape(Hkv, -1, 128)[:, :n])

    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for g in range(len(P)):
        kp, vp = tokens(s["prefix_table"][g], int(P[g]))
        for i in np.nonzero(group == g)[0].tolist():
            if P[g] + S[i] == 0:
                continue
            ks, vs = tokens(s["suffix_table"][i], int(S[i]))
            q = s["q"][i].double().view(Hkv, R, 128)
            x = torch.cat([q @ kp.transpose(1, 2), q @ ks.transpose(1, 2)], 2) * s["scale"]
            p = torch.softmax(x, 2)
            out[i] = (p[:, :, : int(P[g])] @ vp + p[:, :, int(P[g]):] @ vs).reshape(-1, 128)
    return dict(out=out)
