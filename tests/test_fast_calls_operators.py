"""The binding's short way for the 8-bit cache's calls and the norm with rotation, against the long way: the same bytes, the same
refusals, and nothing taken that is not plainly right."""
import pytest
import torch

from paper_2602_09578_amd import binding as B

ENTRIES = ("decode_attn_fp8", "kv_append_fp8", "kv_write_prompt_fp8", "kv_read_pages_fp8", "qk_norm_rope", "qk_norm_rope_backward")


def test_what_is_not_a_device_tensor_goes_the_long_way():
    B.load_library()
    if B._fast is None:
        pytest.skip("torch does not tell the current stream")
    shape, pshape = B.make_shape(2, 1, 4, 2, 3, 1, 1), B.make_prefill_shape(5, 1, 4, 2, 3, 2)
    x = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    for name in ENTRIES:
        f = getattr(B._fast, name)
        for n in range(18):
            for first in (shape, pshape, x):
                for filler in (None, 3, "no", x, shape, False):
                    assert f(*([first] + [filler] * (n - 1) if n else [])) is None


def _calls():
    """(name, function, arguments, outputs among them) of one right call of each entry."""
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()
    Hq, Hkv, pages = 8, 2, 12
    cache = B.alloc_kv_fp8(pages, Hkv, "cuda")
    pshape = B.make_prefill_shape(50, 2, Hq, Hkv, pages, 3)
    prompt = [pshape, rnd(50, Hkv, 128), rnd(50, Hkv, 128), *cache, i32([[0, 1, 2], [3, 4, 5]]), i32([0, 20, 50]), i32([3, 0])]
    B.marl_kv_write_prompt_fp8(*prompt)
    shape = B.make_shape(4, 2, Hq, Hkv, pages, 3, 1, B.MARL_OUT_F32)
    append = [shape, rnd(4, Hkv, 128), rnd(4, Hkv, 128), *cache, i32([[6], [7], [8], [9]]), i32([0, 0, 0, 0])]
    ws = B.alloc_workspace(B.marl_workspace_bytes(shape), "cuda")
    attn = [shape, ws, rnd(4, Hq, 128), *cache, prompt[6], append[6], i32([23, 30]), i32([1, 0, 1, 1]), i32([0, 0, 1, 1]), 0.09, torch.zeros(4, Hq, 128, device="cuda")]
    read = [*cache, i32([0, 3, 5]), i32([2, 0, 1]), torch.zeros(3, Hkv, 16, 128, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(3, Hkv, 128, 16, dtype=torch.bfloat16, device="cuda")]
    qkv = rnd(6, (Hq + 2 * Hkv) * 128)
    q, k = qkv[:, : Hq * 128].view(6, Hq, 128), qkv[:, Hq * 128: (Hq + Hkv) * 128].view(6, Hkv, 128)
    norm = [q, k, rnd(128), rnd(128), torch.rand(40, 64, generator=g).cuda(), i32([0, 39, 4, 5, 6, 7]), 1e-6, torch.zeros(6, Hq, 128, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(6, Hkv, 128, dtype=torch.bfloat16, device="cuda")]
    nws = B.alloc_workspace(B.marl_qk_norm_rope_workspace_bytes(6, Hq, Hkv, 128), "cuda")
    back = [rnd(6, Hq, 128), rnd(6, Hkv, 128), *norm[:7], torch.zeros(6, Hq, 128, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(6, Hkv, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"), nws]
    return [("decode_attn_fp8", B.marl_decode_attn_fp8, attn, [12]), ("kv_append_fp8", B.marl_kv_append_fp8, append, [3, 4, 5, 7]),
            ("kv_write_prompt_fp8", B.marl_kv_write_prompt_fp8, prompt, [3, 4, 5]), ("kv_read_pages_fp8", B.marl_kv_read_pages_fp8, read, [5, 6]),
            ("qk_norm_rope", B.marl_qk_norm_rope, norm, [7, 8]), ("qk_norm_rope_backward", B.marl_qk_norm_rope_backward, back, [9, 10, 11, 12])]


def _bytes(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(len(ENTRIES)), ids=ENTRIES)
def test_the_short_way_makes_the_same_call(which, monkeypatch):
    print("case: fast calls", ENTRIES[which], flush=True)
    B.load_library()
    assert B._fast is not None
    name, call, right, outs = _calls()[which]
    native = getattr(B._fast, name)
    taken = []

    def run(way, args):
        with monkeypatch.context() as m:
            m.setattr(B, "_fast", way)
            try:
                call(*args)
            except Exception as e:
                return f"{type(e).__name__}: {e}"
            torch.cuda.synchronize()
            return [_bytes(args[k]).clone() for k in outs if args[k] is not None]

    class Watched:
        def __getattr__(self, n):
            def f(*a):
                rc = native(*a)
                taken.append(rc)
                return rc
            return f

    def both(args):
        start = {k: _bytes(args[k]).clone() for k in outs if torch.is_tensor(args[k]) and args[k].is_cuda and args[k].is_contiguous()}
        got = []
        for way in (Watched(), None):
            for k, s in start.items():
                args[k].view(torch.uint8).copy_(s.view(args[k].view(torch.uint8).shape))
            got.append(run(way, args))
        return got

    short, long = both(right)
    assert taken == [0] and all(torch.equal(a, b) for a, b in zip(short, long))
    for k, a in enumerate(right):
        if torch.is_tensor(a):
            wrong = [a.to(torch.float64) if a.dtype != B.FP8 else a.float(), a[:-1], a.cpu(), None, 5, a.unsqueeze(0)]
            if a.dtype == torch.uint8:
                wrong = [a[:100], a.cpu(), a[::2]]   # (a workspace: any number of bytes is looked at by the library)
            elif a.dim() > 1 and a.shape[0] > 1 and a.shape[1] > 1:
                wrong.append(a.transpose(0, 1).contiguous().transpose(0, 1))
        elif isinstance(a, float):
            wrong = ["x", float("nan")]
        else:
            wrong = [None, 7]
        for w in wrong:
            short, long = both(right[:k] + [w] + right[k + 1:])
            if isinstance(short, str) or isinstance(long, str):
                assert short == long, (k, short, long)
            else:
                assert all(torch.equal(x, y) for x, y in zip(short, long))


@pytest.mark.gpu
def test_the_operators_stay_bound_where_the_other_functions_are_bound_anew():
    lib = B.load_library()
    B._bind_fast_calls(B._fast, lib.marl_decode_attn, lib.marl_token_logprobs, lib.marl_kv_append, lib.marl_sample_tokens,
                       lib.marl_sample_tokens_top_p, lib.marl_prefill_attn)
    for name, _, right, _ in _calls():
        more = {"qk_norm_rope": [False, None], "qk_norm_rope_backward": [False, None], "decode_attn_fp8": []}.get(name, [None])
        assert getattr(B._fast, name)(*right, *more) == 0
    torch.cuda.synchronize()
