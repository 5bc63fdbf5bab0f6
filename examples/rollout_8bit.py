"""Rollout of one attention layer over an 8-bit KV cache: prompts in two chunks, then decode steps, then the gradient of its norm.

    python examples/rollout_8bit.py [--prompts 4] [--samples 16] [--prompt-tokens 1000] [--steps 64]

What the layer does to a token: a fused projection to queries, keys and values (torch), the norm of every query and key head with rotation by
position (marl_qk_norm_rope, on slices of the projection's result), its key and value into the cache (marl_kv_write_prompt_fp8 for
prompts, marl_kv_append_fp8 for a decode step), attention (marl_prefill_attn over bf16 pages that marl_kv_read_pages_fp8 fills from the
cache; marl_decode_attn_fp8 over the cache itself), the output projection (torch).  A decode step's three calls are captured in a graph
once.  Weights and inputs are random.
"""
from __future__ import annotations

import argparse
import os
import sys
from types import SimpleNamespace

import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_09578_amd import binding as B  # noqa: E402

HQ, HKV, D, HIDDEN, PAGE, EPS = 28, 4, 128, 512, 16, 1e-6
SCALE = D ** -0.5


class Layer:
    def __init__(self, device, max_positions: int, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).to(device)  # noqa: E731
        self.w_in = rnd(HIDDEN, (HQ + 2 * HKV) * D) * HIDDEN ** -0.5
        self.w_out = rnd(HQ * D, HIDDEN) * (HQ * D) ** -0.5
        self.q_weight, self.k_weight = 1 + rnd(D) / 8, 1 + rnd(D) / 8
        angle = torch.arange(max_positions)[:, None] * 10000.0 ** (-torch.arange(D // 2) / (D // 2))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(device)

    def project(self, x):
        """Fused projection of x [tokens, HIDDEN]."""
        return x @ self.w_in

    def heads(self, qkv):
        """Its slices for queries and keys, and a copy of the values (the cache calls take whole rows)."""
        T = qkv.shape[0]
        q, k, v = qkv[:, : HQ * D], qkv[:, HQ * D: (HQ + HKV) * D], qkv[:, (HQ + HKV) * D:]
        return q.view(T, HQ, D), k.view(T, HKV, D), v.view(T, HKV, D)


class QkNormRope(torch.autograd.Function):
    """marl_qk_norm_rope with its gradient.  A weight may be None (ones); there is no second derivative."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos_sin, positions):
        ctx.save_for_backward(q, k, q_weight, k_weight, cos_sin, positions)
        q_out, k_out = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        return B.marl_qk_norm_rope(q, k, q_weight, k_weight, cos_sin, positions, EPS, q_out, k_out)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, cos_sin, positions = ctx.saved_tensors
        wanted = ctx.needs_input_grad
        dq, dk = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        dqw, dkw = (torch.empty(D, dtype=torch.float32, device=q.device) if w else None for w in wanted[2:4])   # (a call writes dq and dk always)
        ws = B.alloc_workspace(B.marl_qk_norm_rope_workspace_bytes(q.shape[0], q.shape[1], k.shape[1], D), q.device)
        B.marl_qk_norm_rope_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, q_weight, k_weight, cos_sin, positions, EPS, dq, dk, dqw, dkw, ws)
        return (dq if wanted[0] else None, dk if wanted[1] else None, dqw.to(q_weight.dtype) if wanted[2] else None,
                dkw.to(k_weight.dtype) if wanted[3] else None, None, None)


def write_prompts(layer, cache, table, lens, x):
    """The prompts' tokens x (one prompt after the other, lens[g] of prompt g), half of each and then the rest.  The rest attends to what
    the cache holds of the first half, as a prompt does whose beginning another turn left there.  Returns the attention's results [tokens, HIDDEN]."""
    dev, G, pages = x.device, len(lens), table.shape[1]
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32).to(dev)  # noqa: E731
    start = [sum(lens[:g]) for g in range(G)]
    out = torch.empty_like(x)
    # bf16 pages for the prompt attention: those of these prompts alone, numbered from 0
    k16 = torch.zeros(G * pages, HKV, PAGE, D, dtype=torch.bfloat16, device=dev)
    v16 = torch.zeros(G * pages, HKV, D, PAGE, dtype=torch.bfloat16, device=dev)
    table16 = i32(torch.arange(G * pages).view(G, pages))
    for part in range(2):
        first = [(n // 2 if part else 0) for n in lens]
        count = [(n - n // 2 if part else n // 2) for n in lens]
        rows = torch.cat([torch.arange(s + f, s + f + c) for s, f, c in zip(start, first, count)]).to(dev)
        positions = torch.cat([torch.arange(f, f + c) for f, c in zip(first, count)]).int().to(dev)
        q_start, q_pos0 = i32([sum(count[:g]) for g in range(G + 1)]), i32(first)
        T = int(rows.numel())
        if T == 0:   # (prompts of one token have no first half)
            continue
        shape = B.make_prefill_shape(T, G, HQ, HKV, G * pages, pages)
        shape8 = B.make_prefill_shape(T, G, HQ, HKV, cache[0].shape[0], pages)
        q, k, v = layer.heads(layer.project(x[rows]))
        q_out, k_out, v = torch.empty(T, HQ, D, dtype=q.dtype, device=dev), torch.empty(T, HKV, D, dtype=q.dtype, device=dev), v.contiguous()
        B.marl_qk_norm_rope(q, k, layer.q_weight, layer.k_weight, layer.cos_sin, positions, EPS, q_out, k_out)
        B.marl_kv_write_prompt_fp8(shape8, k_out, v, *cache, table, q_start, q_pos0)
        # what the cache holds now, this chunk included, so that prompt and decode attention see the same numbers
        B.marl_kv_read_pages_fp8(*cache, table.reshape(-1), table16.reshape(-1), k16, v16)
        o = torch.empty(T, HQ, D, dtype=torch.bfloat16, device=dev)
        B.marl_prefill_attn(shape, B.alloc_workspace(B.marl_prefill_workspace_bytes(shape), dev), q_out, k16, v16, table16, q_start, q_pos0, SCALE, o)
        out[rows] = o.view(T, HQ * D) @ layer.w_out
    return out


class Decoder:
    """Decode steps of a batch: everything that a step needs, allocated once; its calls in a graph."""

    def __init__(self, layer, cache, prefix_table, prefix_lens, suffix_table, group_of_seq):
        dev, NS = layer.w_in.device, suffix_table.shape[0]
        self.layer, self.cache = layer, cache
        self.tables, self.prefix_lens, self.group_of_seq = (prefix_table, suffix_table), prefix_lens, group_of_seq
        self.suffix_lens = torch.zeros(NS, dtype=torch.int32, device=dev)
        self.positions = prefix_lens[group_of_seq.long()].clone()
        self.qkv = torch.zeros(NS, (HQ + 2 * HKV) * D, dtype=torch.bfloat16, device=dev)
        self.q, self.out = (torch.empty(NS, HQ, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.k, self.v = (torch.empty(NS, HKV, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.shape = B.make_shape(NS, prefix_table.shape[0], HQ, HKV, cache[0].shape[0], prefix_table.shape[1], suffix_table.shape[1])
        self.workspace = B.alloc_workspace(B.marl_workspace_bytes(self.shape), dev)
        self.graph = None

    def _calls(self):
        layer = self.layer
        q, k, v = layer.heads(self.qkv)
        self.v.copy_(v)
        B.marl_qk_norm_rope(q, k, layer.q_weight, layer.k_weight, layer.cos_sin, self.positions, EPS, self.q, self.k)
        B.marl_kv_append_fp8(self.shape, self.k, self.v, *self.cache, self.tables[1], self.suffix_lens)   # (suffix_lens grow by one)
        B.marl_decode_attn_fp8(self.shape, self.workspace, self.q, *self.cache, *self.tables, self.prefix_lens, self.suffix_lens, self.group_of_seq,
                               SCALE, self.out)
        self.positions.add_(1)

    def step(self, x):
        """One token x [NS, HIDDEN] of every sequence."""
        torch.matmul(x, self.layer.w_in, out=self.qkv)
        if self.graph is None:     # the first step runs as it is, the graph is recorded for the following ones
            self._calls()
            state = self.suffix_lens.clone(), self.positions.clone()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self._calls()
            assert all(torch.equal(a, b) for a, b in zip(state, (self.suffix_lens, self.positions)))   # (recording runs nothing)
        else:
            self.graph.replay()
        return self.out.view(x.shape[0], HQ * D) @ self.layer.w_out


def run(prompts=4, samples=16, prompt_tokens=1000, steps=64, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(max(1, prompt_tokens // 2), prompt_tokens + 1, (prompts,), generator=g).tolist()
    NS = prompts * samples
    ppages, spages = (max(lens) + PAGE - 1) // PAGE, (steps + PAGE - 1) // PAGE
    total = prompts * ppages + NS * spages
    ids = torch.randperm(total, generator=g).int()
    prefix_table = ids[: prompts * ppages].view(prompts, ppages).to(device)
    suffix_table = ids[prompts * ppages:].view(NS, spages).to(device)
    group_of_seq = torch.arange(prompts, dtype=torch.int32).repeat_interleave(samples).to(device)
    layer = Layer(device, max(lens) + steps, seed)
    cache = B.alloc_kv_fp8(total, HKV, device)
    x = torch.randn(sum(lens), HIDDEN, generator=g).to(torch.bfloat16).to(device)
    prompt_out = write_prompts(layer, cache, prefix_table, lens, x)
    decoder = Decoder(layer, cache, prefix_table, torch.tensor(lens, dtype=torch.int32, device=device), suffix_table, group_of_seq)
    last = torch.tensor([sum(lens[: p + 1]) - 1 for p in range(prompts)], device=device)
    h = prompt_out[last][group_of_seq.long()]
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for t in range(steps):
        if t == 1:
            begin.record()
        noise = torch.randn(NS, HIDDEN, generator=g).to(torch.bfloat16).to(device) if t == 0 else noise.roll(1, 0)
        h = decoder.step(h + noise)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / max(steps - 1, 1) if steps > 1 else float("nan")
    assert steps == 0 or B.marl_attn_read_flags(decoder.workspace) == 0   # (written by an attention call)
    return SimpleNamespace(layer=layer, cache=cache, decoder=decoder, lens=lens, ms_per_step=ms, out=h)


def train_step(layer, x, positions, dq_out, dk_out):
    """Gradients of the layer's projection and norm weights for those of its queries and keys."""
    w_in, q_weight, k_weight = (t.detach().clone().requires_grad_() for t in (layer.w_in, layer.q_weight, layer.k_weight))
    T = x.shape[0]
    qkv = x @ w_in
    qkv.retain_grad()
    q, k = qkv[:, : HQ * D].view(T, HQ, D), qkv[:, HQ * D: (HQ + HKV) * D].view(T, HKV, D)
    torch.autograd.backward(QkNormRope.apply(q, k, q_weight, k_weight, layer.cos_sin, positions), (dq_out, dk_out))
    return SimpleNamespace(qkv=qkv.detach(), dqkv=qkv.grad, w_in=w_in.grad, q_weight=q_weight.grad, k_weight=k_weight.grad)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("prompts", 4), ("samples", 16), ("prompt-tokens", 1000), ("steps", 64)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    r = run(a.prompts, a.samples, a.prompt_tokens, a.steps)
    nbytes = sum(t.numel() * t.element_size() for t in r.cache)
    print(f"{a.prompts} prompts of {min(r.lens)}-{max(r.lens)} tokens x {a.samples} samples, {a.steps} steps: {r.ms_per_step * 1e3:.1f} us a step, "
          f"cache {nbytes / 1e6:.1f} MB ({nbytes / r.cache[0].numel() / 4 * 100:.1f} % of a bf16 one)")
    T = 4 * HIDDEN
    gen = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    g = train_step(r.layer, rnd(T, HIDDEN), torch.arange(T, dtype=torch.int32, device="cuda") % r.layer.cos_sin.shape[0], rnd(T, HQ, D), rnd(T, HKV, D))
    print(f"gradient of {T} tokens: |d w_in| = {g.w_in.float().norm():.4g}, |d q_weight| = {g.q_weight.float().norm():.4g}, |d k_weight| = {g.k_weight.float().norm():.4g}")


if __name__ == "__main__":
    main()
