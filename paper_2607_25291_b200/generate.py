"""Prompts and the tokens after them, through the whole library: `python -m paper_2607_25291_b200.generate`.

A stack of attention layers with random weights (no tokens, no vocabulary: what a step feeds on is its own output) serves a batch of prompts
from page pools.  The prompt: pages planned, keys and values appended, KAP and OSK over the pages.  Each token after it: one page
plan, and in every layer append, page selection (unless --budget 1) and the attention of the new token.  The step is captured into a CUDA
graph, as a serving loop would, and its time printed beside that of the same step over all pages.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as cosa

D = 128


class Stack:
    """Layers, their pools, and the batch's pages."""

    def __init__(self, prompts, new_tokens: int, layers: int = 2, hq: int = 32, hkv: int = 8, page: int = 64, e4m3: bool = False, seed: int = 0):
        dev, gen = "cuda", torch.Generator(device="cuda").manual_seed(seed)
        self.prompts, self.hq, self.hkv, self.page, self.batch = list(prompts), hq, hkv, page, len(prompts)
        hidden = hq * D
        rand = lambda *shape, s: (torch.randn(*shape, generator=gen, device=dev) * s).to(torch.bfloat16)  # noqa: E731
        self.w_qkv = [rand(hidden, (hq + 2 * hkv) * D, s=1.5 * hidden ** -0.5) for _ in range(layers)]
        self.w_out = [rand(hidden, hidden, s=hidden ** -0.5) for _ in range(layers)]
        self.x = rand(self.batch, max(prompts), hidden, s=1.0)
        entries = [-(-(n + new_tokens) // page) for n in prompts]
        pages = sum(entries) + 1
        self.table = torch.full((self.batch, max(entries)), -1, dtype=torch.int32, device=dev)
        self.ring = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        self.lens, self.ring_state = ([torch.zeros(n, dtype=t, device=dev) for _ in range(2)] for n, t in ((self.batch, torch.int32), (2, torch.int64)))
        self.ring_state[0][1] = pages
        self.starts = torch.empty(self.batch + 1, dtype=torch.int32, device=dev)
        kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        scale = torch.full((hkv,), 0.02, device=dev) if e4m3 else None
        self.caches = []
        for _ in range(layers):
            k, v = (torch.zeros(pages, hkv, page, D, dtype=torch.bfloat16, device=dev).to(kind) for _ in range(2))
            bounds = torch.zeros(pages, hkv, 2, D, dtype=torch.bfloat16, device=dev)
            self.caches.append(cosa.make_cache(k, v, self.table, bounds=bounds, k_scale=scale, v_scale=scale))

    def plan(self, grow, slots):
        """Pages for `grow` new tokens of each request; the lengths after it are in self.lens[0]."""
        cosa.cosa_page_plan(self.table, self.page, self.lens[0], grow, self.ring, self.ring_state[0], self.lens[1], self.ring_state[1], self.starts, slots)
        self.lens.reverse()
        self.ring_state.reverse()

    def project(self, layer, x):
        """q, k, v as views [.., heads, d] into one buffer."""
        qkv = (x @ self.w_qkv[layer]).unflatten(-1, (self.hq + 2 * self.hkv, D))
        return qkv.split([self.hq, self.hkv, self.hkv], dim=-2)

    def prefill(self, budget: float = 0.25, tightened: float = 0.10):
        """All prompts at once, padded to the longest; returns the last token's hidden state of each."""
        dev, n = "cuda", max(self.prompts)
        lens = torch.tensor(self.prompts, dtype=torch.int32, device=dev)
        slots = torch.empty(sum(self.prompts), dtype=torch.int32, device=dev)
        self.plan(lens, slots)
        real = torch.arange(n, device=dev) < lens[:, None]      # the tokens that are no padding
        x, dense = self.x, all(c.structs[torch.bfloat16].cache_dtype == cosa.COSA_BF16 for c in self.caches)
        table = self.table[:, :n // self.page].contiguous()
        order = torch.empty(self.batch, self.hq, n // 128, n // 128, dtype=torch.int32, device=dev)
        count = torch.empty(self.batch, self.hq, n // 128, dtype=torch.int32, device=dev)
        out = torch.empty(self.batch, n, self.hq, D, dtype=torch.bfloat16, device=dev)
        for i, cache in enumerate(self.caches):
            q, k, v = self.project(i, x)
            cosa.cosa_cache_append(cache, k[real], v[real], slots)
            opt = cosa.default_options(order_stride=order.shape[-1], seq_lens=lens, skip_scale=0.3 * min(self.prompts))
            heads = lambda t: t.transpose(1, 2)  # noqa: E731
            ks, vs = heads(k), heads(v)
            if dense:      # straight from the pages (an 8-bit cache serves the tokens after the prompt)
                opt.kv_page_table, opt.kv_page_size, opt.kv_num_pages = table.data_ptr(), self.page, cache.num_pages
                ks, vs = cache.tensors[:2]
            cosa.cosa_kap_select(heads(q), ks, budget, order, count, opt=opt)
            cosa.cosa_osk_attention(heads(q), ks, vs, order, count, tightened, heads(out), opt=opt)
            x = x + out.flatten(2) @ self.w_out[i]
        return x[torch.arange(self.batch, device=dev), lens.long() - 1]

    def step(self, x, slots, grow, budget: float, lists=None, window: int = 0, seen=None):
        """One token of each request: x [B, hidden] -> [B, hidden].  `seen`: called with every layer's q, k, v and attention output."""
        self.plan(grow, slots)
        for i, cache in enumerate(self.caches):
            q, k, v = self.project(i, x)
            out = torch.empty(self.batch, self.hq, D, dtype=torch.bfloat16, device="cuda")
            cosa.cosa_cache_append(cache, k, v, slots)
            pages = count = None
            if budget < 1.0:
                pages, count = lists
                cosa.cosa_decode_select(cache, q, self.lens[0], budget, pages, count, min_pages=2, keep_first=1, keep_last=1)
            cosa.cosa_decode_attention(cache, q, self.lens[0], out, pages=pages, count=count, window=window)
            if seen is not None:
                seen(i, q, k, v, out)
            x = x + out.flatten(1) @ self.w_out[i]
        return x / x.float().square().mean(-1, keepdim=True).sqrt().to(x.dtype)

    def lists(self, budget: float):
        most = max(cosa.cosa_budget_count(budget, self.table.shape[1]), 2)
        return (torch.empty(self.batch, self.hkv, most, dtype=torch.int32, device="cuda"),
                torch.empty(self.batch, self.hkv, dtype=torch.int32, device="cuda"))


def step_time(stack: Stack, x, budget: float, tokens: int) -> float:
    """Milliseconds of a step, from one captured graph that takes two tokens (the length buffers change places each step)."""
    slots, grow, lists = torch.empty(stack.batch, dtype=torch.int32, device="cuda"), torch.ones(stack.batch, dtype=torch.int32, device="cuda"), stack.lists(budget)
    state = x.clone()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())

    def two():
        for _ in range(2):
            state.copy_(stack.step(state, slots, grow, budget, lists))

    with torch.cuda.stream(stream):
        two()
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        two()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    graph.replay()
    begin.record()
    for _ in range(tokens // 2):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / (tokens // 2 * 2)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--prompts", default="32768,16384,8192,24576", help="prompt lengths, multiples of 128")
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--page", type=int, default=64)
    p.add_argument("--budget", type=float, default=0.10, help="share of the pages a new token attends to; 1: all")
    p.add_argument("--e4m3", action="store_true", help="8-bit cache")
    a = p.parse_args()
    prompts = [int(n) for n in a.prompts.split(",")]
    if min(prompts) < 1 or any(n % 128 for n in prompts):
        p.error("prompts have to be multiples of 128")
    if a.page < 8 or a.page & (a.page - 1) or max(prompts) % a.page:
        p.error("the page size has to be a power of two from 8 on that divides the longest prompt")
    if a.tokens < 2 or not 0 < a.budget <= 1:
        p.error("at least two tokens, and a budget in (0, 1]")
    torch.cuda.set_device(0)
    for budget in dict.fromkeys((a.budget, 1.0)):
        stack = Stack(prompts, a.tokens + 8, layers=a.layers, page=a.page, e4m3=a.e4m3)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        x = stack.prefill()
        end.record()
        torch.cuda.synchronize()
        first = begin.elapsed_time(end)
        ms = step_time(stack, x, budget, a.tokens)
        status = cosa.cosa_device_status()
        if status:
            raise SystemExit(f"device status {status}")
        print(f"prompts {prompts}, {a.layers} layers, {'e4m3' if a.e4m3 else 'bf16'} pages of {a.page}: prompt {first:.2f} ms (cold), "
              f"token {ms * 1e3:.1f} us over {'all pages' if budget >= 1 else f'{budget:.0%} of the pages'}")


if __name__ == "__main__":
    main()
