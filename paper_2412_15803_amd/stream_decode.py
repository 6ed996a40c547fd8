"""A batch of conversations in a sliding window, from prompt to token, the way a
server runs them on this library:

    python -m paper_2412_15803_amd.stream_decode [--prompts 3] [--samples 2] [--steps 64]

A small decoder with random 4-bit weights reads its prompts (window_attention
over rows of several sequences), forks each into samples (cache_fork), and
generates a token for every sample and step: pages for the tokens that come
(cache_reserve), the 4-bit linears (wq_gemv), the new keys and values
(cache_append), attention of one token each (window_attention), pages that the
window has left behind given back (cache_free), and the next token under
penalties and a mask (process_logits).  At the end some samples leave and the
pool is compacted (cache_compact).

The lengths, tables and tokens stay on the device throughout.  Embeddings, norms
and the gated product are torch operations here; the model has no positions.
"""

from __future__ import annotations

import argparse
import math
import time

import torch

from . import wq


class Decoder:
    """Random 4-bit weights of a small decoder, on one device."""

    def __init__(self, layers=2, hidden=512, q_heads=8, kv_heads=2, dim=64, inter=1024, vocab=2053, seed=0, device="cuda"):
        self.layers, self.hidden, self.q_heads, self.kv_heads, self.dim, self.inter, self.vocab = layers, hidden, q_heads, kv_heads, dim, inter, vocab
        self.device = torch.device(device)
        g = torch.Generator(device=device).manual_seed(seed)
        self.embedding = torch.randn((vocab, hidden), generator=g, device=device).half()
        qkv = (q_heads + 2 * kv_heads) * dim
        self.weights = [[self._pack(g, n, k) for n, k in ((qkv, hidden), (hidden, q_heads * dim), (2 * inter, hidden), (hidden, inter))]
                        for _ in range(layers)]
        self.head = self._pack(g, vocab, hidden)

    def _pack(self, g, n, k):
        w = torch.randn((n, k), generator=g, device=self.device).mul_(1.0 / math.sqrt(k))
        packed = torch.empty((n, k // 8), dtype=torch.int32, device=self.device)
        scales = torch.empty((n, k // 32), dtype=torch.float16, device=self.device)
        wq.wq_pack(w, packed, scales)
        return packed, scales

    def linear(self, weight, x):
        y = torch.empty((x.shape[0], weight[0].shape[0]), dtype=torch.float16, device=self.device)
        wq.wq_gemv(*weight, x, y)
        return y

    @staticmethod
    def norm(x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).half()

    def forward(self, tokens, cache, new_lens, q_starts, max_query_len):
        """Logits [tokens, vocab] of new tokens, whose keys and values go to the cache."""
        h = self.embedding[tokens.long()]
        rows, hq, hkv = tokens.shape[0], self.q_heads, self.kv_heads
        for layer, (qkv_w, o_w, gate_up_w, down_w) in enumerate(self.weights):
            qkv = self.linear(qkv_w, self.norm(h)).view(rows, hq + 2 * hkv, self.dim)
            k_cache, v_cache = cache.layer(layer)
            wq.cache_append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], k_cache, v_cache, cache.table, new_lens, q_starts=q_starts)
            out = torch.empty((rows, hq, self.dim), dtype=torch.float16, device=self.device)
            wq.window_attention(qkv[:, :hq], k_cache, v_cache, cache.table, new_lens, out, 1.0 / math.sqrt(self.dim), cache.max_len,
                                cache.window, sinks=cache.sinks, q_starts=q_starts, max_query_len=max_query_len)
            h = h + self.linear(o_w, out.view(rows, -1))
            gate, up = self.linear(gate_up_w, self.norm(h)).chunk(2, dim=-1)
            h = h + self.linear(down_w, (torch.nn.functional.silu(gate.float()) * up.float()).half())
        return self.linear(self.head, self.norm(h))


class Cache:
    """A paged cache of `slots` sequences that see `window` tokens and the first
    `sinks`; all its state is on the device."""

    def __init__(self, model, slots, max_len, window, sinks, page=16, pages=None):
        self.window, self.sinks, self.page, self.max_len = window, sinks, page, max_len
        width = -(-max_len // page)
        pages = pages or slots * width
        shape = (pages, model.kv_heads, page, model.dim)
        self.arrays = [torch.zeros(shape, dtype=torch.float16, device=model.device) for _ in range(2 * model.layers)]
        self.set = wq.cache_set(self.arrays)
        ints = dict(dtype=torch.int32, device=model.device)
        self.table, self.refs = torch.full((slots, width), -1, **ints), torch.zeros(pages, **ints)
        self.lens, self.shortfall, self.live = torch.zeros(slots, **ints), torch.zeros(1, **ints), torch.zeros(1, **ints)
        self.lacked = torch.zeros(1, **ints)  # the largest shortfall so far
        self.workspace = wq.page_workspace(pages, slots, model.device)

    def layer(self, i):
        return self.arrays[2 * i], self.arrays[2 * i + 1]

    def reserve(self, new_lens):
        wq.cache_reserve(self.table, self.refs, self.lens, new_lens, self.page, self.shortfall, workspace=self.workspace)
        torch.maximum(self.lacked, self.shortfall, out=self.lacked)

    def slide(self, seqs):
        """Give back what the window of the listed sequences has left behind."""
        wq.cache_free(self.table, self.refs, self.lens, seqs, self.page, window=self.window, sinks=self.sinks)

    def drop(self, seqs):
        wq.cache_free(self.table, self.refs, self.lens, seqs, self.page)
        self.lens[seqs.long()] = 0

    def fork(self, src, dst):
        wq.cache_fork(self.set, self.table, self.refs, self.lens, src, dst, self.shortfall, workspace=self.workspace)
        torch.maximum(self.lacked, self.shortfall, out=self.lacked)

    def check(self):
        """Raise if the pool was ever too small (waits for the device)."""
        lacked = int(self.lacked)
        if lacked:
            raise RuntimeError(f"the pool of {self.refs.numel()} pages was {lacked} too small")

    def compact(self):
        wq.cache_compact(self.set, self.table, self.refs, self.table, self.refs, self.live, workspace=self.workspace)


def generate(model, prompts, samples, steps, window, sinks, page=16, allowed=None, repetition=1.1, frequency=0.1, presence=0.1,
             pages=None, room=0):
    """Token histories [len(prompts) * samples] of `steps` generated words each,
    the last step's logits, and the cache.  allowed: a mask as process_logits
    takes it, one row; room: words that the cache can take after the last.
    Raises when the pool of `pages` is too small or a step has no word to choose."""
    if not prompts or not all(len(p) for p in prompts):
        raise ValueError("there must be prompts, and a word in each")
    device = model.device
    ints = dict(dtype=torch.int32, device=device)
    n, slots = len(prompts), len(prompts) * samples
    lens = [len(p) for p in prompts]
    longest = max(lens)
    cache = Cache(model, slots, longest + steps + room, window, sinks, page, pages)
    history = torch.zeros((slots, longest + steps), **ints)
    for i, p in enumerate(prompts):
        history[i, :lens[i]] = torch.tensor(p, **ints)
    history_lens = torch.tensor(lens + [0] * (slots - n), **ints)
    rows = torch.arange(slots, device=device)
    token = torch.zeros(slots, **ints)
    mask = None if allowed is None else allowed.repeat(slots, 1)
    full = lambda x: torch.full((slots,), x, device=device)  # noqa: E731
    penalties = dict(repetition=full(repetition), frequency=full(frequency), presence=full(presence))

    # The prompts: all their tokens at once, then the samples share their pages.
    starts = torch.tensor([sum(lens[:i]) for i in range(n)] + [sum(lens)] * (slots - n + 1), **ints)
    cache.reserve(history_lens)
    flat = torch.cat([history[i, :m] for i, m in enumerate(lens)])
    logits = model.forward(flat, cache, history_lens, starts, longest)
    cache.lens.copy_(history_lens)
    if samples > 1:
        src = torch.arange(n, **ints).repeat_interleave(samples - 1)
        dst = torch.arange(n, slots, **ints)
        cache.fork(src, dst)
        source = torch.cat([torch.arange(n, device=device), src.long()])
    else:
        source = torch.arange(n, device=device)
    cache.check()
    history, prompt_lens = history[source].contiguous(), history_lens[source].contiguous()
    history_lens = prompt_lens.clone()
    logits = logits[starts[1:n + 1].long() - 1][source].contiguous()
    if samples > 1:  # the samples of a prompt differ in their first word
        nth = torch.cat([torch.zeros(n, device=device), 1 + torch.arange(slots - n, device=device) % (samples - 1)]).long()
        best = logits.float().topk(samples, dim=-1).indices
        logits[rows, best[rows, nth]] += 100.0
    every = torch.arange(slots, **ints)
    lowest = torch.zeros_like(token)  # -1 where a step found no word
    for _ in range(steps):
        wq.process_logits(logits, logits, token=token, mask=mask, history=history, history_lens=history_lens, prompt_lens=prompt_lens, **penalties)
        torch.minimum(lowest, token, out=lowest)
        history[rows, history_lens.long()] = token
        history_lens += 1
        cache.reserve(history_lens)
        logits = model.forward(token, cache, history_lens, None, 1)
        cache.lens.copy_(history_lens)
        cache.slide(every)
    cache.check()
    if int(lowest.min()) < 0:
        raise RuntimeError(f"no word was left to choose in sequences {(lowest < 0).nonzero().flatten().tolist()}")
    return history, history_lens, logits, cache


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--prompts", type=int, default=3)
    ap.add_argument("--samples", type=int, default=2)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--window", type=int, default=48)
    ap.add_argument("--sinks", type=int, default=4)
    args = ap.parse_args(argv)
    model = Decoder()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(model.vocab, (20 + 37 * i,), generator=g).tolist() for i in range(args.prompts)]
    generate(model, prompts, args.samples, 2, args.window, args.sinks)  # loads the kernels
    torch.cuda.synchronize()
    start = time.perf_counter()
    history, lens, _, cache = generate(model, prompts, args.samples, args.steps, args.window, args.sinks)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    slots = args.prompts * args.samples
    print(f"{slots} sequences, {args.steps} steps: {slots * args.steps / seconds:.0f} words/s")
    for i in range(slots):
        print(i, history[i, int(lens[i]) - min(12, args.steps):int(lens[i])].tolist())
    used = int((cache.refs > 0).sum())
    cache.drop(torch.arange(0, slots, 2, dtype=torch.int32, device="cuda"))
    cache.compact()
    print(f"pages: {cache.refs.numel()} in the pool, {used} in use, {int(cache.live)} after half of the sequences left, "
          f"highest now {int(cache.table.max())}")


if __name__ == "__main__":
    main()
