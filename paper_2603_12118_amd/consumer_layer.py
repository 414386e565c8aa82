"""The attention part of one layer of the LLM task, over sequences that hold what the encoder task sent.

    python -m paper_2603_12118_amd.consumer_layer [--sequences N] [--steps N] [--block]

Rows of hidden states, text and placed embeddings alike, go through

    QKV (cs_linear_bf16) -> cs_qk_norm_rope -> cs_cache_write -> cs_attention_cache -> output projection (cs_linear_bf16)

first as chunks of a prompt, then one token of every sequence a step, the step recorded as a HIP graph that is replayed while the
lengths on the GPU grow.  ConsumerBlock is the whole layer, on the same pages and steps: the norms before and after (cs_norm_residual), the
projections with packed weights (cs_linear_packed) and a mixture of experts (cs_moe).  A position has three axes (time, height, width): a text token stands at (p, p, p), the tokens of an image at
its time and their place in the grid.  Run as a program it builds a layer of 3584 values, 28 heads on 4 key/value heads of 128, sends
every sequence an image between two texts, generates some tokens, checks the last step against attention over what cs_cache_read
returns, and prints the time of a prompt and of a step; with --block the same of the whole layer.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding as B


def prompt_positions(parts):
    """[tokens, 3] int32 and the next text position.  parts: a number of text tokens, or the (time, height, width) grid of an item."""
    rows, at = [], 0
    for part in parts:
        if isinstance(part, int):
            rows.append(np.repeat(np.arange(at, at + part)[:, None], 3, 1))
            at += part
        else:
            rows.append(at + np.stack(np.meshgrid(*map(np.arange, part), indexing="ij"), -1).reshape(-1, 3))
            at += max(part)
    return np.concatenate(rows).astype(np.int32), at


class PagePool:
    """The pages of the sequences that a layer serves, kept on the host; `table` is their copy on the GPU (-1: no page)."""

    def __init__(self, n_pages: int, page_tokens: int, sequences: int, width: int, device, max_tokens=None):
        """width: pages a sequence may have; max_tokens: tokens, where they end inside the last page."""
        self.max_tokens = width * page_tokens if max_tokens is None else min(max_tokens, width * page_tokens)
        self.page_tokens, self.free = page_tokens, list(range(n_pages))[::-1]
        self.owned, self.lens, self.releases = [[] for _ in range(sequences)], [0] * sequences, [0] * sequences
        self.table = torch.full((sequences, width), -1, dtype=torch.int32, device=device)

    def reserve(self, b: int, tokens: int) -> None:
        """Pages for `tokens` tokens of sequence b in all."""
        self.reserve_all({b: tokens})

    def reserve_all(self, tokens) -> None:
        """Pages for tokens[b] tokens in all of every sequence b of a dict; none for any of them where there is no room for one."""
        new, left = {}, len(self.free)
        for b, n in tokens.items():
            new[b] = max(0, -(-n // self.page_tokens) - len(self.owned[b]))
            left -= new[b]
            if left < 0 or n > self.max_tokens:
                raise RuntimeError(f"no room for {n} tokens of sequence {b}")
        for b, n in new.items():
            if n:
                pages, at = [self.free.pop() for _ in range(n)], len(self.owned[b])
                self.table[b, at:at + n] = torch.tensor(pages, dtype=torch.int32, device=self.table.device)
                self.owned[b] += pages

    def slots(self, b: int, first: int, tokens: int) -> np.ndarray:
        t = np.arange(first, first + tokens)
        return np.asarray(self.owned[b], np.int64)[t // self.page_tokens] * self.page_tokens + t % self.page_tokens

    def release(self, b: int) -> None:
        """Sequence b has ended: its pages are another's to take.  Recorded steps leave it out (DecodeStep.take)."""
        self.free += self.owned[b][::-1]
        self.owned[b], self.lens[b] = [], 0
        self.releases[b] += 1
        self.table[b] = -1


class ConsumerLayer:
    def __init__(self, hidden=3584, n_heads=28, n_kv_heads=4, head_dim=128, sections=(16, 24, 24), theta=1e6, max_position=32768,
                 n_pages=1024, page_tokens=64, sequences=8, max_keys=8192, seed=0, device="cuda:0"):
        g = torch.Generator(device).manual_seed(seed)
        self.hidden, self.n_heads, self.n_kv_heads, self.head_dim, self.sections, self.max_keys = hidden, n_heads, n_kv_heads, head_dim, sections, max_keys
        width, inner = (n_heads + 2 * n_kv_heads) * head_dim, n_heads * head_dim
        bf16 = dict(generator=g, device=device, dtype=torch.bfloat16)
        self.w_qkv, self.w_out = torch.randn(width, hidden, **bf16) * hidden ** -0.5, torch.randn(hidden, inner, **bf16) * inner ** -0.5
        self.b_qkv = torch.randn(width, generator=g, device=device) * 0.1
        self.q_gain, self.k_gain = (1 + 0.1 * torch.randn(head_dim, generator=g, device=device) for _ in range(2))
        pairs = sum(sections)
        angles = torch.arange(max_position, dtype=torch.float64)[:, None] * theta ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
        self.cos_sin = torch.stack((angles.cos(), angles.sin()), -1).float().to(device)
        self.pages = PagePool(n_pages, page_tokens, sequences, -(-max_keys // page_tokens), device, max_keys)
        self.pool = torch.zeros(n_pages, B.cs_cache_query(n_kv_heads, head_dim, page_tokens)[0], dtype=torch.uint8, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.device = device

    def project(self, x, out, name):
        """out = x times the weights `name`, "qkv" (with its bias) or "out"."""
        B.cs_linear_bf16(x, self.w_qkv if name == "qkv" else self.w_out, self.b_qkv if name == "qkv" else None, out)

    def forward(self, x, positions, slots, cu, n_keys, table, max_queries, max_keys):
        """x [T, hidden] bf16 -> [T, hidden] bf16, and the queries and their attention [T, heads, head_dim]; enqueues only."""
        T, h, kv, d = x.shape[0], self.n_heads, self.n_kv_heads, self.head_dim
        qkv = torch.empty(T, h + 2 * kv, d, dtype=torch.bfloat16, device=x.device)
        self.project(x, qkv.view(T, -1), "qkv")
        q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
        B.cs_qk_norm_rope(q, k, self.cos_sin, positions, self.sections, self.q_gain, self.k_gain, q_out=q, k_out=k, err_flag=self.err)
        B.cs_cache_write(self.pool, k, v, slots, self.pages.page_tokens, err_flag=self.err)
        a = B.cs_attention_cache(q, self.pool, table, n_keys, cu, max_queries, max_keys, kv, self.pages.page_tokens, err_flag=self.err)
        out = torch.empty(T, self.hidden, dtype=torch.bfloat16, device=x.device)
        self.project(a.view(T, -1), out, "out")
        return out, q, a

    def prefill(self, which, rows, positions):
        """New tokens of the sequences `which`: rows[i] [n, hidden] bf16 and positions[i] int32 [n, 3] on the GPU.  Returns what forward does.
        Where there is no room, or a call refuses its tensors, no sequence is longer than before."""
        parts, after = [], {}
        for b, x in zip(which, rows):
            first = after.get(b, self.pages.lens[b])
            parts.append((b, first, x.shape[0]))
            after[b] = first + x.shape[0]
        self.pages.reserve_all(after)
        lens, keys = [x.shape[0] for x in rows], [first + n for _, first, n in parts]
        dev = dict(device=self.device)
        got = self.forward(torch.cat(rows), torch.cat(positions), torch.as_tensor(np.concatenate([self.pages.slots(*x) for x in parts]), **dev),
                           torch.as_tensor(np.cumsum([0] + lens, dtype=np.int32), **dev), torch.tensor(keys, dtype=torch.int32, **dev),
                           self.pages.table[torch.tensor(which, **dev)], max(lens), max(keys))
        for b, n in after.items():
            self.pages.lens[b] = n
        return got


class ConsumerBlock(ConsumerLayer):
    """The whole layer.  Rows of the residual stream come in and go out (bf16).  A row without a slot, of a sequence that a step leaves out, is not
    looked at: its stream begins as zeros and goes through no expert, so that without keys to attend to it ends as zeros, whatever x holds there."""

    def __init__(self, hidden=3584, inter=1280, experts=16, top=2, shared=1, score="sigmoid", format="e2m1", residual_scale=1.0, block_scale=1.0,
                 post_norms=True, seed=0, device="cuda:0", **attention):
        """format: of the projections and the experts; post_norms: whether a block's output is normed before it enters the stream."""
        super().__init__(hidden=hidden, seed=seed, device=device, **attention)
        g = torch.Generator(device).manual_seed(seed + 1)
        bf16 = dict(generator=g, device=device, dtype=torch.bfloat16)
        self.packed = {"qkv": B.cs_weights_pack(self.w_qkv, format), "out": B.cs_weights_pack(self.w_out, format)}
        self.router = torch.randn(experts, hidden, **bf16) * hidden ** -0.5
        self.choice_bias = torch.zeros(experts, device=device) if score == "sigmoid" else None
        self.up = B.cs_weights_pack(torch.empty(experts + shared, 2 * inter, hidden, device=device, dtype=torch.bfloat16).normal_(0, hidden ** -0.5, generator=g), format)
        self.down = B.cs_weights_pack(torch.empty(experts + shared, hidden, inter, device=device, dtype=torch.bfloat16).normal_(0, inter ** -0.5, generator=g), format)
        gain = lambda: 1 + 0.1 * torch.randn(hidden, generator=g, device=device)
        self.attention_gain, self.expert_gain, self.next_gain = gain(), gain(), gain()
        self.post_gains = (gain(), gain()) if post_norms else (None, None)
        self.top, self.score, self.scales = top, score, dict(residual_scale=residual_scale, block_scale=block_scale)

    def project(self, x, out, name):
        B.cs_linear_packed(x, self.packed[name], bias=self.b_qkv if name == "qkv" else None, out=out)

    def forward(self, x, positions, slots, cu, n_keys, table, max_queries, max_keys):
        """Rows of the residual stream x [T, hidden] bf16 -> the stream behind the layer, and the queries and their attention; enqueues only.
        What went through is kept in `stages` until the next call: the layers' inputs and outputs and, as `next`, the stream normed for the next layer."""
        live = slots >= 0
        x = torch.where(live[:, None], x, 0)
        # the stream's norm alone: x / 2 + x / 2 is x to the bit, and an infinity stays one (times a block scale of zero it would be a NaN)
        _, y = B.cs_norm_residual(x, x, self.attention_gain, residual_scale=0.5, block_scale=0.5)
        a, q, attended = super().forward(y, positions, slots, cu, n_keys, table, max_queries, max_keys)
        r, z = B.cs_norm_residual(a, x, self.expert_gain, post_gain=self.post_gains[0], **self.scales)
        m, experts, weights = B.cs_moe(z, self.router, self.up, self.down, self.top, score=self.score, choice_bias=self.choice_bias, live=live)
        out, following = B.cs_norm_residual(m, r, self.next_gain, post_gain=self.post_gains[1], **self.scales)
        self.stages = dict(x=x, y=y, a=a, r=r, z=z, live=live, m=m, experts=experts, weights=weights, out=out, next=following)
        return out, q, attended


class DecodeStep:
    """One token of every sequence of a layer, recorded once: fill `x`, call `run`, read `out`.  Lengths, positions and slots stay on the
    GPU and advance in the recording; the host only sees to it that the pages are there.  A sequence that was released is left out: its row of
    `x` goes nowhere, its rows of `out` and `attended` are zeros, until `take` hands the step the sequence that is in its place.  One that was
    given tokens by other calls has to be taken again, too: until then `run` refuses."""

    def __init__(self, layer: ConsumerLayer, next_position):
        """next_position: of every sequence the position of its next token, or None where the step is to leave it out."""
        self.layer, n, dev = layer, len(layer.pages.lens), layer.device
        if len(next_position) != n:
            raise ValueError(f"next_position: expected {n}, one a sequence")
        self.x = torch.zeros(n, layer.hidden, dtype=torch.bfloat16, device=dev)
        self.n_keys, self.ahead = (torch.zeros(n, dtype=torch.int32, device=dev) for _ in range(2))       # ahead: tokens a step adds, 0 or 1
        self.live, self.positions = torch.zeros(n, dtype=torch.bool, device=dev), torch.zeros(n, 3, dtype=torch.int32, device=dev)
        self.serves, self.releases, self.lens, self.next = [False] * n, [0] * n, [0] * n, [0] * n
        self.cu = torch.arange(n + 1, dtype=torch.int32, device=dev)
        # (a warm-up pass runs the calls once outside the recording, on a length of zero and no slot: it changes no cache)
        self.slots, self.no_slot = torch.full((n,), -1, dtype=torch.int64, device=dev), torch.full((n,), -1, dtype=torch.int64, device=dev)
        self._pass(torch.zeros_like(self.n_keys))
        for b, position in enumerate(next_position):
            self.take(b, position)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            P = layer.pages.page_tokens
            page = layer.pages.table.gather(1, (self.n_keys // P).long()[:, None])[:, 0].long()
            torch.where(self.live, torch.add(self.n_keys % P, page, alpha=P), self.no_slot, out=self.slots)
            self.n_keys += self.ahead
            self.out, self.q, self.attended = self._pass(self.n_keys)
            self.positions += self.ahead[:, None]

    def take(self, b: int, next_position) -> None:
        """From now on the step serves sequence b as the layer holds it, its next token at `next_position`, or leaves it out (None)."""
        pages = self.layer.pages
        self.serves[b], self.releases[b], self.lens[b] = next_position is not None, pages.releases[b], pages.lens[b]
        self.live[b] = self.ahead[b] = self.serves[b]
        self.next[b] = next_position if self.serves[b] else 0
        self.n_keys[b], self.positions[b] = pages.lens[b] if self.serves[b] else 0, self.next[b]

    def _pass(self, n_keys):
        layer = self.layer
        return layer.forward(self.x, self.positions, self.slots, self.cu, n_keys, layer.pages.table, 1, layer.max_keys)

    def run(self):
        pages = self.layer.pages
        for b in range(len(pages.lens)):
            if self.serves[b] and self.releases[b] != pages.releases[b]:
                self.take(b, None)
            if self.serves[b] and self.lens[b] != pages.lens[b]:
                raise RuntimeError(f"sequence {b} has {pages.lens[b]} tokens, {self.lens[b]} of them known to the step: take({b}, its next position)")
        served = [b for b in range(len(pages.lens)) if self.serves[b]]
        for b in served:                                      # (the calls would leave its rows as they are and set the flag)
            if not 0 <= self.next[b] < len(self.layer.cos_sin):
                raise RuntimeError(f"sequence {b}: position {self.next[b]} is not in the rotary table of {len(self.layer.cos_sin)}")
        pages.reserve_all({b: pages.lens[b] + 1 for b in served})
        self.graph.replay()
        for b in served:
            pages.lens[b] += 1
            self.lens[b] += 1
            self.next[b] += 1
        return self.out


def attention_of_cached(layer: ConsumerLayer, b: int, q):
    """Attention of the newest queries [n, heads, head_dim] of sequence b in fp32, over what cs_cache_read returns."""
    n = layer.pages.lens[b]
    slots = torch.as_tensor(layer.pages.slots(b, 0, n), device=q.device)
    k, v = B.cs_cache_read(layer.pool, slots, layer.n_kv_heads, layer.head_dim, layer.pages.page_tokens, dtype=torch.float32)
    group = layer.n_heads // layer.n_kv_heads
    k, v = (x.repeat_interleave(group, 1).transpose(0, 1).contiguous() for x in (k, v))
    s = q.float().transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() * layer.head_dim ** -0.5
    seen = torch.arange(n, device=q.device) <= torch.arange(n - q.shape[0], n, device=q.device)[:, None]
    return (s.masked_fill(~seen, float("-inf")).softmax(-1) @ v).transpose(0, 1)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--block", action="store_true", help="the whole layer, with norms and experts")
    a = ap.parse_args()
    grid, before, after = (1, 16, 16), 24, 200
    positions, following = prompt_positions([before, grid, after])
    n = len(positions)
    layer = (ConsumerBlock if a.block else ConsumerLayer)(sequences=a.sequences, max_keys=max(1024, n + a.steps), n_pages=a.sequences * (-(-(n + a.steps) // 64)))
    gen = torch.Generator(layer.device).manual_seed(1)
    rows, placed = [], torch.arange(before, before + grid[1] * grid[2], device=layer.device)
    for _ in range(a.sequences):
        x = torch.randn(n, layer.hidden, generator=gen, device=layer.device, dtype=torch.bfloat16)      # text rows; the image's are overwritten:
        B.cs_forward_embeddings(torch.randn(len(placed), layer.hidden, generator=gen, device=layer.device, dtype=torch.bfloat16), placed, x)
        rows.append(x)
    pos = torch.as_tensor(positions, device=layer.device)
    timer = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    for b in range(a.sequences):
        if b == a.sequences - 1:
            timer[0].record()
        for first in range(0, n, 256):                     # chunks of a prompt
            layer.prefill([b], [rows[b][first:first + 256]], [pos[first:first + 256]])
    timer[1].record()
    step = DecodeStep(layer, [following] * a.sequences)
    timer[2].record()
    for _ in range(a.steps):
        step.x.normal_(generator=gen)
        step.run()
    timer[3].record()
    torch.cuda.synchronize()
    worst = max((step.attended[b:b + 1].float() - attention_of_cached(layer, b, step.q[b:b + 1])).abs().max().item() for b in range(a.sequences))
    print(f"{a.sequences} sequences of {n} tokens ({grid[1] * grid[2]} of an image), {a.steps} generated: prompt {timer[0].elapsed_time(timer[1]):.3f} ms, "
          f"step {timer[2].elapsed_time(timer[3]) / max(a.steps, 1):.3f} ms, cache {layer.pool.numel() / 2 ** 20:.1f} MiB, "
          f"largest difference from attention over cs_cache_read {worst:.4f}, flag {layer.err.item()}")
    if worst > 0.02 or layer.err.item():
        raise SystemExit("the cache's attention and attention over what the cache holds differ")


if __name__ == "__main__":
    main()
