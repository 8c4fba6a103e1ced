"""A decoder block with quantized layers, from prompts to generated tokens.

The seven projections are the package's W4A4 layers; between them run its norms and
residual sums, its head norms and rotation, its paged key-value cache (16, 8 or 4 bits)
and its attentions: of prompts, of the newest token, and of that over a prefix that all
streams share.  The MLP's activation is torch's.  Weights and inputs are random, of
Qwen3-8B's sizes by default.

    python3 examples/decode_block.py --bits 4 --streams 32 --prompt 1000 --tokens 64 --graph
    python3 examples/decode_block.py --streams 32 --shared 8192 --prompt 100 --tokens 64 --graph

prints the time of a decode step.  ``Block`` is what a program would keep.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_01556_amd as tq                                              # noqa: E402


class Pages:
    """Which pages of a cache each stream holds: a program's block manager, at its
    simplest.  `shared` tokens (whole pages) that all streams begin with are held once."""

    def __init__(self, streams: int, tokens: int, page_size: int, seed: int = 0, shared: int = 0):
        assert shared % page_size == 0, "a shared prefix ends with a page"
        self.page_size, self.each, self.shared = page_size, -(-tokens // page_size), shared
        front = shared // page_size
        order = torch.randperm(front + streams * self.each, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.count = order.numel()
        self.prefix, self.table = order[None, :front], order[front:].view(streams, self.each)
        # what a stream's tokens attend to as one sequence: the shared pages, then its own
        self.whole = torch.cat((self.prefix.expand(streams, -1), self.table), 1).contiguous()
        self.members = torch.tensor([0, streams], dtype=torch.int32, device="cuda")
        self.prefix_lengths = torch.tensor([shared], dtype=torch.int32, device="cuda")

    def slots(self, stream, position):
        """Slot numbers of (stream, position) pairs, both int64, positions counted from the
        end of what is shared."""
        page = self.table[stream, position // self.page_size].long()
        return page * self.page_size + position % self.page_size


def rms_norm(x, eps=1e-6):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps)).to(x.dtype)


class Block:
    """One decoder block and its cache."""

    def __init__(self, hidden=4096, mlp=12288, heads=32, kv_heads=8, head_dim=128, rank=64, bits=16,
                 head_norms=True, pages=1024, page_size=16, positions=8192, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def layer(k, n):
            w = torch.randn(n, k, generator=gen, device="cuda").mul_(k ** -0.5).half()
            l1 = torch.randn(k, rank, generator=gen, device="cuda").mul_(0.3 * k ** -0.5).half()
            l2 = torch.randn(rank, n, generator=gen, device="cuda").mul_(0.3 * rank ** -0.5).half()
            return tq.Layer(w, l1, l2)

        d = head_dim
        self.heads, self.kv_heads, self.d = heads, kv_heads, d
        self.qkv = layer(hidden, (heads + 2 * kv_heads) * d)
        self.o, self.up, self.gate, self.down = layer(heads * d, hidden), layer(hidden, mlp), layer(hidden, mlp), layer(mlp, hidden)
        self.q_norm = self.k_norm = None
        if head_norms:
            self.q_norm = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).half()
            self.k_norm = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).half()
        self.attention_norm, self.mlp_norm = (torch.ones(hidden, device="cuda").half() for _ in range(2))
        self.rope = tq.rope_table(positions, d, base=1e6)
        self.cache = tq.empty_kv_cache(pages, page_size, kv_heads, d, bits)

    def heads_of(self, x):
        """q, k and v [tokens, heads, head_dim]: views of the fused projection."""
        y = self.qkv(tq.add_rms_norm(x, weight=self.attention_norm, return_sum=False)).view(x.shape[0], -1, self.d)
        return y.split((self.heads, self.kv_heads, self.kv_heads), 1)

    def rest(self, x, attended):
        x, h = tq.add_rms_norm(self.o(attended.reshape(x.shape[0], -1)), x, self.mlp_norm)
        return tq.add_rms_norm(self.down((torch.nn.functional.silu(self.gate(h).float()) * self.up(h)).half()), x)

    def prompt(self, x, positions, slots, starts, page_table, lengths):
        """x [tokens, hidden]: new tokens of streams, one stream after the other from rows
        `starts` on, the last of each stream's `lengths`: written to the cache, and
        attended to as the cache holds them.  (Exact attention: the layers' 4-bit quantizer
        turns last bits into steps of codes, and a token is to get here what it gets alone.)"""
        q, k, v = self.heads_of(x)
        q = tq.qk_norm_rope_append(self.cache, q, k, v, positions, self.rope, slots, self.q_norm, self.k_norm)
        return self.rest(x, tq.prompt_attention(self.cache, q, starts, page_table, lengths, exact=True))

    def decode(self, x, positions, slots, page_table, lengths, pages=None):
        """x [streams, hidden]: one new token of every stream, at `positions` and in
        `slots`; lengths count it.  pages: whose prefix the streams share."""
        q, k, v = self.heads_of(x)
        q = tq.qk_norm_rope_append(self.cache, q, k, v, positions, self.rope, slots, self.q_norm, self.k_norm)
        if pages is None:
            return self.rest(x, tq.paged_attention(self.cache, q, page_table, lengths))
        return self.rest(x, tq.shared_prefix_attention(self.cache, q, pages.members, pages.prefix, pages.prefix_lengths,
                                                       page_table, lengths, exact=True))


def captured(block, *tensors):
    """A graph of one decode step over these tensors, and the tensor of its result."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                 # everything the step loads or sets up, first
        block.decode(*tensors)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.decode(*tensors)
    return graph, y


def generate(block, pages, x, tokens, graph=False, shared=None):
    """The block's outputs for prompts x [streams, length, hidden] and for `tokens` new
    tokens of each stream (the block's last output taken as its next input, as there
    is no vocabulary here): [streams, length + tokens, hidden], and seconds a token.
    shared [pages.shared, hidden]: what all prompts begin with, computed once."""
    streams, length, hidden = x.shape
    front = pages.shared
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    if front:
        position = torch.arange(front, device="cuda")
        slots = pages.prefix[0, position // pages.page_size].long() * pages.page_size + position % pages.page_size
        block.prompt(shared, position.to(torch.int32), slots, ints(0, front), pages.prefix, ints(front))
    stream = torch.arange(streams, device="cuda")
    position = torch.arange(length, device="cuda")
    slots = pages.slots(stream.repeat_interleave(length), position.repeat(streams))
    starts = torch.arange(0, streams * length + 1, length, dtype=torch.int32, device="cuda")
    y = block.prompt(x.reshape(-1, hidden), (front + position).repeat(streams).to(torch.int32), slots, starts, pages.whole,
                     torch.full((streams,), front + length, dtype=torch.int32, device="cuda"))
    out = [y.view(streams, length, hidden)]
    # what a step reads: kept tensors, which a graph needs
    new = rms_norm(out[0][:, -1]).contiguous()
    lengths = torch.full((streams,), length + 1, dtype=torch.int32, device="cuda")
    positions, slots = lengths + (front - 1), pages.slots(stream, (lengths - 1).long())
    args = (new, positions, slots, pages.table, lengths, pages if front else None)
    step = captured(block, *args) if graph else None
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for t in range(tokens):
        if step is not None:
            step[0].replay()
            y = step[1].clone()
        else:
            y = block.decode(*args)
        out.append(y[:, None])
        if t + 1 < tokens:
            new.copy_(rms_norm(y))
            positions += 1
            lengths += 1
            slots.copy_(pages.slots(stream, (lengths - 1).long()))
    torch.cuda.synchronize()
    return torch.cat(out, 1), (time.perf_counter() - begin) / max(tokens, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, default=16, choices=(16, 8, 4))
    ap.add_argument("--streams", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--page-size", type=int, default=16)
    ap.add_argument("--shared", type=int, default=0, help="tokens that all prompts begin with, held once")
    ap.add_argument("--graph", action="store_true", help="replay a captured step")
    a = ap.parse_args()
    pages = Pages(a.streams, a.prompt + a.tokens, a.page_size, shared=a.shared)
    block = Block(bits=a.bits, pages=pages.count, page_size=a.page_size, positions=a.shared + a.prompt + a.tokens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.streams, a.prompt, 4096, generator=gen, device="cuda").half()
    shared = torch.randn(a.shared, 4096, generator=gen, device="cuda").half()
    generate(block, pages, x[:, :8], 2, a.graph, shared)
    y, seconds = generate(block, pages, x, a.tokens, a.graph, shared)
    print(f"{a.streams} streams of {a.shared} shared + {a.prompt} + {a.tokens} tokens, {a.bits}-bit cache: "
          f"{seconds * 1e6:.0f} us per decode step of one block; output rms {y.float().square().mean().sqrt():.3f}")


if __name__ == "__main__":
    main()
