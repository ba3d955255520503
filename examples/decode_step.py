"""A decoder block's decode step on the library's operators.

One block of a Llama-shaped model serves several streams at once, one new token each per step:

    rms_norm -> q, k, v (additive-codebook layers, one launch) -> each stream's own low-rank adapter beside q and v
    -> rotary positions and the cache's writing (one launch) -> paged attention -> o (additive-codebook layer)
    -> rms_norm with the residual, int8 output -> gate, up (4-bit layers on the int8 rows) -> silu * -> down (4-bit layer)

and a head's logits are answered with the log probabilities of chosen tokens, the entropy and alternatives,

with the precision level k of the additive-codebook layers chosen per step, the cache's pages
handed out by PagePool, and a stream forked in mid-decode (its pages shared until one of the two
writes). Silu and the head are plain torch. Run it on a GPU: ``python examples/decode_step.py``.
"""
from __future__ import annotations

import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_12876_amd as A  # noqa: E402


class DecodeBlock:
    """Weights, cache and one step of a block. ``aq``: QuantLinear layers by name (q, k, v, o); ``w4``:
    W4Linear layers by name (gate, up, down); ``norms``: two bf16 vectors; ``adapters``: Adapters by the names of
    layers in aq (q, k, v), of which a step's ``index`` picks each stream's."""

    def __init__(self, aq, w4, norms, heads: int, kv_heads: int, cache: A.KVCache, eps: float = 1e-5, adapters=None):
        self.aq, self.w4, self.norms, self.cache, self.eps, self.adapters = aq, w4, norms, cache, eps, adapters or {}
        self.rotary = A.Rotary.scaled(cache.head_dim)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, cache.head_dim
        self.hidden = norms[0].numel()

    def step(self, h, k_level: int, positions, slots, table, lengths, max_length: int, index=None):
        """h [n][hidden] bf16 -> the block's output; positions, slots int64 [n], table, lengths int32; index int32 [n]:
        each stream's adapter, -1 for none."""
        n, dev = h.shape[0], h.device
        x = torch.empty_like(h)
        A.rms_norm(h, self.norms[0], x, eps=self.eps)
        q, k, v = (torch.empty((n, heads, self.dim), dtype=h.dtype, device=dev)
                   for heads in (self.heads, self.kv_heads, self.kv_heads))
        A.gemv_multi([self.aq[name].handle for name in "qkv"], k_level, x, A.DType.BF16, n, [q, k, v], A.DType.BF16)
        if index is not None:
            for name, t in zip("qkv", (q, k, v)):
                if name in self.adapters:
                    self.adapters[name].add(x, index, t.view(n, -1), t.view(n, -1))
        self.cache.rotary_append(self.rotary, q, k, v, positions, slots, q)      # q in place
        o = torch.empty_like(q)
        self.cache.attention(q, table, lengths, o, max_length=max_length, scale=self.dim ** -0.5)
        a = self.aq["o"](o.view(n, -1), k_level)
        # the residual's addition, the norm and the scaling to int8 are one kernel
        x8 = torch.empty((n, self.hidden), dtype=torch.int8, device=dev)
        group = self.w4["gate"].group_size
        xs = torch.empty((n, -(-self.hidden // group)), dtype=torch.float32, device=dev)
        h2 = torch.empty_like(h)
        A.rms_norm(a, self.norms[1], x8, eps=self.eps, residual=h, residual_out=h2, scales=xs, scale_group=group)
        gate, up = self.w4["gate"](x8, xs), self.w4["up"](x8, xs)
        return h2 + self.w4["down"](torch.nn.functional.silu(gate) * up)


class Streams:
    """The streams of a server: page tables and lengths of one step, from a PagePool."""

    def __init__(self, pool: A.PagePool, caches, device="cuda"):
        self.pool, self.caches, self.device = pool, caches, device
        self.ready = {}                     # slots of streams extended in a step that then ran out of pages

    def copy(self, pairs):
        if pairs:
            src, dst = (torch.tensor(p, dtype=torch.int32).to(self.device) for p in zip(*pairs))
            A.kv_copy_pages(self.caches, src, dst)

    def free(self, seq):
        self.ready.pop(seq, None)
        self.pool.free(seq)

    def advance(self, seqs):
        """One more token for every stream: (positions, slots, table, lengths, max_length) on the GPU. Where the
        pool runs out of pages (ENOMEM), free a stream and call again."""
        pairs = []
        try:
            for s in seqs:
                if s not in self.ready:
                    self.ready[s], copies = self.pool.extend(s, 1)
                    pairs += copies
        finally:                            # what was given out stands, and a free may follow
            self.copy(pairs)
        slots = [self.ready.pop(s) for s in seqs]
        lengths = torch.tensor([self.pool.length(s) for s in seqs], dtype=torch.int32)
        tables = [self.pool.table(s) for s in seqs]
        table = torch.full((len(seqs), max(len(t) for t in tables)), -1, dtype=torch.int32)
        for i, t in enumerate(tables):
            table[i, :len(t)] = t
        return (lengths.long().to(self.device) - 1, torch.cat(slots).to(self.device), table.to(self.device),
                lengths.to(self.device), int(lengths.max()))


def answer(h, head, targets, n_top: int = 3):
    """What a stream's token gets back: (log probability of the given token, entropy, ids and log probabilities of
    the likeliest ones), from the head's logits of the rows h."""
    logits, n = h @ head, h.shape[0]
    lp, entropy = (torch.empty((n,), dtype=torch.float32, device=h.device) for _ in range(2))
    ids = torch.empty((n, n_top), dtype=torch.int64, device=h.device)
    tops = torch.empty((n, n_top), dtype=torch.float32, device=h.device)
    A.log_probs(logits, targets, lp, entropy=entropy, top_ids=ids, top_logprobs=tops)
    return lp, entropy, ids, tops


def random_adapters(block, n: int = 4, rank: int = 16, seed: int = 0):
    """n adapters beside q and v."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def make(d_out):
        a = torch.randn((n, rank, block.hidden), generator=g, device="cuda") * block.hidden ** -0.5
        b = torch.randn((n, d_out, rank), generator=g, device="cuda") * 0.3 * rank ** -0.5
        return A.Adapters(a.bfloat16(), b.bfloat16(), 0.5 + torch.rand((n,), generator=g, device="cuda"))

    return {"q": make(block.heads * block.dim), "v": make(block.kv_heads * block.dim)}


def random_block(hidden=512, heads=8, kv_heads=2, dim=64, ffn=1376, pages=64, page=16, cache_dtype=torch.bfloat16, seed=0):
    """A block with random weights, and its raw tensors for whoever wants to check it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    raw = {}

    def aq(name, d_out, d_in, M=4):
        codes = torch.randint(0, 256, (M, d_out, d_in // 8), generator=g, device="cuda").to(torch.uint8)
        books = (torch.randn((M, 256, 8), generator=g, device="cuda") * (0.5 / (M * d_in) ** 0.5)).to(torch.float16)
        scales = (0.5 + torch.rand((d_out,), generator=g, device="cuda")).to(torch.float16)
        raw[name] = (codes, books, scales)
        return A.QuantLinear(codes, books, scales)

    def w4(name, d_out, d_in, group=32):
        w = torch.randint(0, 256, (d_out, d_in // 2), generator=g, device="cuda").to(torch.uint8)
        s = (torch.rand((d_out, -(-d_in // group)), generator=g, device="cuda") * (0.4 / d_in ** 0.5)).to(torch.float16)
        raw[name] = (w, s)
        return A.W4Linear(w, s, group_size=group)

    layers = {"q": aq("q", heads * dim, hidden), "k": aq("k", kv_heads * dim, hidden), "v": aq("v", kv_heads * dim, hidden),
              "o": aq("o", hidden, heads * dim)}
    mlp = {"gate": w4("gate", ffn, hidden), "up": w4("up", ffn, hidden), "down": w4("down", hidden, ffn)}
    norms = [(1 + 0.1 * torch.randn((hidden,), generator=g, device="cuda")).bfloat16() for _ in range(2)]
    cache = A.KVCache.allocate(pages, page, kv_heads, dim, cache_dtype)
    return DecodeBlock(layers, mlp, norms, heads, kv_heads, cache), raw


def main():
    torch.manual_seed(0)
    block, _ = random_block(hidden=4096, heads=32, kv_heads=32, dim=128, ffn=11008, pages=256, cache_dtype=torch.float8_e4m3fn)
    block.adapters = random_adapters(block)
    head = (torch.randn((block.hidden, 32000), device="cuda") * 0.02).bfloat16()
    pool = A.PagePool(256, 16, 8)
    streams = Streams(pool, [block.cache])
    live = [pool.add() for _ in range(3)]
    for step in range(40):
        if step == 20:
            live.append(pool.fork(live[0]))          # shares its pages with stream 0 until either writes
        if step == 30:
            streams.free(live.pop(1))
            streams.copy(pool.compact())
        h = torch.randn((len(live), block.hidden), device="cuda").bfloat16()
        index = torch.tensor([s % 5 - 1 for s in live], dtype=torch.int32).to("cuda")      # stream 0 has no adapter
        h = block.step(h, 4 if step % 2 else 2, *streams.advance(live), index=index)
        lp, entropy, ids, _ = answer(h, head, torch.zeros((len(live),), dtype=torch.int64, device="cuda"))
        if step % 10 == 9:
            print(f"step {step + 1}: {len(live)} streams of {[pool.length(s) for s in live]} tokens, "
                  f"{pool.counts()[0]} pages free, |h| = {h.float().norm(dim=1).mean().item():.3f}, entropy "
                  f"{entropy.mean().item():.3f}, likeliest tokens {ids[:, 0].tolist()}")


if __name__ == "__main__":
    main()
