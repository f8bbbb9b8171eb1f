"""Decoding with a hybrid model: recurrent (Phalanx) layers and attention layers.

A layer takes the normed sum of the residual stream and the last layer's output in
8 bits (``swr_rms_norm``), projects it with 4-bit weights (``swr_fp4_linear``),
mixes over the sequence, and projects the result back:

  * a recurrent layer mixes with the sliding window recurrence, carrying its two
    states a channel (``swr_step``);
  * an attention layer appends the token's key and value to its paged cache
    (``swr_cache_append``) and attends over the request's pages
    (``swr_paged_attention``).  ``swr_block_tables`` hands out pages and slots, once a
    step for all of the layers.

The weights are random: what it shows is how the calls fit together, and what a
step takes.  Run it on a GPU:

    python examples/hybrid_decode.py [--layers RRARRA] [--batch 8] [--tokens 200]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import torch  # noqa: E402

import paper_2512_13921_amd as swr  # noqa: E402

BLOCK = 16   # of the recurrence's jagged window


class HybridDecoder:
    """``layers``: a string of R (recurrence of ``heads`` heads) and A (attention of
    ``q_heads`` heads of ``dim`` over ``kv_heads``)."""

    def __init__(self, layers, batch, width, heads, q_heads, kv_heads, dim, vocab, max_tokens, page_size=16, seed=0,
                 device="cuda:0"):
        self.layers, self.batch, self.width, self.heads = layers, batch, width, heads
        self.q_heads, self.kv_heads, self.dim, self.page_size = q_heads, kv_heads, dim, page_size
        rng = torch.Generator(device="cpu").manual_seed(seed)

        def packed(n, k):
            w = torch.randn(n, k, generator=rng) * k ** -0.5
            return swr.swr_fp4_pack(w.to(device, torch.bfloat16))

        self.embedding = torch.randn(vocab, width, generator=rng).to(device, torch.bfloat16)
        self.norms = [(1 + 0.1 * torch.randn(width, generator=rng)).to(device, torch.bfloat16) for _ in layers + "F"]
        self.into, self.out = [], []
        for kind in layers:
            mixed = width if kind == "R" else q_heads * dim
            # x, b, c and a decay a head; or queries, keys and values
            self.into.append(packed(3 * width + heads if kind == "R" else (q_heads + 2 * kv_heads) * dim, width))
            self.out.append(packed(width, mixed))
        self.head = packed(vocab, width)

        def i32(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)

        pages = -(-max_tokens // page_size)
        self.table = i32(batch, pages)
        self.table.fill_(-1)
        self.free = torch.arange(batch * pages, dtype=torch.int32, device=device)
        self.free_count = torch.full((1,), batch * pages, dtype=torch.int32, device=device)
        self.lengths, self.one_more = i32(batch), i32(batch) + 1
        cache = (batch * pages, page_size, kv_heads, dim)
        self.caches = [[torch.zeros(cache, dtype=torch.bfloat16, device=device) for _ in "kv"] if kind == "A" else None
                       for kind in layers]
        self.states = [torch.zeros(batch, heads, 2, width // heads, device=device) if kind == "R" else None
                       for kind in layers]
        self.position = 0

    def recurrence(self, i, z):
        """z [batch, 3 width + heads]: x, b, c and the decays' logits of one token."""
        width, shape = self.width, (self.batch, 1, self.heads, self.width // self.heads)
        x, b, c = (z[:, j * width:(j + 1) * width].unflatten(1, shape[1:]) for j in range(3))
        y, _ = swr.swr_step(x, z[:, None, 3 * width:], b, c, BLOCK, self.position, self.states[i], sigmoid_decay=True,
                            sigmoid_pregate=True)
        return y.reshape(self.batch, width)

    def attention(self, i, z, slots, lengths):
        """z [batch, (q_heads + 2 kv_heads) dim]: queries, keys and values of one token."""
        z = z.unflatten(1, (-1, self.dim))
        q, k, v = z.split((self.q_heads, self.kv_heads, self.kv_heads), 1)
        swr.swr_cache_append(k, v, *self.caches[i], slots)
        return swr.swr_paged_attention(q, *self.caches[i], self.table, lengths).flatten(1)

    def step(self, tokens):
        """Logits [batch, vocab] (float32) after one more token of each request."""
        slots, _, self.lengths, self.free_count = swr.swr_block_tables(
            self.lengths, self.one_more, self.table, self.free, self.free_count, self.page_size, self.batch)
        h, y = self.embedding[tokens], None
        for i, kind in enumerate(self.layers):
            if y is None:
                u, scale = swr.swr_rms_norm(h, self.norms[i], fp8=True)
            else:
                u, scale, h = swr.swr_rms_norm(h, self.norms[i], y, fp8=True)
            z = swr.swr_fp4_linear(u, *self.into[i], scale)
            z = self.recurrence(i, z) if kind == "R" else self.attention(i, z, slots, self.lengths)
            y = swr.swr_fp4_linear(z, *self.out[i])
        u, _ = swr.swr_rms_norm(h, self.norms[-1], y)
        self.position += 1
        return swr.swr_fp4_linear(u, *self.head, out_dtype=torch.float32)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", default="RRARRA")
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=200)
    args = ap.parse_args()
    if not args.layers or set(args.layers) - set("RA") or args.batch < 1 or args.tokens < 1:
        ap.error("layers must be a string of R and A, batch and tokens positive")
    model = HybridDecoder(args.layers, args.batch, width=2048, heads=32, q_heads=16, kv_heads=2, dim=128, vocab=8192,
                          max_tokens=args.tokens + 1)
    tokens = torch.arange(args.batch, device="cuda:0")
    tokens = model.step(tokens).argmax(1)   # (first calls load the kernels)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(args.tokens):
        tokens = model.step(tokens).argmax(1)
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"{len(args.layers)} layers ({args.layers}), {args.batch} requests, {args.tokens} tokens each: "
          f"{1e6 * took / args.tokens:.0f} us a step, {args.batch * args.tokens / took:.0f} tokens/s")


if __name__ == "__main__":
    main()
