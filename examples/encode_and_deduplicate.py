"""Documents to duplicates on one GPU: a small text encoder built from the
package's operators turns packed token embeddings into unit rows, an IVF index
is laid out over them and every document is searched against the others.  With
``--train`` the encoder first takes a few gradient steps that pull the rows of
known duplicates together.

    python examples/encode_and_deduplicate.py [--docs 4000] [--train 3]

The documents are synthetic: random token embeddings, a tenth of them copies
of another document with some tokens changed.  The encoder's weights are
random, so the rows show near-copies only; what matters here is the path.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_03199_gb300 as sieve  # noqa: E402

WIDTH, HEADS, DIM, BUCKETS, REACH = 256, 4, 64, 32, 128


class Block:
    """Pre-norm attention with a residual: h + attention(norm(h)) projected."""

    def __init__(self, device, seed=0):
        g = torch.Generator(device).manual_seed(seed)

        def randn(*shape, scale):
            return scale * torch.randn(*shape, generator=g, device=device)

        self.norm_w = torch.ones(WIDTH, device=device)
        self.norm_b = torch.zeros(WIDTH, device=device)
        self.w_in = randn(WIDTH, 3 * HEADS * DIM, scale=WIDTH ** -0.5).bfloat16()
        self.w_out = randn(HEADS * DIM, WIDTH, scale=0.3 * (HEADS * DIM) ** -0.5).bfloat16()
        self.table = randn(BUCKETS, HEADS, scale=0.2)
        self.buckets = sieve.relative_buckets(BUCKETS, REACH, device=device)

    def forward(self, h, offsets):
        y, mean, rstd = sieve.layer_norm(h, self.norm_w, self.norm_b)
        qkv = (y @ self.w_in).view(-1, 3, HEADS, DIM)
        o, lse = sieve.attention(qkv[:, 0], qkv[:, 1], qkv[:, 2], offsets, table=self.table, buckets=self.buckets)
        out = h + o.view(-1, HEADS * DIM) @ self.w_out
        return out, (h, y, mean, rstd, qkv, o, lse)

    def backward(self, dout, saved, offsets):
        """Gradients by name; the input's under "h"."""
        h, y, mean, rstd, qkv, o, lse = saved
        o2 = o.view(-1, HEADS * DIM)
        do = (dout @ self.w_out.t()).view_as(o)
        dqkv = torch.empty_like(qkv)
        *_, dtable = sieve.attention_backward(do, qkv[:, 0], qkv[:, 1], qkv[:, 2], o, lse, offsets, table=self.table,
                                              buckets=self.buckets, grads=(dqkv[:, 0], dqkv[:, 1], dqkv[:, 2]))
        dqkv2 = dqkv.view(-1, 3 * HEADS * DIM)
        dh, dw, db = sieve.layer_norm_backward(dqkv2 @ self.w_in.t(), h, self.norm_w, mean, rstd)
        return {"norm_w": dw, "norm_b": db, "w_in": y.t() @ dqkv2, "w_out": o2.t() @ dout, "table": dtable,
                "h": dh + dout}

    def step(self, grads, rate):
        for name, grad in grads.items():
            if name != "h":
                getattr(self, name).sub_(rate * grad)


def encode(block, tokens, offsets):
    h, saved = block.forward(tokens, offsets)
    rows, norms = sieve.unit_pool(h, offsets)
    return rows, (h, saved, norms)


def train_step(block, tokens, offsets, pairs, rate):
    """One step on the loss mean(1 - row_a . row_b) over known duplicates."""
    rows, (h, saved, norms) = encode(block, tokens, offsets)
    a, b = pairs[:, 0], pairs[:, 1]
    loss = (1 - (rows[a] * rows[b]).sum(1)).mean()
    drows = torch.zeros_like(rows)
    drows.index_add_(0, a, -rows[b] / len(pairs)).index_add_(0, b, -rows[a] / len(pairs))
    dh = sieve.unit_pool_backward(drows, rows, norms, offsets, h.shape[0], dtype=h.dtype)
    grads = block.backward(dh, saved, offsets)
    block.step(grads, rate)
    return loss, grads


def documents(n, device, seed=1):
    """Token embeddings of n documents of 1 to 200 tokens, their offsets, and
    the pairs (copy, original) planted among them."""
    g = torch.Generator(device).manual_seed(seed)
    lengths = torch.randint(1, 201, (n,), generator=g, device=device)
    copies = n // 10
    lengths[n - copies:] = lengths[:copies]
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)]).int()
    tokens = torch.randn(int(offsets[-1]), WIDTH, generator=g, device=device)
    head = int(offsets[copies])
    tail = int(offsets[n - copies])
    changed = torch.rand(head, generator=g, device=device) < 0.03
    tokens[tail:] = torch.where(changed[:, None], tokens[tail:], tokens[:head])
    pairs = torch.stack([torch.arange(n - copies, n, device=device), torch.arange(copies, device=device)], 1)
    return tokens.bfloat16(), offsets, pairs


def build_index(rows, nlist):
    """An index over the rows: sampled rows as centroids, every row with its nearest."""
    pick = torch.linspace(0, len(rows) - 1, nlist, device=rows.device).long()
    centroids = rows[pick].contiguous()
    assign = (rows @ centroids.t()).argmax(1).int()
    return sieve.build_layout(rows, assign, nlist, centroids)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--docs", type=int, default=4000)
    ap.add_argument("--train", type=int, default=0, help="gradient steps before the search")
    args = ap.parse_args(argv)
    device = torch.device("cuda:0")
    tokens, offsets, pairs = documents(args.docs, device)
    block = Block(device)
    losses = [float(train_step(block, tokens, offsets, pairs, rate=0.05)[0]) for _ in range(args.train)]
    rows, _ = encode(block, tokens, offsets)
    index = build_index(rows, nlist=max(1, args.docs // 100))
    nprobe = min(16, max(1, args.docs // 100))
    ids, scores, count, _ = sieve.search(index, rows, tau=0.9, k=5, nprobe=nprobe, W=min(4, nprobe),
                                         query_ids=torch.arange(args.docs, device=device))
    found = (ids[pairs[:, 0]] == pairs[:, 1:]).any(1)
    print(f"{args.docs} documents, {tokens.shape[0]} tokens: {int((count > 0).sum())} have a duplicate, "
          f"{int(found.sum())} of {len(pairs)} planted copies found"
          + (f"; loss {losses[0]:.4f} -> {losses[-1]:.4f} over {len(losses)} steps" if losses else ""))
    return dict(rows=rows, found=float(found.float().mean()), losses=losses)


if __name__ == "__main__":
    main()
