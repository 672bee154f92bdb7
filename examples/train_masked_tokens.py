"""Training a text encoder on its own tokens, on one GPU: token ids become rows
of a table, blocks of attention and a feed-forward layer add to the residual
stream between two norms each, and the rows of masked tokens are scored
against the same table under a cross entropy.  After the steps every document is
pooled into the unit row that the deduplication search takes.

    python examples/train_masked_tokens.py [--docs 2000] [--steps 5]

The documents are synthetic: words drawn as often as in text, so a few steps
already learn their frequencies.  What matters here is the path: every operator
between the plain matrix products is the package's, forward and backward, and the
table's two gradients (as input and as output) add up in one tensor.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_03199_gb300 as sieve  # noqa: E402

WIDTH, HEADS, DIM, INNER, BUCKETS, REACH = 256, 4, 64, 512, 32, 128
MASK = 0                                            # the id that stands for a masked token


class Encoder:
    """Two blocks: h -> h + gate norm(attention(x)), h -> h + gate norm(feed-forward(x)),
    x the norm of the stream before each; master weights fp32, products bf16."""

    def __init__(self, vocab, device, seed=0):
        g = torch.Generator(device).manual_seed(seed)

        def randn(*shape, scale):
            return scale * torch.randn(*shape, generator=g, device=device)

        self.p = {"table": randn(vocab, WIDTH, scale=WIDTH ** -0.5), "out_bias": torch.zeros(vocab, device=device),
                  "w_qkv": randn(WIDTH, 3 * HEADS * DIM, scale=WIDTH ** -0.5),
                  "w_o": randn(HEADS * DIM, WIDTH, scale=(HEADS * DIM) ** -0.5),
                  "w_up": randn(WIDTH, INNER, scale=WIDTH ** -0.5), "w_down": randn(INNER, WIDTH, scale=INNER ** -0.5),
                  "rel": randn(BUCKETS, HEADS, scale=0.2)}
        for i in range(3):                          # before attention, before the feed-forward layer, before the loss
            self.p[f"norm{i}"] = torch.ones(WIDTH, device=device)
        for i in range(2):
            self.p[f"post{i}"], self.p[f"gate{i}"] = torch.ones(WIDTH, device=device), torch.full((WIDTH,), 0.5, device=device)
        self.buckets = sieve.relative_buckets(BUCKETS, REACH, device=device)

    def step_args(self, i):
        return dict(weight=self.p[f"norm{i + 1}"], post_weight=self.p[f"post{i}"], gate=self.p[f"gate{i}"], rms=True)

    def forward(self, ids, offsets):
        """The normed last rows, and what the backward pass needs."""
        w = {k: v.bfloat16() for k, v in self.p.items() if k.startswith("w_") or k == "table"}
        h0 = sieve.embed(ids, w["table"], scale=math.sqrt(WIDTH))
        x0, mean, rstd = sieve.layer_norm(h0, self.p["norm0"])
        qkv = (x0 @ w["w_qkv"]).view(-1, 3, HEADS, DIM)
        o, lse = sieve.attention(qkv[:, 0], qkv[:, 1], qkv[:, 2], offsets, table=self.p["rel"], buckets=self.buckets)
        y0 = o.view(-1, HEADS * DIM) @ w["w_o"]
        h1, x1, stats0 = sieve.residual_norm(h0, y0, **self.step_args(0))
        up = x1 @ w["w_up"]
        y1 = torch.relu(up) @ w["w_down"]
        h2, x2, stats1 = sieve.residual_norm(h1, y1, **self.step_args(1))
        return x2, (w, h0, x0, mean, rstd, qkv, o, lse, y0, h1, x1, stats0, up, y1, stats1)

    def backward(self, dx2, saved, ids, offsets, grads):
        """Adds to ``grads`` by name; the table's holds the loss' part already."""
        w, h0, x0, mean, rstd, qkv, o, lse, y0, h1, x1, stats0, up, y1, stats1 = saved
        dh1, dy1, grads["norm2"], _, grads["post1"], _, grads["gate1"] = sieve.residual_norm_backward(
            None, dx2, h1, y1, stats1, **self.step_args(1))
        act = torch.relu(up)
        grads["w_down"] = act.t() @ dy1
        dup = (dy1 @ w["w_down"].t()) * (up > 0)
        grads["w_up"] = x1.t() @ dup
        dh0, dy0, grads["norm1"], _, grads["post0"], _, grads["gate0"] = sieve.residual_norm_backward(
            dh1, dup @ w["w_up"].t(), h0, y0, stats0, **self.step_args(0))
        grads["w_o"] = o.view(-1, HEADS * DIM).t() @ dy0
        dqkv = torch.empty_like(qkv)
        *_, grads["rel"] = sieve.attention_backward(
            (dy0 @ w["w_o"].t()).view_as(o), qkv[:, 0], qkv[:, 1], qkv[:, 2], o, lse, offsets, table=self.p["rel"],
            buckets=self.buckets, grads=(dqkv[:, 0], dqkv[:, 1], dqkv[:, 2]))
        dqkv = dqkv.view(-1, 3 * HEADS * DIM)
        grads["w_qkv"] = x0.t() @ dqkv
        dx0, grads["norm0"], _ = sieve.layer_norm_backward(dqkv @ w["w_qkv"].t(), h0, self.p["norm0"], mean, rstd, need_dbias=False)
        sieve.embed_backward(dx0 + dh0, ids, self.p["table"].shape[0], scale=math.sqrt(WIDTH), out=grads["table"], accumulate=True)

    def loss_and_grads(self, ids, targets, offsets):
        """The mean loss over the tokens with a target, and every weight's gradient."""
        x, saved = self.forward(ids, offsets)
        table, bias = saved[0]["table"], self.p["out_bias"]
        loss, lse = sieve.cross_entropy(x, table, targets, bias=bias)
        share = 1 / (targets >= 0).sum().clamp(min=1)
        grads = {"table": torch.empty_like(self.p["table"])}
        dx, _, grads["out_bias"] = sieve.cross_entropy_backward(share.expand(len(loss)).contiguous(), x, table, targets, loss, lse,
                                                               bias=bias, dweight=grads["table"])
        self.backward(dx, saved, ids, offsets, grads)
        return loss.sum() * share, grads

    def rows(self, ids, offsets):
        return sieve.unit_pool(self.forward(ids, offsets)[0], offsets)[0]


def documents(n, vocab, device, seed=1):
    """Ids of n packed documents of 1 to 120 words (id 0 is the mask) and their offsets."""
    g = torch.Generator(device).manual_seed(seed)
    lengths = torch.randint(1, 121, (n,), generator=g, device=device)
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)]).int()
    u = torch.rand(int(offsets[-1]), generator=g, device=device).double()
    return torch.exp(u * math.log(vocab - 1)).long().clamp_(1, vocab - 1), offsets


def masked(ids, share, seed):
    """The ids with some hidden, and the hidden ones as targets (-1 elsewhere)."""
    g = torch.Generator(ids.device).manual_seed(seed)
    hide = torch.rand(ids.shape, generator=g, device=ids.device) < share
    return torch.where(hide, MASK, ids), torch.where(hide, ids, -1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--docs", type=int, default=2000)
    ap.add_argument("--vocab", type=int, default=20_000)
    ap.add_argument("--steps", type=int, default=5)
    args = ap.parse_args(argv)
    device = torch.device("cuda:0")
    ids, offsets = documents(args.docs, args.vocab, device)
    model = Encoder(args.vocab, device)
    losses = []
    for step in range(args.steps):
        hidden, targets = masked(ids, 0.15, seed=step)
        loss, grads = model.loss_and_grads(hidden, targets, offsets)
        for name, grad in grads.items():
            model.p[name].sub_(0.03 * grad)
        losses.append(float(loss))
    rows = model.rows(ids, offsets)
    print(f"{args.docs} documents, {len(ids)} tokens, {args.vocab} words; loss "
          + " ".join(f"{x:.3f}" for x in losses) + f"; {len(rows)} unit rows")
    return dict(losses=losses, rows=rows)


if __name__ == "__main__":
    main()
