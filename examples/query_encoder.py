"""A query encoder in front of the index, trained and used on one GPU: tokens -> embedding rows -> layer norm -> projection to the
index's D dimensions (8-bit blocks) -> one vector a token, which the index is built from and asked with.

The texts are synthetic: a passage has a topic, half of its words belong to that topic and the others to none.  The encoder learns to bring
a topic's words near a point of their own (so many random points of D dimensions); then the words of held-out passages are the queries, and
the nearest database words vote for the passage's topic.

    python examples/query_encoder.py [--steps 60] [--topics 64] [--dims 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1702_05911_amd as pqt  # noqa: E402

LENGTH = 24              # words of a passage; shorter ones are padded with -1
WORDS_PER_TOPIC = 50


def passages(count, topics, seed, device):
    """(tokens count x LENGTH, topics count): half of a passage's words are its topic's, the others common ones."""
    g = torch.Generator().manual_seed(seed)
    topic = torch.randint(0, topics, (count,), generator=g)
    own = topic[:, None] * WORDS_PER_TOPIC + torch.randint(0, WORDS_PER_TOPIC, (count, LENGTH), generator=g)
    common = topics * WORDS_PER_TOPIC + torch.randint(0, 1000, (count, LENGTH), generator=g)
    tokens = torch.where(torch.rand((count, LENGTH), generator=g) < 0.5, own, common)
    tokens[torch.arange(LENGTH)[None, :] >= torch.randint(LENGTH // 2, LENGTH + 1, (count, 1), generator=g)] = -1
    return tokens.to(device), topic.to(device)


class Encoder:
    """Embedding, layer norm and projection; weights in fp32, what the operators read in bf16 and 8-bit blocks."""

    def __init__(self, vocabulary, width, dims, device, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.table = (0.02 * torch.randn((vocabulary, width), generator=g)).to(device)
        self.gain, self.shift = torch.ones(width, device=device), torch.zeros(width, device=device)
        self.weight = (torch.randn((dims, width), generator=g) / width ** 0.5).to(device)
        self.bias = torch.zeros(dims, device=device)
        self.scale = width ** 0.5
        self.values = (self.table, self.gain, self.shift, self.weight, self.bias)
        self.optimizer = torch.optim.Adam(self.values, lr=0.01)
        self.lay_out()

    def lay_out(self):
        """Once after each update: the table's bf16 copy, the projection's blocks and those of its transpose."""
        self.rows = self.table.to(torch.bfloat16)
        self.blocks, self.blocks_t = pqt.pqt_block_quantize(self.weight, columns=True)

    def encode(self, tokens):
        """One vector of `dims` floats a token."""
        y, _, _ = pqt.pqt_layer_norm(pqt.pqt_embed(self.rows, tokens, self.scale), self.gain, self.shift)
        return pqt.pqt_block_product(pqt.pqt_block_quantize(y), self.blocks, bias=self.bias, out_dtype=torch.float32)

    def step(self, tokens, target):
        """One training step on the mean squared distance to `target`; returns it.  The normalised rows are kept for the backward
        pass as the 8-bit blocks of their transpose."""
        x = pqt.pqt_embed(self.rows, tokens, self.scale)
        y, mean, rstd = pqt.pqt_layer_norm(x, self.gain, self.shift)
        y, kept = pqt.pqt_block_quantize(y, columns=True)
        off = pqt.pqt_block_product(y, self.blocks, bias=self.bias, out_dtype=torch.float32) - target
        off[tokens < 0] = 0.0
        grad = off * (2.0 / max(1, int((tokens >= 0).sum())))
        g, g_t = pqt.pqt_block_quantize(grad, columns=True)
        d_weight = pqt.pqt_block_product(g_t, kept, out_dtype=torch.float32)
        d_y = pqt.pqt_block_product(g, self.blocks_t, out_dtype=torch.bfloat16)
        d_x, d_gain, d_shift = pqt.pqt_layer_norm_gradient(d_y, x, self.gain, mean, rstd)
        d_table = pqt.pqt_embed_gradient(d_x, tokens, self.table.shape[0], self.scale)
        for value, d in zip(self.values, (d_table, d_gain, d_shift, d_weight, grad.sum(0))):
            value.grad = d
        self.optimizer.step()
        self.lay_out()
        return float(off.square().sum(1)[tokens >= 0].mean())


def run(steps=60, topics=64, dims=64, width=256, passages_per_step=512, device=0, say=print):
    """Returns (first and last loss, share of held-out passages whose topic the index finds)."""
    dev = torch.device("cuda", device)
    vocabulary = topics * WORDS_PER_TOPIC + 1000
    encoder = Encoder(vocabulary, width, dims, dev)
    points = torch.randn((topics, dims), generator=torch.Generator().manual_seed(1)).to(dev)
    losses = []
    for step in range(steps):
        tokens, topic = passages(passages_per_step, topics, 100 + step, dev)
        target = points[topic].repeat_interleave(LENGTH, 0)
        losses.append(encoder.step(tokens.flatten(), target))
        if step % 20 == 0 or step == steps - 1:
            say(f"step {step}: mean squared distance {losses[-1]:.3f}")
    # the database: the words of 4,000 passages
    tokens, topic = passages(4000, topics, 7, dev)
    words = tokens.flatten()
    there = words >= 0
    vectors, of_topic = encoder.encode(words[there]), topic.repeat_interleave(LENGTH)[there]
    index = pqt.builder.build_index_native(vectors, P=2, k1=16, k2=8, M=8, T=1024, C=2048, train_n=min(20_000, vectors.shape[0]), iters=10,
                                           device=device)
    # held-out passages: every word asks for its ten nearest, whose topics vote
    tokens, topic = passages(500, topics, 8, dev)
    words = tokens.flatten()
    ids, _ = pqt.pqt_query_batch(index, encoder.encode(words), 10, 8)
    votes = torch.zeros((500, topics), device=dev)
    valid = (ids >= 0) & (words >= 0)[:, None]
    passage = torch.arange(500, device=dev).repeat_interleave(LENGTH)[:, None].expand_as(ids)
    votes.index_put_((passage[valid], of_topic[ids[valid]]), torch.ones(int(valid.sum()), device=dev), accumulate=True)
    right = float((votes.argmax(1) == topic).float().mean())
    say(f"{vectors.shape[0]} words in the index; topic found for {100 * right:.1f} % of 500 held-out passages")
    pqt.pqt_index_free(index)
    return losses[0], losses[-1], right


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--topics", type=int, default=64)
    ap.add_argument("--dims", type=int, default=64)
    a = ap.parse_args()
    run(a.steps, a.topics, a.dims)
