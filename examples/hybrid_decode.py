"""Speculative decoding of a small hybrid -- one Gated DeltaNet layer and one attention layer -- with every step of both
layers in the library:

    python examples/hybrid_decode.py [--sequences 4] [--tokens 24] [--nodes 12]

Each sequence is decoded twice.  First token by token: the attention layer appends the token's key and value to its paged
cache (rotated on the way) and attends to it.  Then with draft trees: rotate, verify the tree through both layers, accept
the longest path whose tokens the model would have chosen, commit that path to the state and to the cache.  The two
have to produce the same tokens.  Weights are random; the drafts are the first run's tokens cut short at random
places among random distractors, so that some are right and most are not.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2608_20961_b200 import attention as at  # noqa: E402
from paper_2608_20961_b200 import binding as tw  # noqa: E402

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HIDDEN, VOCAB, H_GDN, HQ, HKV, D, PAGE, PAGES = 256, 211, 2, 4, 2, 128, 16, 8


class Hybrid:
    """hidden -> GDN layer -> attention layer -> logits, for the rows of a batch of draft trees."""

    def __init__(self, B, dev, seed=0):
        gen = torch.Generator().manual_seed(seed)
        w = lambda i, o: (torch.randn((i, o), generator=gen) / math.sqrt(i)).to(BF16).to(dev)
        self.B, self.dev = B, dev
        self.embed = torch.randn((VOCAB, HIDDEN), generator=gen).to(BF16).to(dev)
        self.gdn_in, self.gdn_out = w(HIDDEN, 3 * H_GDN * 128 + 2 * H_GDN), w(H_GDN * 128, HIDDEN)
        self.attn_in, self.attn_out = w(HIDDEN, (HQ + 2 * HKV) * D), w(HQ * D, HIDDEN)
        freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
        angle = torch.arange(PAGES * PAGE, dtype=torch.float64)[:, None] * freq
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(dev)
        self.reset()

    def reset(self):
        B, dev = self.B, self.dev
        self.state = torch.zeros((B, H_GDN, 128, 128), dtype=BF16, device=dev)
        kv = lambda: torch.zeros((B * PAGES, PAGE, HKV, D), dtype=BF16, device=dev)
        table = torch.randperm(B * PAGES, generator=torch.Generator().manual_seed(1)).to(I32).view(B, PAGES).to(dev)
        self.cache = at.KVCache(kv(), kv(), table, torch.zeros(B, dtype=I32, device=dev))
        self.layer = at.AttentionLayer(self.cache, HQ, self.cos_sin)
        self.status = torch.zeros(B, dtype=I32, device=dev)

    @staticmethod
    def _norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def verify(self, tokens, parent, offsets, append=False):
        """Logits [T, VOCAB] of every node; keeps what commit needs.  append: trees of one node, whose key and value
        go to the cache at once."""
        dev, T = self.dev, tokens.numel()
        tree = tw.Tree.empty(offsets, parent, H_GDN, int((offsets[1:] - offsets[:-1]).max()))
        x = self.embed[tokens]
        p = self._norm(x) @ self.gdn_in
        q, k, v = (p[:, i * H_GDN * 128:(i + 1) * H_GDN * 128].reshape(T, H_GDN, 128) for i in range(3))
        unit = lambda t: torch.nn.functional.normalize(t.float(), dim=-1).to(BF16).contiguous()
        alpha = 0.9 + 0.0999 * torch.sigmoid(p[:, -2 * H_GDN:-H_GDN].float()).contiguous()
        beta = torch.sigmoid(p[:, -H_GDN:].float()).contiguous()
        self.gdn_k = unit(k)
        O, self.gdn_U = torch.empty((T, H_GDN, 128), dtype=BF16, device=dev), torch.empty((T, H_GDN, 128), device=dev)
        tw.treewy_tree_prepare(tree, alpha, self.status)
        tw.treewy_verify(self.state, unit(q), self.gdn_k, v.contiguous(), beta, tree, H_GDN, O, self.gdn_U, self.status)
        x = x + O.view(T, -1) @ self.gdn_out
        # the attention layer: positions are the context plus the depth in the tree
        qkv = self._norm(x) @ self.attn_in
        q = qkv[:, :HQ * D].unflatten(1, (HQ, D))
        k = qkv[:, HQ * D:(HQ + HKV) * D].unflatten(1, (HKV, D))
        v = qkv[:, (HQ + HKV) * D:].unflatten(1, (HKV, D))
        seq = torch.repeat_interleave(torch.arange(self.B, device=dev), offsets[1:] - offsets[:-1])
        positions = (self.cache.context_len[seq] + tree.depth[:T]).to(I32)
        if append:
            O = self.layer.append_and_attend(tree, positions, q, k, v, self.status)
        else:
            O = self.layer.verify(tree, positions, q, k, v, self.status)
        self.tree, self.attn_k, self.attn_v = tree, k, v
        x = x + O.view(T, -1) @ self.attn_out
        assert not self.status.any(), self.status.tolist()
        return self._norm(x).float() @ self.embed.float().T

    def commit(self, accepted):
        tw.treewy_commit(self.state, self.gdn_U, self.gdn_k, self.tree, H_GDN, accepted, None, self.status)
        self.layer.commit(self.tree, self.attn_k, self.attn_v, accepted, self.status)


def one_by_one(model, first, n):
    model.reset()
    B, dev = model.B, model.dev
    offsets, parent = torch.arange(B + 1, dtype=I32, device=dev), torch.full((B,), -1, dtype=I32, device=dev)
    tokens, out = first, []
    for _ in range(n):
        logits = model.verify(tokens, parent, offsets, append=True)
        tw.treewy_commit(model.state, model.gdn_U, model.gdn_k, model.tree, H_GDN, torch.zeros(B, dtype=I32, device=dev), None, model.status)
        tokens = logits.argmax(-1)
        out.append(tokens)
    return torch.stack(out, 1).tolist()


def speculative(model, first, n, nodes, known, seed=0):
    """known: the drafts' source (what a good draft model would propose)."""
    model.reset()
    gen = torch.Generator().manual_seed(seed)
    rand = lambda hi: int(torch.randint(hi, (1,), generator=gen))
    dev = model.dev
    out, root, rounds = [[] for _ in range(model.B)], first.tolist(), 0
    while min(len(o) for o in out) < n:
        tokens, parents, offsets = [], [], [0]
        for b in range(model.B):
            # the right path first, then distractors anywhere
            path = known[b][len(out[b]):len(out[b]) + rand(5)]
            t, p = [root[b]] + path, list(range(-1, len(path)))
            while len(t) < nodes:
                p.append(rand(len(t)))
                t.append(rand(VOCAB))
            tokens, parents = tokens + t, parents + p
            offsets.append(len(tokens))
        logits = model.verify(torch.tensor(tokens, device=dev), torch.tensor(parents, dtype=I32, device=dev),
                              torch.tensor(offsets, dtype=I32, device=dev))
        choice, accepted = logits.argmax(-1).tolist(), []
        for b in range(model.B):
            lo, node = offsets[b], 0
            while True:
                want = choice[lo + node]
                out[b].append(want)
                kids = [i for i in range(node + 1, offsets[b + 1] - lo) if parents[lo + i] == node and tokens[lo + i] == want]
                if not kids:
                    break
                node = kids[0]
            accepted.append(node)
            root[b] = out[b][-1]
        model.commit(torch.tensor(accepted, dtype=I32, device=dev))
        rounds += 1
    return [o[:n] for o in out], rounds


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=24)
    ap.add_argument("--nodes", type=int, default=12)
    args = ap.parse_args(argv)
    assert args.tokens + args.nodes <= PAGE * PAGES
    model = Hybrid(args.sequences, torch.device("cuda:0"))
    first = torch.arange(args.sequences, device=model.dev) + 1
    plain = one_by_one(model, first, args.tokens)
    spec, rounds = speculative(model, first, args.tokens, args.nodes, plain)
    same = plain == spec
    print(f"{args.tokens} tokens of {args.sequences} sequences: {args.tokens} steps one by one, {rounds} rounds of trees of "
          f"{args.nodes} nodes; the same tokens: {same}")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
