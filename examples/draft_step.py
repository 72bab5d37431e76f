"""A small decoder that drafts: several sequences, a tree of guessed tokens for each in one pass.

    python examples/draft_step.py [--seqs 4] [--steps 16] [--branch 2] [--cache bf16]

The layers of decode_step.py with a norm of every query and key head, an embedding and an output projection.  A step
draws a tree of tokens from a cheap draft model (here a table: the token after each token), runs all of its nodes
through the layers at once, keeps those that the layers' own probabilities allow, and moves their keys and values
together behind the sequence:

    q          = kv_append_norm  heads normed and rotated by their depth, stored in the tree's slots
    a          = attn_tree       every node over the sequence and the nodes above it
    path, next = verify_drafts   from given random numbers
                 kv_copy         in every layer's cache

The tokens follow the layers' probabilities whatever was drafted.  A prompt runs through the same calls as a chain.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import decode_step as base  # noqa: E402
import paper_1909_02765_amd as ilpm  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM, PAGE = base.WIDTH, base.HEADS, base.KV_HEADS, base.DIM, base.PAGE
VOCAB = 500


def make_weights(seed, device="cuda"):
    """decode_step's, with head norms, an embedding, an output projection and the draft model's table, all f32."""
    w = base.make_weights(seed, device)
    g = torch.Generator().manual_seed(seed + 1)
    for layer in w["layers"]:
        layer["q_norm"], layer["k_norm"] = ((1 + 0.1 * torch.randn(DIM, generator=g)).to(device) for _ in range(2))
    w["embed"] = torch.randn((VOCAB, WIDTH), generator=g).to(device)
    w["head"] = (torch.randn((VOCAB, WIDTH, 1, 1), generator=g) * 2.0 * WIDTH ** -0.5).to(device)
    w["draft"] = torch.softmax(torch.randn((VOCAB, VOCAB), generator=g) * 2.0, -1).to(device)
    return w


def tree_of(nodes, branch):
    """The parents of a tree whose node i hangs below node (i - 1) // branch, and its nodes' depths."""
    parents = [-1] + [(i - 1) // branch for i in range(1, nodes)]
    depths = [0]
    for p in parents[1:]:
        depths.append(depths[p] + 1)
    return parents, depths


class Decoder:
    """Some sequences: their cache pages, and on the GPU how many tokens each holds."""

    def __init__(self, weights, seqs, most_tokens, cache=torch.float32):
        self.w, self.seqs, self.most, self.bound = weights, seqs, most_tokens, 0
        self.cos, self.sin = base.angles(most_tokens)
        pages = -(-most_tokens // PAGE)
        # The pages of the sequences lie where the pool had room.
        order = torch.randperm(seqs * pages, generator=torch.Generator().manual_seed(1))
        self.table = order.to(torch.int32).view(seqs, pages).cuda()
        self.pools = [[torch.empty((seqs * pages, PAGE, KV_HEADS, DIM), dtype=cache, device="cuda") for _ in range(2)]
                      for _ in weights["layers"]]
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.ids = torch.arange(seqs, dtype=torch.int32, device="cuda")

    @staticmethod
    def _project(w, z, epilogue=0):
        """z [rows, C_in] through a 1x1 convolution of a 1 x rows map: [rows, C_out]."""
        x = z.t().contiguous().view(1, z.shape[1], 1, z.shape[0])
        return ilpm.conv2d_epilogue(x, w, None, 1, 0, epilogue).view(w.shape[0], -1).t().contiguous()

    def forward(self, tokens, parents, depths):
        """tokens [seqs, nodes] int32 in trees of these parents: the logits after every node [seqs, nodes, VOCAB].  Their
        keys and values lie behind the sequences then; what of them is kept is up to keep()."""
        n, t = tokens.shape
        if self.bound + t > self.most:  # (the cache would leave them out)
            raise ValueError(f"{t} nodes after up to {self.bound} tokens are more than the {self.most} that this decoder was made for")
        slots = (self.lengths[:, None] + torch.arange(t, dtype=torch.int32, device="cuda")).view(-1)
        places = (self.lengths[:, None] + torch.tensor(depths, dtype=torch.int32, device="cuda")).view(-1)
        seq = self.ids[:, None].expand(n, t).reshape(-1)
        tree = torch.tensor(parents, dtype=torch.int32, device="cuda").expand(n, t).contiguous()
        r, z = ilpm.residual_norm(self.w["embed"][tokens.view(-1).long()], pre="rms", pre_w=self.w["first"])
        for layer, pool in zip(self.w["layers"], self.pools):
            qkv = self._project(layer["qkv"], z).view(n * t, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
            ilpm.kv_append_norm(k, v, *pool, self.table, seq, places, slots=slots, q=q, norm="rms", q_w=layer["q_norm"],
                                k_w=layer["k_norm"], cos=self.cos, sin=self.sin, q_out=q)
            a = ilpm.attn_tree(q, *pool, self.table, self.lengths, tree, max_len=self.bound)
            r, z = ilpm.residual_norm(r, self._project(layer["out"], a.reshape(n * t, HEADS * DIM)), post="rms",
                                      post_w=layer["attn_post"], gate=layer["attn_gate"], scale=0.7, pre="rms", pre_w=layer["attn_next"])
            up = self._project(layer["up"], z, ilpm.EPI_RELU)
            r, z = ilpm.residual_norm(r, self._project(layer["down"], up), post="rms", post_w=layer["ffn_post"],
                                      gate=layer["ffn_gate"], scale=0.7, pre="rms", pre_w=layer["ffn_next"])
        return self._project(self.w["head"], z).view(n, t, VOCAB)

    def keep(self, counts, most, path=None):
        """The first counts[s] nodes of each sequence (or those of its path), at most `most`, become its last tokens."""
        if path is not None:
            for k, v in self.pools:
                ilpm.kv_copy(k, v, self.table, self.table, self.lengths, self.lengths, counts, path=path)
        self.lengths = self.lengths + counts
        self.bound += most

    def prompt(self, tokens):
        """tokens [seqs, n] int32: the logits after the last of them."""
        for at in range(0, tokens.shape[1], ilpm.MAX_NODES):
            part = tokens[:, at:at + ilpm.MAX_NODES].contiguous()
            parents, depths = tree_of(part.shape[1], 1)
            logits = self.forward(part, parents, depths)
            self.keep(torch.full_like(self.lengths, part.shape[1]), part.shape[1])
        return logits[:, -1]

    def step(self, last, nodes, branch, generator):
        """One drafted step behind the tokens `last` [seqs]: (tokens [seqs, nodes] of the tree, path, counts, the next
        tokens).  The kept nodes are the sequences' own from then on; the next tokens are the next step's `last`."""
        parents, depths = tree_of(nodes, branch)
        tokens = torch.empty((self.seqs, nodes), dtype=torch.int32, device="cuda")
        tokens[:, 0] = last
        for i in range(1, nodes):  # (each from its parent's row, independently)
            tokens[:, i] = torch.multinomial(self.w["draft"][tokens[:, parents[i]].long()], 1, generator=generator)[:, 0].to(torch.int32)
        target = torch.softmax(self.forward(tokens, parents, depths), -1)
        tree = torch.tensor(parents, dtype=torch.int32, device="cuda").expand(self.seqs, nodes).contiguous()
        numbers = torch.rand((self.seqs, nodes), generator=generator, device="cuda")
        path, counts, after = ilpm.verify_drafts(tokens, tree, target, numbers, draft=self.w["draft"][tokens.long()])
        self.keep(counts, max(depths) + 1, path)
        return tokens, path, counts, after


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=40)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--nodes", type=int, default=15)
    ap.add_argument("--branch", type=int, default=2)
    ap.add_argument("--cache", choices=("f32", "f16", "bf16"), default="bf16")
    args = ap.parse_args()
    cache = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[args.cache]
    deepest = max(tree_of(args.nodes, args.branch)[1]) + 1
    d = Decoder(make_weights(0), args.seqs, args.prompt + args.steps * deepest + args.nodes, cache)
    g = torch.Generator(device="cuda").manual_seed(2)
    tokens = torch.randint(0, VOCAB, (args.seqs, args.prompt), generator=g, device="cuda", dtype=torch.int32)
    last = torch.multinomial(torch.softmax(d.prompt(tokens), -1), 1, generator=g)[:, 0].to(torch.int32)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(args.steps):
        last = d.step(last, args.nodes, args.branch, g)[3]
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / args.steps * 1e6
    made = (d.lengths - args.prompt).float().mean().item()
    print(f"{args.seqs} sequences, trees of {args.nodes} nodes: {us:.0f} us a step, {made / args.steps:.2f} tokens a step and sequence "
          f"({len(d.pools)} layers, {args.cache} cache)")


if __name__ == "__main__":
    main()
