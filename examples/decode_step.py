"""A small decoder answering token by token on the library's operators.

    python examples/decode_step.py [--tokens 64] [--cache bf16]

Each layer keeps an f32 residual stream.  Projections are 1x1 convolutions (the
tokens of a call are the pixels of a 1 x T map, so one token is a 1 x 1 map) on
weights packed once; between them lie the decoder-step operators:

    z                     the block's input, the norm of the stream
    q, k, v  = conv(z)    one packed projection, sliced
    q        = kv_append  keys and values into the paged cache, q and k rotated
    a        = attn_decode
    r, z     = residual_norm(r, conv(a))     norm, gate, residual sum, next norm
    r, z     = residual_norm(r, conv(relu(conv(z))))

A prompt runs through the same calls: its tokens are rows that share one page
table, and row t sees t + 1 keys.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1909_02765_amd as ilpm  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM, FFN, LAYERS, PAGE = 256, 8, 2, 64, 512, 2, 16


def make_weights(seed, device="cuda"):
    """He-normal projections [C_out, C_in, 1, 1] and near-1 norm weights, all f32."""
    g = torch.Generator().manual_seed(seed)

    def matrix(c_out, c_in):
        return (torch.randn((c_out, c_in, 1, 1), generator=g) * c_in ** -0.5).to(device)

    def vector(mean, std):
        return (mean + std * torch.randn(WIDTH, generator=g)).to(device)

    layers = [{"qkv": matrix((HEADS + 2 * KV_HEADS) * DIM, WIDTH), "out": matrix(WIDTH, HEADS * DIM),
               "up": matrix(FFN, WIDTH), "down": matrix(WIDTH, FFN),
               **{k: vector(1.0, 0.1) for k in ("attn_post", "attn_next", "ffn_post", "ffn_next")},
               "attn_gate": vector(0.5, 0.1), "ffn_gate": vector(0.5, 0.1)} for _ in range(LAYERS)]
    return {"first": vector(1.0, 0.1), "layers": layers}


def angles(positions, device="cuda"):
    rate = 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
    a = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    return a.cos().float().to(device), a.sin().float().to(device)


class Decoder:
    """One sequence: its weights packed for one token, its cache pages, and how many tokens they hold."""

    def __init__(self, weights, most_tokens, cache=torch.float32):
        self.w, self.length, self.most = weights, 0, most_tokens
        self.cos, self.sin = angles(most_tokens)
        pages = -(-most_tokens // PAGE)
        # The pages of a sequence lie where the pool had room.
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(1))
        self.table = order.to(torch.int32).view(1, pages).cuda()
        self.pools = [[torch.empty((pages, PAGE, KV_HEADS, DIM), dtype=cache, device="cuda") for _ in range(2)]
                      for _ in range(LAYERS)]
        self.packed = [{k: self._pack(layer[k], ilpm.EPI_RELU if k == "up" else 0) for k in ("qkv", "out", "up", "down")}
                       for layer in weights["layers"]]

    @staticmethod
    def _pack(w, epilogue):
        plan = ilpm.plan_for(w.shape[1], 1, 1, w.shape[0], 1, 1, 0, epilogue, prepacked=True)
        return plan, ilpm.prepack_weights(w, plan)

    def _project(self, layer, name, z):
        """z [T, C_in] through a 1x1 convolution of a 1 x T map: [T, C_out]."""
        w = self.w["layers"][layer][name]
        epilogue = ilpm.EPI_RELU if name == "up" else 0
        if z.shape[0] == 1:  # channels first and rows are the same for one token
            plan, packed = self.packed[layer][name]
            y = ilpm.conv2d_prepacked_epilogue(z.view(1, -1, 1, 1), packed, w.shape[0], 1, None, 1, 0, epilogue, plan=plan)
            return y.view(1, -1)
        x = z.t().contiguous().view(1, z.shape[1], 1, z.shape[0])
        return ilpm.conv2d_epilogue(x, w, None, 1, 0, epilogue).view(w.shape[0], -1).t().contiguous()

    def step(self, x):
        """x [T, WIDTH], the next T tokens' embeddings: their outputs [T, WIDTH]."""
        t = x.shape[0]
        if self.length + t > self.most:  # (the cache would leave them out)
            raise ValueError(f"{t} tokens after {self.length} are more than the {self.most} that this decoder was made for")
        pos = torch.arange(self.length, self.length + t, dtype=torch.int32, device="cuda")
        seq, lengths = torch.zeros_like(pos), pos + 1
        rows = self.table.expand(t, -1)  # every token of the call reads the one sequence's pages
        r, z = ilpm.residual_norm(x, pre="rms", pre_w=self.w["first"])
        for i, layer in enumerate(self.w["layers"]):
            qkv = self._project(i, "qkv", z).view(t, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
            ilpm.kv_append(k, v, *self.pools[i], self.table, seq, pos, q=q, cos=self.cos, sin=self.sin, q_out=q)
            a = ilpm.attn_decode(q, *self.pools[i], rows, lengths, max_len=self.length + t)
            r, z = ilpm.residual_norm(r, self._project(i, "out", a.reshape(t, HEADS * DIM)), post="rms", post_w=layer["attn_post"],
                                      gate=layer["attn_gate"], scale=0.7, pre="rms", pre_w=layer["attn_next"])
            r, z = ilpm.residual_norm(r, self._project(i, "down", self._project(i, "up", z)), post="rms", post_w=layer["ffn_post"],
                                      gate=layer["ffn_gate"], scale=0.7, pre="rms", pre_w=layer["ffn_next"])
        self.length += t
        return z


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompt", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--cache", choices=("f32", "f16", "bf16"), default="bf16")
    args = ap.parse_args()
    cache = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[args.cache]
    d = Decoder(make_weights(0), args.prompt + args.tokens, cache)
    x = torch.randn((args.prompt, WIDTH), generator=torch.Generator().manual_seed(2)).cuda()
    z = d.step(x)[-1:]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(args.tokens):
        z = d.step(z)  # (a model would sample a token and embed it here)
    torch.cuda.synchronize()
    us = (time.perf_counter() - began) / args.tokens * 1e6
    print(f"{args.prompt} prompt tokens, then {args.tokens} one by one: {us:.0f} us a token ({LAYERS} layers, {args.cache} cache); "
          f"the last output's norm is {z.norm().item():.4f}")


if __name__ == "__main__":
    main()
