"""GPU: the example decoder (projections as 1x1 convolutions, paged cache,
single-token attention, norms) against the same layers written densely in 64
bits, prompt and single tokens alike."""
import importlib.util
import os

import pytest
import torch

from gpu_common import note, torch_cuda

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    torch_cuda()
    spec = importlib.util.spec_from_file_location("decode_step_example", os.path.join(ROOT, "examples", "decode_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(m, w, x):
    """All tokens at once, causal, in 64 bits on the CPU."""
    def rms(v, weight):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * weight

    t = x.shape[0]
    cos, sin = (a.double() for a in m.angles(t, "cpu"))
    half = m.DIM // 2

    def turn(v):  # [T, heads, DIM]
        a, b = v[..., :half], v[..., half:]
        c, s = cos[:, None], sin[:, None]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    r = x
    z = rms(r, w["first"])
    causal = torch.ones(t, t, dtype=torch.bool).tril()
    for layer in w["layers"]:
        lin = {k: layer[k].view(layer[k].shape[0], -1) for k in ("qkv", "out", "up", "down")}
        qkv = (z @ lin["qkv"].T).view(t, -1, m.DIM)
        q, k, v = turn(qkv[:, :m.HEADS]), turn(qkv[:, m.HEADS:m.HEADS + m.KV_HEADS]), qkv[:, m.HEADS + m.KV_HEADS:]
        k, v = (u.repeat_interleave(m.HEADS // m.KV_HEADS, 1) for u in (k, v))
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0)) * m.DIM ** -0.5
        p = torch.softmax(s.masked_fill(~causal, -torch.inf), -1)
        a = (p @ v.transpose(0, 1)).transpose(0, 1).reshape(t, -1)
        r = r + 0.7 * layer["attn_gate"] * rms(a @ lin["out"].T, layer["attn_post"])
        z = rms(r, layer["attn_next"])
        r = r + 0.7 * layer["ffn_gate"] * rms((z @ lin["up"].T).clamp_min(0) @ lin["down"].T, layer["ffn_post"])
        z = rms(r, layer["ffn_next"])
    return z


# With an f32 cache each of the 2 x 4 projections may be 1e-4 off (the bound that convolutions are held to), of outputs
# of magnitude 1; a 16-bit cache rounds keys and values by up to its unit, which attention averages, in each layer.
@pytest.mark.parametrize("cache,bound", [(torch.float32, 1e-3), (torch.float16, 4 * 2.0 ** -11 + 1e-3), (torch.bfloat16, 4 * 2.0 ** -8 + 1e-3)],
                         ids=str)
def test_decoder_agrees_with_dense_layers(cache, bound):
    m = example()
    weights = m.make_weights(5, "cpu")
    steps = [37, 1, 1, 5, 1, 1]
    total = sum(steps)
    x = torch.randn((total, m.WIDTH), generator=torch.Generator().manual_seed(6))
    d = m.Decoder(m.make_weights(5), total, cache)
    got, at = [], 0
    for n in steps:
        note(f"[example] {cache}, tokens {at} to {at + n}")
        got.append(d.step(x[at:at + n].cuda()))
        at += n
    torch.cuda.synchronize()
    dbl = {"first": weights["first"].double(), "layers": [{k: v.double() for k, v in l.items()} for l in weights["layers"]]}
    want = dense(m, dbl, x.double())
    off = (torch.cat(got).double().cpu() - want).abs().max().item()
    assert off <= bound * max(1.0, want.abs().max().item()), off


def test_decoder_refuses_more_tokens_than_it_was_made_for():
    """What its cache and angles have no place for would be left out, and the outputs be those of other tokens."""
    m = example()
    d = m.Decoder(m.make_weights(5), 20)
    x = torch.randn((24, m.WIDTH), generator=torch.Generator().manual_seed(6)).cuda()
    z = d.step(x[:18])
    with pytest.raises(ValueError, match="more than the 20"):
        d.step(x[18:21])
    last = d.step(x[18:20])   # a refused call changed nothing
    with pytest.raises(ValueError):
        d.step(x[20:21])
    again = m.Decoder(m.make_weights(5), 20).step(x[:20])
    torch.cuda.synchronize()
    assert (torch.cat((z, last)) - again).abs().max() < 1e-3
