"""GPU: the operators of a drafted decoder step together, as the example decoder
calls them: trees against the same layers written densely in 64 bits along each
node's own branch, the kept tokens against the walk's definition, and what the
cache holds after it was moved together."""
import importlib.util
import os
import sys

import pytest
import torch

import draft_ref as ref
from gpu_common import note, torch_cuda

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    torch_cuda()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        spec = importlib.util.spec_from_file_location("draft_step_example", os.path.join(ROOT, "examples", "draft_step.py"))
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
    finally:
        sys.path.pop(0)
    return m


def dense(m, w, tokens):
    """The logits after each of a row of tokens, causal, in 64 bits on the CPU."""
    def rms(v, weight):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * weight

    t = len(tokens)
    cos, sin = (a.double() for a in m.base.angles(t, "cpu"))
    half = m.DIM // 2

    def turn(v):  # [T, heads, DIM]
        a, b = v[..., :half], v[..., half:]
        c, s = cos[:, None], sin[:, None]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    r = w["embed"][torch.tensor(tokens)]
    z = rms(r, w["first"])
    causal = torch.ones(t, t, dtype=torch.bool).tril()
    for layer in w["layers"]:
        lin = {k: layer[k].view(layer[k].shape[0], -1) for k in ("qkv", "out", "up", "down")}
        qkv = (z @ lin["qkv"].T).view(t, -1, m.DIM)
        q, k, v = qkv[:, :m.HEADS], qkv[:, m.HEADS:m.HEADS + m.KV_HEADS], qkv[:, m.HEADS + m.KV_HEADS:]
        q, k = turn(rms(q, layer["q_norm"])), turn(rms(k, layer["k_norm"]))
        k, v = (u.repeat_interleave(m.HEADS // m.KV_HEADS, 1) for u in (k, v))
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0)) * m.DIM ** -0.5
        p = torch.softmax(s.masked_fill(~causal, -torch.inf), -1)
        a = (p @ v.transpose(0, 1)).transpose(0, 1).reshape(t, -1)
        r = r + 0.7 * layer["attn_gate"] * rms(a @ lin["out"].T, layer["attn_post"])
        z = rms(r, layer["attn_next"])
        r = r + 0.7 * layer["ffn_gate"] * rms((z @ lin["up"].T).clamp_min(0) @ lin["down"].T, layer["ffn_post"])
        z = rms(r, layer["ffn_next"])
    return z @ w["head"].view(m.VOCAB, -1).T


def doubles(w):
    return {k: [{n: v.double() for n, v in layer.items()} for layer in v] if k == "layers" else v.double() for k, v in w.items()}


# The example's f32 projections may be 1e-4 off each (the bound that convolutions are held to) of outputs of magnitude 1,
# and the last one has logits of magnitude 2 and more; a 16-bit cache rounds keys and values by up to its unit, which
# attention averages, in each of two layers.
@pytest.mark.parametrize("cache,bound", [(torch.float32, 3e-3), (torch.float16, 8 * 2.0 ** -11 + 3e-3), (torch.bfloat16, 8 * 2.0 ** -8 + 3e-3)],
                         ids=str)
def test_drafted_steps_agree_with_dense_layers(cache, bound):
    m = example()
    w = doubles(m.make_weights(5, "cpu"))
    seqs, steps, nodes, branch = 3, 5, 12, 2
    d = m.Decoder(m.make_weights(5), seqs, 300, cache)
    g = torch.Generator(device="cuda").manual_seed(6)
    prompt = torch.randint(0, m.VOCAB, (seqs, 70), generator=g, device="cuda", dtype=torch.int32)   # two parts
    logits = d.prompt(prompt)
    text = prompt.tolist()
    parents, depths = m.tree_of(nodes, branch)
    above = ref.above(parents)
    last = logits.argmax(-1).to(torch.int32)

    def near(got, want, what):
        off = (got.double().cpu() - want).abs().max().item()
        assert off <= bound * max(1.0, want.abs().max().item()), (what, off)

    for s in range(seqs):
        near(logits[s], dense(m, w, text[s])[-1], "prompt")
    kept = 0
    for step in range(steps):
        note(f"[draft example] {cache}, step {step}")
        before = d.lengths.tolist()
        seen = {}
        forward, verify = d.forward, m.ilpm.verify_drafts
        d.forward = lambda *a: seen.setdefault("logits", forward(*a))

        def spy(tokens, tree, target, numbers, draft=None):
            seen.update(tree=tree, target=target, numbers=numbers, draft=draft)
            return verify(tokens, tree, target, numbers, draft=draft)

        m.ilpm.verify_drafts = spy
        try:
            tokens, path, counts, after = d.step(last, nodes, branch, g)
        finally:
            m.ilpm.verify_drafts, d.forward = verify, forward
        torch.cuda.synchronize()
        assert before == [len(t) for t in text]
        tree = tokens.tolist()
        for s in range(seqs):
            for i in (0, 1, 2, 5, nodes - 1):   # nodes of every depth, each along its own branch
                near(seen["logits"][s, i], dense(m, w, text[s] + [tree[s][a] for a in above[i]])[-1], f"node {i}")
        want = ref.verify(tokens.cpu(), seen["tree"].cpu(), seen["target"].cpu(), seen["numbers"].cpu(), seen["draft"].cpu())
        assert (path.tolist(), counts.tolist(), after.tolist()) == tuple(want)
        for s, (way, n) in enumerate(zip(path.tolist(), counts.tolist())):
            text[s] += [tree[s][i] for i in way[:n]]
            kept += n - 1
        last = after
    assert d.lengths.tolist() == [len(t) for t in text]
    assert kept > 0   # (else nothing was moved)


def test_decoder_refuses_more_nodes_than_it_was_made_for():
    m = example()
    d = m.Decoder(m.make_weights(5), 2, 40)
    g = torch.Generator(device="cuda").manual_seed(6)
    prompt = torch.randint(0, m.VOCAB, (2, 30), generator=g, device="cuda", dtype=torch.int32)
    last = d.prompt(prompt).argmax(-1).to(torch.int32)
    with pytest.raises(ValueError, match="more than the 40"):
        d.step(last, 11, 2, g)
    d.step(last, 10, 3, g)
    with pytest.raises(ValueError):
        d.step(last, 10, 3, g)
