"""Norm, projection, head norms, attention and their gradients together, as they are used."""

import importlib.util
import math
import os

import pytest
import torch

import paper_2607_02461_amd as oq

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16 = torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_runs():
    losses = _example().main(lengths=(70, 33, 1), steps=2)
    assert len(losses) == 2 and all(math.isfinite(v) for v in losses)


def _attend(q, k, v, lengths, scale):
    """Causal attention of packed prompts in fp64."""
    out, first, G = [], 0, q.shape[1] // k.shape[1]
    for n in lengths:
        a, b, c = (t[first:first + n].transpose(0, 1) for t in (q, k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)))
        s = (a @ b.transpose(1, 2) * scale).masked_fill(torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1), -math.inf)
        out.append((torch.softmax(s, -1) @ c).transpose(0, 1))
        first += n
    return torch.cat(out)


def _turned(x, weight, pos, D):
    n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight
    angle = pos.double() * 10000.0 ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    z = torch.view_as_complex(n.reshape(*n.shape[:-1], D // 2, 2).contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.view_as_real(z).flatten(-2)


def _close(name, got, want, steps):
    """Norm-wise: each of `steps` roundings to bf16 on the way is off by at most 2^-8 of what it rounds."""
    off = float((got.double() - want).norm() / want.norm())
    assert off <= steps * 2.0 ** -8, f"{name}: {off}"


def test_gradients_through_the_chain():
    # the example's gradients against differentiation in fp64, with the projection that its adapters stand beside replaced
    # by what the quantized one gave (its gradient goes through the unquantized weight on both sides)
    e = _example()
    lengths = (90, 1, 37)
    tokens = sum(lengths)
    pos, rope = e.positions(lengths), oq.rope_plan((e.D,), (max(lengths) + 1,))
    plan = oq.attention_plan(lengths, heads=e.HEADS, kv_heads=e.KV_HEADS, causal=True)
    adapter = oq.lora_plan(tokens, [0], [0], [e.RANK], [1.0])
    block = e.Block()
    g = torch.Generator(device=DEV).manual_seed(3)
    block.B.normal_(0.0, 0.05, generator=g)
    block.q_weight.uniform_(0.5, 2.0, generator=g)
    block.k_weight.uniform_(0.5, 2.0, generator=g)
    x = torch.randn((tokens, e.WIDTH), generator=g, device=DEV).to(BF16)
    target = torch.randn((tokens, e.HEADS, e.D), generator=g, device=DEV)
    loss, grads = e.gradients(block, x, plan, rope, pos, adapter, target)

    leaves = dict(A=block.A, B=block.B, q_weight=block.q_weight, k_weight=block.k_weight, scale=block.scale_shift()[0], shift=block.scale_shift()[1])
    leaves = {n: t.detach().double().requires_grad_() for n, t in leaves.items()}
    xd = x.double()
    centred = xd - xd.mean(-1, keepdim=True)
    y = centred * torch.rsqrt(centred.square().mean(-1, keepdim=True) + 1e-6) * (1 + leaves["scale"]) + leaves["shift"]
    dense = y @ block.qkv_weight.double().t()
    quantized = block.linear(oq.layer_norm_modulate(x, *block.scale_shift()), block.qkv_codes).double()
    qkv = dense + (quantized - dense).detach() + (y @ leaves["A"][0].t()) @ leaves["B"][0].t()
    q, k, v = qkv.view(tokens, -1, e.D).split((e.HEADS, e.KV_HEADS, e.KV_HEADS), dim=1)
    q, k = _turned(q, leaves["q_weight"], pos, e.D), _turned(k, leaves["k_weight"], pos, e.D)
    want = (_attend(q, k, v, lengths, e.D ** -0.5) - target.double()).square().mean()
    assert abs(float(loss) - want.item()) <= 6 * 2.0 ** -8 * want.item()
    # on the way to a gradient: y, qkv, q or k, p, o, the output's gradient, ds, dq, its projection's, and dy; twice that for
    # the scores, which two of them make
    for (name, got), exact in zip(grads.items(), torch.autograd.grad(want, [leaves[n] for n in grads])):
        _close(name, got, exact, 20)


def test_tokens_one_by_one_and_in_chunks_give_a_prompts_rows():
    # a cache that grows token by token, or by a chunk, against the whole prompt at once
    H, Hk, D, n = 8, 2, 128, 333
    g = torch.Generator(device=DEV).manual_seed(4)
    q, k, v = (torch.randn((n, h, D), generator=g, device=DEV).to(BF16) for h in (H, Hk, Hk))
    whole = oq.attention(oq.attention_plan([n], heads=H, kv_heads=Hk, causal=True), q, k, v, out_dtype=torch.float32)
    for first, rows in [(i, 1) for i in (0, 1, 31, 32, 127, 128, 332)] + [(5, 60), (300, 33), (0, 333)]:
        plan = oq.attention_plan([rows], [first + rows], heads=H, kv_heads=Hk, causal=True)
        got = oq.attention(plan, q[first:first + rows], k, v, out_dtype=torch.float32)
        # both have p in bf16 beside v, measured from maxima that may differ: 2^-8 of sum p |v| each
        size = _attend(q.double(), k.double(), v.double().abs(), (n,), D ** -0.5)[first:first + rows]
        assert float(((got - whole[first:first + rows]).abs().double() - 2.1 * 2.0 ** -8 * size).max()) <= 0.0


def test_the_chain_in_a_graph():
    e = _example()
    lengths = (64, 30)
    tokens = sum(lengths)
    pos, rope = e.positions(lengths), oq.rope_plan((e.D,), (max(lengths) + 1,))
    plan = oq.attention_plan(lengths, heads=e.HEADS, kv_heads=e.KV_HEADS, causal=True)
    adapter = oq.lora_plan(tokens, [0], [0], [e.RANK], [1.0])
    block = e.Block()
    x = torch.randn((tokens, e.WIDTH), device=DEV).to(BF16)
    e.serve(block, x, plan, rope, pos, adapter)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _, _ = e.serve(block, x, plan, rope, pos, adapter)
    for seed in range(3):
        x.copy_(torch.randn((tokens, e.WIDTH), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, e.serve(block, x, plan, rope, pos, adapter)[0])
