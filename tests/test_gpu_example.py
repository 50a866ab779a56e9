"""The example that runs the adapters, the head norms and the rotary positions together, as they are used."""

import importlib.util
import os

import pytest
import torch

import paper_2607_02461_amd as oq

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("adapted_attention_input", os.path.join(ROOT, "examples", "adapted_attention_input.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_training_lowers_the_loss():
    losses = _example().main(steps=12)
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.99 * losses[0]


def test_serving_against_plain_torch():
    e = _example()
    tokens = 4 + 2 * 3 * 5
    pos = e.positions(2, 3, 5, 4)
    rope = oq.rope_plan(e.DIMS, (2, 3, 5))
    layer = e.Layer(adapters=1)
    layer.B.normal_(0.0, 0.1)
    layer.q_weight.uniform_(0.5, 2.0)
    plan = oq.lora_plan(2 * tokens, [0, tokens], [0, -1], [e.RANK], [0.5])
    x = torch.randn((2 * tokens, e.WIDTH), device="cuda").to(torch.bfloat16)
    q, k, v = e.serve(layer, x, 2, plan, rope, pos)
    # the projection again without adapters, then each step in plain fp32
    none = oq.lora_plan(2 * tokens, [], [], [e.RANK], [0.5])
    base = layer.project(x, none).float()
    base[:tokens] += 0.5 * (x[:tokens].float() @ layer.A[0].float().t()) @ layer.B[0].float().t()
    heads = base.view(2, tokens, 3, e.HEADS, e.D)
    angles = torch.cat([pos[:, a:a + 1].double() * 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda") / d) for a, d in enumerate(e.DIMS)], 1)
    for i, (got, w) in enumerate(((q, layer.q_weight), (k, layer.k_weight))):
        n = heads[:, :, i] * torch.rsqrt(heads[:, :, i].square().mean(-1, keepdim=True) + 1e-6) * w
        z = torch.view_as_complex(n.double().reshape(2, tokens, e.HEADS, e.D // 2, 2)) * torch.polar(torch.ones_like(angles), angles)[:, None]
        want = torch.view_as_real(z).flatten(-2)
        # the adapted projection is rounded to bf16 before the norm, and the result after it: 2^-8 of a value twice,
        # and of its pair's other one once
        size = torch.hypot(want[..., 0::2], want[..., 1::2]).repeat_interleave(2, dim=-1)
        assert float(((got.double() - want).abs() - 2.0 ** -6 * size).max()) <= 0.0
    assert torch.equal(v, heads[:, :, 2].to(torch.bfloat16)) or float((v.float() - heads[:, :, 2]).abs().max()) <= 2.0 ** -7 * float(heads[:, :, 2].abs().max())
