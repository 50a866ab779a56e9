"""The attention half of a transformer block on prompts of different lengths, served, and a training step of what is not
frozen in it.

    python examples/attention_block.py

Serving: the modulated norm, the quantized QKV projection with an adapter, the head norms with the rotation, attention over
each prompt, the quantized output projection.  Then one more token of each prompt over the keys and values so far.  Training:
the same down to attention's output, and the gradients in the opposite order: of the adapter, the head norms' weights, and
the modulation's scale and shift.
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_02461_amd as oq  # noqa: E402

DEV = "cuda"
HEADS, KV_HEADS, D = 16, 4, 64
WIDTH, QKV = HEADS * D, (HEADS + 2 * KV_HEADS) * D
RANK = 16


class Block:
    """The frozen projections, quantized, and what is trained beside them."""

    def __init__(self, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def weight(n, k):
            return torch.randn((n, k), generator=g, device=DEV).mul_(k ** -0.5).to(torch.bfloat16)

        self.qkv_weight, self.out_weight = weight(QKV, WIDTH), weight(WIDTH, WIDTH)
        self.rotation, self.codebook = oq.rpbh_plan(WIDTH, 128, seed), oq.lloydmax_codebook(4, WIDTH)
        self.qkv_codes = oq.quantize_weights_offline(self.rotation, self.codebook, self.qkv_weight)
        self.out_codes = oq.quantize_weights_offline(self.rotation, self.codebook, self.out_weight)
        self.modulation = 0.1 * torch.randn((1, 6 * WIDTH), generator=g, device=DEV)   # one conditioning for the batch
        self.q_weight, self.k_weight = torch.ones(D, device=DEV), torch.ones(D, device=DEV)
        self.A = weight(RANK, WIDTH)[None].contiguous()
        self.B = torch.zeros((1, QKV, RANK), dtype=torch.bfloat16, device=DEV)

    def linear(self, x, codes):
        """x times a quantized projection, bf16."""
        x_codes, x_norm = oq.rpbh_quantize_act(self.rotation, self.codebook, x)
        return oq.orbit_qlinear_ex(self.codebook, x_codes, x_norm, self.codebook, *codes, out_dtype=torch.bfloat16)

    def scale_shift(self):
        return self.modulation.chunk(6, dim=-1)[:2]

    def heads(self, x, adapter, h=None):
        """The modulated norm of tokens x and queries, keys and values as the projection leaves them."""
        y = oq.layer_norm_modulate(x, *self.scale_shift())
        qkv = self.linear(y, self.qkv_codes)
        oq.lora_add(adapter, y, self.A, self.B, qkv, out=qkv, h=h)
        return y, qkv.view(-1, HEADS + 2 * KV_HEADS, D).split((HEADS, KV_HEADS, KV_HEADS), dim=1)


def positions(lengths):
    return torch.cat([torch.arange(n) for n in lengths]).to(torch.int32)[:, None].to(DEV)


def serve(block, x, plan, rope, pos, adapter):
    """(the half block's output, its keys and values) of packed prompts."""
    _, (q, k, v) = block.heads(x, adapter)
    q, k = oq.qk_norm_rope(rope, q, k, pos, block.q_weight, block.k_weight, q_out=q, k_out=k)   # in place
    o = oq.attention(plan, q, k, v)
    return block.linear(o.flatten(1), block.out_codes), k, v


def next_token(block, x, lengths, rope, keys, values, place):
    """One token of each prompt: its keys and values go behind the prompt's in a cache of `place` tokens a prompt."""
    n = len(lengths)
    adapter = oq.lora_plan(n, [0], [0], [RANK], [1.0])
    pos = torch.tensor(lengths, dtype=torch.int32, device=DEV)[:, None]
    _, (q, k, v) = block.heads(x, adapter)
    q, k = oq.qk_norm_rope(rope, q, k, pos, block.q_weight, block.k_weight, q_out=q, k_out=k)
    at = torch.arange(n, device=DEV) * place + pos[:, 0]
    keys[at], values[at] = k, v
    plan = oq.attention_plan([1] * n, [m + 1 for m in lengths], heads=HEADS, kv_heads=KV_HEADS, causal=True,
                             k_starts=[i * place for i in range(n)])
    return block.linear(oq.attention(plan, q, keys, values).flatten(1), block.out_codes)


def gradients(block, x, plan, rope, pos, adapter, target):
    """(mean squared distance of attention's output from target, gradients by name).  The projection's own gradient goes
    through its unquantized weight."""
    h = torch.empty((x.shape[0], RANK), dtype=torch.float32, device=DEV)
    y, (q, k, v) = block.heads(x, adapter, h)
    nq, nk = oq.qk_norm_rope(rope, q, k, pos, block.q_weight, block.k_weight)
    lse = torch.empty((x.shape[0], HEADS), dtype=torch.float32, device=DEV)
    o = oq.attention(plan, nq, nk, v, lse=lse)
    error = o.float() - target
    d_qkv = torch.empty((x.shape[0], HEADS + 2 * KV_HEADS, D), dtype=torch.bfloat16, device=DEV)
    dq, dk, dv = d_qkv.split((HEADS, KV_HEADS, KV_HEADS), dim=1)
    dnq, dnk, _ = oq.attention_backward(plan, (error * (2 / error.numel())).to(torch.bfloat16), nq, nk, v, o, lse, v_grad=dv)
    _, _, d_qw, d_kw = oq.qk_norm_rope_backward(rope, dnq, dnk, q, k, pos, block.q_weight, block.k_weight, q_grad=dq, k_grad=dk)
    d_qkv = d_qkv.flatten(1)
    dy, dA, dB = oq.lora_add_backward(adapter, d_qkv, y, block.A, block.B, h, base=d_qkv @ block.qkv_weight)
    _, d_scale, d_shift = oq.layer_norm_modulate_backward(dy, x, block.scale_shift()[0])
    return error.square().mean(), dict(A=dA, B=dB, q_weight=d_qw, k_weight=d_kw, scale=d_scale, shift=d_shift)


def main(lengths=(300, 77, 129), steps=3, rate=1e-3):
    tokens = sum(lengths)
    pos, rope = positions(lengths), oq.rope_plan((D,), (max(lengths) + 1,))
    plan = oq.attention_plan(lengths, heads=HEADS, kv_heads=KV_HEADS, causal=True)
    adapter = oq.lora_plan(tokens, [0], [0], [RANK], [1.0])
    block = Block()
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((tokens, WIDTH), generator=g, device=DEV).to(torch.bfloat16)
    out, k, v = serve(block, x, plan, rope, pos, adapter)
    print(f"served {len(lengths)} prompts of {lengths} tokens: {tuple(out.shape)}")

    place = max(lengths) + 1
    keys = torch.empty((len(lengths) * place, KV_HEADS, D), dtype=torch.bfloat16, device=DEV)
    values = torch.empty_like(keys)
    first = 0
    for i, n in enumerate(lengths):
        keys[i * place:i * place + n], values[i * place:i * place + n] = k[first:first + n], v[first:first + n]
        first += n
    more = torch.randn((len(lengths), WIDTH), generator=g, device=DEV).to(torch.bfloat16)
    print(f"and one more token of each: {tuple(next_token(block, more, lengths, rope, keys, values, place).shape)}")

    target = torch.randn((tokens, HEADS, D), generator=g, device=DEV)
    losses = []
    for _ in range(steps):
        loss, grads = gradients(block, x, plan, rope, pos, adapter, target)
        losses.append(float(loss))
        for name, grad in grads.items():
            weight = dict(scale=block.scale_shift()[0], shift=block.scale_shift()[1]).get(name, getattr(block, name, None))
            weight.copy_(weight.float() - rate * grad / (grad.square().mean().sqrt() + 1e-30))
    print("distance by step:", " ".join(f"{v:.5f}" for v in losses))
    return losses


if __name__ == "__main__":
    main()
