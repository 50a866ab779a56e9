"""From tokens to attention's queries, keys and values in an image transformer whose requests bring adapters, and a
training step of those adapters beside the frozen quantized projection.

    python examples/adapted_attention_input.py

Serving: rotate and quantize the tokens, run the quantized QKV projection, add each request's low-rank adapter, then the
norms of query and key heads with the rotation by (time, row, column) in one pass.  Training: the same calls, then their
gradients in the opposite order, down to the adapters' and the norms' weights.
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_02461_amd as oq  # noqa: E402

DEV = "cuda"
HEADS, D = 24, 128
WIDTH = HEADS * D
RANK = 16
DIMS = (16, 56, 56)              # values of a head that turn with time, row and column


class Layer:
    """One attention input: a quantized QKV projection, the norms' weights, and a pool of adapters."""

    def __init__(self, adapters, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        weight = torch.randn((3 * WIDTH, WIDTH), generator=g, device=DEV).mul_(WIDTH ** -0.5).to(torch.bfloat16)
        self.rotation = oq.rpbh_plan(WIDTH, 128, seed)
        self.codebook = oq.lloydmax_codebook(4, WIDTH)
        self.codes, self.norms = oq.quantize_weights_offline(self.rotation, self.codebook, weight)
        self.q_weight = torch.ones(D, device=DEV)
        self.k_weight = torch.ones(D, device=DEV)
        self.A = torch.randn((adapters, RANK, WIDTH), generator=g, device=DEV).mul_(WIDTH ** -0.5).to(torch.bfloat16)
        self.B = torch.zeros((adapters, 3 * WIDTH, RANK), dtype=torch.bfloat16, device=DEV)

    def project(self, x, plan, h=None):
        """The adapted QKV projection of tokens x, bf16 [rows, 3 WIDTH]."""
        codes, norms = oq.rpbh_quantize_act(self.rotation, self.codebook, x)
        M, N, K = x.shape[0], self.codes.shape[0], x.shape[1]
        workspace = torch.empty((max(16, oq.orbit_qlinear_workspace_size(M, N, K)),), dtype=torch.uint8, device=DEV)
        qkv = oq.orbit_qlinear_ws(self.codebook, codes, norms, self.codebook, self.codes, self.norms, workspace,
                                  out_dtype=torch.bfloat16)
        return oq.lora_add(plan, x, self.A, self.B, qkv, out=qkv, h=h)

    def heads(self, qkv, batch):
        """Views of queries, keys and values, [batch, token, head, D]."""
        return qkv.view(batch, -1, 3, HEADS, D).unbind(2)


def positions(frames, rows, columns, text):
    """int32 [token, 3]: text tokens at the origin, then the grid of image tokens."""
    grid = torch.cartesian_prod(torch.arange(frames), torch.arange(rows), torch.arange(columns))
    return torch.cat([torch.zeros((text, 3), dtype=torch.int64), grid]).to(torch.int32).to(DEV)


def serve(layer, x, batch, plan, rope, pos):
    """Queries and keys ready for attention, values as they come."""
    q, k, v = layer.heads(layer.project(x, plan), batch)
    q, k = oq.qk_norm_rope(rope, q, k, pos, layer.q_weight, layer.k_weight, q_out=q, k_out=k)   # in place
    return q, k, v


def train_step(layer, x, batch, plan, rope, pos, target_q, target_k, rate):
    """One step down the mean squared distance of q and k from their targets, each weight's as long as `rate`
    times the square root of its size; returns the distance before it."""
    h = torch.empty((x.shape[0], RANK), dtype=torch.float32, device=DEV)
    qkv = layer.project(x, plan, h=h)
    q, k, _ = layer.heads(qkv, batch)
    yq, yk = oq.qk_norm_rope(rope, q, k, pos, layer.q_weight, layer.k_weight, out_dtype=torch.float32)
    eq, ek = yq - target_q, yk - target_k
    n = eq.numel() + ek.numel()
    loss = (eq.square().sum() + ek.square().sum()) / n
    d_qkv = torch.zeros_like(qkv)
    dq, dk, _ = layer.heads(d_qkv, batch)
    _, _, d_qw, d_kw = oq.qk_norm_rope_backward(rope, eq * (2 / n), ek * (2 / n), q, k, pos, layer.q_weight, layer.k_weight,
                                                q_grad=dq, k_grad=dk)
    _, dA, dB = oq.lora_add_backward(plan, d_qkv, x, layer.A, layer.B, h)
    for weight, grad in ((layer.A, dA), (layer.B, dB), (layer.q_weight, d_qw), (layer.k_weight, d_kw)):
        weight.copy_(weight.float() - rate * grad / (grad.square().mean().sqrt() + 1e-30))
    return loss


def main(steps=20):
    frames, rows, columns, text = 1, 16, 16, 32
    tokens, requests = text + frames * rows * columns, 4
    pos = positions(frames, rows, columns, text)
    rope = oq.rope_plan(DIMS, (frames, rows, columns))
    # three of four requests have an adapter, two of them the same one
    plan = oq.lora_plan(requests * tokens, [i * tokens for i in range(requests)], [0, 1, -1, 0], [RANK, RANK // 2], [1.0, 2.0])
    layer = Layer(adapters=2)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((requests * tokens, WIDTH), generator=g, device=DEV).to(torch.bfloat16)

    q, k, v = serve(layer, x, requests, plan, rope, pos)
    print(f"served {requests} requests of {tokens} tokens: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    target_q, target_k = q.float().roll(1, dims=-1), k.float().roll(1, dims=-1)
    losses = [float(train_step(layer, x, requests, plan, rope, pos, target_q, target_k, rate=1e-3)) for _ in range(steps)]
    print("loss by step:", " ".join(f"{v:.4f}" for v in losses))
    return losses


if __name__ == "__main__":
    main()
