"""What a transformer block has around its quantized projections, as cases that can be timed and compared:

    norm         layer_norm / layer_norm_modulate: the norm in front of a projection, with weights, or with a scale and
                 a shift for each batch
    norm_train   the same and its backward pass: gradients of the rows and of weight and bias, or scale and shift
    attn         attention over packed sequences of any lengths: whole prompts, chunks, single tokens, other sequences'
                 keys; grouped heads, causal or not
    attn_train   attention and its backward pass

Widths and token counts are those of the workloads this repository states (an image DiT: hidden 3072 in 24 heads of 128,
4096 image tokens + up to 512 text tokens, two guidance branches; a video DiT: hidden 5120 in 40 heads of 128, 21 frames
of 30 x 52 tokens + 512 text tokens), or generic where grouped heads and causal masks come in.  All inputs are made from
the seed alone; a case's lengths go by the case.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
MOST_NORM = 33272 * 5120              # values of the largest norm, and of the largest training step of one
MOST_PAIRS = 40 * 32760 * 32760 * 128     # heads x pairs of tokens x head size of the largest attention
MOST_TRAIN = 24 * 2 * 4429 * 4429 * 128   # and of its training step
MOST_ROWS = 32760 * 40 * 128          # values of the largest q, k or v
SCORES = 1 << 32                      # of the plain form at a time: 16 GiB
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def listed():
    return [
        # one conditioning token for each guidance branch: all latency and launch
        dict(name="norm_token", kind="norm", B=2, L=1, N=5120, modulate=True, dtype="bf16", out="bf16"),
        # a text encoder's output under a weight and a bias, rows of an odd length
        dict(name="norm_odd", kind="norm", B=3, L=333, N=1999, modulate=False, dtype="bf16", out="fp32"),
        # the video model's residual stream, kept in fp32, in front of the quantizer
        dict(name="norm_video", kind="norm", B=1, L=33272, N=5120, modulate=True, dtype="fp32", out="bf16"),
        # a training step of the image model's modulated norm, 333 prompt tokens
        dict(name="norm_train_image", kind="norm_train", B=2, L=4429, N=3072, modulate=True, dtype="bf16", out="bf16"),
        # of the video model's norm in front of the cross attention, which has a weight and a bias
        dict(name="norm_train_video", kind="norm_train", B=1, L=32760, N=5120, modulate=False, dtype="fp32", out="bf16"),
        # 16 requests with one new token each over what they have so far, up to 8192 tokens, grouped heads
        dict(name="attn_token", kind="attn", B=16, Lq=1, Lk=8192, ragged=True, H=32, Hk=8, D=128, causal=True),
        # an image step: two guidance branches
        dict(name="attn_image", kind="attn", B=2, Lq=0, Lk=4608, ragged=False, H=24, Hk=24, D=128, causal=False),
        # the video model's tokens over a prompt
        dict(name="attn_cross", kind="attn", B=1, Lq=32760, Lk=512, ragged=False, H=40, Hk=40, D=128, causal=False),
        # twelve prompts of 300 to 4096 tokens, packed, causal, grouped heads
        dict(name="attn_packed", kind="attn", B=12, Lq=0, Lk=4096, ragged=True, H=32, Hk=8, D=128, causal=True),
        # the whole clip: the largest call
        dict(name="attn_video", kind="attn", B=1, Lq=0, Lk=32760, ragged=False, H=40, Hk=40, D=128, causal=False),
        # a training step of the image model, 333 prompt tokens: a ragged count
        dict(name="attn_train_image", kind="attn_train", B=2, Lq=0, Lk=4429, ragged=False, H=24, Hk=24, D=128, causal=False),
        # a training step on packed sequences, causal, grouped heads of 64
        dict(name="attn_train_packed", kind="attn_train", B=7, Lq=0, Lk=2048, ragged=True, H=16, Hk=4, D=64, causal=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "attn", "attn", "attn_train", "attn_train"])
    if kind.startswith("norm"):
        N = rng.choice([5120, 8 * _log_int(rng, 16, 1536), _log_int(rng, 100, 12288)])
        B = rng.randint(1, 4)
        L = max(1, min(_log_int(rng, 1, 33272), MOST_NORM // (B * N)))
        return dict(kind=kind, B=B, L=L, N=N, modulate=rng.random() < 0.6, dtype=rng.choice(["bf16", "fp32"]), out=rng.choice(["bf16", "bf16", "fp32"]))
    Hk = rng.choice([8, 24, 40, rng.randint(1, 16)])
    H = Hk * rng.choice([1, 1, 2, 4, 5, 8])
    D = rng.choice([128, 128, 64, 96, 80, 40])
    B, ragged, causal = _log_int(rng, 1, 32), rng.random() < 0.6, rng.random() < 0.6
    Lk = _log_int(rng, 1, 32760)
    Lk = max(1, min(Lk, MOST_ROWS // (B * H * D)))
    most = MOST_PAIRS if kind == "attn" else MOST_TRAIN
    if rng.random() < 0.5:
        Lq = 0                                              # as many queries as keys
        Lk = max(1, min(Lk, int(math.sqrt(most / (B * H * D)))))
    else:                                                   # a chunk, single tokens, or more queries than keys
        Lq = 1 if rng.random() < 0.4 and kind == "attn" else _log_int(rng, 1, 4096)
        Lq = max(1, min(Lq, MOST_ROWS // (B * H * D), most // (B * H * D * Lk)))
    return dict(kind=kind, B=B, Lq=Lq, Lk=Lk, ragged=ragged, H=H, Hk=Hk, D=D, causal=causal)


# --- inputs ---------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + stream) % (1 << 62))
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _lengths(case):
    """Queries and keys of each sequence.  Ragged: from a B-th of the longest to the longest, the longest first."""
    n = case["B"]
    k = [max(1, case["Lk"] * (n - i) // n - 3 * i) if case["ragged"] else case["Lk"] for i in range(n)]
    return (k if case["Lq"] == 0 else [case["Lq"]] * n), k


def _rows(case, seed):
    """The residual stream [B, L, N]: channels of different size and place, a scale for each token."""
    g = _gen(seed, 1)
    B, L, N = case["B"], case["L"], case["N"]
    x = _randn((B, L, N), g).mul_(torch.exp(0.5 * _randn((N,), g))).add_(0.5 * _randn((N,), g))
    return x.mul_(torch.exp(0.5 * _randn((B, L, 1), g))).to(TYPE[case["dtype"]])


def _norm_weights(case, seed):
    """Weight and bias, bf16 [N]; or scale and shift of each batch, views of the modulation projection's fp32 output."""
    g = _gen(seed, 2)
    if case["modulate"]:
        return (0.3 * _randn((case["B"], 6 * case["N"]), g)).chunk(6, dim=-1)[:2]
    return (1 + 0.2 * _randn((case["N"],), g)).to(torch.bfloat16), (0.2 * _randn((case["N"],), g)).to(torch.bfloat16)


def _norm_grad(case, seed):
    return _randn((case["B"], case["L"], case["N"]), _gen(seed, 3)).mul_(0.01).to(TYPE[case["out"]])


def _unit(x):
    """Heads as a norm with weights around 1.3 leaves them."""
    return x.mul_(torch.rsqrt(x.square().mean(-1, keepdim=True))).mul_(1.3)


def _heads(case, seed):
    """q [rows, H, D], k and v [rows, Hk, D]: views of the fused projection's output; of the queries' and of the
    keys' and values' where they are other tokens."""
    g = _gen(seed, 4)
    q, k = (sum(n) for n in _lengths(case))
    H, Hk, D = case["H"], case["Hk"], case["D"]
    kv = _randn((k, 2 * Hk, D), g)
    kv[:, :Hk] = _unit(kv[:, :Hk])
    kv[:, Hk:].mul_(torch.exp(0.5 * _randn((Hk, D), g)))
    queries = _unit(_randn((q, H, D), g))
    if case["Lq"] == 0:
        qkv = torch.cat([queries, kv], dim=1).to(torch.bfloat16)
        return qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    kv = kv.to(torch.bfloat16)
    return queries.to(torch.bfloat16), kv[:, :Hk], kv[:, Hk:]


def _heads_grad(case, seed):
    return _randn((sum(_lengths(case)[0]), case["H"], case["D"]), _gen(seed, 5)).mul_(0.01).to(torch.bfloat16)


def prepare(case, seed):
    kind = case["kind"]
    state = dict(case=case)
    if kind.startswith("norm"):
        state["x"], (state["w"], state["b"]) = _rows(case, seed), _norm_weights(case, seed)
        if kind == "norm_train":
            state["dy"] = _norm_grad(case, seed)
        return state
    state["q"], state["k"], state["v"] = _heads(case, seed)
    if kind == "attn_train":
        state["do"] = _heads_grad(case, seed)
    nq, nk = _lengths(case)
    if own:
        import paper_2607_02461_amd as oq
        state["plan"] = oq.attention_plan(nq, nk, heads=case["H"], kv_heads=case["Hk"], causal=case["causal"])
        return state
    # sequences side by side, [B, longest]: each place's row of the packed tensors, and each row's place
    for name, n in (("q", nq), ("k", nk)):
        n = torch.tensor(n, device=DEV)
        at = torch.arange(int(n.max()), device=DEV)
        state[name + "_len"] = n
        state[name + "_row"] = (n.cumsum(0) - n)[:, None] + torch.minimum(at, n[:, None] - 1)
        state[name + "_place"] = (at < n[:, None]).flatten().nonzero()[:, 0]
    return state


# --- plain forms ----------------------------------------------------------------------------------
def _normed(s):
    """Normed rows, 1 / deviation and the gain, in fp32."""
    x, w = s["x"].float(), s["w"].float()
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r, (1 + w)[:, None] if s["case"]["modulate"] else w


def _plain_norm(s):
    case = s["case"]
    n, r, gain = _normed(s)
    b = s["b"].float()
    y = (n * gain + (b[:, None] if case["modulate"] else b)).to(TYPE[case["out"]])
    if case["kind"] == "norm":
        return y
    dy = s["dy"].float()
    over = 1 if case["modulate"] else (0, 1)
    dw, db = (dy * n).sum(over), dy.sum(over)
    g = dy * gain
    dx = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    return y, dx.to(s["x"].dtype), dw, db


def _side_by_side(s, t, rows):
    """[B, heads, longest, D] in fp32 of packed heads."""
    return s[t][s[rows]].float().transpose(1, 2).contiguous()


def _packed(x, place, like):
    return x.transpose(1, 2).flatten(0, 1)[place].to(like.dtype)


def _plain_attention(s):
    """Scores of as many heads at a time as memory has room for."""
    case = s["case"]
    B, H, Hk, D = case["B"], case["H"], case["Hk"], case["D"]
    G, Lq, Lk = H // Hk, s["q_row"].shape[1], s["k_row"].shape[1]
    scale = D ** -0.5
    j = torch.arange(Lk, device=DEV)
    last = s["k_len"][:, None] - 1
    if case["causal"]:
        last = torch.minimum(last, torch.arange(Lq, device=DEV) + (s["k_len"] - s["q_len"])[:, None])
    hidden = (j > last[..., None])[:, None, None]                      # [B, 1, 1, Lq or 1, Lk]
    train = case["kind"] == "attn_train"
    q, k, v = _side_by_side(s, "q", "q_row"), _side_by_side(s, "k", "k_row"), _side_by_side(s, "v", "k_row")
    o = torch.empty_like(q)
    if train:
        do = s["do"].float()[s["q_row"]] * (torch.arange(Lq, device=DEV) < s["q_len"][:, None])[..., None, None]
        do = do.transpose(1, 2).contiguous()
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    step = max(1, SCORES // (B * G * Lq * Lk))
    for h in range(0, Hk, step):
        here, of = slice(h, h + step), slice(h * G, (h + step) * G)
        kt, qs = k[:, here], q[:, of].reshape(B, -1, G * Lq, D)
        p = (qs @ kt.transpose(2, 3)).mul_(scale)
        p.view(B, -1, G, Lq, Lk).masked_fill_(hidden, -math.inf)
        most = p.amax(-1, keepdim=True)
        p.sub_(most.masked_fill_(most == -math.inf, 0.0)).exp_()
        total = p.sum(-1, keepdim=True)
        total.masked_fill_(total == 0, 1.0)                            # rows that see no key: zeros
        if not train:
            o[:, of] = (p @ v[:, here]).div_(total).view(B, -1, Lq, D)
            continue
        p.div_(total)
        out, grad = p @ v[:, here], do[:, of].reshape(B, -1, G * Lq, D)
        o[:, of] = out.view(B, -1, Lq, D)
        dv[:, here] = p.transpose(2, 3) @ grad
        ds = (grad @ v[:, here].transpose(2, 3)).sub_((grad * out).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        dq[:, of] = (ds @ kt).view(B, -1, Lq, D)
        dk[:, here] = ds.transpose(2, 3) @ qs
    o = _packed(o, s["q_place"], s["q"])
    if not train:
        return o
    return o, _packed(dq, s["q_place"], s["q"]), _packed(dk, s["k_place"], s["k"]), _packed(dv, s["k_place"], s["v"])


def run(state):
    s, case = state, state["case"]
    if not own:
        return _plain_norm(s) if case["kind"].startswith("norm") else _plain_attention(s)
    import paper_2607_02461_amd as oq
    if case["kind"].startswith("norm"):
        forward, backward = (oq.layer_norm_modulate, oq.layer_norm_modulate_backward) if case["modulate"] else (oq.layer_norm, oq.layer_norm_backward)
        y = forward(s["x"], s["w"], s["b"], eps=EPS, out_dtype=TYPE[case["out"]])
        return y if case["kind"] == "norm" else (y,) + tuple(backward(s["dy"], s["x"], s["w"], eps=EPS))
    if case["kind"] == "attn":
        return oq.attention(s["plan"], s["q"], s["k"], s["v"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=s["q"].device)
    o = oq.attention(s["plan"], s["q"], s["k"], s["v"], lse=lse)
    return (o,) + tuple(oq.attention_backward(s["plan"], s["do"], s["q"], s["k"], s["v"], o, lse))


def _pairs(case):
    """Pairs of a query and a key that it sees, over all sequences."""
    if not case["causal"]:
        return sum(q * k for q, k in zip(*_lengths(case)))
    live = [np.clip(np.arange(q, dtype=np.int64) + 1 + k - q, 0, k) for q, k in zip(*_lengths(case))]
    return int(sum(v.sum() for v in live))


def work(case):
    if case["kind"].startswith("norm"):
        B, L, N = case["B"], case["L"], case["N"]
        one, other = SIZE[case["dtype"]], SIZE[case["out"]]
        weights = 8 * B * N if case["modulate"] else 4 * N
        got = {"bytes": (one + other) * B * L * N + weights, "flops": 8 * B * L * N}
        if case["kind"] == "norm_train":
            got["bytes"] += (other + one) * B * L * N + 8 * N * (B if case["modulate"] else 1)
            got["flops"] += 14 * B * L * N
        return got
    q, k = (sum(n) for n in _lengths(case))
    wide, narrow, D = 2 * q * case["H"] * case["D"], 4 * k * case["Hk"] * case["D"], case["D"]
    per = case["H"] * D * _pairs(case)
    if case["kind"] == "attn":
        return {"bytes": 2 * wide + narrow, "flops": 4 * per}
    return {"bytes": 4 * wide + 2 * narrow, "flops": 14 * per}


# --- the definitions in 64 bits -------------------------------------------------------------------
def _exact_norm(case, seed):
    x, (w, b) = _rows(case, seed).double(), (t.double() for t in _norm_weights(case, seed))
    train = case["kind"] == "norm_train"
    x, w, b = (t.requires_grad_(train) for t in (x, w, b))
    gain, offset = (1 + w.unsqueeze(1), b.unsqueeze(1)) if case["modulate"] else (w, b)
    y = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS) * gain + offset
    if not train:
        return y
    return (y.detach(),) + torch.autograd.grad(y, (x, w, b), _norm_grad(case, seed).double())


def exact(case, seed):
    if case["kind"].startswith("norm"):
        return _exact_norm(case, seed)
    train, G, D = case["kind"] == "attn_train", case["H"] // case["Hk"], case["D"]
    q, k, v = _heads(case, seed)
    results = [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in ((q, q, k, v) if train else (q,))]
    do = _heads_grad(case, seed) if train else None
    q0 = k0 = 0
    for nq, nk in zip(*_lengths(case)):
        first = max(0, nq - nk) if case["causal"] else 0            # queries before it see nothing
        rows, keys = slice(q0 + first, q0 + nq), slice(k0, k0 + nk)
        q0, k0 = q0 + nq, k0 + nk
        hidden = None
        if case["causal"]:
            n = nq - first
            hidden = torch.ones((n, nk), dtype=torch.bool, device=DEV).triu(nk - n + 1)
        for h in range(case["H"]):
            mine = [t.double() for t in (q[rows, h], k[keys, h // G], v[keys, h // G])]
            mine = [t.requires_grad_(train) for t in mine]
            z = mine[0] @ mine[1].t() / math.sqrt(D)
            o = torch.softmax(z if hidden is None else z.masked_fill(hidden, -math.inf), dim=-1) @ mine[2]
            results[0][rows, h] = o.detach()
            if train:
                dq, dk, dv = torch.autograd.grad(o, mine, do[rows, h].double())
                results[1][rows, h] = dq
                results[2][keys, h // G] += dk
                results[3][keys, h // G] += dv
    return tuple(results) if train else results[0]
