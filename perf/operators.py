"""What stands between a quantized QKV projection and attention, and beside a projection when requests bring
their own adapters, as cases that can be timed and compared:

    rope            axial_rope: rotary positions with one to three axes (time, height, width)
    norm_rope       qk_norm_rope: RMS norms of queries and keys for each head, with the rotation in the same pass
    norm_rope_bwd   qk_norm_rope_backward: gradients of q, k and of both norms' weights
    lora            lora_add: low-rank adapters of many requests on the output of the projection they share
    lora_train      lora_add, then lora_add_backward: a training step's two directions

Widths and token counts are those of the workloads this repository states: an image DiT (hidden 3072 in 24 heads
of 128, feed-forward 12288, 4096 image tokens + up to 512 text tokens, two guidance branches) and a video DiT
(hidden 5120 in 40 heads of 128, feed-forward 13824, 21 frames of 30 x 52 tokens + 512 text tokens).  All inputs
are made from the seed alone.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 10000.0
MOST_ROPE = 32760 * 40 * 128          # elements of the largest rotation, and of q in the largest norm
MOST_BACK = 9216 * 24 * 128           # of q in the largest norm's backward pass
MOST_LORA = 33272 * (5120 + 13824)    # M (K + N) of the largest adapters' call, and of their training step
MOST_TRAIN = 9216 * (3072 + 9216)
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


def listed():
    return [
        # one modulated text token's heads: the smallest call, all latency and launch
        dict(name="rope_token", kind="rope", B=1, L=1, H=24, D=128, axes="16,56,56", halves=False, dtype="bf16", inverse=False),
        # the video model's queries, whole clip: time, height and width axes
        dict(name="rope_video", kind="rope", B=1, L=32760, H=40, D=128, axes="44,42,42", halves=False, dtype="bf16", inverse=False),
        # the rotation's gradient in fp32 for half-split pairs, a part of the head rotated, ragged token count
        dict(name="rope_grad", kind="rope", B=3, L=2777, H=16, D=96, axes="16,24,24", halves=True, dtype="fp32", inverse=True),
        # one token per guidance branch
        dict(name="norm_token", kind="norm_rope", B=2, L=1, Hq=24, Hk=24, D=128, axes="16,56,56", halves=False, dtype="bf16", out="bf16"),
        # queries and keys of an image step, views of the fused QKV projection's bf16 output
        dict(name="norm_image", kind="norm_rope", B=2, L=4608, Hq=24, Hk=24, D=128, axes="16,56,56", halves=False, dtype="bf16", out="bf16"),
        # the video model's, from the fp32 output of the quantized projection
        dict(name="norm_video", kind="norm_rope", B=1, L=32760, Hq=40, Hk=40, D=128, axes="44,42,42", halves=False, dtype="fp32", out="bf16"),
        # training the norms of the image model, 333 prompt tokens: a ragged count
        dict(name="norm_image_bwd", kind="norm_rope_bwd", B=2, L=4429, Hq=24, Hk=24, D=128, axes="16,56,56", halves=False, dtype="bf16", out="bf16"),
        # modulation projections of 16 requests, a token and an adapter each
        dict(name="lora_token", kind="lora", M=16, K=3072, N=18432, R=16, adapters=16, requests=16, ragged=False, idle=False, out="fp32"),
        # two images' fused QKV projection, each under its own adapter
        dict(name="lora_image", kind="lora", M=9216, K=3072, N=9216, R=32, adapters=2, requests=2, ragged=False, idle=False, out="bf16"),
        # the video feed-forward with one adapter of rank 64, on the projection's fp32 output
        dict(name="lora_video", kind="lora", M=33272, K=5120, N=13824, R=64, adapters=1, requests=1, ragged=False, idle=False, out="fp32"),
        # a short training step: 5 ragged requests of 333 rows in all, three adapters of ranks 8, 4 and 2
        dict(name="train_short", kind="lora_train", M=333, K=3072, N=3072, R=8, adapters=3, requests=5, ragged=True, idle=True, out="bf16"),
        # a training step on two images, adapters of rank 32 on the fused QKV projection
        dict(name="train_image", kind="lora_train", M=9216, K=3072, N=9216, R=32, adapters=2, requests=2, ragged=False, idle=False, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "norm_rope", "norm_rope", "norm_rope_bwd", "norm_rope_bwd", "lora", "lora", "lora_train", "lora_train"])
    if kind.startswith("lora"):
        K, N = (rng.choice([3072, 5120, 8 * _log_int(rng, 64, 1536)]) for _ in range(2))
        if rng.random() < 0.3:
            N = _log_int(rng, 512, 18432)
        M = _log_int(rng, 1, 33272)
        M = max(1, min(M, (MOST_LORA if kind == "lora" else MOST_TRAIN) // (K + N)))
        requests = min(M, _log_int(rng, 1, 64))
        adapters = rng.randint(1, min(16, requests))
        return dict(kind=kind, M=M, K=K, N=N, R=8 * rng.choice([1, 2, 2, 4, 4, 6, 8]), adapters=adapters, requests=requests,
                    ragged=rng.random() < 0.7, idle=rng.random() < 0.4, out="bf16" if kind == "lora_train" else rng.choice(["bf16", "fp32"]))
    D, axes = rng.choice([(128, "16,56,56"), (128, "44,42,42"), (128, "64,64"), (128, "128"), (64, "16,24,24"), (96, "16,24,24"),
                          (80, "40,40"), (256, "64,96,96")])
    H = rng.choice([24, 40, rng.randint(1, 48)])
    B = rng.randint(1, 4)
    L = _log_int(rng, 1, 32760)
    most = MOST_BACK if kind == "norm_rope_bwd" else MOST_ROPE
    L = max(1, min(L, most // (B * H * D)))
    case = dict(kind=kind, B=B, L=L, D=D, axes=axes, halves=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if kind == "rope":
        return case | dict(H=H, inverse=rng.random() < 0.5)
    return case | dict(Hq=H, Hk=rng.choice([H, H, max(1, H // 4)]), out="bf16" if case["dtype"] == "bf16" else rng.choice(["bf16", "fp32"]))


# --- inputs ---------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + stream) % (1 << 62))
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def _lengths(case):
    """Positions that each axis has a table for: frames, rows and columns of tokens."""
    return {1: [34832], 2: [672, 52], 3: [32, 64, 64]}[len(_axes(case))]


def _positions(case, seed):
    """int32 [L, axes]: an eighth of the tokens, at most 512, are text at the origin, the others lie on a grid from
    some place in its first frame on."""
    L, axes = case["L"], len(_axes(case))
    text = min(512, L // 8)
    i = torch.arange(L, device=DEV) - text
    at = i + int(np.random.default_rng(seed).integers(1, 30 * 52))
    grid = {1: [at], 2: [at // 52, at % 52], 3: [at // (30 * 52), at // 52 % 30, at % 52]}[axes]
    return torch.where((i >= 0)[:, None], torch.stack(grid, dim=1), 0).to(torch.int32).contiguous()


def _frequencies(case):
    """Per axis, theta^(-2 j / dim) in 64 bits."""
    return [THETA ** (-2.0 * np.arange(d // 2) / d) for d in _axes(case)]


def _heads(case, seed):
    """q and k, [B, L, heads, D]: views of one fused projection's output, as it lies in memory (q, k, v side by side);
    channels of different size, and a scale for each token."""
    g = _gen(seed, 1)
    B, L, D = case["B"], case["L"], case["D"]
    Hq, Hk = case["Hq"], case["Hk"]
    qkv = _randn((B, L, Hq + 2 * Hk, D), g).mul_(torch.exp(0.5 * _randn((Hq + 2 * Hk, D), g)))
    qkv = qkv.mul_(torch.exp(0.3 * _randn((B, L, 1, 1), g))).to(TYPE[case["dtype"]])
    return qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk]


def _norm_weights(case, seed):
    g = _gen(seed, 2)
    return [(1.0 + 0.2 * _randn((case["D"],), g)).to(torch.bfloat16) for _ in range(2)]


def _norm_grads(case, seed):
    g = _gen(seed, 3)
    return [_randn((case["B"], case["L"], h, case["D"]), g).mul_(0.01).to(TYPE[case["out"]]) for h in (case["Hq"], case["Hk"])]


def _rows(case, seed):
    """First row of each request, its adapter (-1: none) and each adapter's rank and scale."""
    r = np.random.default_rng(seed)
    M, n, req = case["M"], case["adapters"], case["requests"]
    starts = np.sort(r.integers(0, M + 1, req - 1)) if case["ragged"] else np.arange(1, req) * M // req
    adapter = r.permutation(req) % n
    if case["idle"]:
        adapter = np.where(r.random(req) < 0.2, -1, adapter)
    ranks = [max(1, case["R"] >> (a % 3)) if case["ragged"] else case["R"] for a in range(n)]
    scales = [float(np.float32(s)) for s in r.choice([0.5, 1.0, 2.0], n)]
    return [0] + [int(s) for s in starts], [int(a) for a in adapter], ranks, scales


def _tokens(M, K, seed):
    """bf16 tokens with heavy tails (Student-t, 4 degrees of freedom) and 1% outlier channels."""
    g = _gen(seed, 4)
    scale = torch.ones((K,), device=DEV)
    scale[torch.randperm(K, generator=g, device=DEV)[: max(1, K // 100)]] = 20.0
    chi2 = torch.zeros((M, K), device=DEV)
    for _ in range(4):
        chi2 += _randn((M, K), g).square_()
    return chi2.reciprocal_().mul_(4.0).sqrt_().mul_(_randn((M, K), g)).mul_(scale).to(torch.bfloat16)


def _pools(case, seed):
    """Adapters A [n, R, K] and B [n, N, R]."""
    g = _gen(seed, 5)
    n, R, K, N = case["adapters"], case["R"], case["K"], case["N"]
    return (_randn((n, R, K), g) / math.sqrt(K)).to(torch.bfloat16), (_randn((n, N, R), g) * 0.1).to(torch.bfloat16)


def _base(case, seed):
    """The shared projection's output."""
    return _randn((case["M"], case["N"]), _gen(seed, 6)).to(TYPE[case["out"]])


def _out_grad(case, seed):
    return _randn((case["M"], case["N"]), _gen(seed, 7)).mul_(0.01).to(torch.bfloat16)


def _single(case, seed):
    return _heads(case | dict(Hq=case["H"], Hk=0), seed)[0]


def prepare(case, seed):
    kind = case["kind"]
    state = dict(case=case)
    if kind.startswith("lora"):
        starts, adapter, ranks, scales = _rows(case, seed)
        state["x"], state["base"] = _tokens(case["M"], case["K"], seed), _base(case, seed)
        state["a"], state["b"] = _pools(case, seed)
        if kind == "lora_train":
            state["dy"] = _out_grad(case, seed)
        if own:
            import paper_2607_02461_amd as oq
            state["plan"] = oq.lora_plan(case["M"], starts, adapter, ranks, scales)
            return state
        # the scale that each row gives to each column of all adapters' ranks together
        of_row = torch.tensor(np.repeat(adapter, np.diff(starts + [case["M"]])), device=DEV)
        column = torch.arange(case["adapters"] * case["R"], device=DEV)
        live = column % case["R"] < torch.tensor(ranks, device=DEV)[column // case["R"]]
        scale = torch.tensor(scales, dtype=torch.float32, device=DEV)[column // case["R"]]
        state["gate"] = torch.where((of_row[:, None] == column // case["R"]) & live, scale, 0.0)
        return state
    state["positions"] = _positions(case, seed)
    if kind == "rope":
        state["x"] = _single(case, seed)
    else:
        state["q"], state["k"] = _heads(case, seed)
        state["wq"], state["wk"] = _norm_weights(case, seed)
        if kind == "norm_rope_bwd":
            state["dq"], state["dk"] = _norm_grads(case, seed)
    if own:
        import paper_2607_02461_amd as oq
        state["plan"] = oq.rope_plan(_axes(case), _lengths(case), theta=THETA, halves=case["halves"])
        return state
    # one table of angles for all axes, row by row of the longest, and where each pair looks in it
    pairs = [len(f) for f in _frequencies(case)]
    angle = [np.arange(n)[:, None] * f for n, f in zip(_lengths(case), _frequencies(case))]
    table = np.concatenate([np.pad(a, ((0, max(_lengths(case)) - len(a)), (0, 0))) for a in angle], axis=1)
    state["cos"] = torch.tensor(np.cos(table), dtype=torch.float32, device=DEV)
    state["sin"] = torch.tensor(np.sin(table), dtype=torch.float32, device=DEV)
    state["axis"] = torch.tensor(np.repeat(np.arange(len(pairs)), pairs), device=DEV)
    return state


# --- plain forms ----------------------------------------------------------------------------------
def _turn(s, x, sign):
    """The rotation of fp32 heads [B, L, H, D] by sign * angle."""
    row = s["positions"].long()[:, s["axis"]]
    cos, sin = s["cos"].gather(0, row)[:, None], s["sin"].gather(0, row)[:, None] * sign
    n = cos.shape[-1]
    u, v = (x[..., :n], x[..., n:2 * n]) if s["case"]["halves"] else (x[..., :2 * n:2], x[..., 1:2 * n:2])
    a, b = u * cos - v * sin, u * sin + v * cos
    turned = torch.cat([a, b], dim=-1) if s["case"]["halves"] else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _norm_turn(s, x, w):
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()
    return _turn(s, y, 1.0).to(TYPE[s["case"]["out"]])


def _norm_turn_grad(s, dy, x, w):
    g, x = _turn(s, dy.float(), -1.0), x.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    unit = x * r
    dw = (g * unit).sum(dim=(0, 1, 2))
    g = g * w.float()
    return (r * (g - unit * (g * unit).mean(dim=-1, keepdim=True))).to(s["q"].dtype), dw


def _adapters(s):
    """All adapters side by side, [n R, K] and [n R, N], and the rows' products with A, scaled where they are the
    row's own and zero elsewhere."""
    a = s["a"].flatten(0, 1).float()
    b = s["b"].transpose(1, 2).flatten(0, 1).float()
    x = s["x"].float()
    return x, a, b, (x @ a.t()) * s["gate"]


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rope":
        return _turn(s, s["x"].float(), -1.0 if case["inverse"] else 1.0).to(s["x"].dtype)
    if kind == "norm_rope":
        return _norm_turn(s, s["q"], s["wq"]), _norm_turn(s, s["k"], s["wk"])
    if kind == "norm_rope_bwd":
        return _norm_turn_grad(s, s["dq"], s["q"], s["wq"]) + _norm_turn_grad(s, s["dk"], s["k"], s["wk"])
    x, a, b, h = _adapters(s)
    y = (s["base"].float() + h @ b).to(TYPE[case["out"]])
    if kind == "lora":
        return y
    dy = s["dy"].float()
    g = (dy @ b.t()) * s["gate"]
    n, R = case["adapters"], case["R"]
    return y, (g @ a).to(torch.bfloat16), (g.t() @ x).view(n, R, -1), (h.t() @ dy).view(n, R, -1).transpose(1, 2).contiguous()


def run(state):
    if not own:
        return _plain(state)
    import paper_2607_02461_amd as oq
    s, case = state, state["case"]
    kind = case["kind"]
    if kind == "rope":
        return oq.axial_rope(s["plan"], s["x"], s["positions"], inverse=case["inverse"])
    if kind == "norm_rope":
        return oq.qk_norm_rope(s["plan"], s["q"], s["k"], s["positions"], s["wq"], s["wk"], eps=EPS, out_dtype=TYPE[case["out"]])
    if kind == "norm_rope_bwd":
        dq, dk, dwq, dwk = oq.qk_norm_rope_backward(s["plan"], s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["wq"], s["wk"], eps=EPS)
        return dq, dwq, dk, dwk
    if kind == "lora":
        return oq.lora_add(s["plan"], s["x"], s["a"], s["b"], s["base"])
    h = torch.empty((case["M"], case["R"]), dtype=torch.float32, device=s["x"].device)
    y = oq.lora_add(s["plan"], s["x"], s["a"], s["b"], s["base"], h=h)
    return (y,) + tuple(oq.lora_add_backward(s["plan"], s["dy"], s["x"], s["a"], s["b"], h))


def work(case):
    kind = case["kind"]
    if kind.startswith("lora"):
        M, K, N, R, n = (case[v] for v in ("M", "K", "N", "R", "adapters"))
        pools = n * R * (K + N)
        got = {"bytes": 2 * M * K + 2 * SIZE[case["out"]] * M * N + 2 * pools, "flops": 2 * M * R * (K + N) + 2 * M * N}
        if kind == "lora_train":
            got["bytes"] += 2 * M * N + 2 * M * K + 4 * pools
            got["flops"] += 4 * M * R * (K + N)
        return got
    B, L, D = case["B"], case["L"], case["D"]
    axes = _axes(case)
    fixed = 4 * L * len(axes) + sum(4 * n * d for n, d in zip(_lengths(case), axes))
    if kind == "rope":
        x = B * L * case["H"] * D
        return {"bytes": 2 * SIZE[case["dtype"]] * x + fixed, "flops": 3 * x}
    x = B * L * (case["Hq"] + case["Hk"]) * D
    one, other = SIZE[case["dtype"]], SIZE[case["out"]]
    if kind == "norm_rope":
        return {"bytes": (one + other) * x + fixed + 4 * D, "flops": 7 * x}
    return {"bytes": (2 * one + other) * x + fixed + 12 * D, "flops": 16 * x}


# --- the definitions in 64 bits -------------------------------------------------------------------
def _factors(case, seed, sign):
    """exp(i sign angle) of each token and pair, 1 for what is not rotated, complex128 [L, 1, D / 2]."""
    pos = _positions(case, seed).double()
    f = [torch.tensor(v, device=DEV) for v in _frequencies(case)]
    angle = torch.cat([pos[:, a:a + 1] * f[a] for a in range(len(f))], dim=1)
    angle = torch.nn.functional.pad(angle, (0, case["D"] // 2 - angle.shape[1]))
    return torch.polar(torch.ones_like(angle), sign * angle)[:, None]


def _exact_turn(case, seed, x, sign):
    """Pairs as complex numbers, in the order of the head's elements."""
    n, D = sum(_axes(case)), case["D"]
    order = torch.arange(D, device=x.device)
    if case["halves"]:
        order[:n] = order[:n].view(2, n // 2).t().reshape(-1)
    z = torch.view_as_complex(x[..., order].reshape(x.shape[:-1] + (D // 2, 2))) * _factors(case, seed, sign)
    return torch.view_as_real(z).flatten(-2)[..., torch.argsort(order)]


def _exact_norm(case, seed, x, w):
    return _exact_turn(case, seed, w * x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS), 1.0)


def exact(case, seed):
    kind = case["kind"]
    if kind == "rope":
        return _exact_turn(case, seed, _single(case, seed).double(), -1.0 if case["inverse"] else 1.0)
    if kind.startswith("norm"):
        heads, weights = _heads(case, seed), _norm_weights(case, seed)
        if kind == "norm_rope":
            return tuple(_exact_norm(case, seed, x.double(), w.double()) for x, w in zip(heads, weights))
        out = []
        for x, w, dy in zip(heads, weights, _norm_grads(case, seed)):
            x, w = x.double().requires_grad_(), w.double().requires_grad_()
            _exact_norm(case, seed, x, w).backward(dy.double())
            out += [x.grad, w.grad]
        return tuple(out)
    starts, adapter, ranks, scales = _rows(case, seed)
    x, (a, b) = _tokens(case["M"], case["K"], seed), _pools(case, seed)
    y = _base(case, seed).double()
    train = kind == "lora_train"
    if train:
        dy = _out_grad(case, seed)
        dx = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
        da, db = (torch.zeros(p.shape, dtype=torch.float64, device=DEV) for p in (a, b))
    for first, end, i in zip(starts, starts[1:] + [case["M"]], adapter):
        if i < 0 or first == end:
            continue
        r, xs = ranks[i], x[first:end].double()
        ai, bi = a[i, :r].double(), b[i, :, :r].double()
        h = xs @ ai.t()
        y[first:end] += scales[i] * (h @ bi.t())
        if train:
            gs = dy[first:end].double() * scales[i]
            g = gs @ bi
            dx[first:end] = g @ ai
            da[i, :r] += g.t() @ xs
            db[i, :, :r] += gs.t() @ h
    return (y, dx, da, db) if train else y
