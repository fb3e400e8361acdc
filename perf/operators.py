"""The 16-bit projection with its epilogue and linear attention with a decay per head, as cases with their inputs, one
pass each in a plain form and through the library, and what a pass cannot do without.

    linear    out = act(x W^T + bias) + residual
    prefill   S_t = exp(min(g_t, 0)) S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t  over a prompt, S carried in fp32
    step      the same for one token of every sequence

Sizes are the ones the repository is configured, tested and benchmarked at: widths 768 / 1536 (130M layer), 2560 / 5120
(2.8B layer, 64 sequences in generation, 2048-token and 4 x 4096-token prompts), 4096 / 8192 (Jamba-shaped layer, 16384
tokens), cut into heads of 64 or 128 columns, and odd ones.  `listed` fixes twelve points, `draw` gives others of the
same ranges.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh", "sigmoid"]
CHUNK = 128  # tokens per block of the plain form
BEHIND = 1.0  # what output rows behind a sequence's end hold before (and after) the call
MAX_LINEAR, MAX_PREFILL, MAX_STEP = 1.1e12, 7e10, 1.7e8  # a drawn case stays at or below the largest listed ones


def listed():
    return [
        # smallest call: one token through a projection of the small layer; launch latency
        {"name": "linear_1x768x1536", "op": "linear", "M": 1, "K": 768, "N": 1536, "type": "f16", "out": "f16",
         "act": "silu", "bias": True, "residual": False, "pad": 0},
        # generation, one sequence, input projection of the 2.8B layer: reading the weight
        {"name": "linear_1x2560x10240", "op": "linear", "M": 1, "K": 2560, "N": 10240, "type": "bf16", "out": "bf16",
         "act": "silu", "bias": True, "residual": False, "pad": 0},
        # generation, serving batch, output projection onto the residual stream
        {"name": "linear_64x5120x2560", "op": "linear", "M": 64, "K": 5120, "N": 2560, "type": "bf16", "out": "bf16",
         "act": "none", "bias": False, "residual": True, "pad": 0},
        # the headline prompt through the input projection
        {"name": "linear_2048x2560x10240", "op": "linear", "M": 2048, "K": 2560, "N": 10240, "type": "bf16",
         "out": "bf16", "act": "silu", "bias": True, "residual": False, "pad": 0},
        # long context through the widest layer's output projection
        {"name": "linear_16384x8192x4096", "op": "linear", "M": 16384, "K": 8192, "N": 4096, "type": "f16",
         "out": "f16", "act": "none", "bias": False, "residual": True, "pad": 0},
        # odd sizes, rows of a wider tensor, fp32 out: a gate's projection over a few prompts
        {"name": "linear_2103x1283x835", "op": "linear", "M": 2103, "K": 1283, "N": 835, "type": "f16", "out": "f32",
         "act": "gelu", "bias": True, "residual": True, "pad": 3},
        # a short prompt, few small heads, fixed decay per head
        {"name": "prefill_1x256_12x64x64", "op": "prefill", "batch": 1, "length": 256, "key_heads": 12, "heads": 12,
         "dk": 64, "dv": 64, "type": "f16", "decay": "head", "ragged": False},
        # the headline prompt: 80 value heads that share one key head, decay by token
        {"name": "prefill_1x2048_80x128x64", "op": "prefill", "batch": 1, "length": 2048, "key_heads": 1, "heads": 80,
         "dk": 128, "dv": 64, "type": "bf16", "decay": "token", "ragged": False},
        # several prompts of unequal length, odd heads, one of them empty
        {"name": "prefill_7x701_10x96x80", "op": "prefill", "batch": 7, "length": 701, "key_heads": 2, "heads": 10,
         "dk": 96, "dv": 80, "type": "f16", "decay": "token", "ragged": True},
        # long context, wide heads
        {"name": "prefill_1x16384_64x128x128", "op": "prefill", "batch": 1, "length": 16384, "key_heads": 64,
         "heads": 64, "dk": 128, "dv": 128, "type": "bf16", "decay": "token", "ragged": False},
        # generation, one sequence: launch latency
        {"name": "step_1_12x64x64", "op": "step", "batch": 1, "key_heads": 12, "heads": 12, "dk": 64, "dv": 64,
         "type": "f16", "decay": "head"},
        # generation, serving batch: reading and writing the states
        {"name": "step_64_80x128x64", "op": "step", "batch": 64, "key_heads": 1, "heads": 80, "dk": 128, "dv": 64,
         "type": "bf16", "decay": "token"},
    ]


def _log_int(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(["linear", "prefill", "step"], weights=[5, 5, 2])[0]
    while True:
        c = {"op": op, "type": rng.choice(["f16", "bf16"])}
        if op == "linear":
            c["M"], c["K"], c["N"] = _log_int(rng, 1, 16384), _log_int(rng, 64, 8192), _log_int(rng, 64, 16384)
            if rng.random() < 0.7:  # widths of layers are mostly multiples of 64
                c["K"], c["N"] = max(64, c["K"] // 64 * 64), max(64, c["N"] // 64 * 64)
            c["out"] = rng.choice([c["type"], c["type"], "f32"])
            c["act"], c["bias"], c["residual"] = rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.5
            c["pad"] = rng.choice([0, 0, 8, 5])
        else:
            c["dk"], c["dv"] = rng.choice([64, 128, 128, rng.randint(16, 256)]), rng.choice([64, 128, rng.randint(16, 256)])
            c["key_heads"] = _log_int(rng, 1, 32)
            c["heads"] = c["key_heads"] * _log_int(rng, 1, max(1, 64 // c["key_heads"]))
            c["decay"] = rng.choice(["token", "token", "head", "none"])
            c["batch"] = _log_int(rng, 1, 256 if op == "step" else 16)
            if op == "prefill":
                c["length"] = _log_int(rng, 16, max(16, 16384 // c["batch"]))
                c["ragged"] = c["batch"] > 1 and rng.random() < 0.4
        w = work(c)
        if w["flops"] <= {"linear": MAX_LINEAR, "prefill": MAX_PREFILL, "step": MAX_STEP}[op]:
            return c


def _lens(case):
    """Lengths of a ragged batch: the longest fills the tensor, the last is empty."""
    B, L = case["batch"], case["length"]
    rng = random.Random(B * 100003 + L)
    return [L] + [rng.randint(1, L) for _ in range(B - 2)] + [0]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPE[case["type"]]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=DEV) * std

    s = dict(case)
    if case["op"] == "linear":
        M, K, N, pad = case["M"], case["K"], case["N"], case["pad"]
        out = DTYPE[case["out"]]
        s["x"] = normal(M, K + pad).to(dt)[:, :K]
        s["W"] = normal(N, K, std=K ** -0.5).to(dt)
        s["bias_v"] = normal(N) if case["bias"] else None
        s["res"] = normal(M, N + pad).to(out)[:, :N] if case["residual"] else None
        s["y"] = torch.empty((M, N), dtype=out, device=DEV)
        return s
    B, L, Hk, H, dk, dv = case["batch"], case.get("length", 1), case["key_heads"], case["heads"], case["dk"], case["dv"]
    # q | k | v as one projection leaves them: columns of one row per token
    s["qkv"] = normal(B * L, 2 * Hk * dk + H * dv).to(dt)
    if case["decay"] == "token":  # time step, log-uniform in [1e-3, 1e-1], times a rate per head from 1 to 16
        step = torch.exp(torch.rand((B * L, H), generator=g, device=DEV) * math.log(100.0) + math.log(1e-3))
        s["g"] = -step * (1 + 15 * torch.rand(H, generator=g, device=DEV))
    elif case["decay"] == "head":  # memories of 32 to 4096 tokens
        s["g"] = torch.log1p(-torch.exp2(-5 - 7 * torch.rand(H, generator=g, device=DEV)))
    else:
        s["g"] = None
    s["scale"] = dk ** -0.5
    s["state"] = normal(B, H, dk, dv, std=3.0)
    s["y"] = torch.full((B * L, H * dv), BEHIND, dtype=dt, device=DEV)
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV) if case.get("ragged") else None
    return s


def _activate(v, act):
    if act == "relu":
        return torch.clamp(v, min=0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-v))
    return v


def _plain_linear(s):
    v = s["x"].float() @ s["W"].float().t()
    if s["bias_v"] is not None:
        v = v + s["bias_v"]
    v = _activate(v, s["act"])
    if s["res"] is not None:
        v = v + s["res"].float()
    return v.to(s["y"].dtype)


def _plain_attention(s):
    """Blocks of tokens: products inside a block, the blocks' states joined by one product with their decays."""
    B, L, Hk, H, dk, dv = s["batch"], s.get("length", 1), s["key_heads"], s["heads"], s["dk"], s["dv"]
    C = min(CHUNK, L)
    n = -(-L // C)
    x = s["qkv"].view(B, L, -1).float()
    q, k, v = x.split([Hk * dk, Hk * dk, H * dv], dim=2)
    g = torch.zeros((B, L, H), dtype=torch.float64, device=DEV) if s["g"] is None else s["g"].double().expand(B * L, H).reshape(B, L, H)
    g = torch.clamp(g, min=-1e4, max=0)
    if s["lens"] is not None:  # tokens behind the end change nothing
        on = torch.arange(L, device=DEV)[None, :] < s["lens"][:, None]
        k = torch.where(on[:, :, None], k, torch.zeros_like(k))
        g = torch.where(on[:, :, None], g, torch.zeros_like(g))

    def blocks(t, heads, width):  # [B, L, heads * width] -> [B, H, n, C, width], keys shared by H / Hk value heads
        t = torch.cat([t, t.new_zeros((B, n * C - L, heads * width))], 1)
        t = t.view(B, n, C, heads, width).permute(0, 3, 1, 2, 4)
        return t if heads == H else t.repeat_interleave(H // heads, dim=1)

    q, k, v, g = blocks(q, Hk, dk), blocks(k, Hk, dk), blocks(v, H, dv), blocks(g, H, 1)[..., 0]
    G = torch.cumsum(g, 3)  # within the block, 64 bits
    D = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill_(~torch.ones((C, C), dtype=torch.bool, device=DEV).tril(), -math.inf))
    inside = torch.matmul(torch.matmul(q, k.transpose(3, 4)) * D.float(), v)
    kw = k * torch.exp(G[..., -1:] - G).float()[..., None]
    U = torch.matmul(kw.transpose(3, 4), v)  # what each block adds to the state
    U = torch.cat([s["state"][:, :, None], U], 2).view(B, H, n + 1, dk * dv)
    T = torch.cat([torch.zeros((B, H, 1), dtype=G.dtype, device=DEV), torch.cumsum(G[..., -1], 2)], 2)
    J = (T[..., :, None] - T[..., None, :]).masked_fill_(~torch.ones((n + 1, n + 1), dtype=torch.bool, device=DEV).tril(), -math.inf)
    S = torch.matmul(torch.exp(J).float(), U).view(B, H, n + 1, dk, dv)
    o = s["scale"] * (inside + torch.exp(G).float()[..., None] * torch.matmul(q, S[:, :, :n]))
    o = o.permute(0, 2, 3, 1, 4).reshape(B, n * C, H * dv)[:, :L].to(s["y"].dtype)
    y = s["y"].view(B, L, H * dv)
    y.copy_(o if s["lens"] is None else torch.where(on[:, :, None], o, y))
    s["state"].copy_(S[:, :, n])
    return {"out": s["y"], "state": s["state"]}


def run(s):
    if not own:
        return {"out": _plain_linear(s)} if s["op"] == "linear" else _plain_attention(s)
    import paper_2410_13229_amd as Q

    kind = {"f16": Q.TYPE_F16, "bf16": Q.TYPE_BF16, "f32": Q.TYPE_F32}
    st = torch.cuda.current_stream().cuda_stream
    if s["op"] == "linear":
        M, N, K = s["M"], s["N"], s["K"]
        if "ws" not in s:  # kept from call to call, as the buffers are
            s["ws"] = torch.empty(max(256, Q.quamba_linear_workspace_bytes(M, N, K)), dtype=torch.uint8, device=DEV)
            s["a"] = getattr(Q, "ACT_" + s["act"].upper())
        res = s["res"]
        Q.quamba_linear(kind[s["type"]], s["x"], s["x"].stride(0), s["W"], K, s["bias_v"], res,
                        0 if res is None else res.stride(0), M, N, K, s["a"], kind[s["out"]], s["y"], N, s["ws"], st)
        return {"out": s["y"]}
    B, Hk, H, dk, dv, x, g = s["batch"], s["key_heads"], s["heads"], s["dk"], s["dv"], s["qkv"], s["g"]
    ld, esz, at = x.stride(0), x.element_size(), x.data_ptr()
    q, k, v = at, at + Hk * dk * esz, at + 2 * Hk * dk * esz
    ldg = 0 if g is None or g.dim() == 1 else H
    if s["op"] == "step":
        Q.quamba_linattn_step(kind[s["type"]], q, ld, k, ld, v, ld, g, ldg, B, Hk, H, dk, dv, s["scale"], s["y"], H * dv,
                              s["state"], st)
    else:
        L = s["length"]
        if "ws" not in s:
            s["ws"] = torch.empty(max(256, Q.quamba_linattn_workspace_bytes(B, L, Hk, H, dk, dv)), dtype=torch.uint8, device=DEV)
        Q.quamba_linattn_prefill(kind[s["type"]], q, ld, k, ld, v, ld, g, ldg, s["lens"], B, L, Hk, H, dk, dv, s["scale"],
                                 s["y"], H * dv, s["state"], s["ws"], st)
    return {"out": s["y"], "state": s["state"]}


def work(case):
    """linear: operands, bias, residual and output once, 2 M N K operations.  Attention: q, k, v, decays and outputs of the
    tokens that count, the states read and written; per token and head the update and the product with the state."""
    esz = {"f16": 2, "bf16": 2, "f32": 4}
    if case["op"] == "linear":
        M, K, N, o = case["M"], case["K"], case["N"], esz[case["out"]]
        return {"bytes": 2 * (M * K + N * K) + (4 * N if case["bias"] else 0) + M * N * o * (2 if case["residual"] else 1),
                "flops": 2.0 * M * N * K}
    B, L, Hk, H, dk, dv = case["batch"], case.get("length", 1), case["key_heads"], case["heads"], case["dk"], case["dv"]
    T = sum(_lens(case)) if case.get("ragged") else B * L
    decays = {"token": 4 * T * H, "head": 4 * H, "none": 0}[case["decay"]]
    return {"bytes": 2 * T * (2 * Hk * dk + 2 * H * dv) + decays + 8 * B * H * dk * dv, "flops": 4.0 * T * H * dk * dv}


def exact(case, seed):
    """The definitions in 64 bits: one product, and the recurrence token by token."""
    s = prepare(case, seed)
    if case["op"] == "linear":
        v = torch.addmm(torch.zeros((), dtype=torch.float64, device=DEV) if s["bias_v"] is None else s["bias_v"].double(),
                        s["x"].double(), s["W"].double().t())
        v = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t), "gelu": lambda t: t * torch.special.ndtr(t),
             "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh"), "sigmoid": torch.sigmoid}[case["act"]](v)
        return {"out": v if s["res"] is None else v + s["res"].double()}
    B, L, Hk, H, dk, dv = case["batch"], case.get("length", 1), case["key_heads"], case["heads"], case["dk"], case["dv"]
    S = s["state"].double()
    rows = s["qkv"].view(B, L, -1)
    y = s["y"].double().view(B, L, H, dv)
    for t in range(L):
        row = rows[:, t].double()
        q = row[:, : Hk * dk].view(B, Hk, 1, dk).expand(B, Hk, H // Hk, dk).reshape(B, H, dk)
        k = row[:, Hk * dk: 2 * Hk * dk].view(B, Hk, 1, dk).expand(B, Hk, H // Hk, dk).reshape(B, H, dk)
        v = row[:, 2 * Hk * dk:].view(B, H, dv)
        new = k[..., :, None] * v[..., None, :]
        if s["g"] is None:
            new += S
        else:
            a = torch.exp(torch.minimum(s["g"].double().expand(B * L, H).reshape(B, L, H)[:, t], torch.zeros((), dtype=torch.float64, device=DEV)))
            new += a[..., None, None] * S
        o = case["dk"] ** -0.5 * (q[..., :, None] * new).sum(2)
        if s["lens"] is None:
            S, y[:, t] = new, o
        else:
            on = (t < s["lens"])[:, None, None]
            S, y[:, t] = torch.where(on[..., None], new, S), torch.where(on, o, y[:, t])
    return {"out": y.view(B * L, H * dv), "state": S}
