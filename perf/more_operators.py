"""The operators that serve a feed-forward sub-block, dense or as a mixture of experts, and that clip its
gradients: measured cases, plain forms and exact values.

Operators (T tokens, D channels, F hidden channels, E experts; matrices are row-major):
  qnorm   r' = scale r + gate * norm(y) * w_post;  x = norm(r') * w_pre, as 8-bit values (e4m3) and the scale of
          each 1 x 128 block: s = max|x| / 448, q = x / s
  int4    C[m,n] = sum_g scale[n,g] sum_{k in group g} (q[n,k] - zero[n,g]) X[m,k], q of 4 bits, zero 8 if absent
  moe     the k largest of x Wr^T choose experts e_j, with softmax weights p_j: y = sum_j p_j ffn_{e_j}(x)
  clip    norm over all elements of a list of gradients; each times min(1, max_norm / (norm + eps))

``run`` computes them with elementary torch operations in 32 bits (own = False) or through the
library's entry points (own = True).
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MOST_EXPERT_BYTES = 1 << 30  # of a layer's experts in a drawn case


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # one token of a served model, in front of an 8-bit projection: latency
        dict(name="qnorm_one_token", op="qnorm", T=1, D=4096, type="bf16", gate="all", rows=0, post=True),
        # a ragged batch of a small model, fp16
        dict(name="qnorm_ragged", op="qnorm", T=777, D=1000, type="fp16", gate="none", rows=0, post=False),
        # a long prompt, a gate for each sequence of 2048 tokens
        dict(name="qnorm_prompt", op="qnorm", T=16384, D=4096, type="bf16", gate="groups", rows=2048, post=True),
        # one token against 4-bit weights: the weights are read once, nothing else counts
        dict(name="int4_one_token", op="int4", M=1, N=8192, K=4096, group=128, type="bf16", scale="bf16", zero=False),
        # the square projection of a smaller model, small groups with zero points: latency
        dict(name="int4_small", op="int4", M=4, N=2048, K=2048, group=32, type="fp16", scale="fp16", zero=True),
        # a batch of answers, ragged in every direction
        dict(name="int4_batch", op="int4", M=23, N=5000, K=4200, group=64, type="bf16", scale="bf16", zero=True),
        # a prompt
        dict(name="int4_prompt", op="int4", M=2048, N=8192, K=4096, group=128, type="bf16", scale="bf16", zero=False),
        # one token through a mixture of 64 experts, 8 of them chosen
        dict(name="moe_one_token", op="moe", T=1, D=2048, F=1024, E=64, k=8, type="bf16", act="silu", normalize=True),
        # a ragged handful of tokens, few experts
        dict(name="moe_ragged", op="moe", T=5, D=1000, F=1304, E=10, k=3, type="fp16", act="gelu", normalize=False),
        # a batch of answers that between them choose nearly every expert
        dict(name="moe_batch", op="moe", T=32, D=2048, F=2048, E=32, k=4, type="bf16", act="silu", normalize=True),
        # the gradients of a small model, 40 tensors, clipped
        dict(name="clip_small", op="clip", layers=8, D=256, F=700, type="mixed", clipped=True),
        # the gradients of a large one in 16 bits, clipped
        dict(name="clip_model", op="clip", layers=12, D=2048, F=8192, type="bf16", clipped=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng, lo, hi):
    """Mostly multiples of 64, as layers have; some of 8; some of nothing."""
    n, u = _log_int(rng, lo, hi), rng.random()
    step = 64 if u < 0.6 else 8 if u < 0.85 else 1
    return max(step, min(hi, (n + step // 2) // step * step))


def draw(rng):
    op = rng.choice(["qnorm", "int4", "int4", "moe", "moe", "clip"])
    if op == "qnorm":
        D = _channels(rng, 64, 8192)
        T = _log_int(rng, 1, min(16384, 16384 * 4096 // D))
        gate = rng.choice(["none", "all", "groups", "tokens"])
        rows = {"none": 0, "all": 0, "groups": rng.randint(1, T), "tokens": 1}[gate]
        return dict(op=op, T=T, D=D, type=rng.choice(["bf16", "bf16", "fp16"]), gate=gate, rows=rows, post=rng.random() < 0.7)
    if op == "int4":
        ty = rng.choice(["bf16", "bf16", "fp16"])
        return dict(op=op, M=_log_int(rng, 1, 2048), N=_channels(rng, 64, 8192), K=_channels(rng, 64, 4096),
                    group=rng.choice([32, 64, 128, 128]), type=ty, scale=rng.choice([ty, ty, "fp32"]), zero=rng.random() < 0.5)
    if op == "moe":
        D, F, E = _channels(rng, 64, 4096), _channels(rng, 64, 4096), _log_int(rng, 4, 128)
        while 6 * E * D * F > MOST_EXPERT_BYTES // 2:
            E = max(4, E // 2)
            F = max(64, F // 128 * 64)
        return dict(op=op, T=_log_int(rng, 1, 64), D=D, F=F, E=E, k=rng.randint(1, min(8, E)),
                    type=rng.choice(["bf16", "bf16", "fp16"]), act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]),
                    normalize=rng.random() < 0.5)
    D, F = _channels(rng, 64, 2048), _channels(rng, 64, 8192)
    most = max(1, min(60, 12 * 2048 * 8192 // (D * F) // 2))
    return dict(op=op, layers=_log_int(rng, 1, most), D=D, F=F, type=rng.choice(["bf16", "fp16", "fp32", "mixed"]),
                clipped=rng.random() < 0.7)


# ---- inputs -------------------------------------------------------------------------------------

def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)


def _stream_values(gen, T, D, dtype):
    """Activations of a residual stream: unit variance, with one channel in 64 twenty times as large."""
    v = torch.randn((T, D), generator=gen, device="cuda")
    loud = torch.rand((D,), generator=gen, device="cuda") < 1 / 64
    return (v * torch.where(loud, 20.0, 1.0)).to(dtype)


def _cdiv(a, b):
    return -(-a // b)


def _gradient_shapes(case):
    """(shape, type) of every gradient: three matrices and two vectors a layer, as a sub-block has."""
    D, F, ty = case["D"], case["F"], case["type"]
    wide, narrow = ("bf16", "fp32") if ty == "mixed" else (ty, ty)
    return [((F, D), wide), ((F, D), wide), ((D, F), wide), ((D,), narrow), ((D,), narrow)] * case["layers"]


def _views(flat, shapes):
    """The gradients as they lie in their type's buffer, one behind the other."""
    at, out = dict.fromkeys(flat, 0), []
    for shape, ty in shapes:
        n = math.prod(shape)
        out.append(flat[ty][at[ty]:at[ty] + n].view(shape))
        at[ty] += n
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    op = case["op"]
    s = dict(case=dict(case))
    dtype = TYPES.get(case["type"])
    new = lambda *shape, t=dtype: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    if op == "qnorm":
        T, D = case["T"], case["D"]
        s["rows"] = case["rows"] if case["gate"] in ("groups", "tokens") else T
        s["scale"] = 1.0 if D % 3 else 0.875
        s["w_pre"] = (1.0 + 0.1 * torch.randn((D,), generator=gen, device="cuda")).to(dtype)
        s["w_post"] = (1.0 + 0.1 * torch.randn((D,), generator=gen, device="cuda")).to(dtype) if case["post"] else None
        s["gate"] = _normal(gen, (_cdiv(T, s["rows"]), D), dtype, 0.5) if case["gate"] != "none" else None
        s["block"] = _normal(gen, (T, D), dtype, 0.7)
        s["resid"] = _stream_values(gen, T, D, dtype)
        s["resid_out"], s["q"] = new(T, D), new(T, D, t=torch.float8_e4m3fn)
        s["q_scale"] = new(T, _cdiv(D, 128), t=torch.float32)
    elif op == "int4":
        M, N, K = case["M"], case["N"], case["K"]
        groups = _cdiv(K, case["group"])
        s["x"] = _normal(gen, (M, K), dtype)
        s["q"] = torch.randint(0, 256, (N, _cdiv(K, 2)), generator=gen, device="cuda", dtype=torch.uint8)
        s["scale"] = (torch.exp(0.3 * torch.randn((N, groups), generator=gen, device="cuda")) * (0.2 * K ** -0.5)).to(TYPES[case["scale"]])
        s["zero"] = None
        if case["zero"]:
            s["zero"] = (8 + 1.5 * torch.randn((N, groups), generator=gen, device="cuda")).round().clamp_(0, 15).to(torch.uint8)
        s["out"] = new(M, N)
    elif op == "moe":
        T, D, F, E = case["T"], case["D"], case["F"], case["E"]
        s["x"] = _normal(gen, (T, D), dtype)
        s["w_router"] = _normal(gen, (E, D), dtype, D ** -0.5)
        s["w_gate"] = _normal(gen, (E, F, D), dtype, D ** -0.5)
        s["w_up"] = _normal(gen, (E, F, D), dtype, D ** -0.5)
        s["w_down"] = _normal(gen, (E, D, F), dtype, F ** -0.5)
        s["out"] = new(T, D)
        s["ids"], s["weights"] = new(T, case["k"], t=torch.int32), new(T, case["k"], t=torch.float32)
    else:
        shapes = _gradient_shapes(case)
        total = {}
        for shape, ty in shapes:
            total[ty] = total.get(ty, 0) + math.prod(shape)
        s["flat"] = {ty: _normal(gen, (n,), TYPES[ty], 0.01) for ty, n in total.items()}
        s["flat_out"] = {ty: torch.empty_like(v) for ty, v in s["flat"].items()}
        s["norm"] = new(1, t=torch.float32)
        # the norm is near 0.01 sqrt(elements)
        s["max_norm"] = 0.01 * sum(total.values()) ** 0.5 * (0.3 if case["clipped"] else 3.0)
        s["grads"], s["outs"] = _views(s["flat"], shapes), _views(s["flat_out"], shapes)
        if own:
            from paper_1802_06905_b200 import block
            s["grads"], s["outs"] = block.TensorList(s["grads"]), block.TensorList(s["outs"])
    return s


# ---- the operators ------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_1802_06905_b200 import block
    c = s["case"]
    op = c["op"]
    if op == "qnorm":
        block.residual_norm_quantize(s["resid"], s["resid_out"], s["q"], s["q_scale"], block=s["block"], w_post=s["w_post"],
                                     gate=s["gate"], w_pre=s["w_pre"], rows_per_gate=s["rows"], scale=s["scale"], eps=EPS)
        return [s["resid_out"], s["q"], s["q_scale"]]
    if op == "int4":
        return block.int4_product(s["x"], s["q"], s["scale"], s["out"], zero=s["zero"], group=c["group"])
    if op == "moe":
        block.moe_forward(s["x"], s["w_router"], s["w_gate"], s["w_up"], s["w_down"], s["out"], s["ids"], s["weights"],
                          act=block.ACTS[c["act"]], normalize=c["normalize"])
        return [s["out"], s["ids"], s["weights"]]
    block.clip_gradients(s["grads"], s["max_norm"], s["norm"], outs=s["outs"], eps=EPS)
    return {"norm": s["norm"], **s["flat_out"]}


def _act(name, g):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * (1 + torch.erf(g * 2 ** -0.5))
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh((2 / math.pi) ** 0.5 * (g + 0.044715 * g * g * g)))
    return g * (g > 0).to(g.dtype)


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    dtype = TYPES.get(c["type"])
    f = lambda name: None if s.get(name) is None else s[name].float()  # noqa: E731
    if op == "qnorm":
        T, D = c["T"], c["D"]
        n = f("block")
        if s["w_post"] is not None:
            n = n * torch.rsqrt((n * n).mean(1, keepdim=True) + EPS) * f("w_post")
        if s["gate"] is not None:
            n = f("gate")[torch.arange(T, device="cuda") // s["rows"]] * n
        r = s["scale"] * f("resid") + n
        x = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * f("w_pre")
        cb = _cdiv(D, 128)
        x = torch.nn.functional.pad(x, (0, cb * 128 - D)).reshape(T, cb, 128)
        scale = x.abs().amax(2, keepdim=True) / E4M3_MAX
        q = x / torch.where(scale == 0, torch.ones_like(scale), scale)
        return [r.to(dtype), q.reshape(T, cb * 128)[:, :D].contiguous().to(torch.float8_e4m3fn), scale.reshape(T, cb)]
    if op == "int4":
        N, K, g = c["N"], c["K"], c["group"]
        groups = _cdiv(K, g)
        w = torch.stack([s["q"] & 15, s["q"] >> 4], 2).reshape(N, -1)[:, :K].float()
        w = torch.nn.functional.pad(w, (0, groups * g - K)).reshape(N, groups, g)
        zero = f("zero")[:, :, None] if c["zero"] else 8.0
        w = ((w - zero) * f("scale")[:, :, None]).reshape(N, groups * g)[:, :K]
        return (f("x") @ w.T).to(dtype)
    if op == "moe":
        return _plain_moe(s, c)
    flat = {ty: v.float() for ty, v in s["flat"].items()}
    sums = torch.stack([v.square().sum(dtype=torch.float64) for v in flat.values()])
    norm = sums.sum().sqrt().float().reshape(1)
    factor = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    return {"norm": norm, **{ty: (v * factor).to(TYPES[ty]) for ty, v in flat.items()}}


def _plain_moe(s, c):
    T, E, k = c["T"], c["E"], c["k"]
    logits = s["x"].double() @ s["w_router"].double().T  # which experts are chosen hangs on close values
    ids = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k]
    chosen = logits.gather(1, ids)
    p = torch.exp(chosen - logits.amax(1, keepdim=True))
    p = p / (p if c["normalize"] else torch.exp(logits - logits.amax(1, keepdim=True))).sum(1, keepdim=True)
    p = p.float()
    x = s["x"].float()
    if T * k <= E:  # few pairs of token and expert: their matrices alone
        pick = lambda name: s[name][ids.reshape(-1)].float()  # noqa: E731
        xs = x.repeat_interleave(k, 0)[:, :, None]
        h = _act(c["act"], pick("w_gate") @ xs) * (pick("w_up") @ xs)
        y = ((pick("w_down") @ h).reshape(T, k, -1) * p[:, :, None]).sum(1)
    else:  # every token through every expert, and a weight of 0 for those that it has not chosen
        full = torch.zeros((T, E), device="cuda").scatter_(1, ids, p)
        mul = lambda v, name: v @ s[name].float().transpose(1, 2)  # noqa: E731
        h = _act(c["act"], mul(x[None], "w_gate")) * mul(x[None], "w_up")
        y = (mul(h, "w_down") * full.T[:, :, None]).sum(0)
    return [y.to(TYPES[c["type"]]), ids.to(torch.int32), p]


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    op = case["op"]
    e = 4 if case["type"] == "fp32" else 2
    if op == "qnorm":
        T, D = case["T"], case["D"]
        groups = 0 if case["gate"] == "none" else 1 if case["gate"] == "all" else _cdiv(T, case["rows"])
        weights = (1 + bool(case["post"]) + groups) * D
        return {"bytes": e * (3 * T * D + weights) + T * D + 4 * T * _cdiv(D, 128), "flops": 14 * T * D}
    if op == "int4":
        M, N, K = case["M"], case["N"], case["K"]
        a_group = (4 if case["scale"] == "fp32" else 2) + bool(case["zero"])
        return {"bytes": N * _cdiv(K, 2) + a_group * N * _cdiv(K, case["group"]) + e * M * (N + K), "flops": 2 * M * N * K}
    if op == "moe":
        T, D, F, E, k = case["T"], case["D"], case["F"], case["E"], case["k"]
        used = E * (1 - (1 - k / E) ** T)  # experts that T tokens choose between them, on average
        return {"bytes": int(e * (E * D + 2 * T * D + 3 * used * D * F) + 8 * T * k), "flops": 2 * T * E * D + 6 * T * k * D * F}
    count = {"bf16": 0, "fp32": 0}
    for shape, ty in _gradient_shapes(case):
        count["fp32" if ty == "fp32" else "bf16"] += math.prod(shape)
    return {"bytes": 4 * count["bf16"] + 8 * count["fp32"], "flops": 3 * (count["bf16"] + count["fp32"])}


# ---- the same values from the definitions, in 64 bits -------------------------------------------

def _exact_act(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * torch.special.ndtr(g)
    if name == "gelu_tanh":
        return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return torch.clamp(g, min=0)


def _e4m3_round(v):
    """The nearest e4m3 value (ties to even), of 64-bit values of at most 448 in size."""
    m, ex = torch.frexp(v)                                # v = m 2^ex, 0.5 <= |m| < 1
    step = torch.ldexp(torch.ones_like(v), torch.clamp(ex - 4, min=-9))  # 3 mantissa bits; subnormals below 2^-6
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    d = lambda name: None if s.get(name) is None else s[name].double()  # noqa: E731
    op = case["op"]
    if op == "qnorm":
        T, D = case["T"], case["D"]
        n = d("block")
        if case["post"]:
            n = n / torch.sqrt(torch.mean(n ** 2, dim=-1, keepdim=True) + EPS) * d("w_post")
        if s["gate"] is not None:
            n = torch.repeat_interleave(d("gate"), s["rows"], dim=0)[:T] * n
        r = s["scale"] * d("resid") + n
        x = r / torch.sqrt(torch.mean(r ** 2, dim=-1, keepdim=True) + EPS) * d("w_pre")
        at = (torch.arange(D, device="cuda") // 128)[None].expand(T, D)
        amax = torch.zeros(s["q_scale"].shape, dtype=torch.float64, device="cuda").scatter_reduce_(1, at, x.abs(), "amax")
        scale = amax / E4M3_MAX
        return [r, _e4m3_round(x / torch.where(scale == 0, 1.0, scale).gather(1, at)), scale]
    if op == "int4":
        k = torch.arange(case["K"], device="cuda")
        code = torch.bitwise_and(torch.bitwise_right_shift(s["q"][:, k // 2].int(), 4 * (k % 2)), 15).double()
        at = k // case["group"]
        w = (code - (d("zero")[:, at] if case["zero"] else 8.0)) * d("scale")[:, at]
        return torch.einsum("mk,nk->mn", d("x"), w)
    if op == "moe":
        T, k, E = case["T"], case["k"], case["E"]
        x = d("x")
        logits = torch.einsum("td,ed->te", x, d("w_router"))
        left, ids = logits.clone(), []
        for _ in range(k):
            best = left.argmax(1)
            ids.append(best)
            left[torch.arange(T, device="cuda"), best] = -math.inf
        ids = torch.stack(ids, 1)
        p = torch.softmax(logits, 1).gather(1, ids)
        if case["normalize"]:
            p = p / p.sum(1, keepdim=True)
        y = torch.zeros_like(x)
        for e in range(E):
            row, slot = (ids == e).nonzero(as_tuple=True)
            h = _exact_act(case["act"], x[row] @ s["w_gate"][e].double().T) * (x[row] @ s["w_up"][e].double().T)
            y.index_add_(0, row, (h @ s["w_down"][e].double().T) * p[row, slot, None])
        return [y, ids.to(torch.int32), p]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(v, dtype=torch.float64) for v in s["flat"].values()]))
    factor = min(1.0, s["max_norm"] / (norm.item() + EPS))
    return {"norm": norm.reshape(1), **{ty: v.double() * factor for ty, v in s["flat"].items()}}
