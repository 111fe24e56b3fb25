"""The operators of a pruned feed-forward block, as cases that can be timed and compared.

  op "linear"  a pruned linear layer on token-major activations, y = act(x W^T + b) + r, W in CSR (density 1 - sparsity);
               gated: y = act(x Wg^T + bg) * (x Wu^T + bu) + r, the rows of Wg before those of Wu in one CSR of 2M rows
  op "norm"    the residual stream between two blocks, h = alpha x + beta gate * post(y), n = pre(h)
  op "block"   n = pre(x), g = gated(n), d = g Wd^T, then h and the next block's n as above

The plan of a linear layer is built and uploaded once, as a program that serves a model does; a pass is the calls on
activations that are already on the GPU.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _linear(name, T, K, M, type, sparsity, act="none", bias=False, residual=False, gated=False):
    return dict(name=name, op="linear", T=T, K=K, M=M, type=type, sparsity=sparsity, act=act, bias=bias, residual=residual, gated=gated)


def _norm(name, T, D, type, post="rms", pre="rms", gate="vector", bias=False, y=True):
    return dict(name=name, op="norm", T=T, D=D, type=type, post=post, pre=pre, gate=gate, bias=bias, y=y)


def listed():
    return [
        # the smallest product: one token through a small head, where the launch is most of it
        _linear("token_small", 1, 512, 768, "bf16", 0.80, act="relu", bias=True),
        # one token of a single user through the wide half of a feed-forward block: bound by the weights' bytes
        _linear("token_gated", 1, 4096, 12288, "bf16", 0.50, act="silu", gated=True),
        # a serving batch through the narrow half, the residual stream added
        _linear("batch_down", 16, 12288, 4096, "bf16", 0.70, residual=True),
        # a ragged batch of drafted tokens through a projection, other type
        _linear("batch_fp16", 53, 2560, 2560, "f16", 0.60, bias=True, residual=True),
        # fp32 with odd sizes everywhere: rows that start at any word
        _linear("odd_fp32", 333, 1001, 1503, "f32", 0.80, act="gelu", bias=True),
        # one chunk of a prompt, fp16
        _linear("chunk_gated", 250, 2560, 6912, "f16", 0.65, act="gelu_tanh", gated=True),
        # a long prompt through both halves: bound by the matrix cores
        _linear("prompt_gated", 4096, 4096, 12288, "bf16", 0.50, act="silu", gated=True),
        _linear("prompt_down", 2000, 12288, 4096, "bf16", 0.50, residual=True),
        # one token's residual stream between two blocks
        _norm("norm_token", 1, 4096, "bf16"),
        # the same for a long prompt
        _norm("norm_prompt", 8192, 4096, "bf16"),
        # layer norms with odd rows in fp32, every token with a gate of its own
        _norm("norm_odd", 1023, 5003, "f32", post="layer", pre="layer", gate="token", bias=True),
        # a whole feed-forward block for a serving batch
        dict(name="block_batch", op="block", T=32, D=2048, F=5632, type="bf16", sparsity=0.60),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to thousands, any widths (odd ones among them), all types, sparsities that
    pruning leaves, every epilogue."""
    type = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["linear", "linear", "linear", "norm", "norm", "block"])
    while True:
        T = _log_int(rng, 1, 8192)
        if op == "norm":
            kinds = rng.choice([("rms", "rms"), ("none", "rms"), ("layer", "layer"), ("none", "layer"), ("rms", "none")])
            case = _norm("", T, _log_int(rng, 64, 16384), type, kinds[0], kinds[1], rng.choice(["none", "vector", "token"]),
                         bias=rng.random() < 0.5, y=kinds[0] != "none" or rng.random() < 0.7)
            size = {"f32": 4}.get(type, 2)
            fits = case["T"] * case["D"] * size <= 8192 * 4096 * 2
        elif op == "linear":
            step = rng.choice([1, 8, 64])
            K, M = (max(step, _log_int(rng, 128, 12288) // step * step) for _ in range(2))
            case = _linear("", T, K, M, type, round(rng.uniform(0.5, 0.95), 3), rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                           bias=rng.random() < 0.5, residual=rng.random() < 0.5, gated=rng.random() < 0.4)
            rows = M * (2 if case["gated"] else 1)
            fits = T * K * rows <= 4096 * 4096 * 24576 / (16 if type == "f32" else 1) and K * rows <= 4096 * 24576
        else:
            case = dict(name="", op="block", T=T, D=_log_int(rng, 128, 4096), F=_log_int(rng, 256, 12288), type=type,
                        sparsity=round(rng.uniform(0.5, 0.95), 3))
            fits = T * case["D"] * case["F"] * 3 <= 4096 * 4096 * 24576 / (16 if type == "f32" else 1)
        if fits:
            del case["name"]
            return case


# ---- inputs -------------------------------------------------------------------------------------------------------------

ALPHA, BETA, EPS = 1.0, 0.5, 1e-5


def _weight(gen, rows, K, sparsity, dtype):
    """A pruned weight matrix: every weight kept with probability 1 - sparsity, rows that keep a signal's size."""
    w = torch.randn((rows, K), device="cuda", generator=gen).mul_(1.0 / math.sqrt(max(1.0, K * (1.0 - sparsity))))
    w *= torch.rand((rows, K), device="cuda", generator=gen) >= sparsity
    return w.to(dtype)


def _randn(gen, shape, dtype, scale=1.0, shift=0.0):
    return torch.randn(shape, device="cuda", generator=gen).mul_(scale).add_(shift).to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, T = TYPES[case["type"]], case["T"]
    s = {}
    if case["op"] == "linear":
        K, M = case["K"], case["M"]
        rows = 2 * M if case["gated"] else M
        s["x"] = _randn(gen, (T, K), dt)
        s["w"] = _weight(gen, rows, K, case["sparsity"], dt)
        s["bias"] = _randn(gen, (rows,), dt, 0.1) if case["bias"] else None
        s["residual"] = _randn(gen, (T, M), dt) if case["residual"] else None
    elif case["op"] == "norm":
        D = case["D"]
        s["x"] = _randn(gen, (T, D), dt, 2.0, 0.1)
        s["y"] = _randn(gen, (T, D), dt, 1.5, -0.2) if case["y"] else None
        gate = {"none": None, "vector": (D,), "token": (T, D)}[case["gate"]] if case["y"] else None
        s["gate"] = _randn(gen, gate, dt, 0.2, 0.8) if gate else None
        for which in ("post", "pre"):
            used = case[which] != "none" and (which == "pre" or case["y"])
            s[which + "_weight"] = _randn(gen, (D,), dt, 0.1, 1.0) if used else None
            s[which + "_bias"] = _randn(gen, (D,), dt, 0.1) if used and case["bias"] else None
    else:
        D, F = case["D"], case["F"]
        s["x"] = _randn(gen, (T, D), dt, 2.0)
        s["w_up"] = _weight(gen, 2 * F, D, case["sparsity"], dt)
        s["w_down"] = _weight(gen, D, F, case["sparsity"], dt)
        for k in ("pre_weight", "post_weight", "next_weight"):
            s[k] = _randn(gen, (D,), dt, 0.1, 1.0)
        s["gate"] = _randn(gen, (D,), dt, 0.2, 0.8)
    return s


def _csr(w):
    """The CSR of a pruned matrix on the host, as it comes out of a checkpoint."""
    rows = w.shape[0]
    kept = w != 0
    rowptr = np.zeros(rows + 1, dtype=np.int32)
    rowptr[1:] = torch.cumsum(kept.sum(1), 0).to(torch.int32).cpu().numpy()
    colidx = torch.arange(w.shape[1], dtype=torch.int32, device=w.device).expand(w.shape)[kept].cpu().numpy()
    return rowptr, colidx, w[kept].float().cpu().numpy()


def _plan(w, T, M, type, gated):
    import paper_1802_10280_amd as esc

    desc = esc.make_linear_desc(T, w.shape[1], M, {"f32": esc.T_F32, "f16": esc.T_F16, "bf16": esc.T_BF16}[type], gated)
    rowptr, colidx, value = _csr(w)
    plan = esc.escoin_linear_plan_build(desc, rowptr, colidx, value)
    return dict(desc=desc, plan=plan, d_plan=torch.from_numpy(plan).cuda())


def _norm_desc(T, D, type, post, pre, gate="vector"):
    import paper_1802_10280_amd as esc

    kinds = {"none": esc.NORM_NONE, "rms": esc.NORM_RMS, "layer": esc.NORM_LAYER}
    return esc.make_norm_desc(T, D, {"f32": esc.T_F32, "f16": esc.T_F16, "bf16": esc.T_BF16}[type], kinds[post], kinds[pre],
                              gate_rows=int(gate == "token"), eps=EPS, alpha=ALPHA, beta=BETA)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    import paper_1802_10280_amd as esc

    new = lambda *shape: torch.empty(shape, dtype=TYPES[case["type"]], device="cuda")
    T = case["T"]
    if case["op"] == "linear":
        flags = {"none": 0, "relu": esc.F_RELU, "silu": esc.F_SILU, "gelu": esc.F_GELU, "gelu_tanh": esc.F_GELU_TANH}[case["act"]]
        s["flags"] = flags | (esc.F_BIAS if case["bias"] else 0) | (esc.F_RESIDUAL if case["residual"] else 0)
        s["layer"] = _plan(s.pop("w"), T, case["M"], case["type"], case["gated"])
        s["out"] = new(T, case["M"])
    elif case["op"] == "norm":
        s["desc"] = _norm_desc(T, case["D"], case["type"], case["post"] if case["y"] else "none", case["pre"], case["gate"])
        s["h"] = new(T, case["D"]) if case["y"] else None
        s["n"] = new(T, case["D"]) if case["pre"] != "none" else None
    else:
        D, F = case["D"], case["F"]
        s["up"] = _plan(s.pop("w_up"), T, F, case["type"], True)
        s["down"] = _plan(s.pop("w_down"), T, D, case["type"], False)
        s["first"] = _norm_desc(T, D, case["type"], "none", "rms")
        s["last"] = _norm_desc(T, D, case["type"], "rms", "rms")
        s["out"] = [new(T, D), new(T, F), new(T, D), new(T, D), new(T, D)]
    return s


# ---- the framework's calls ----------------------------------------------------------------------------------------------


def _forward(layer, x, out, bias, residual, flags):
    import paper_1802_10280_amd as esc

    esc.escoin_linear_forward(layer["desc"], layer["plan"], layer["d_plan"], x, out, bias, residual, flags)


def _run_own(s):
    import paper_1802_10280_amd as esc

    case = s["case"]
    if case["op"] == "linear":
        _forward(s["layer"], s["x"], s["out"], s["bias"], s["residual"], s["flags"])
        return s["out"]
    if case["op"] == "norm":
        esc.escoin_norm_forward(s["desc"], s["x"], s["h"], s["n"], d_y=s["y"], d_gate=s["gate"], d_post_weight=s["post_weight"],
                                d_post_bias=s["post_bias"], d_pre_weight=s["pre_weight"], d_pre_bias=s["pre_bias"])
        return [t for t in (s["h"], s["n"]) if t is not None]
    n, g, d, h, n2 = s["out"]
    esc.escoin_norm_forward(s["first"], s["x"], None, n, d_pre_weight=s["pre_weight"])
    _forward(s["up"], n, g, None, None, esc.F_SILU)
    _forward(s["down"], g, d, None, None, 0)
    esc.escoin_norm_forward(s["last"], s["x"], h, n2, d_y=d, d_gate=s["gate"], d_post_weight=s["post_weight"], d_pre_weight=s["next_weight"])
    return [h, n2]


# ---- the plain form: elementary torch operations in 32 bits, rounded once an operator -------------------------------------


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain_linear(x, w, bias, residual, act, gated):
    z = x.float() @ w.float().t()
    if bias is not None:
        z = z + bias.float()
    if gated:
        half = z.shape[1] // 2
        z = _act(z[:, :half], act) * z[:, half:]
    else:
        z = _act(z, act)
    if residual is not None:
        z = z + residual.float()
    return z.to(x.dtype)


def _plain_kind(v, kind, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    if weight is not None:
        v = v * weight.float()
    return v if bias is None else v + bias.float()


def _plain_norm(x, y, gate, post, post_weight, post_bias, pre, pre_weight, pre_bias):
    h = ALPHA * x.float()
    if y is not None:
        b = _plain_kind(y.float(), post, post_weight, post_bias)
        h = h + BETA * (b if gate is None else gate.float() * b)
    n = _plain_kind(h, pre, pre_weight, pre_bias)
    return h.to(x.dtype), n.to(x.dtype)


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    if case["op"] == "linear":
        return _plain_linear(s["x"], s["w"], s["bias"], s["residual"], case["act"], case["gated"])
    if case["op"] == "norm":
        h, n = _plain_norm(s["x"], s["y"], s["gate"], case["post"], s["post_weight"], s["post_bias"], case["pre"], s["pre_weight"], s["pre_bias"])
        return ([h] if case["y"] else []) + ([n] if case["pre"] != "none" else [])
    n = _plain_norm(s["x"], None, None, "none", None, None, "rms", s["pre_weight"], None)[1]
    g = _plain_linear(n, s["w_up"], None, None, "silu", True)
    d = _plain_linear(g, s["w_down"], None, None, "none", False)
    return list(_plain_norm(s["x"], d, s["gate"], "rms", s["post_weight"], None, "rms", s["next_weight"], None))


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------


def _double(t):
    return None if t is None else t.double()


def _exact_product(x, w, bias):
    """The product by blocks of rows, so that no 64-bit copy of all weights is needed."""
    step = max(1, (1 << 25) // w.shape[1])
    z = torch.cat([torch.matmul(w[r:r + step].double(), x.t()) for r in range(0, w.shape[0], step)]).t()
    return z if bias is None else z + bias


def _exact_gate(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return z * torch.special.expit(z * (1.0 + 0.044715 * z.square()) * math.sqrt(8.0 / math.pi))
    return z


def _exact_linear(x, w, bias, residual, act, gated):
    z = _exact_product(x, w, bias)
    out = _exact_gate(z[:, :z.shape[1] // 2], act) * z[:, z.shape[1] // 2:] if gated else _exact_gate(z, act)
    return out if residual is None else out.add(residual)


def _exact_kind(v, kind, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        spread, centre = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
        v = (v - centre) * (spread + EPS).rsqrt()
    else:
        v = v * (torch.linalg.vector_norm(v, dim=1, keepdim=True).square() / v.shape[1] + EPS).rsqrt()
    if weight is not None:
        v = weight * v
    return v if bias is None else v + bias


def _exact_norm(x, y, gate, post, post_weight, post_bias, pre, pre_weight, pre_bias):
    h = x * ALPHA
    if y is not None:
        b = _exact_kind(y, post, post_weight, post_bias) * BETA
        h = h + (b if gate is None else b * gate)
    return h, _exact_kind(h, pre, pre_weight, pre_bias)


def exact(case, seed):
    s = {k: v if k.startswith("w") else _double(v) for k, v in _inputs(case, seed).items()}
    if case["op"] == "linear":
        return _exact_linear(s["x"], s["w"], s["bias"], s["residual"], case["act"], case["gated"])
    if case["op"] == "norm":
        h, n = _exact_norm(s["x"], s["y"], s["gate"], case["post"], s["post_weight"], s["post_bias"], case["pre"], s["pre_weight"], s["pre_bias"])
        return ([h] if case["y"] else []) + ([n] if case["pre"] != "none" else [])
    n = _exact_norm(s["x"], None, None, "none", None, None, "rms", s["pre_weight"], None)[1]
    g = _exact_linear(n, s["w_up"], None, None, "silu", True)
    d = _exact_linear(g, s["w_down"], None, None, "none", False)
    return list(_exact_norm(s["x"], d, s["gate"], "rms", s["post_weight"], None, "rms", s["next_weight"], None))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------


def _product_work(T, K, rows, out, size, sparsity):
    """The kept weights with a bit a place for where they stand, input and output once; a multiply and an add per kept weight
    and token."""
    kept = K * rows * (1.0 - sparsity)
    return kept * size + K * rows / 8.0 + (T * K + T * out) * size, 2.0 * T * kept


def _norm_work(T, D, size, reads, writes, vectors, flops):
    return (T * D * (reads + writes) + D * vectors) * size, float(T * D * flops)


def work(case):
    size, T = {"f32": 4}.get(case["type"], 2), case["T"]
    if case["op"] == "linear":
        rows = case["M"] * (2 if case["gated"] else 1)
        b, f = _product_work(T, case["K"], rows, case["M"], size, case["sparsity"])
        b += (rows if case["bias"] else 0) * size + (T * case["M"] if case["residual"] else 0) * size
    elif case["op"] == "norm":
        normed = (case["post"] != "none" and case["y"]) + (case["pre"] != "none")
        per_token = case["y"] and case["gate"] == "token"
        vector = case["y"] and case["gate"] == "vector"
        b, f = _norm_work(T, case["D"], size, 1 + case["y"] + per_token, case["y"] + (case["pre"] != "none"),
                          normed * (2 if case["bias"] else 1) + vector, 4 * normed + 3 * case["y"] + 1)
    else:
        D, F = case["D"], case["F"]
        parts = [_norm_work(T, D, size, 1, 0, 1, 4), _product_work(T, D, 2 * F, 0, size, case["sparsity"]),
                 _product_work(0, F, D, 0, size, case["sparsity"]), _norm_work(T, D, size, 0, 2, 3, 11)]
        b = sum(p[0] for p in parts) - T * D * size
        f = sum(p[1] for p in parts) + 2.0 * T * F * D * (1.0 - case["sparsity"])
    return {"bytes": float(b), "flops": float(f)}
