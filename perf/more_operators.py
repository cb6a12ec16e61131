"""Calls of a training step's other operators around the mixer: layer norm, the gated feed-forward half,
and the clipping of a step's gradients by their common norm.

With T tokens, K channels in and N hidden channels:

    op "norm"        h = x + residual;  y = (h - mean(h)) / sqrt(var(h) + eps) * w + b      (rows of K channels)
       "norm_bwd"    dx, dw, db of that y from the stored h; dh is the gradient that reaches h directly
       "gated"       g = x wg^T + bg;  u = x wu^T + bu;  y = act(g) u;  w = [wg; wu] is [2 N, K]; in training
                     p = [g, u] is stored beside y
       "gated_bwd"   dx, dw and the bias's db from the stored p
       "norm_gated"  "norm" to 8 bits (e4m3, one scale a token) and "gated" on those 8 bits and 8-bit weights (one
                     scale an output channel): the first half of a feed-forward block in serving
       "clip"        norm = sqrt(sum of all squares of a list of tensors);  each tensor times min(1, max_norm / (norm + 1e-6))

Where `own` is false, ``run`` computes them from elementary operations in 32 bits (the sum of a step's squares in 64),
rounded once.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
CLIP_EPS = 1e-6
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
E4M3_MAX = 448.0


def _case(name, op, T, K, N=0, dtype="bf16", act="none", residual=False, preact=False):
    return {"name": name, "op": op, "T": T, "K": K, "N": N, "dtype": dtype, "act": act, "residual": residual, "preact": preact}


def _layer_tensors(tokens, channels, hidden):
    """One layer's gradients, as text: the mixer's weights and gains, two norms, the gated half and the product behind it."""
    return (f"bf16:{channels * channels} f32:{tokens * channels} bf16:{channels * channels} f32:{channels} f32:{channels} f32:{channels} "
            f"f32:{channels} bf16:{2 * hidden * channels} f32:{2 * hidden} bf16:{hidden * channels} f32:{channels}")


def listed():
    return [
        # one token of a recurrent or streaming user: launch and latency
        _case("norm_token_bf16", "norm", 1, 256, residual=True),
        # two 135 x 240 maps of 128 channels, before the feed-forward half of a layer
        _case("norm_fullimage_bf16", "norm", 64800, 128, residual=True),
        # a training step's norm inside a residual stream (dh arrives beside dy)
        _case("norm_bwd_train_bf16", "norm_bwd", 16 * 8192, 256, residual=True),
        # 4000-token sequences of an odd width in float32, the first norm of a stack (no dh)
        _case("norm_bwd_odd_f32", "norm_bwd", 16 * 4000, 77, dtype="f32"),
        # one token through the gated half: the weights are read once
        _case("gated_token_bf16", "gated", 1, 1024, 2736, act="silu"),
        # norm and gated half for 24 requests of one token each, 8-bit weights and activations
        _case("norm_gated_batch_e4m3", "norm_gated", 24, 4096, 8192, act="silu", residual=True),
        # the full image in training, both pre-activations stored: 128 -> 344 channels
        _case("gated_fullimage_train_bf16", "gated", 64800, 128, 344, act="gelu", preact=True),
        # a prompt of 8192 tokens through a wide layer: the matrix products themselves
        _case("gated_large_bf16", "gated", 8192, 4096, 8192, act="silu"),
        # a training step's gated half: [16, 8192, 256] -> 688 channels
        _case("gated_bwd_train_bf16", "gated_bwd", 16 * 8192, 256, 688, act="silu"),
        # every size odd
        _case("gated_bwd_odd_bf16", "gated_bwd", 3001, 1003, 777, act="gelu"),
        # the gradients of one small layer
        {"name": "clip_layer", "op": "clip", "tensors": _layer_tensors(256, 64, 176), "max_norm": 1.0},
        # those of five layers of 2048 channels over 4096 tokens: 0.6 GB in 55 tensors
        {"name": "clip_stack", "op": "clip", "tensors": " ".join([_layer_tensors(4096, 2048, 5464)] * 5), "max_norm": 1.0},
    ]


MAX_FLOPS, MAX_BYTES = 1.1e12, 1.1e9  # a drawn case costs no more than the largest listed ones


def _spread(rng, lo, hi):
    """A size spread over [lo, hi] by its logarithm; two in three are whole multiples of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, v - v % 8) if rng.random() < 2 / 3 and v >= 8 else v


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "gated", "gated_bwd", "norm_gated", "clip"])
    while True:
        if op == "clip":
            largest = _spread(rng, 64, 1 << 26)
            tensors = " ".join(f"{rng.choice(['f32', 'bf16'])}:{_spread(rng, 1, largest)}" for _ in range(_spread(rng, 1, 60)))
            case = {"op": op, "tensors": tensors, "max_norm": rng.choice([0.1, 1.0, 1e6])}
        else:
            T, K = _spread(rng, 1, 131072), _spread(rng, 64, 8192)
            N = 0 if op in ("norm", "norm_bwd") else _spread(rng, 64, 8192)
            dtype = rng.choice(["f32", "bf16"]) if N == 0 else "bf16"
            act = "none" if N == 0 else rng.choice(["none", "relu", "gelu", "silu"])
            case = {"op": op, "T": T, "K": K, "N": N, "dtype": dtype, "act": act,
                    "residual": op in ("norm", "norm_bwd", "norm_gated") and rng.random() < 0.5, "preact": op == "gated" and rng.random() < 0.5}
        need = work(case)
        if need["flops"] <= MAX_FLOPS and need["bytes"] <= MAX_BYTES:
            return case


def _tensors(case):
    return [(dtype, int(n)) for dtype, n in (t.split(":") for t in case["tensors"].split())]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    state = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if case["op"] == "clip":
        # gradients of unequal size from tensor to tensor, and the buffers that the clipped ones go to
        state["grads"] = [(normal(n) * 10.0 ** (-3 + 2 * (i % 7) / 6)).to(TORCH_DTYPE[t]) for i, (t, n) in enumerate(_tensors(case))]
        state["clipped"] = [torch.empty_like(g) for g in state["grads"]]
        return state
    op, T, K, N = case["op"], case["T"], case["K"], case["N"]
    dt = TORCH_DTYPE[case["dtype"]]
    if op in ("norm", "norm_bwd", "norm_gated"):
        # activations: channels of unequal size and mean, as in a trained network
        x = ((normal(T, K) + 0.5 * normal(K)) * torch.exp(0.5 * normal(K))).to(dt)
        state["gain"] = 1.0 + 0.1 * normal(K)
        if op == "norm_bwd":
            state["h"] = x
            state["dy"] = normal(T, K).to(dt)
            state["dh"] = normal(T, K).to(dt) if case["residual"] else None
        else:
            state["x"] = x
            state["shift"] = 0.1 * normal(K)
            state["residual"] = normal(T, K).to(dt) if case["residual"] else None
    if op in ("gated", "gated_bwd"):
        state["x"] = normal(T, K).to(dt)
        state["w"] = (normal(2 * N, K) / math.sqrt(K)).to(dt)
    if op == "gated":
        state["bias"] = 0.1 * normal(2 * N)
    if op == "gated_bwd":
        state["dy"] = normal(T, N).to(dt)
        # the pre-activations that the forward stored
        state["p"] = normal(T, 2 * N).to(dt)
    if op == "norm_gated":
        # weights laid out in 8 bits once, when they are loaded
        w = normal(2 * N, K) / math.sqrt(K)
        state["w_scale"] = w.abs().amax(1) / E4M3_MAX
        state["w"] = (w / state["w_scale"][:, None]).to(torch.float8_e4m3fn)
        state["bias"] = 0.1 * normal(2 * N)
    return state


# ---- the plain forms, in 32 bits ----

GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(p, act):
    """The activation and its slope."""
    if act == "relu":
        return p.clamp_min(0.0), (p > 0).to(p.dtype)
    if act == "none":
        return p, torch.ones_like(p)
    if act == "silu":
        s, du = 1.0 / (1.0 + torch.exp(-p)), 1.0
    else:
        s = 1.0 / (1.0 + torch.exp(-2.0 * GELU_A * (p + GELU_B * p * p * p)))
        du = 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * p * p)
    return p * s, s * (1.0 + p * (1.0 - s) * du)


def _plain_norm(x, residual, gain, shift):
    h = x.float() if residual is None else x.float() + residual.float()
    c = h - h.mean(1, keepdim=True)
    return h, c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * gain + shift


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "clip":
        norm = torch.sqrt(sum((g.double() * g.double()).sum() for g in s["grads"]))
        factor = torch.clamp_max(case["max_norm"] / (norm + CLIP_EPS), 1.0).float()
        return {"clipped": [(g.float() * factor).to(g.dtype) for g in s["grads"]], "norm": norm.float()}
    dt, N, act = TORCH_DTYPE[case["dtype"]], case["N"], case["act"]
    if op == "norm":
        h, y = _plain_norm(s["x"], s["residual"], s["gain"], s["shift"])
        return {"y": y.to(dt)} if s["residual"] is None else {"y": y.to(dt), "h": h.to(dt)}
    if op == "norm_bwd":
        h, dy = s["h"].float(), s["dy"].float()
        c = h - h.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
        n = c * rstd
        a = dy * s["gain"]
        dx = rstd * (a - a.mean(1, keepdim=True) - n * (a * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(dt), "dw": (dy * n).sum(0), "db": dy.sum(0)}
    if op == "gated":
        p = torch.matmul(s["x"].float(), s["w"].float().t()) + s["bias"]
        y = (_act(p[:, :N], act)[0] * p[:, N:]).to(dt)
        return {"y": y, "p": p.to(dt)} if case["preact"] else {"y": y}
    if op == "gated_bwd":
        dy, g, u = s["dy"].float(), s["p"][:, :N].float(), s["p"][:, N:].float()
        value, slope = _act(g, act)
        dp = torch.cat([dy * u * slope, dy * value], 1)
        return {"dx": torch.matmul(dp, s["w"].float()).to(dt), "dw": torch.matmul(dp.t(), s["x"].float()).to(dt), "db": dp.sum(0)}
    # norm_gated
    h, y = _plain_norm(s["x"], s["residual"], s["gain"], s["shift"])
    scale = y.abs().amax(1, keepdim=True) / E4M3_MAX
    q = (y / scale).to(torch.float8_e4m3fn).float() * scale
    p = torch.matmul(q, (s["w"].float() * s["w_scale"][:, None]).t()) + s["bias"]
    out = {"y": (_act(p[:, :N], act)[0] * p[:, N:]).to(dt)}
    if s["residual"] is not None:
        out["h"] = h.to(dt)
    return out


# ---- the framework's calls ----

def _framework(s):
    from paper_2607_25234_gb300 import whtmix

    case = s["case"]
    op = case["op"]
    if op == "clip":
        clipped, norm = whtmix.clip_by_global_norm(s["grads"], case["max_norm"], out=s["clipped"])
        return {"clipped": clipped, "norm": norm}
    act = case["act"]
    if op == "norm":
        if s["residual"] is None:
            return {"y": whtmix.layer_norm(s["x"], s["gain"], s["shift"], eps=EPS)}
        y, h = whtmix.layer_norm(s["x"], s["gain"], s["shift"], residual=s["residual"], eps=EPS)
        return {"y": y, "h": h}
    if op == "norm_bwd":
        dx, dw, db = whtmix.layer_norm_backward(s["h"], s["gain"], s["dy"], dh=s["dh"], eps=EPS)
        return {"dx": dx, "dw": dw, "db": db}
    if op == "gated":
        if not case["preact"]:
            return {"y": whtmix.gated_linear(s["x"], s["w"], s["bias"], act)}
        y, p = whtmix.gated_linear(s["x"], s["w"], s["bias"], act, preact=True)
        return {"y": y, "p": p}
    if op == "gated_bwd":
        dx, dw, db = whtmix.gated_linear_backward(s["x"], s["w"], s["dy"], s["p"], act)
        return {"dx": dx, "dw": dw, "db": db}
    normed = whtmix.layer_norm(s["x"], s["gain"], s["shift"], residual=s["residual"], eps=EPS, out_dtype=torch.float8_e4m3fn)
    q, scale = normed[:2]
    out = {"y": whtmix.gated_linear(q, s["w"], s["bias"], act, x_scale=scale, w_scale=s["w_scale"])}
    if s["residual"] is not None:
        out["h"] = normed[2]
    return out


def run(state):
    return _framework(state) if own else _plain(state)


def work(case):
    op = case["op"]
    if op == "clip":
        sizes = _tensors(case)
        return {"bytes": 2 * sum(BYTES[t] * n for t, n in sizes) + 4, "flops": 3 * sum(n for _, n in sizes)}
    T, K, N, e, r = case["T"], case["K"], case["N"], BYTES[case["dtype"]], 1 if case["residual"] else 0
    if op == "norm":
        return {"bytes": T * K * e * (2 + 2 * r) + 8 * K, "flops": 8 * T * K}
    if op == "norm_bwd":
        return {"bytes": T * K * e * (3 + r) + 12 * K, "flops": 16 * T * K}
    if op == "gated":
        return {"bytes": (T * K + 2 * N * K + T * N * (3 if case["preact"] else 1)) * e + 8 * N, "flops": 4 * T * K * N}
    if op == "gated_bwd":
        return {"bytes": (2 * T * K + 4 * N * K + 3 * T * N) * e + 8 * N, "flops": 8 * T * K * N}
    # norm_gated: the 8-bit activations stay between the two calls
    return {"bytes": T * K * e * (1 + 2 * r) + 2 * N * K + T * N * e + 8 * K + 16 * N, "flops": 4 * T * K * N + 8 * T * K}


# ---- the definitions in 64 bits ----

def _nearest_e4m3(v):
    """The e4m3 value nearest to each v (|v| <= 448), ties to even: steps of 2^(e-3), e >= -6."""
    _, e = torch.frexp(v.abs().clamp_min(2.0 ** -6))  # v = m 2^e with m in [1/2, 1)
    step = torch.ldexp(torch.ones_like(v), e - 4)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        squares = torch.stack([g.double().square().sum() for g in s["grads"]]).sum()
        norm = squares.sqrt()
        factor = min(1.0, case["max_norm"] / (float(norm) + CLIP_EPS))
        return {"clipped": [g.double() * factor for g in s["grads"]], "norm": norm}
    s = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    N, act = case["N"], case["act"]

    def phi(z):
        if act == "none":
            return z
        if act == "relu":
            return torch.where(z > 0, z, 0.0)
        return z * torch.sigmoid(z if act == "silu" else 2 * GELU_A * (z + GELU_B * z ** 3))

    def slope(z):
        if act in ("none", "relu"):
            return torch.where((z > 0) | (act == "none"), 1.0, 0.0).double()
        u, du = (z, 1.0) if act == "silu" else (2 * GELU_A * (z + GELU_B * z ** 3), 2 * GELU_A * (1 + 3 * GELU_B * z ** 2))
        return torch.sigmoid(u) * (1 + z * torch.sigmoid(-u) * du)

    if op in ("norm", "norm_gated"):
        h = s["x"] if s["residual"] is None else s["x"] + s["residual"]
        y = s["shift"] + s["gain"] * (h - h.mean(1, keepdim=True)) * torch.rsqrt(h.var(1, keepdim=True, unbiased=False) + EPS)
        out = {}
        if s["residual"] is not None:
            out["h"] = h
        if op == "norm":
            return {**out, "y": y}
        top = y.abs().max(1, keepdim=True).values / E4M3_MAX
        z = (_nearest_e4m3(y / top) * top) @ (s["w"] * s["w_scale"].unsqueeze(1)).T + s["bias"]
        return {**out, "y": phi(z[:, :N]) * z[:, N:]}
    if op == "norm_bwd":
        h, dy = s["h"], s["dy"]
        inv = torch.rsqrt(h.var(1, keepdim=True, unbiased=False) + EPS)
        n = (h - h.mean(1, keepdim=True)) * inv
        a = dy * s["gain"]
        dx = inv * (a - a.sum(1, keepdim=True) / case["K"] - n * (a * n).sum(1, keepdim=True) / case["K"])
        return {"dx": dx if s["dh"] is None else dx + s["dh"], "dw": (dy * n).sum(0), "db": dy.sum(0)}
    if op == "gated":
        p = s["x"] @ s["w"].T + s["bias"]
        y = phi(p[:, :N]) * p[:, N:]
        return {"y": y, "p": p} if case["preact"] else {"y": y}
    g, u = s["p"][:, :N], s["p"][:, N:]
    dp = torch.cat([s["dy"] * u * slope(g), s["dy"] * phi(g)], 1)
    return {"dx": dp @ s["w"], "dw": dp.T @ s["x"], "db": dp.sum(0)}
