"""The calls by which the layer operators around the mixer are judged: RMS norm with the residual's
addition, and the matrix product with bias, activation and residual in its epilogue.

A layer around the mixer is  h = x + block(norm(x));  y = h + W2 act(W1 norm(h) + b1) + b2, and its
calls are, with T tokens:

    op "norm"         h = x + residual;  y = h / sqrt(mean(h^2) + eps) * w          (rows of K channels)
       "norm_bwd"     dx and dw of that y from the stored h; dh is the gradient that reaches h directly
       "linear"       y = act(x w^T + bias) + residual                              (K -> N channels)
       "linear_bwd"   dx, dw and the bias's db from the stored pre-activation p
       "norm_linear"  "norm" to 8 bits (e4m3, one scale a token) and "linear" on those 8 bits and
                      8-bit weights (one scale an output channel): the layer's first half in serving

Where `own` is false, ``run`` computes them from elementary operations in 32 bits, rounded once.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3_MAX = 448.0


def _case(name, op, T, K, N=0, dtype="bf16", act="none", residual=False):
    return {"name": name, "op": op, "T": T, "K": K, "N": N, "dtype": dtype, "act": act, "residual": residual}


def listed():
    return [
        # one token of a recurrent or streaming user: launch and latency
        _case("norm_token_bf16", "norm", 1, 256, residual=True),
        # two 135 x 240 maps of 128 channels, before the feed-forward half of a layer
        _case("norm_fullimage_bf16", "norm", 64800, 128, residual=True),
        # a prompt of a wide model, its width odd (rows that start at any two-byte address)
        _case("norm_wide_odd_bf16", "norm", 2000, 5001, residual=True),
        # a batch of 4000-token sequences in training, float32, the first norm of a stack (no dh)
        _case("norm_bwd_longseq_f32", "norm_bwd", 32 * 4000, 64, dtype="f32"),
        # a training step's norm inside a residual stream (dh arrives beside dy)
        _case("norm_bwd_train_bf16", "norm_bwd", 16 * 8192, 256, residual=True),
        # one token through a feed-forward product: the weights are read once
        _case("linear_token_bf16", "linear", 1, 1024, 4096, act="silu"),
        # the layer's first half for 24 requests of one token each, 8-bit weights and activations
        _case("norm_linear_batch_e4m3", "norm_linear", 24, 4096, 8192, act="silu", residual=True),
        # the feed-forward's first product on the full image: 128 -> 512 channels
        _case("ffn_up_fullimage_bf16", "linear", 64800, 128, 512, act="gelu"),
        # a prompt of 8192 tokens through a wide layer: the matrix product itself
        _case("linear_large_bf16", "linear", 8192, 4096, 4096, act="silu", residual=True),
        # the same width in 8 bits, from the residual stream on, a ragged number of tokens
        _case("norm_linear_large_e4m3", "norm_linear", 8000, 4096, 4096, act="gelu", residual=True),
        # every size odd
        _case("linear_odd_bf16", "linear", 3001, 1003, 777, act="gelu", residual=True),
        # a training step's feed-forward product: [16, 8192, 256] -> 1024 channels
        _case("linear_bwd_train_bf16", "linear_bwd", 16 * 8192, 256, 1024, act="gelu"),
    ]


MAX_FLOPS, MAX_BYTES = 2.7e11, 6.6e8  # a drawn case costs no more than the largest listed ones


def _spread(rng, lo, hi):
    """A size spread over [lo, hi] by its logarithm; two in three are whole multiples of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, v - v % 8) if rng.random() < 2 / 3 and v >= 8 else v


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "linear", "linear_bwd", "norm_linear"])
    while True:
        T, K = _spread(rng, 1, 131072), _spread(rng, 64, 8192)
        N = 0 if op in ("norm", "norm_bwd") else _spread(rng, 64, 8192)
        dtype = rng.choice(["f32", "bf16"]) if op in ("norm", "norm_bwd") else "bf16"
        act = "none" if N == 0 else rng.choice(["none", "relu", "gelu", "silu"])
        case = {"op": op, "T": T, "K": K, "N": N, "dtype": dtype, "act": act,
                "residual": op != "linear_bwd" and rng.random() < 0.5}
        need = work(case)
        if need["flops"] <= MAX_FLOPS and need["bytes"] <= MAX_BYTES:
            return case


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    op, T, K, N = case["op"], case["T"], case["K"], case["N"]
    dt = TORCH_DTYPE[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    state = {"case": case}
    # activations: channels of unequal size, as in a trained network
    x = normal(T, K) * torch.exp(0.5 * normal(K))
    if op in ("norm", "norm_linear"):
        state["x"] = x.to(dt)
        state["residual"] = normal(T, K).to(dt) if case["residual"] else None
        state["gain"] = 1.0 + 0.1 * normal(K)
    if op == "norm_bwd":
        state["h"] = x.to(dt)
        state["gain"] = 1.0 + 0.1 * normal(K)
        state["dy"] = normal(T, K).to(dt)
        state["dh"] = normal(T, K).to(dt) if case["residual"] else None
    if op in ("linear", "linear_bwd"):
        state["x"] = normal(T, K).to(dt)
        state["w"] = (normal(N, K) / math.sqrt(K)).to(dt)
    if op == "linear":
        state["bias"] = 0.1 * normal(N)
        state["residual"] = normal(T, N).to(dt) if case["residual"] else None
    if op == "linear_bwd":
        state["dy"] = normal(T, N).to(dt)
        # the pre-activation that the forward stored
        state["p"] = normal(T, N).to(dt)
    if op == "norm_linear":
        # weights laid out in 8 bits once, when they are loaded
        w = normal(N, K) / math.sqrt(K)
        state["w_scale"] = w.abs().amax(1) / E4M3_MAX
        state["w"] = (w / state["w_scale"][:, None]).to(torch.float8_e4m3fn)
        state["bias"] = 0.1 * normal(N)
    return state


# ---- the plain forms, in 32 bits ----

GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(p, act):
    if act == "relu":
        return p.clamp_min(0.0)
    if act == "silu":
        return p / (1.0 + torch.exp(-p))
    if act == "gelu":
        return p / (1.0 + torch.exp(-2.0 * GELU_A * (p + GELU_B * p * p * p)))
    return p


def _act_slope(p, act):
    if act == "relu":
        return (p > 0).to(p.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-p))
        return s * (1.0 + p * (1.0 - s))
    if act == "gelu":
        s = 1.0 / (1.0 + torch.exp(-2.0 * GELU_A * (p + GELU_B * p * p * p)))
        return s * (1.0 + p * (1.0 - s) * 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * p * p))
    return torch.ones_like(p)


def _plain_norm(x, residual, gain):
    h = x.float() if residual is None else x.float() + residual.float()
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * gain


def _plain(s):
    case = s["case"]
    op, act = case["op"], case["act"]
    dt = TORCH_DTYPE[case["dtype"]]
    if op == "norm":
        h, y = _plain_norm(s["x"], s["residual"], s["gain"])
        return {"y": y.to(dt)} if s["residual"] is None else {"y": y.to(dt), "h": h.to(dt)}
    if op == "norm_bwd":
        h, dy = s["h"].float(), s["dy"].float()
        rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        n = h * rstd
        a = dy * s["gain"]
        dx = rstd * (a - n * (a * n).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(dt), "dw": (dy * n).sum(0)}
    if op == "linear":
        y = _act(torch.matmul(s["x"].float(), s["w"].float().t()) + s["bias"], act)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt)}
    if op == "linear_bwd":
        dp = s["dy"].float() * _act_slope(s["p"].float(), act)
        return {"dx": torch.matmul(dp, s["w"].float()).to(dt), "dw": torch.matmul(dp.t(), s["x"].float()).to(dt),
                "db": dp.sum(0)}
    # norm_linear
    h, y = _plain_norm(s["x"], s["residual"], s["gain"])
    scale = y.abs().amax(1, keepdim=True) / E4M3_MAX
    q = (y / scale).to(torch.float8_e4m3fn).float() * scale
    z = torch.matmul(q, (s["w"].float() * s["w_scale"][:, None]).t()) + s["bias"]
    out = {"y": _act(z, act).to(dt)}
    if s["residual"] is not None:
        out["h"] = h.to(dt)
    return out


# ---- the framework's calls ----

def _framework(s):
    from paper_2607_25234_gb300 import whtmix

    case = s["case"]
    op, act = case["op"], case["act"]
    if op == "norm":
        if s["residual"] is None:
            return {"y": whtmix.rms_norm(s["x"], s["gain"], eps=EPS)}
        y, h = whtmix.rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS)
        return {"y": y, "h": h}
    if op == "norm_bwd":
        dx, dw = whtmix.rms_norm_backward(s["h"], s["gain"], s["dy"], dh=s["dh"], eps=EPS)
        return {"dx": dx, "dw": dw}
    if op == "linear":
        return {"y": whtmix.linear(s["x"], s["w"], bias=s["bias"], activation=act, residual=s["residual"])}
    if op == "linear_bwd":
        dx, dw, db = whtmix.linear_backward(s["x"], s["w"], s["dy"], p=s["p"], activation=act)
        return {"dx": dx, "dw": dw, "db": db}
    # norm_linear
    got = whtmix.rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS, out_dtype=torch.float8_e4m3fn)
    y = whtmix.linear(got[0], s["w"], bias=s["bias"], activation=act, x_scale=got[1], w_scale=s["w_scale"])
    return {"y": y} if s["residual"] is None else {"y": y, "h": got[2]}


def run(state):
    return _framework(state) if own else _plain(state)


def work(case):
    op, T, K, N = case["op"], case["T"], case["K"], case["N"]
    e = 4 if case["dtype"] == "f32" else 2
    r = 1 if case["residual"] else 0
    if op == "norm":
        return {"bytes": T * K * e * (2 + 2 * r) + 4 * K, "flops": 5 * T * K}
    if op == "norm_bwd":
        return {"bytes": T * K * e * (3 + r) + 8 * K, "flops": 12 * T * K}
    if op == "linear":
        return {"bytes": (T * K + N * K + T * N * (1 + r)) * e + 4 * N, "flops": 2 * T * K * N}
    if op == "linear_bwd":
        p = 0 if case["act"] == "none" else 1
        return {"bytes": (2 * T * K + 2 * N * K + T * N * (1 + p)) * e + 4 * N, "flops": 4 * T * K * N}
    # norm_linear: the 8-bit activations stay between the two calls
    return {"bytes": T * K * e * (1 + 2 * r) + N * K + T * N * e + 4 * K + 8 * N, "flops": 2 * T * K * N + 5 * T * K}


# ---- the definitions in 64 bits ----

def _nearest_e4m3(v):
    """The e4m3 value nearest to each v (|v| <= 448), ties to even: steps of 2^(e-3), e >= -6."""
    _, e = torch.frexp(v.abs().clamp_min(2.0 ** -6))  # v = m 2^e with m in [1/2, 1)
    step = torch.ldexp(torch.ones_like(v), e - 4)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in prepare(case, seed).items()}
    op, act = case["op"], case["act"]
    sigmoid = torch.sigmoid

    def phi(z):  # the activation and its derivative
        if act == "none":
            return z, torch.ones_like(z)
        if act == "relu":
            return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
        u, du = (z, 1.0) if act == "silu" else (2 * GELU_A * (z + GELU_B * z ** 3), 2 * GELU_A * (1 + 3 * GELU_B * z ** 2))
        g = sigmoid(u)
        return z * g, g + z * g * sigmoid(-u) * du

    if op in ("norm", "norm_linear"):
        h = s["x"] if s["residual"] is None else s["x"] + s["residual"]
        y = s["gain"] * h * torch.rsqrt(h.square().sum(1, keepdim=True) / case["K"] + EPS)
        out = {}
        if s["residual"] is not None:
            out["h"] = h
        if op == "norm":
            return {**out, "y": y}
        top = y.abs().max(1, keepdim=True).values / E4M3_MAX
        z = (_nearest_e4m3(y / top) * top) @ (s["w"] * s["w_scale"].unsqueeze(1)).T + s["bias"]
        return {**out, "y": phi(z)[0]}
    if op == "norm_bwd":
        h, dy = s["h"], s["dy"]
        inv = torch.rsqrt(h.square().sum(1, keepdim=True) / case["K"] + EPS)
        a = dy * s["gain"]
        dx = a * inv - h * inv ** 3 * (a * h).sum(1, keepdim=True) / case["K"]
        return {"dx": dx if s["dh"] is None else dx + s["dh"], "dw": (dy * h * inv).sum(0)}
    if op == "linear":
        y = phi(s["x"] @ s["w"].T + s["bias"])[0]
        return {"y": y if s["residual"] is None else y + s["residual"]}
    dp = s["dy"] * phi(s["p"])[1]
    return {"dx": dp @ s["w"], "dw": dp.T @ s["x"], "db": dp.sum(0)}
