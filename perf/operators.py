"""The operators of a language model's 4-bit layers, as measurable cases.

norm    residual addition and RMS norm whose rows leave as 8-bit codes with a scale each (``dsq_rms_norm``):
        what a serving program runs before a layer that takes 8-bit rows.
train   the same norm in a training step: forward to floats, then ``dsq_rms_norm_bwd`` with gradients of both outputs.
w4      float rows times 4-bit weights with a scale and a zero point per group of input channels
        (``dsq_linear_w4``): one token, a few, a prompt.
w4a8    8-bit rows times the same weights (``dsq_linear_w4a8``).

Weights are packed once in ``prepare``, as a program does when it loads its model.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6

# Largest drawn cases: elements of a norm, weights of a product, multiply-accumulates of a product.
MAX_NORM = 8192 * 4096
MAX_WEIGHTS = 8192 * 32768
MAX_MACS = 2048 * 4096 * 8192


def listed():
    return [
        # One token through the norm of a middle-sized model: the smallest call, latency.
        dict(name="norm.token.4096", kind="norm", rows=1, dim=4096, dtype="bf16"),
        # A prompt, or the tokens of many requests.
        dict(name="norm.prompt.4096", kind="norm", rows=2048, dim=4096, dtype="bf16"),
        # A training step's norm over a micro-batch.
        dict(name="train.4096", kind="train", rows=8192, dim=4096, dtype="bf16"),
        # Rows of an odd, small width in full precision, many of them.
        dict(name="train.odd.f32", kind="train", rows=20000, dim=251, dtype="f32"),
        # One token through a square projection: 8 MB of weights, launch and latency.
        dict(name="w4.token.4096-4096", kind="w4", M=1, K=4096, N=4096, group=128, bias=False, dtype="bf16"),
        # One token through the largest layer: the weights come from memory.
        dict(name="w4.token.8192-32768", kind="w4", M=1, K=8192, N=32768, group=128, bias=False, dtype="bf16"),
        # The fully connected head of VGG-16 with a few requests in flight.
        dict(name="w4.head.25088-4096", kind="w4", M=4, K=25088, N=4096, group=64, bias=True, dtype="f16"),
        # Ragged sizes, small groups, full-precision activations.
        dict(name="w4.odd.4100-1000.f32", kind="w4", M=3, K=4100, N=1000, group=32, bias=True, dtype="f32"),
        # A short prompt with float activations.
        dict(name="w4.prompt.4096-4096", kind="w4", M=256, K=4096, N=4096, group=128, bias=False, dtype="bf16"),
        # A decoding batch on 8-bit rows.
        dict(name="w4a8.batch.4096-12288", kind="w4a8", M=16, K=4096, N=12288, group=128, bias=False, dtype="bf16"),
        # Ragged sizes and small groups.
        dict(name="w4a8.odd.5000-1000", kind="w4a8", M=333, K=5000, N=1000, group=32, bias=True, dtype="f16"),
        # A prompt on 8-bit rows: the matrix units' case.
        dict(name="w4a8.prompt.4096-8192", kind="w4a8", M=2048, K=4096, N=8192, group=128, bias=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "train", "w4", "w4", "w4", "w4a8", "w4a8"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("norm", "train"):
        dim = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        most = MAX_NORM // (2 if dtype == "f32" else 1)
        return dict(kind=kind, rows=_log(rng, 1, max(2, min(16384, most // dim))), dim=dim, dtype=dtype)
    while True:
        K, N = _log(rng, 256, 25088), _log(rng, 64, 32768)
        if rng.random() < 0.6:
            K, N = max(256, K // 128 * 128), max(64, N // 64 * 64)
        M = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 16, 2048)])
        if K * N <= MAX_WEIGHTS and M * K * N <= MAX_MACS // (1 if kind == "w4a8" else 2 if dtype != "f32" else 16):
            return dict(kind=kind, M=M, K=K, N=N, group=rng.choice([32, 64, 128, 128]), bias=rng.random() < 0.5,
                        dtype=dtype)


# ---- inputs --------------------------------------------------------------------------------------

def _inputs(case, seed):
    """The tensors of a case, from its seed: activations with a few large channels, as a model's have, and weights
    whose codes gather in the middle of their range."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    dt = DTYPES[case["dtype"]]
    if case["kind"] in ("norm", "train"):
        rows, dim = case["rows"], case["dim"]
        large = 1.0 + 8.0 * (torch.rand(dim, generator=g, device="cuda") < 0.01)
        d = {"x": normal(rows, dim).to(dt), "residual": (normal(rows, dim) * large * 2.0).to(dt),
             "weight": (1.0 + 0.2 * normal(dim)).to(dt)}
        if case["kind"] == "train":
            d["grad_y"] = normal(rows, dim).to(dt)
            d["grad_sum"] = normal(rows, dim).to(dt)
        return d
    M, K, N, G = case["M"], case["K"], case["N"], -(-case["K"] // case["group"])
    d = {"codes": torch.randint(0, 16, (N, K), generator=g, device="cuda", dtype=torch.uint8),
         "scale": 0.003 * torch.exp(0.3 * normal(N, G)).half().float(),
         "zero": torch.randint(6, 11, (N, G), generator=g, device="cuda", dtype=torch.uint8)}
    if case["bias"]:
        d["bias"] = normal(N).to(dt)
    if case["kind"] == "w4":
        d["x"] = normal(M, K).to(dt)
    else:
        d["q"] = (normal(M, K) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
        d["q_scale"] = 0.02 * torch.exp(0.3 * normal(M))
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = {"case": case, "in": d}
    if own:
        from paper_1908_05033_amd import binding as B
        dt, u8 = DTYPES[case["dtype"]], dict(dtype=torch.uint8, device="cuda")
        state["B"] = B
        if case["kind"] in ("norm", "train"):
            rows, dim = case["rows"], case["dim"]
            state["sum"] = torch.empty(rows, dim, dtype=dt, device="cuda")
            if case["kind"] == "norm":
                state["q"] = torch.empty(rows, B.dsq_code_row_bytes(dim), dtype=torch.int8, device="cuda")
                state["q_scale"] = torch.empty(rows, device="cuda")
                state["q_row"], state["q_step"] = state["q"][:, :dim], state["q_scale"][:, None]
            else:
                state["y"], state["grad_x"] = torch.empty_like(state["sum"]), torch.empty_like(state["sum"])
                state["rstd"] = torch.empty(rows, device="cuda")
                state["grad_weight"] = torch.empty(dim, device="cuda")
                state["workspace"] = torch.empty(B.dsq_rms_norm_bwd_bytes(rows, dim), **u8)
        else:
            M, K, N, group = case["M"], case["K"], case["N"], case["group"]
            state["w"] = torch.empty(B.dsq_w4_packed_bytes(N, K), **u8)
            state["s"] = torch.empty(B.dsq_w4_scale_bytes(N, K, group), **u8)
            B.dsq_pack_weights_w4(None, d["codes"], d["scale"], d["zero"], N, K, group, state["w"], state["s"])
            state["out"] = torch.empty(M, N, dtype=dt, device="cuda")
            if case["kind"] == "w4a8":       # rows as dsq_rms_norm writes them
                state["q"] = torch.zeros(M, B.dsq_code_row_bytes(K), dtype=torch.int8, device="cuda")
                state["q"][:, :K] = d["q"]
    return state


# ---- one pass ------------------------------------------------------------------------------------

def _own(state):
    case, d, B = state["case"], state["in"], state["B"]
    if case["kind"] == "norm":
        B.dsq_rms_norm(d["x"], d["residual"], d["weight"], EPS, state["sum"], None, state["q"], state["q_scale"], None)
        return {"sum": state["sum"], "values": state["q_row"] * state["q_step"]}
    if case["kind"] == "train":
        B.dsq_rms_norm(d["x"], d["residual"], d["weight"], EPS, state["sum"], state["y"], None, None, state["rstd"])
        B.dsq_rms_norm_bwd(state["sum"], d["weight"], state["rstd"], d["grad_y"], d["grad_sum"], state["grad_x"],
                           state["grad_weight"], state["workspace"])
        return {k: state[k] for k in ("sum", "y", "grad_x", "grad_weight")}
    if case["kind"] == "w4":
        B.dsq_linear_w4(d["x"], state["w"], state["s"], case["N"], case["K"], case["group"], d.get("bias"), state["out"])
    else:
        B.dsq_linear_w4a8(state["q"], d["q_scale"], state["w"], state["s"], case["N"], case["K"], case["group"],
                          d.get("bias"), state["out"])
    return {"out": state["out"]}


def run(state):
    if own:
        return _own(state)
    case, d = state["case"], state["in"]
    dt = DTYPES[case["dtype"]]
    if case["kind"] in ("norm", "train"):
        h = (d["x"].float() + d["residual"].float()).to(dt)
        hf, w = h.float(), d["weight"].float()
        r = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
        if case["kind"] == "norm":
            # (a code is a rounding: which side of a half a value is on is decided in 64 bits)
            p = h.double() * w.double()
            amax = p.abs().amax(1, keepdim=True)
            code = torch.round(127.0 * p / amax.clamp_min(1e-300))
            return {"sum": h, "values": code.float() * (amax.float() * r / 127.0)}
        y = (hf * r * w).to(dt)
        gy = d["grad_y"].float()
        n = hf * r
        t = gy * w
        gx = r * (t - n * (t * n).mean(1, keepdim=True)) + d["grad_sum"].float()
        return {"sum": h, "y": y, "grad_x": gx.to(dt), "grad_weight": (gy * n).sum(0)}
    of_k = torch.arange(case["K"], device="cuda") // case["group"]
    w = (d["codes"].float() - d["zero"].float()[:, of_k]) * d["scale"][:, of_k]
    x = d["x"].float() if case["kind"] == "w4" else d["q"].float()
    out = x @ w.t()
    if case["kind"] == "w4a8":
        out = out * d["q_scale"][:, None]
    if case["bias"]:
        out = out + d["bias"].float()
    return {"out": out.to(dt)}


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("norm", "train"):
        n, rows, dim = case["rows"] * case["dim"], case["rows"], case["dim"]
        if case["kind"] == "norm":
            # x, residual, weight; the sum, 8-bit codes, scales
            return {"bytes": n * (3 * e + 1) + dim * e + 4 * rows, "flops": 8 * n}
        # forward: x, residual, sum, y, 1/rms; backward: sum, both gradients, grad_x; the weight and its gradient
        return {"bytes": n * 8 * e + dim * (2 * e + 4) + 8 * rows, "flops": 18 * n}
    M, K, N, G = case["M"], case["K"], case["N"], -(-case["K"] // case["group"])
    rows = M * K * e if case["kind"] == "w4" else M * (K + 4)
    return {"bytes": N * K // 2 + 4 * N * G + rows + M * N * e + (N * e if case["bias"] else 0), "flops": 2 * M * N * K}


# ---- the definition in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    d = {k: v.double() if v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    dt = DTYPES[case["dtype"]]
    if case["kind"] in ("norm", "train"):
        # (the sum is an output of its own and held in its type; what follows reads that)
        h = (d["x"] + d["residual"]).to(dt).double()
        rms = torch.sqrt(torch.sum(h ** 2, dim=1) / case["dim"] + EPS)[:, None]
        if case["kind"] == "norm":
            v = h * d["weight"]
            step = torch.max(torch.abs(v), dim=1).values[:, None] / 127
            return {"sum": h, "values": torch.round(v / step) * (step / rms)}
        unit = h / rms
        t = d["grad_y"] * d["weight"]
        along = torch.sum(t * unit, dim=1, keepdim=True) / case["dim"]
        return {"sum": h, "y": unit * d["weight"], "grad_x": (t - unit * along) / rms + d["grad_sum"],
                "grad_weight": torch.sum(d["grad_y"] * unit, dim=0)}
    rows = d["x"] if case["kind"] == "w4" else d["q"].double() * d["q_scale"][:, None]
    out = torch.zeros(case["M"], case["N"], dtype=torch.float64, device="cuda")
    for c in range(0, case["N"], 4096):
        # (whole groups of channels at a time: the weights in 64 bits take eight bytes each)
        level = d["codes"][c:c + 4096].double() - torch.repeat_interleave(d["zero"][c:c + 4096].double(), case["group"], 1)[:, :case["K"]]
        level *= torch.repeat_interleave(d["scale"][c:c + 4096], case["group"], 1)[:, :case["K"]]
        out[:, c:c + 4096] = torch.matmul(rows, level.t())
    if case["bias"]:
        out += d["bias"]
    return {"out": out}
