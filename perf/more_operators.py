"""Cases of the projections in 8-bit integers: rows to 8-bit codes with a scale each, the RMS norm that adds the residual and
leaves such rows, and the product of two such matrices, each in a plain form (elementary torch operations) and, where `own` is
true, through the package's calls.

A row x of d values has A = max |x|, the scale A / 127 and the codes rint(127 x / A), ties to even, of the quotient as a real
number; the codes stand for code * scale. Codes come back as those values: the cases that make them read them back.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1.0e-6
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    gemm, norm, quant = dict(op="gemm"), dict(op="norm"), dict(op="quantize")
    return [
        # one new token through the fused query/key/value projection of the 1.5B-shaped verifier: latency
        dict(gemm, name="gemm_1x2048x1536", M=1, N=2048, K=1536, epi="store", out="f16"),
        # a decode step of 16 sequences through the 7B-shaped down projection, onto the fp32 residual stream
        dict(gemm, name="gemm_16x3584x18944_add", M=16, N=3584, K=18944, epi="add", out="f32"),
        # a decode step of 8 sequences through the 7B-shaped gate and up projections: bound by reading the weights
        dict(gemm, name="gated_8x18944x3584", M=8, N=18944, K=3584, epi="gated", out="f16"),
        # the decode-shaped verification batch (64 steps of 5 to 8 tokens), output projection of the 1.7B-shaped verifier
        dict(gemm, name="gemm_421x2048x2048", M=421, N=2048, K=2048, epi="store", out="bf16"),
        # the headline batch's down projection: few tiles, a long sum
        dict(gemm, name="gemm_1163x1536x8960", M=1163, N=1536, K=8960, epi="store", out="f16"),
        # the headline batch's gate and up projections
        dict(gemm, name="gated_1163x8960x1536", M=1163, N=8960, K=1536, epi="gated", out="f16"),
        # the same of the batch of 64 steps: bound by the tensor cores
        dict(gemm, name="gated_5377x8960x1536", M=5377, N=8960, K=1536, epi="gated", out="bf16"),
        # one token's norm: latency
        dict(norm, name="norm_1x1536", M=1, d=1536, x="f32", delta="f16", out="f16"),
        # the headline batch's norm
        dict(norm, name="norm_1163x1536", M=1163, d=1536, x="f32", delta="f16", out="f16"),
        # a long prompt through the 7B-shaped model with a 16-bit residual stream
        dict(norm, name="norm_8191x3584_bf16", M=8191, d=3584, x="bf16", delta="bf16", out="bf16"),
        # a decode step's gated hidden rows
        dict(quant, name="quantize_37x8960", M=37, d=8960, x="f16", out="f16"),
        # those of the batch of 64 steps
        dict(quant, name="quantize_5377x8960_bf16", M=5377, d=8960, x="bf16", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "norm", "quantize"])
    m = _log_int(rng, 1, 8191)
    if op == "gemm":
        epi = rng.choice(["store", "add", "gated"])
        out = "f32" if epi == "add" else rng.choice(["f16", "bf16"])
        return dict(op=op, M=m, N=_log_int(rng, 64, 18944), K=16 * _log_int(rng, 4, 1184), epi=epi, out=out)
    case = dict(op=op, M=m, d=16 * _log_int(rng, 4, 1184), out=rng.choice(["f16", "bf16"]))
    if op == "quantize":
        return dict(case, x=rng.choice(["f16", "bf16", "f32"]))
    x, delta = rng.choice([("f32", "f16"), ("f32", "bf16"), ("f32", "none"), ("f16", "f16"), ("bf16", "bf16")])
    return dict(case, x=x, delta=delta)


def draw(rng):
    """One case of the listed ones' ranges that moves and computes no more than the largest of its kind."""
    while True:
        case = _drawn(rng)
        w, most = work(case), [work(c) for c in listed() if c["op"] == case["op"]]
        if all(w[k] <= max(m[k] for m in most) for k in w):
            return case


def work(case):
    m = case["M"]
    if case["op"] == "gemm":
        n, k, two = case["N"], case["K"], 2 if case["epi"] == "gated" else 1
        held = 4 * m * n if case["epi"] == "add" else 0
        return {"bytes": m * k + two * n * k + 4 * (m + two * n) + held + m * n * SIZE[case["out"]], "flops": 2 * two * m * n * k}
    d = case["d"]
    back = m * (2 * (d + 4) + d * SIZE[case["out"]])              # codes and scales written and read, their values written
    if case["op"] == "quantize":
        return {"bytes": m * d * SIZE[case["x"]] + back, "flops": 4 * m * d}
    added = 0 if case["delta"] == "none" else m * d * (SIZE[case["delta"]] + SIZE[case["x"]])
    return {"bytes": m * d * SIZE[case["x"]] + added + 4 * d + back, "flops": 8 * m * d}


# ------------------------------------------------------------------------------------------------------------ inputs
def _coded(x):
    """8-bit codes and fp32 scales of fp32 rows, as a program has them of its weights and activations."""
    scale = x.abs().amax(-1) / 127.0
    return torch.round(x / scale[:, None]).clamp(-127, 127).to(torch.int8), scale


def _draws(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    m = case["M"]
    if case["op"] == "gemm":
        n, k = case["N"], case["K"]
        # channels of the activations differ in size, rows of the weights less so
        a, a_scale = _coded(normal(m, k) * torch.exp(0.5 * normal(k)))
        d = dict(a=a, a_scale=a_scale)
        for name in ("w", "w2")[: 2 if case["epi"] == "gated" else 1]:
            d[name], d[name + "_scale"] = _coded(0.02 * torch.exp(0.1 * normal(n, 1)) * normal(n, k))
        if case["epi"] == "add":
            d["add"] = 4.0 * normal(m, n)
        return d
    wide = torch.exp(0.7 * normal(case["d"]))
    d = dict(x=(normal(m, case["d"]) * wide).to(TYPES[case["x"]]))
    if case["op"] == "norm":
        d["gain"] = torch.exp(0.3 * normal(case["d"]))
        if case["delta"] != "none":
            d["delta"] = (0.5 * normal(m, case["d"])).to(TYPES[case["delta"]])
    return d


def prepare(case, seed):
    state = dict(_draws(case, seed), case=case)
    if own:
        from paper_2602_18447_b200 import binding
        dev, m = torch.device("cuda"), case["M"]
        state["B"] = binding
        state["out"] = torch.empty(m, case["N"] if case["op"] == "gemm" else case["d"], dtype=TYPES[case["out"]], device=dev)
        if case["op"] != "gemm":
            state["codes"] = torch.empty(m, case["d"], dtype=torch.int8, device=dev)
            state["scales"] = torch.empty(m, dtype=torch.float32, device=dev)
        if "delta" in state:
            state["x_out"] = torch.empty_like(state["x"])
    return state


# -------------------------------------------------------------------------------------------------------- plain forms
def _quantize(y):
    """Codes (as fp32 numbers) and largest magnitudes of fp32 rows. The quotient is taken in 64 bits, where a border between
    two codes is never crossed by its rounding."""
    most = y.abs().amax(-1)
    safe = torch.where(most > 0, most, torch.ones_like(most)).double()
    return torch.round(127.0 * y.double() / safe[:, None]).float(), most


def _product(a, a_scale, w, w_scale):
    return (a.float() @ w.float().T) * a_scale[:, None] * w_scale[None, :]


def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    dt = TYPES[case["out"]]
    if case["op"] == "gemm":
        y = _product(state["a"], state["a_scale"], state["w"], state["w_scale"])
        if case["epi"] == "add":
            y = state["add"] + y
        elif case["epi"] == "gated":
            y = y / (1.0 + torch.exp(-y)) * _product(state["a"], state["a_scale"], state["w2"], state["w2_scale"])
        return {"out": y.to(dt)}
    x = state["x"]
    if case["op"] == "quantize":
        codes, most = _quantize(x.float())
        scale = most / 127.0
        return {"values": (codes * scale[:, None]).to(dt), "scales": scale}
    found = {}
    if "delta" in state:
        x = (x.float() + state["delta"].float()).to(x.dtype)
        found["x"] = x
    x = x.float()
    r = 1.0 / torch.sqrt((x * x).mean(-1) + EPS)
    codes, most = _quantize(x * state["gain"])
    scale = r * most / 127.0
    return dict(found, values=(codes * scale[:, None]).to(dt), scales=scale)


def _run_own(state):
    case, B = state["case"], state["B"]
    if case["op"] == "gemm":
        B.cs_gemm_i8(state["a"], state["a_scale"], state["w"], state["w_scale"], state["out"], w2=state.get("w2"),
                     w2_scales=state.get("w2_scale"), add=state.get("add"))
        return {"out": state["out"]}
    found = {"values": state["out"], "scales": state["scales"]}
    if case["op"] == "quantize":
        B.cs_quantize_i8(state["x"], state["codes"], state["scales"])
    else:
        B.cs_rmsnorm_i8(state["x"], state["gain"], state["codes"], state["scales"], EPS, delta=state.get("delta"),
                        x_out=state.get("x_out"))
        if "delta" in state:
            found = dict(x=state["x_out"], **found)
    B.cs_dequantize_i8(state["codes"], state["scales"], state["out"])
    return found


# -------------------------------------------------------------------------------------------------------------- exact
def _codes64(y):
    top = torch.linalg.vector_norm(y, float("inf"), dim=1, keepdim=True)
    return torch.where(top == 0, torch.zeros_like(y), torch.round(y * 127 / top)), top[:, 0] / 127


def exact(case, seed):
    d = _draws(case, seed)
    if case["op"] == "gemm":
        if case["M"] * case["N"] * case["K"] > 2 ** 38:
            return None
        row = torch.einsum("mk,m->mk", d["a"].double(), d["a_scale"].double())
        y = torch.mm(row, torch.einsum("nk,n->kn", d["w"].double(), d["w_scale"].double()))
        if case["epi"] == "gated":
            up = torch.mm(row, torch.einsum("nk,n->kn", d["w2"].double(), d["w2_scale"].double()))
            y = y * torch.special.expit(y) * up
        elif case["epi"] == "add":
            y += d["add"]
        return {"out": y}
    if case["op"] == "quantize":
        codes, step = _codes64(d["x"].double())
        return {"values": codes * step[:, None], "scales": step}
    x, out = d["x"].double(), {}
    if "delta" in d:
        x = x + d["delta"].double()
        out["x"] = x
        # the row that is normed is the one that the program keeps, in the type of x
        x = x.float().to(d["x"].dtype).double()
    # the gained row is held in 32 bits, by definition: codes are its own
    codes, step = _codes64((x * d["gain"].double()).float().double())
    step = step * torch.rsqrt(x.square().sum(1) / case["d"] + EPS)
    return dict(out, values=codes * step[:, None], scales=step)
