"""Cases of the 4-bit context cache: attention over it, appending to a paged cache with the rotary turn on the way, and
reading rows of a cache back, each in a plain form (elementary torch operations) and, where `own` is true, through the
package's calls.

The 4-bit format. The 128 or 64 channels of one (token, kv head) row of K or V are cut into groups of 64 consecutive
channels. A group keeps an fp16 offset o (its smallest value) and an fp16 scale s (a fifteenth of its range, at most
1023.5); channel x is the code c = rint((x - o) / s) in 0 .. 15 and stands for s c + o. K is rotated before that.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GROUP = 64
PAGE = 16
MAX_SCALE = 1023.5
THETA = 1.0e6


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    att = dict(op="attention", new="cached")
    return [
        # one conversation, one new token: the call whose latency a user waits for
        dict(att, name="attend_1x512", B=1, hq=12, hkv=2, hd=128, ctx_lo=512, ctx_hi=512, n_lo=1, n_hi=1, pick=1),
        # the 1.5B-shaped verifier's batch, decoding one token per request
        dict(att, name="attend_16x2048", B=16, hq=12, hkv=2, hd=128, ctx_lo=512, ctx_hi=2048, n_lo=1, n_hi=1, pick=202),
        # long reasoning traces, one token per request
        dict(att, name="attend_8x32768", B=8, hq=12, hkv=2, hd=128, ctx_lo=8192, ctx_hi=32768, n_lo=1, n_hi=1, pick=404),
        # the decode-shaped verification batch: short steps whose own keys are not in the cache yet
        dict(att, name="attend_64x8192_steps", new="given", B=64, hq=16, hkv=8, hd=128, ctx_lo=2048, ctx_hi=8192, n_lo=5,
             n_hi=8, pick=707),
        # small heads, one query head per kv head, contexts down to nothing, steps that end inside a page
        dict(att, name="attend_7x300_hd64", new="given", src="bf16", B=7, hq=4, hkv=4, hd=64, ctx_lo=0, ctx_hi=300, n_lo=1,
             n_hi=37, pick=101),
        # the 7B-shaped verifier on whole steps: many query rows per kv head (7 heads a group)
        dict(att, name="attend_8x4096_chunk", B=8, hq=28, hkv=4, hd=128, ctx_lo=1024, ctx_hi=4096, n_lo=24, n_hi=96,
             pick=505),
        # a decode step's tokens go into the cache: a few hundred KB, bound by latency
        dict(op="append", name="append_64x1_4bit", fmt="int4", src="f16", B=64, hq=16, hkv=8, hd=128, ctx_lo=2048,
             ctx_hi=8192, n_lo=1, n_hi=1, pick=808),
        # accepted steps into the 8-bit cache
        dict(op="append", name="append_33x96_e4m3", fmt="e4m3", src="bf16", B=33, hq=12, hkv=2, hd=128, ctx_lo=0, ctx_hi=2048,
             n_lo=17, n_hi=96, pick=33),
        # a prompt's chunk into the 16-bit cache
        dict(op="append", name="append_16x2048_16bit", fmt="16bit", src="f16", B=16, hq=12, hkv=2, hd=128, ctx_lo=0, ctx_hi=40,
             n_lo=512, n_hi=2048, pick=606),
        # the same into the 4-bit cache, with more heads
        dict(op="append", name="append_16x2048_4bit", fmt="int4", src="f16", B=16, hq=16, hkv=8, hd=128, ctx_lo=0, ctx_hi=40,
             n_lo=512, n_hi=2048, pick=606),
        # a short context read back (to check it, or to move it to another format)
        dict(op="read", name="read_3x400_hd64", fmt="int4", src="f16", B=3, hq=4, hkv=2, hd=64, ctx_lo=20, ctx_hi=400, n_lo=0,
             n_hi=0, pick=9),
        # a batch's whole contexts read back
        dict(op="read", name="read_16x4096", fmt="int4", src="f16", B=16, hq=16, hkv=8, hd=128, ctx_lo=512, ctx_hi=4096,
             n_lo=0, n_hi=0, pick=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["attention", "attention", "append", "read"])
    hkv = rng.choice([1, 2, 3, 4, 8])
    case = dict(op=op, src=rng.choice(["f16", "bf16"]), B=_log_int(rng, 1, 64), hq=hkv * rng.choice([1, 2, 3, 4, 6, 7, 8]),
                hkv=hkv, hd=rng.choice([64, 128, 128]), pick=rng.randrange(1 << 20))
    if op == "attention":
        n = _log_int(rng, 1, 96)
        hi = _log_int(rng, 1, 32768)
        return dict(case, new=rng.choice(["cached", "given"]), ctx_lo=rng.randint(0, hi), ctx_hi=hi, n_lo=rng.randint(1, n),
                    n_hi=n)
    case["fmt"] = rng.choice(["int4", "int4", "e4m3", "e5m2", "16bit"])
    n = _log_int(rng, 1, 4096)
    if op == "append":
        hi = _log_int(rng, 1, 16384)
        return dict(case, ctx_lo=rng.randint(0, hi), ctx_hi=hi, n_lo=rng.randint(1, n), n_hi=n)
    return dict(case, ctx_lo=rng.randint(1, n), ctx_hi=n, n_lo=0, n_hi=0)


def draw(rng):
    """One case of the listed ones' ranges that reads, writes and computes no more than the largest of its kind."""
    while True:
        case = _drawn(rng)
        w, most = work(case), [work(c) for c in listed() if c["op"] == case["op"]]
        if all(w[k] <= max(m[k] for m in most) for k in w):
            return case


def _lens(case):
    g = np.random.RandomState(case["pick"])
    ctx = g.randint(case["ctx_lo"], case["ctx_hi"] + 1, size=case["B"])
    new = g.randint(case["n_lo"], case["n_hi"] + 1, size=case["B"])
    return ctx.astype(np.int64), new.astype(np.int64)


def _row_bytes(case):
    """Bytes of one (token, kv head) row of K or of V in the cache."""
    hd = case["hd"]
    return {"int4": hd // 2 + 4 * (hd // GROUP), "e4m3": hd, "e5m2": hd, "16bit": 2 * hd}[case.get("fmt", "int4")]


def work(case):
    ctx, new = _lens(case)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    t = int(new.sum())
    if case["op"] == "attention":
        cached = int(ctx.sum()) + (t if case["new"] == "cached" else 0)
        given = 0 if case["new"] == "cached" else t
        seen = int((ctx * new + new * (new + 1) // 2).sum())
        return {"bytes": 2 * cached * hkv * _row_bytes(case) + 4 * given * hkv * hd + 4 * t * hq * hd,
                "flops": 4 * seen * hq * hd}
    if case["op"] == "append":
        # q in and out, k and v in, the cosines and sines of every position, the rows written and read back
        back = 0 if case["fmt"] == "16bit" else 4 * hd
        return {"bytes": t * (4 * hq * hd + 4 * hd + hkv * (4 * hd + 2 * _row_bytes(case) + back)),
                "flops": 3 * t * hd * (hq + hkv)}
    rows = int(ctx.sum()) * hkv
    return {"bytes": rows * (2 * _row_bytes(case) + 4 * hd), "flops": 4 * rows * hd}


# ------------------------------------------------------------------------------------------------------------ inputs
def _draws(case, seed):
    """What both forms start from: lengths, pages, and the fp16 or bf16 rows."""
    ctx, new = _lens(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    hq, hkv, hd, b = case["hq"], case["hkv"], case["hd"], case["B"]
    dt = torch.bfloat16 if case.get("src") == "bf16" else torch.float16
    total = ctx + new
    pages = -(-total // PAGE)
    n_pages, width = int(pages.sum()) + 3, max(1, int(pages.max()))
    order = torch.randperm(n_pages, generator=g, device=dev).cpu().numpy()
    first = np.concatenate([[0], np.cumsum(pages)])
    table = np.zeros((b, width), dtype=np.int64)
    at = np.arange(width)[None, :] < pages[:, None]
    table[at] = order[:first[-1]]
    t = int(new.sum())
    d = dict(case=case, ctx=ctx, new=new, table=table, pages=pages, n_pages=n_pages, dev=dev, dt=dt)
    # channels of K differ in size, as the rotary pairs of a trained model's keys do
    spread = torch.exp(0.5 * torch.randn(hkv, hd, generator=g, device=dev))
    rows = lambda n, h: torch.randn(n, h, hd, generator=g, device=dev)  # noqa: E731
    d["q"] = rows(t, hq).to(dt)
    d["k"] = (0.78 * spread * rows(t, hkv)).to(dt)
    d["v"] = (0.78 * rows(t, hkv)).to(dt)
    if case["op"] != "append":
        n = int(total.sum()) if case.get("new") == "cached" else int(ctx.sum())
        d["cached_k"] = (0.78 * spread * rows(n, hkv)).to(dt)
        d["cached_v"] = (0.78 * rows(n, hkv)).to(dt)
    return d


def _token_places(lens, start):
    """Sequence and position of every token of a ragged batch, in order."""
    seq = np.repeat(np.arange(len(lens)), lens)
    pos = np.arange(int(lens.sum())) - np.repeat(np.cumsum(lens) - lens, lens) + np.repeat(start, lens)
    return seq, pos


def _filled(d):
    """How many tokens of each sequence the cache holds before the call."""
    case = d["case"]
    if case["op"] == "append":
        return np.zeros_like(d["ctx"])
    return d["ctx"] + d["new"] if case.get("new") == "cached" else d["ctx"]


def prepare(case, seed):
    d = _draws(case, seed)
    dev = d["dev"]
    seq, pos = _token_places(d["new"], d["ctx"])
    state = {"case": case, "q": d["q"], "k": d["k"], "v": d["v"]}
    if case["op"] == "read":
        seq, pos = _token_places(d["ctx"], np.zeros_like(d["ctx"]))
    state["seq"] = torch.from_numpy(seq).to(dev)
    state["pos"] = torch.from_numpy(pos).to(dev)
    if own:
        return _prepare_own(d, state)
    if case["op"] == "append":
        # the rotary table of the new tokens' positions, as the plan of a step keeps it for all layers
        angle = state["pos"].double()[:, None] * _frequencies(case["hd"]).to(dev)
        state["cos"], state["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    state["table"] = torch.from_numpy(d["table"]).to(dev)
    state["ctx"] = torch.from_numpy(d["ctx"]).to(dev)
    state["new"] = torch.from_numpy(d["new"]).to(dev)
    shape = (d["n_pages"], PAGE, case["hkv"])
    if case.get("fmt", "int4") == "int4":
        groups = case["hd"] // GROUP
        for name in ("k", "v"):
            state["code_" + name] = torch.zeros(*shape, case["hd"], dtype=torch.uint8, device=dev)
            state["scale_" + name] = torch.zeros(*shape, groups, dtype=torch.float16, device=dev)
            state["offset_" + name] = torch.zeros(*shape, groups, dtype=torch.float16, device=dev)
    elif case["fmt"] == "16bit":
        # the 16-bit pool's own layout: [layer][K, V][page][kv head][slot][channel]
        state["pool"] = torch.zeros(1, 2, d["n_pages"], case["hkv"], PAGE, case["hd"], dtype=torch.float16, device=dev)
    else:
        kind = torch.float8_e4m3fn if case["fmt"] == "e4m3" else torch.float8_e5m2
        for name in ("k", "v"):
            state["code_" + name] = torch.zeros(*shape, case["hd"], dtype=torch.uint8, device=dev).view(kind)
    held = _filled(d)
    if held.sum():
        at_seq, at_pos = _token_places(held, np.zeros_like(held))
        places = (torch.from_numpy(at_seq).to(dev), torch.from_numpy(at_pos).to(dev))
        _store(state, "k", d["cached_k"].float(), *places)
        _store(state, "v", d["cached_v"].float(), *places)
    return state


class _Handles:
    """A one-layer model (its matrices are not used by these calls), a cache and a plan, freed with the state."""

    def __init__(self, d):
        from paper_2602_18447_b200 import binding as B
        from workloads.configs import ModelShape
        case = d["case"]
        self.B = B
        m = ModelShape("heads", 1, 256, case["hq"], case["hkv"], case["hd"], 256, 512, THETA)
        z = lambda r: np.zeros((r, 256), dtype=np.uint16)  # noqa: E731
        layer = dict(wq=z(m.q_dim), wk=z(m.kv_dim), wv=z(m.kv_dim), wo=np.zeros((256, m.q_dim), dtype=np.uint16), wg=z(256),
                     wu=z(256), wd=z(256), norm1=np.ones(256, np.float32), norm2=np.ones(256, np.float32))
        self.model = B.cs_model_load(m, dict(embed=z(512), lm_head=z(512), final_norm=np.ones(256, np.float32),
                                             layers=[layer]))
        fmt, width = case.get("fmt", "int4"), d["table"].shape[1]
        self.pool = None
        if fmt == "16bit":
            self.pool = torch.zeros(1, 2, d["n_pages"], case["hkv"], PAGE, case["hd"], dtype=torch.float16, device=d["dev"])
            self.kv = B.cs_kv_alloc(self.model, d["n_pages"], PAGE, case["B"], width, self.pool)
        elif fmt == "int4":
            self.kv = B.cs_kv_alloc_4bit(self.model, d["n_pages"], PAGE, case["B"], width)
        else:
            self.kv = B.cs_kv_alloc_8bit(self.model, d["n_pages"], PAGE, case["B"], width, fmt)
        self.plan = B.cs_plan_create(self.kv)
        held = _filled(d)
        self.set(d, np.zeros_like(held))
        if held.sum():
            some = np.flatnonzero(held)
            B.cs_plan_set(self.plan, some, held[some])
            B.cs_kv_append(self.plan, 0, d["cached_k"], d["cached_v"], rotate=False)
        self.set(d, d["ctx"])
        self.seqs, self.lens = np.arange(case["B"], dtype=np.int32), d["new"].astype(np.int32)
        self.given = case.get("new") == "given"
        torch.cuda.synchronize()

    def set_plan(self):
        """What a program does anew for every step's lengths, before its layers: here the one layer pays for all of it."""
        self.B.cs_plan_set(self.plan, self.seqs, self.lens, given=self.given)

    def set(self, d, ctx):
        for i in range(d["case"]["B"]):
            self.B.cs_kv_set_seq(self.kv, i, d["table"][i, :d["pages"][i]], int(ctx[i]))

    def __del__(self):
        self.B.cs_plan_free(self.plan)
        self.B.cs_kv_free(self.kv)
        self.B.cs_model_free(self.model)


def _prepare_own(d, state):
    case = d["case"]
    state["h"] = h = _Handles(d)
    state["seq"], state["pos"] = state["seq"].int(), state["pos"].int()
    n = len(state["seq"])
    like = lambda t: torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
    if case["op"] == "attention":
        state["out"] = like(d["q"])
    else:
        state["q_out"] = like(d["q"])
        shape = (n, case["hkv"], case["hd"])
        state["k_out"] = torch.empty(shape, dtype=torch.float16, device=d["dev"])
        state["v_out"] = torch.empty(shape, dtype=torch.float16, device=d["dev"])
    state["B"] = h.B
    return state


# -------------------------------------------------------------------------------------------------------- plain forms
def _frequencies(hd):
    return torch.tensor([THETA ** (-2.0 * j / hd) for j in range(hd // 2)], dtype=torch.float64)


def _rotate(x, cos, sin):
    """Pairs (j, j + hd / 2) turned by the position's angle."""
    half = x.shape[-1] // 2
    a, b = x[..., :half].float(), x[..., half:].float()
    c, s = cos[:, None, :], sin[:, None, :]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _quantise(x):
    """Codes, scales and offsets of fp32 rows [..., hd]."""
    g = x.unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    offset = lo.half()
    scale = ((hi - lo) / 15.0).clamp(max=MAX_SCALE).half()
    s = scale.float()[..., None]
    steps = (g - offset.float()[..., None]) / torch.where(s > 0, s, torch.ones_like(s))
    code = torch.round(torch.where(s > 0, steps, torch.zeros_like(steps))).clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), scale, offset


def _store(state, name, x, seq, pos):
    """fp32 rows x of K ("k") or V ("v") into the pages of their positions."""
    page, slot = state["table"][seq, pos // PAGE], pos % PAGE
    fmt = state["case"].get("fmt", "int4")
    if fmt == "int4":
        code, scale, offset = _quantise(x)
        state["code_" + name][page, slot] = code
        state["scale_" + name][page, slot] = scale
        state["offset_" + name][page, slot] = offset
    elif fmt == "16bit":
        state["pool"][0, 0 if name == "k" else 1].transpose(1, 2)[page, slot] = x.bfloat16().half()
    else:
        most = 448.0 if fmt == "e4m3" else 57344.0
        pool = state["code_" + name]
        pool.view(torch.uint8)[page, slot] = x.clamp(-most, most).to(pool.dtype).view(torch.uint8)


def _load(state, name, page, slot):
    """fp32 values of the rows at (page, slot)."""
    fmt = state["case"].get("fmt", "int4")
    if fmt == "16bit":
        return state["pool"][0, 0 if name == "k" else 1].transpose(1, 2)[page, slot].float()
    code = state["code_" + name]
    if fmt != "int4":
        return code.view(torch.uint8)[page, slot].view(code.dtype).float()
    c = code[page, slot].float().unflatten(-1, (-1, GROUP))
    s, o = state["scale_" + name][page, slot].float(), state["offset_" + name][page, slot].float()
    return (c * s[..., None] + o[..., None]).flatten(-2)


def _attend(state):
    case = state["case"]
    hq, hkv, hd, b = case["hq"], case["hkv"], case["hd"], case["B"]
    ctx, new, table = state["ctx"], state["new"], state["table"]
    dev = ctx.device
    seq, pos = state["seq"], state["pos"]
    t_in = pos - ctx[seq]                                        # index of each token within its step
    width = case["n_hi"]
    q = torch.zeros(b, width, hq, hd, device=dev)
    q[seq, t_in] = state["q"].float()
    q = q.view(b, width, hkv, hq // hkv, hd)
    key = torch.arange(table.shape[1] * PAGE, device=dev)
    page, slot = table[:, key // PAGE], (key % PAGE).expand(b, -1)
    k, v = _load(state, "k", page, slot), _load(state, "v", page, slot)
    step = torch.arange(width, device=dev)
    if case["new"] == "cached":
        sees = key[None, None, :] <= ctx[:, None, None] + step[None, :, None]
    else:
        k_new, v_new = torch.zeros(b, width, hkv, hd, device=dev), torch.zeros(b, width, hkv, hd, device=dev)
        k_new[seq, t_in], v_new[seq, t_in] = state["k"].float(), state["v"].float()
        k, v = torch.cat([k, k_new], 1), torch.cat([v, v_new], 1)
        sees = torch.cat([(key < ctx[:, None])[:, None, :].expand(-1, width, -1),
                          (step[None, :] <= step[:, None]).expand(b, -1, -1)], -1)
    s = torch.einsum("bthgd,bkhd->bhgtk", q, k) / math.sqrt(hd)
    s = s.masked_fill(~sees[:, None, None], float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.einsum("bhgtk,bkhd->bthgd", p, v) / p.sum(-1).permute(0, 3, 1, 2)[..., None]
    return o.reshape(b, width, hq, hd)[seq, t_in].to(state["q"].dtype)


def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    if case["op"] == "attention":
        return {"out": _attend(state)}
    if case["op"] == "append":
        q = _rotate(state["q"], state["cos"], state["sin"]).to(state["q"].dtype)
        _store(state, "k", _rotate(state["k"], state["cos"], state["sin"]), state["seq"], state["pos"])
        _store(state, "v", state["v"].float(), state["seq"], state["pos"])
        if case["fmt"] == "16bit":
            return {"q": q, "pool": state["pool"]}
    page, slot = state["table"][state["seq"], state["pos"] // PAGE], state["pos"] % PAGE
    out = {"k": _load(state, "k", page, slot).half(), "v": _load(state, "v", page, slot).half()}
    return dict(out, q=q) if case["op"] == "append" else out


def _run_own(state):
    case, B, h = state["case"], state["B"], state["h"]
    if case["op"] != "read":
        h.set_plan()
    if case["op"] == "attention":
        new = (state["k"], state["v"]) if case["new"] == "given" else (None, None)
        B.cs_attention_4bit(h.plan, 0, state["q"], state["out"], *new)
        return {"out": state["out"]}
    if case["op"] == "append":
        B.cs_kv_append(h.plan, 0, state["k"], state["v"], q=state["q"], q_out=state["q_out"])
        if case["fmt"] == "16bit":
            return {"q": state["q_out"], "pool": h.pool}
    B.cs_kv_read(h.kv, 0, state["seq"], state["pos"], state["k_out"], state["v_out"])
    out = {"k": state["k_out"], "v": state["v_out"]}
    return dict(out, q=state["q_out"]) if case["op"] == "append" else out


# -------------------------------------------------------------------------------------------------------------- exact
def _as_held(x, fmt):
    """The values that a cache of this format holds for the rows x (64 bits in and out)."""
    if fmt == "16bit":
        return x.bfloat16().double()
    if fmt in ("e4m3", "e5m2"):
        mantissa, low, most = (3, -6, 448.0) if fmt == "e4m3" else (2, -14, 57344.0)
        x = x.clamp(-most, most)
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** low))) - mantissa)
        return torch.round(x / step) * step
    hd = x.shape[-1]
    rows = x.reshape(-1, GROUP)
    low = rows.min(dim=1, keepdim=True).values
    top = rows.max(dim=1, keepdim=True).values
    o = low.half().double()
    s = torch.minimum((top - low) / 15, torch.full_like(low, MAX_SCALE)).half().double()
    n = torch.round((rows - o) / torch.where(s == 0, torch.ones_like(s), s)).clamp(0, 15)
    return (torch.where(s == 0, torch.zeros_like(n), n) * s + o).reshape(*x.shape[:-1], hd)


def _turned(x, pos):
    """x [n, heads, hd] as complex pairs times exp(i pos theta^(-2j/hd))."""
    hd = x.shape[-1]
    j = torch.arange(hd // 2, dtype=torch.float64, device=x.device)
    phase = pos.double()[:, None] * torch.exp(-2.0 * j / hd * math.log(THETA))
    z = torch.complex(x[..., : hd // 2].double(), x[..., hd // 2:].double()) * torch.polar(torch.ones_like(phase), phase)[:, None]
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    d = _draws(case, seed)
    dev, fmt = d["dev"], case.get("fmt", "int4")
    if case["op"] == "read":
        # every row is read back in order
        return {"k": _as_held(d["cached_k"].double(), fmt), "v": _as_held(d["cached_v"].double(), fmt)}
    if case["op"] == "append":
        seq, pos = _token_places(d["new"], d["ctx"])
        at = torch.from_numpy(pos).to(dev)
        q, k, v = _turned(d["q"], at), _as_held(_turned(d["k"], at), fmt), _as_held(d["v"].double(), fmt)
        if fmt != "16bit":
            return {"k": k, "v": v, "q": q}
        pool = torch.zeros(1, 2, d["n_pages"], case["hkv"], PAGE, case["hd"], dtype=torch.float64, device=dev)
        page, slot = torch.from_numpy(d["table"][seq, pos // PAGE]).to(dev), at % PAGE
        for h in range(case["hkv"]):
            pool[0, 0, page, h, slot] = k[:, h]
            pool[0, 1, page, h, slot] = v[:, h]
        return {"q": q, "pool": pool}
    group = case["hq"] // case["hkv"]
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device=dev)
    held = _filled(d)
    a = b = 0
    for i in range(case["B"]):
        n, c, m = int(d["new"][i]), int(held[i]), int(d["ctx"][i])
        k, v = (_as_held(d[x][a:a + c].double(), fmt) for x in ("cached_k", "cached_v"))
        if case["new"] == "given":
            k, v = torch.cat([k, d["k"][b:b + n].double()]), torch.cat([v, d["v"][b:b + n].double()])
        for h in range(case["hq"]):
            s = d["q"][b:b + n, h].double() @ k[:, h // group].T * case["hd"] ** -0.5
            s += torch.full_like(s, float("-inf")).triu(m + 1)
            out[b:b + n, h] = torch.softmax(s, -1) @ v[:, h // group]
        a, b = a + c, b + n
    return {"out": out}
