"""Plain statement in 64 bits of rows in 8-bit codes, of the norm that makes them and of their products."""
from __future__ import annotations

import numpy as np

EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # half a step, relative to the value
LOW = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}       # half a step below the normal range


def torch_type(name):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


def quantise(y):
    """Rows (any float type) -> (codes, largest magnitudes) as float64; a row with something that is no number: zeros, NaN.
    The quotient of numbers of 24 bits is a half only where it is one exactly, and 64 bits tell."""
    y = np.asarray(y, np.float64)
    most = np.abs(y).max(-1)
    good = np.isfinite(y).all(-1)
    q = 127.0 * np.where(good[:, None], y, 0.0) / np.where(good & (most > 0), most, 1.0)[:, None]
    return np.rint(q), np.where(good, most, np.nan)


def scale_of(most):
    """The scale in 64 bits and how far fp32 may be off it: one rounding."""
    return most / 127.0, EPS["f32"] * np.abs(most / 127.0) + LOW["f32"]


def add_rows(x, delta, kind):
    """x + delta as the residual keeps it: an fp32 sum, then the type of x. float64 of those values."""
    import torch
    s = (torch.from_numpy(np.asarray(x, np.float32)) + torch.from_numpy(np.asarray(delta, np.float32))).to(torch_type(kind))
    return s.double().numpy()


def norm(x, gain, eps, threads_chain):
    """Codes, scales and the scales' bound of the norm of rows x (float64 of what is held). threads_chain: the longest chain of
    additions in the sum of squares; all terms are positive, so each addition is off by 2^-24 of the sum at most, the root halves
    that, and mean, eps, root and two divisions round once each."""
    with np.errstate(over="ignore", invalid="ignore"):
        y = np.asarray(x, np.float32) * np.asarray(gain, np.float32)[None, :]
    codes, most = quantise(y)
    ms = (np.asarray(x, np.float64) ** 2).mean(-1) + eps
    scale = np.where(most > 0, most / np.sqrt(np.where(ms > 0, ms, 1.0)) / 127.0, most)
    return codes, scale, (threads_chain / 2 + 6) * EPS["f32"] * np.abs(scale) + LOW["f32"]


def product(a, sa, w, sw):
    """y and its bound: the sum is exact, then it, and the two products with the scales, are rounded to fp32."""
    acc = np.asarray(a, np.float64) @ np.asarray(w, np.float64).T
    y = acc * np.asarray(sa, np.float64)[:, None] * np.asarray(sw, np.float64)[None, :]
    return y, 3.01 * EPS["f32"] * np.abs(y) + 2 * LOW["f32"]


def gated(y1, b1, y2, b2):
    """silu(y1) y2 and its bound: the fast exponential is off by (2 + 1.173 |y|) 2^-23 (CUDA's bound, in steps of the result), the
    sum by 2^-24, the fast division by two steps (2^-22), the product with y2 by 2^-24; an error of y1 is magnified by at most
    1 + |y1| (y silu'(y) / silu(y)). A divisor beyond 2^126 counts as infinite."""
    e = np.exp(np.minimum(-y1, 700.0))
    silu = y1 / (1.0 + e)
    rel = (2 + 1.173 * np.abs(y1)) * 2.0 ** -23 + 2.0 ** -24 + 2.0 ** -22
    b = rel * np.abs(silu) + (1 + np.abs(y1)) * np.where(y1 != 0, np.abs(silu / np.where(y1 != 0, y1, 1.0)), 0.5) * b1
    b = b + np.abs(y1) * 2.0 ** -125
    out = silu * y2
    return out, 1.01 * (b * np.abs(y2) + np.abs(silu) * b2 + 2.0 ** -24 * np.abs(out)) + b * b2


def rounded(want, bound, kind):
    """The bound after rounding to `kind`."""
    return bound + EPS[kind] * (np.abs(want) + bound) + LOW[kind]


def check(got, want, bound, what=""):
    got = np.asarray(got, np.float64)
    bad = np.where(np.isnan(want), ~np.isnan(got), ~(np.abs(got - want) <= bound))      # no number is met by no number alone
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4], np.argwhere(bad)[:4].tolist())


def codes_of(g, rows, d, limit=127):
    """Random codes and scales as quantised rows have them."""
    c = g.integers(-limit, limit + 1, size=(rows, d)).astype(np.int8)
    return c, np.exp(g.normal(size=rows) * 0.5 - 6.0).astype(np.float32)


# ----------------------------------------------------------------------------------- the pass over 8-bit projections
def as_held(y):
    """Rows in 64 bits as their codes and scales stand for them."""
    codes, most = quantise(y)
    return codes * (most / 127.0)[:, None]


def layer_weights(O):
    """O.LayerWeights with its matrices as the library holds them after cs_model_quantize_i8: fp16 values, then codes."""
    class Weights(O.LayerWeights):
        def __init__(self, layer):
            super().__init__(layer)
            for name in ("wq", "wk", "wv", "wo", "wg", "wu", "wd"):
                setattr(self, name, as_held(getattr(self, name).astype(np.float16).astype(np.float64)))
    return Weights


def decoder_layer(O, noise=None):
    """O.decoder_layer_extend with rows quantised in front of each projection. noise: a generator, with which every value that the
    library rounds to fp16 is off by up to half a step (2^-11 relative), at random."""
    def off(y):
        return y if noise is None else y * (1.0 + 2.0 ** -11 * noise.uniform(-1, 1, size=y.shape))

    def layer(x, lw, shape, ctx_len, k_ctx, v_ctx):
        n = x.shape[0]
        hq, hkv, hd = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
        if n == 0:
            return x, np.zeros((0, hkv, hd)), np.zeros((0, hkv, hd))
        pos = ctx_len + np.arange(n)

        def normed(rows, gain):
            return as_held(rows * gain) / np.sqrt((rows * rows).mean(-1, keepdims=True) + shape.rms_eps)

        a = normed(x, lw.norm1)
        q, k, v = (off(a @ w.T).reshape(n, h, hd) for w, h in ((lw.wq, hq), (lw.wk, hkv), (lw.wv, hkv)))
        if lw.q_norm is not None:
            q, k = O.rmsnorm(q, lw.q_norm, shape.rms_eps), O.rmsnorm(k, lw.k_norm, shape.rms_eps)
        q, k = off(O.rope(q, pos, shape.rope_theta)), off(O.rope(k, pos, shape.rope_theta))
        o = off(O.attention_extend(q, k_ctx, v_ctx, k, v).reshape(n, hq * hd))
        x = x + off(as_held(o) @ lw.wo.T)
        b = normed(x, lw.norm2)
        h = off(O.silu(b @ lw.wg.T) * (b @ lw.wu.T))
        return x + off(as_held(h) @ lw.wd.T), k, v
    return layer
