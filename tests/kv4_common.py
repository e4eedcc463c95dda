"""Plain statement of the 4-bit cache format and of attention over it in 64 bits, and small handles to run the calls on."""
from __future__ import annotations

import numpy as np

GROUP, PAGE, MAX_SCALE = 64, 16, 1023.5


def quantise(x):
    """float64 rows [..., hd] -> (codes, scales, offsets); scales and offsets are fp16 values [..., hd / 64]. The subtraction and
    the fifteenth are taken in fp32, as the format has them."""
    x = np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=65504.0, neginf=-65504.0).clip(-65504, 65504)
    g = x.astype(np.float32).reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = g.min(-1), g.max(-1)
    o = lo.astype(np.float16)
    s = np.minimum((hi - lo) * np.float32(1.0 / 15.0), np.float32(MAX_SCALE)).astype(np.float16)
    sf = s.astype(np.float64)[..., None]
    steps = (g.astype(np.float64) - o.astype(np.float64)[..., None]) / np.where(sf > 0, sf, 1.0)
    c = np.where(sf > 0, np.rint(steps).clip(0, 15), 0)
    return c.reshape(x.shape), s.astype(np.float64), o.astype(np.float64)


def values(c, s, o):
    g = c.reshape(*c.shape[:-1], -1, GROUP)
    return (g * s[..., None] + o[..., None]).reshape(c.shape)


def rotate(x, pos, theta):
    """float64 rows [n, heads, hd] turned by their positions, pairs (j, j + hd / 2)."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    a = np.asarray(pos, np.float64)[:, None] * float(np.float32(theta)) ** (-np.arange(half) / half)[None, :]
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    return np.concatenate([x[..., :half] * c - x[..., half:] * s, x[..., half:] * c + x[..., :half] * s], -1)


def attend(q, k, v, v_steps, k_mag, seen, scale, expanded=False):
    """One step in 64 bits: q [n, hq, hd], k, v [m, hkv, hd]; token t sees keys < seen[t]. Returns (out, bound): the bound counts
    the roundings that the kernel's formats make, per output:
      p to fp16 (2^-11 of each term's |p v|), p s to fp16 (2^-11 of p s |c - 8|, at most p |c s| = v_steps), the output (2^-11, or
      2^-8 for bf16: added by the caller); below fp16's normal range p is off by 2^-25 and p s by 2^-25 too, times 8 codes,
      where the largest p of a row is at least 2^2: m 2^-27 |v| and m 2^-24 together for m keys; the score's fp32 sums: hd + 8
      additions of terms q (64 + c) s and q o, each off by at most 2^-23 of the sum of magnitudes (k_mag [m, hkv] = max over
      groups of 79 s + |o|); 2^x to 2^-18.
    expanded: the keys and values were rounded to fp16 first: 2^-11 of every |q_d k_d| in the score, 2^-11 of every |p v|; the sums
    run over the values themselves.
    """
    n, hq, hd = q.shape
    group = hq // k.shape[1]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(hq):
        kh, vh, st, mag = k[:, h // group], v[:, h // group], v_steps[:, h // group], k_mag[:, h // group]
        for t in range(n):
            m = seen[t]
            if m <= 0:
                continue
            s = kh[:m] @ q[t, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[t, h] = p @ vh[:m]
            delta = (hd + 8) * 2.0 ** -23 * scale * np.abs(q[t, h]).sum() * mag[:m].max() + 2.0 ** -18
            spread = p @ np.abs(vh[:m])
            if expanded:
                delta += 2.0 ** -11 * scale * (np.abs(kh[:m]) @ np.abs(q[t, h])).max()
            bound[t, h] = (2.0 ** -11 * (spread * (2 if expanded else 1) + p @ st[:m]) + m * 2.0 ** -27 * np.abs(vh[:m]).max() + m * 2.0 ** -24
                           + 2 * delta * spread + 2 * delta * np.abs(out[t, h]))
    return out, bound


class Cache:
    """A one-layer model of the given heads (its matrices are not used), a cache of one format and a plan."""

    def __init__(self, hq, hkv, hd, n_seqs=4, pages_each=8, fmt="int4", layers=1, theta=1.0e4, share=None, seed=5):
        import torch
        from paper_2602_18447_b200 import binding as B
        from workloads.configs import ModelShape
        self.B, self.torch = B, torch
        self.hq, self.hkv, self.hd, self.theta = hq, hkv, hd, theta
        m = ModelShape("heads", layers, 256, hq, hkv, hd, 256, 512, theta)
        z = lambda r, c=256: np.zeros((r, c), np.uint16)  # noqa: E731
        one = np.ones(256, np.float32)
        layer = dict(wq=z(m.q_dim), wk=z(m.kv_dim), wv=z(m.kv_dim), wo=z(256, m.q_dim), wg=z(256), wu=z(256), wd=z(256),
                     norm1=one, norm2=one)
        self.model = B.cs_model_load(m, dict(embed=z(512), lm_head=z(512), final_norm=one, layers=[layer] * layers))
        self.n_pages = n_seqs * pages_each + 3
        self.pool = None
        if fmt == "int4":
            self.kv = B.cs_kv_alloc_4bit(self.model, self.n_pages, PAGE, n_seqs, pages_each)
        elif fmt == "16bit":
            self.pool = torch.zeros(layers, 2, self.n_pages, hkv, PAGE, hd, dtype=torch.float16, device="cuda")
            self.kv = B.cs_kv_alloc(self.model, self.n_pages, PAGE, n_seqs, pages_each, self.pool)
        else:
            self.kv = B.cs_kv_alloc_8bit(self.model, self.n_pages, PAGE, n_seqs, pages_each, fmt)
        order = np.random.default_rng(seed).permutation(self.n_pages)[:n_seqs * pages_each]
        self.pages = order.reshape(n_seqs, pages_each).astype(np.int32)
        self.plan = B.cs_plan_create(self.kv)
        self.n_seqs = n_seqs
        self.set(np.zeros(n_seqs, int))

    def set(self, ctx):
        for i, c in enumerate(ctx):
            self.B.cs_kv_set_seq(self.kv, i, self.pages[i], int(c))

    def read(self, seq, pos, layer=0):
        t = self.torch
        n = len(seq)
        k = t.full((n, self.hkv, self.hd), 7.0, dtype=t.float16, device="cuda")
        v = t.full_like(k, 7.0)
        self.B.cs_kv_read(self.kv, layer, t.tensor(np.asarray(seq), dtype=t.int32, device="cuda"),
                          t.tensor(np.asarray(pos), dtype=t.int32, device="cuda"), k, v)
        t.cuda.synchronize()
        return k.double().cpu().numpy(), v.double().cpu().numpy()

    def close(self):
        self.B.cs_plan_free(self.plan)
        self.B.cs_kv_free(self.kv)
        self.B.cs_model_free(self.model)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def places(lens, start):
    seq = np.repeat(np.arange(len(lens)), lens)
    pos = np.concatenate([np.arange(n) + s for n, s in zip(lens, start)]) if len(lens) else np.zeros(0, int)
    return seq, pos
