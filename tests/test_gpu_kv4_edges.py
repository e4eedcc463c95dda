"""The calls on the 4-bit cache at the ends of their ranges: large queries, small values, what other calls leave behind."""
import numpy as np
import pytest

import kv4_common as K

pytestmark = pytest.mark.gpu


def _dev(x, dtype):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).to(getattr(torch, dtype)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _attend(q, kc, vc, ctx, lens, given, scale, dtype, kn=None, vn=None):
    """Attention of given float64 rows through a cache that holds `kc`, `vc` -> (outputs, and the same in 64 bits with the bound of
    K.attend but for the output's own rounding)."""
    import torch
    q, kc, vc = (_dev(x, dtype) for x in (q, kc, vc))
    kn, vn = (_dev(x, dtype) for x in (kn, vn)) if given else (None, None)
    hq, hkv, hd = q.shape[1], kc.shape[1], q.shape[2]
    ctx, lens = np.asarray(ctx), np.asarray(lens)
    held = ctx + (0 if given else lens)
    with K.Cache(hq, hkv, hd, n_seqs=len(ctx), pages_each=int((ctx + lens).max()) // 16 + 1) as c:
        c.B.cs_plan_set(c.plan, np.flatnonzero(held), held[held > 0])
        c.B.cs_kv_append(c.plan, 0, kc, vc, rotate=False)
        c.set(ctx)
        c.B.cs_plan_set(c.plan, np.arange(len(ctx)), lens, given=given)
        out = torch.full_like(q, float("nan"))
        c.B.cs_attention_4bit(c.plan, 0, q, out, kn, vn, scale=scale)
        torch.cuda.synchronize()
        c.B.cs_last_status(c.model)
    (ck, sk, ok), (cv, sv, ov) = K.quantise(_np(kc)), K.quantise(_np(vc))
    rows = [K.values(ck, sk, ok), K.values(cv, sv, ov), K.values(cv, sv, 0 * ov), (79 * sk + np.abs(ok)).max(-1)]
    want, bound = np.zeros(q.shape), np.zeros(q.shape)
    a = b = 0
    for i in range(len(ctx)):
        at, m = slice(b, b + lens[i]), int(held[i])
        parts = [z[a:a + m] for z in rows]
        if given:
            own_k, own_v = _np(kn[at]), _np(vn[at])
            parts = [np.concatenate(z) for z in zip(parts, (own_k, own_v, np.abs(own_v), np.abs(own_k).max(-1)))]
        want[at], bound[at] = K.attend(_np(q[at]), *parts, int(ctx[i]) + np.arange(lens[i]) + 1, scale or hd ** -0.5,
                                       max(lens) * hq // hkv > 96)
        a, b = a + m, b + lens[i]
    return _np(out), want, bound


def _out_eps(dtype):
    return 2.0 ** -11 if dtype == "float16" else 2.0 ** -8


def _large_query(kind, n, hq, hd, rng):
    q = np.zeros((n, hq, hd))
    if kind == "one":                                 # a single channel, one of those held as 64 + c among them
        for t in range(n):
            for h in range(hq):
                q[t, h, (7 * t + 5 * h) % hd] = 1030.0 if (t + h) % 2 else -2047.0
    elif kind == "mixed":                             # an ordinary row beside a large one in the same tile
        q = rng.standard_normal(q.shape).astype(np.float16).astype(np.float64)
        q[::2, ::3] = -70.0
    else:
        q[:] = float(kind)
        q[:, 1::2] *= -1.0
    return q


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("kind", ["64", "70", "100", "2047", "65504", "one", "mixed"])
@pytest.mark.parametrize("hd,hq,hkv,n", [(128, 6, 2, 2), (64, 6, 2, 2), (128, 6, 2, 5), (64, 7, 1, 9), (128, 5, 5, 1)])
def test_queries_of_every_fp16_magnitude(hd, hq, hkv, n, kind, given):
    """Sums over a row's channels far beyond fp16's range; the scale brings the scores back to a few units, so that the softmax
    is an ordinary one. The bound is K.attend's; a row that is taken times 2^-e for its sums loses at most 2^-25 2^e of a channel, with
    e the smallest that brings 64 x 16 max |q| below 2^15: 2^-25 2^e <= 2^-29 max |q|, in each of hd products with at most k_mag."""
    rng = np.random.default_rng(hd + n)
    dtype = "bfloat16" if kind in ("64", "70", "100") else "float16"
    ctx, lens = np.array([37, 200, 0, 16]), np.array([n, 1, n, 2])
    t, held = int(lens.sum()), ctx + (0 if given else lens)
    q = _large_query(kind, t, hq, hd, rng)
    k, v = (0.78 * rng.standard_normal((int(held.sum()), hkv, hd)) for _ in range(2))
    kn, vn = (0.78 * rng.standard_normal((t, hkv, hd)) for _ in range(2))
    scale = 24.0 / np.abs(q).sum(-1).max()
    got, want, bound = _attend(q, k, v, ctx, lens, given, scale, dtype, kn, vn)
    delta = hd * 2.0 ** -29 * scale * np.abs(q).max() * (79 * 8 * 0.78 / 15 + 4.5 * 0.78)
    spread = 4.5 * 0.78
    bound = bound + 2 * delta * 2 * spread + _out_eps(dtype) * np.abs(want) + 2.0 ** -25
    err = np.abs(got - want)
    assert np.all(np.isfinite(got))
    assert np.all(err <= bound), (float(np.max(err / bound)), np.argwhere(~(err <= bound))[:4])
    assert float(np.median(bound)) < 0.1              # the bound says something
