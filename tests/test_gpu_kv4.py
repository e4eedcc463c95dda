"""Rows into and out of the caches (every format) and attention over the 4-bit one, against plain statements in 64 bits."""
import numpy as np
import pytest

import kv4_common as K

pytestmark = pytest.mark.gpu


def _rows(rng, n, h, hd, dtype, scale=1.0, device="cuda"):
    import torch
    x = torch.from_numpy(rng.standard_normal((n, h, hd)) * scale)
    return x.to(getattr(torch, dtype)).to(device)


def _np(t):
    return t.double().cpu().numpy()


def _held(c, s, o):
    """What cs_kv_read gives for these codes: the value, exact in 64 bits, rounded to fp16 once."""
    return K.values(c, s, o).astype(np.float16).astype(np.float64)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_append_4bit_holds_the_codes_of_the_formula(hd, dtype):
    """Unrotated rows: fp16 and bf16 inputs make every step of the quantiser exact up to the quotient, so the codes are those
    of the formula in 64 bits. Steps that begin and end anywhere in a page, whole pages among them."""
    rng = np.random.default_rng(hd)
    ctx, lens = np.array([0, 5, 16, 31]), np.array([1, 40, 16, 2])
    with K.Cache(4, 2, hd) as c:
        c.set(ctx)
        k, v = (_rows(rng, lens.sum(), 2, hd, dtype, 3.0) for _ in range(2))
        k[3] = 1.5                                       # a constant group: scale 0
        k[4] = 2.0 ** -20                                # ranges below fp16's normal range
        v[5, 0, 3] = 60000.0 if dtype == "float16" else 59904.0      # beyond what one scale spans: saturates
        c.B.cs_plan_set(c.plan, np.arange(4), lens)
        c.B.cs_kv_append(c.plan, 0, k, v, rotate=False)
        got_k, got_v = c.read(*K.places(lens, ctx))
        assert np.array_equal(got_k, _held(*K.quantise(_np(k))))
        assert np.array_equal(got_v, _held(*K.quantise(_np(v))))
        # nothing else was written: slots in front of and behind the new tokens still hold zeros
        before = [(i, p) for i in range(4) for p in range(128) if not ctx[i] <= p < ctx[i] + lens[i]]
        rest_k, rest_v = c.read(*zip(*before))
        assert not rest_k.any() and not rest_v.any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("far", [0, 100000])
def test_append_4bit_turns_the_keys(hd, dtype, far):
    """|held - turned| <= s / 2, plus at the ends of the range the roundings of s (15 s 2^-11) and o (2^-11 |min|), plus the fp16
    rounding of what is read (2^-11) and fp32 in the turn: two products, a sum and the table's cos and sin, 2^-22 of |a| + |b|."""
    rng = np.random.default_rng(7)
    lens, ctx = np.array([33, 3]), np.array([far + 7, far])
    pages = (far + 64) // 16
    with K.Cache(6, 3, hd, n_seqs=2, pages_each=pages) as c:
        c.set(ctx)
        n = lens.sum()
        q, k, v = _rows(rng, n, 6, hd, dtype), _rows(rng, n, 3, hd, dtype, 2.0), _rows(rng, n, 3, hd, dtype)
        q_out = c.torch.empty_like(q)
        c.B.cs_plan_set(c.plan, [0, 1], lens)
        c.B.cs_kv_append(c.plan, 0, k, v, q=q, q_out=q_out)
        seq, pos = K.places(lens, ctx)
        got_k, got_v = c.read(seq, pos)
        want = K.rotate(_np(k), pos, c.theta)
        g = want.reshape(n, 3, -1, K.GROUP)
        lo, span = g.min(-1, keepdims=True), np.ptp(g, axis=-1, keepdims=True)
        s = span / 15 * (1 + 2.0 ** -11)
        mag = np.abs(_np(k)).max()
        bound = (s * (0.5 + 15 * 2.0 ** -11) + 2.0 ** -11 * np.abs(lo) + 2.0 ** -11 * (np.abs(g) + s) + 2.0 ** -21 * mag)
        assert np.all(np.abs(got_k - want) <= np.broadcast_to(bound, g.shape).reshape(want.shape))
        assert np.array_equal(got_v, _held(*K.quantise(_np(v))))
        eps = 2.0 ** -11 if dtype == "float16" else 2.0 ** -8
        want_q = K.rotate(_np(q), pos, c.theta)
        assert np.all(np.abs(_np(q_out) - want_q) <= eps * np.abs(want_q) + 2.0 ** -21 * np.abs(_np(q)).max() + 2.0 ** -25)


@pytest.mark.parametrize("hd", [64, 128])
def test_append_one_by_one_equals_append_at_once(hd):
    rng = np.random.default_rng(3)
    n = 37
    k, v = _rows(rng, n, 2, hd, "float16"), _rows(rng, n, 2, hd, "float16")
    with K.Cache(2, 2, hd, n_seqs=2) as c:
        c.set([3, 3])
        c.B.cs_plan_set(c.plan, [0], [n])
        c.B.cs_kv_append(c.plan, 0, k, v)
        for t in range(n):
            c.B.cs_plan_set(c.plan, [1], [1])
            c.B.cs_kv_append(c.plan, 0, k[t:t + 1], v[t:t + 1])
            c.B.cs_kv_commit(c.plan)
        pos = np.arange(n) + 3
        a, b = c.read(np.zeros(n, int), pos), c.read(np.ones(n, int), pos)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1]) and a[0].any()


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3", "e5m2"])
def test_append_takes_slices_of_a_fused_projection(fmt):
    """q, k and v as column ranges of one [T, n_qkv] matrix, q turned in place; equal to contiguous copies."""
    import torch
    rng = np.random.default_rng(4)
    hq, hkv, hd, n = 6, 2, 128, 21
    with K.Cache(hq, hkv, hd, n_seqs=2, fmt=fmt) as c:
        fused = _rows(rng, n, hq + 2 * hkv, hd, "bfloat16")
        q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        q_out = torch.empty(n, hq, hd, dtype=torch.bfloat16, device="cuda")
        c.set([9, 9])
        c.B.cs_plan_set(c.plan, [0], [n])
        c.B.cs_kv_append(c.plan, 0, k.contiguous(), v.contiguous(), q=q.contiguous(), q_out=q_out)
        c.B.cs_plan_set(c.plan, [1], [n])
        keep = fused[:, hq:].clone()
        c.B.cs_kv_append(c.plan, 0, k, v, q=q, q_out=q)
        torch.cuda.synchronize()
        assert torch.equal(q, q_out) and torch.equal(fused[:, hq:], keep)
        a, b = (c.read(np.full(n, i), np.arange(n) + 9) for i in (0, 1))
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("hd", [64, 128])
def test_append_16bit_equals_fill(hd):
    """The 16-bit cache gets the cells that cs_kv_fill writes, and nothing else."""
    import torch
    rng = np.random.default_rng(5)
    n = 50
    with K.Cache(4, 2, hd, n_seqs=1, fmt="16bit") as c:
        k, v = _rows(rng, n, 2, hd, "bfloat16"), _rows(rng, n, 2, hd, "bfloat16")
        c.B.cs_plan_set(c.plan, [0], [n])
        c.B.cs_kv_append(c.plan, 0, k, v, rotate=False)
        torch.cuda.synchronize()
        mine = c.pool.clone()
        c.pool.zero_()
        c.set([n])
        c.B.cs_kv_fill(c.kv, 0, 0, k.view(torch.uint16).cpu().numpy(), v.view(torch.uint16).cpu().numpy())
        assert torch.equal(mine, c.pool) and mine.any()
        got = c.read(np.zeros(n, int), np.arange(n))
        assert np.array_equal(got[0], _np(k.half())) and np.array_equal(got[1], _np(v.half()))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("hd", [64, 128])
def test_append_8bit_rounds_to_the_nearest_value(fmt, hd):
    from oracle import confspec_oracle as O
    from workloads import generate
    rng = np.random.default_rng(6)
    n = 45
    encode = generate.e4m3_codes_from_f32 if fmt == "e4m3" else generate.e5m2_codes_from_f32
    decode = O.widen_e4m3 if fmt == "e4m3" else O.widen_e5m2
    with K.Cache(4, 2, hd, n_seqs=1, fmt=fmt) as c:
        k, v = _rows(rng, n, 2, hd, "float16", 4.0), _rows(rng, n, 2, hd, "float16", 2.0 ** -6)
        k[0, 0, 0], k[1, 1, 1] = 60000.0, -60000.0                       # saturate
        c.set([11])
        c.B.cs_plan_set(c.plan, [0], [n])
        c.B.cs_kv_append(c.plan, 0, k, v, rotate=False)
        got = c.read(np.zeros(n, int), np.arange(n) + 11)
        for g, x in zip(got, (k, v)):
            assert np.array_equal(g, decode(encode(x.float().cpu().numpy())).astype(np.float64))


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3", "e5m2"])
def test_append_stores_only_finite_values(fmt):
    """NaN counts as 0 and infinities saturate, so that a row behind another sequence's end cannot spoil it."""
    import torch
    with K.Cache(2, 2, 128, n_seqs=1, fmt=fmt) as c:
        k = torch.ones(18, 2, 128, dtype=torch.float16, device="cuda")
        k[0, 0, 5], k[1, 1, 6], k[2, 0, 7], k[17, 1, 100] = float("nan"), float("inf"), float("-inf"), float("nan")
        c.B.cs_plan_set(c.plan, [0], [18])
        c.B.cs_kv_append(c.plan, 0, k, k, rotate=False)
        most = {"int4": 65504.0, "16bit": 65504.0, "e4m3": 448.0, "e5m2": 57344.0}[fmt]
        for x in c.read(np.zeros(18, int), np.arange(18)):
            assert np.all(np.isfinite(x)) and np.all(np.abs(x) <= most)
            assert np.all(x[3:17] == 1.0)
            if fmt == "int4":
                assert np.array_equal(x, _held(*K.quantise(_np(k))))
            else:
                assert x[0, 0, 5] == 0.0 and x[1, 1, 6] == most and x[2, 0, 7] == -most


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3", "e5m2"])
def test_read_outside_the_table_gives_zeros_and_a_status(fmt):
    rng = np.random.default_rng(8)
    with K.Cache(2, 2, 64, n_seqs=2, pages_each=2, fmt=fmt) as c:
        k = _rows(rng, 20, 2, 64, "float16")
        c.B.cs_plan_set(c.plan, [1], [20])
        c.B.cs_kv_append(c.plan, 0, k, k, rotate=False)
        good, _ = c.read([1, 1], [0, 19])
        c.B.cs_last_status(c.model)
        got, _ = c.read([1, -1, 2, 1, 1, 1], [0, 0, 0, -1, 32, 19])
        assert np.array_equal(got[[0, 5]], good) and not got[1:5].any()
        with pytest.raises(c.B.ConfSpecError) as e:
            c.B.cs_last_status(c.model)
        assert e.value.status == c.B.CS_ERANGE
        c.B.cs_last_status(c.model)


def _attention_case(hq, hkv, hd, ctx, lens, given, dtype, q_scale=1.0, kv_scale=0.78, scale=0.0, seed=1, pages_each=None):
    import torch
    rng = np.random.default_rng(seed)
    ctx, lens = np.asarray(ctx), np.asarray(lens)
    n, held = int(lens.sum()), ctx + (0 if given else lens)
    pages_each = pages_each or int((ctx + lens).max()) // 16 + 1
    with K.Cache(hq, hkv, hd, n_seqs=len(ctx), pages_each=pages_each) as c:
        q = _rows(rng, n, hq, hd, dtype, q_scale)
        kc, vc = (_rows(rng, held.sum(), hkv, hd, dtype, kv_scale) for _ in range(2))
        kn, vn = (_rows(rng, n, hkv, hd, dtype, kv_scale) for _ in range(2))
        some = np.flatnonzero(held)
        if len(some):
            c.B.cs_plan_set(c.plan, some, held[some])
            c.B.cs_kv_append(c.plan, 0, kc, vc, rotate=False)
        c.set(ctx)
        c.B.cs_plan_set(c.plan, np.arange(len(ctx)), lens, given=given)
        out = torch.full_like(q, float("nan"))
        new = (kn, vn) if given else (None, None)
        c.B.cs_attention_4bit(c.plan, 0, q, out, *new, scale=scale)
        torch.cuda.synchronize()
        first = out.clone()
        c.B.cs_attention_4bit(c.plan, 0, q, out, *new, scale=scale)
        torch.cuda.synchronize()
        assert torch.equal(first, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.B.cs_attention_4bit(c.plan, 0, q, out, *new, scale=scale)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, out)
        c.B.cs_last_status(c.model)
    got = _np(out)
    (ck, sk, ok), (cv, sv, ov) = K.quantise(_np(kc)), K.quantise(_np(vc))
    xk, xv = K.values(ck, sk, ok), K.values(cv, sv, ov)
    steps, mag = K.values(cv, sv, 0 * ov), (79 * sk + np.abs(ok)).max(-1)
    a = b = 0
    for i in range(len(ctx)):
        at, m = slice(b, b + lens[i]), int(held[i])
        parts = [z[a:a + m] for z in (xk, xv, steps, mag)]
        if given:
            own_k, own_v = _np(kn[at]), _np(vn[at])
            parts = [np.concatenate(z) for z in zip(parts, (own_k, own_v, np.abs(own_v), np.abs(own_k).max(-1)))]
        seen = int(ctx[i]) + np.arange(lens[i]) + 1
        want, bound = K.attend(_np(q[at]), *parts, seen, scale or hd ** -0.5, max(lens) * hq // hkv > 96)
        bound = bound + (2.0 ** -11 if dtype == "float16" else 2.0 ** -8) * np.abs(want) + 2.0 ** -25
        err = np.abs(got[at] - want)
        assert np.all(err <= bound), (i, float(np.nanmax(err / bound)), np.argwhere(~(err <= bound))[:4])
        a, b = a + m, b + lens[i]
    return got


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("hq,hkv,hd", [(12, 2, 128), (2, 2, 64), (16, 8, 128), (7, 1, 64), (5, 5, 128)])
def test_attention_one_token(hq, hkv, hd, given):
    _attention_case(hq, hkv, hd, [0, 1, 15, 16, 17, 63, 200, 511], np.ones(8, int), given, "float16")


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("hq,hkv,hd,dtype", [(12, 2, 128, "float16"), (14, 2, 128, "bfloat16"), (4, 4, 64, "bfloat16"),
                                             (16, 8, 128, "float16")])
def test_attention_steps_of_every_length(hq, hkv, hd, dtype, given):
    """Row tiles of 8 and 16, several tiles, and the expanded form: steps of 1 to 100 tokens, pages that end inside a step,
    contexts down to nothing."""
    for lens in ([1, 2, 1, 1], [1, 2, 3, 2], [5, 4, 1, 3], [8, 1, 3, 13], [8, 1, 17, 100]):
        _attention_case(hq, hkv, hd, [0, 7, 48, 130], lens, given, dtype, seed=sum(lens))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ctx", [[100], [600], [1500, 40], [250, 3, 700]])
def test_attention_of_few_contexts_shared_by_clusters(ctx, hd):
    """One to three conversations: the pieces of a context are the CTAs of one cluster (2, 4 or 8 of them)."""
    _attention_case(12, 2, hd, ctx, [1] * len(ctx), False, "float16")
    _attention_case(6, 2, hd, ctx, [5] * len(ctx), True, "bfloat16")


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("hd,lens", [(128, [1, 1]), (128, [3, 5]), (64, [20, 1])])
def test_attention_long_contexts_cut_into_pieces(hd, lens, given):
    _attention_case(4, 2, hd, [9001, 4111], lens, given, "float16")


@pytest.mark.parametrize("q_scale,kv_scale,scale", [(8.0, 4.0, 0.0), (0.01, 0.01, 0.0), (30.0, 30.0, 0.02), (1.0, 200.0, 0.001)])
def test_attention_over_a_range_of_magnitudes(q_scale, kv_scale, scale):
    """Sharp and flat distributions, small and large values."""
    _attention_case(6, 2, 128, [70, 300], [2, 4], False, "float16", q_scale, kv_scale, scale)
    _attention_case(6, 2, 64, [70, 300], [2, 4], True, "float16", q_scale, kv_scale, scale)


def test_attention_reads_nothing_behind_a_sequence():
    """A page's slots behind the last token hold another sequence's rows, some of them made of infinities and NaN: the output is
    the same as over clean pages, and the other rows of the output stay as they were."""
    import torch
    rng = np.random.default_rng(9)
    outs = []
    for dirty in (False, True):
        rng = np.random.default_rng(9)
        with K.Cache(4, 2, 128, n_seqs=2, pages_each=3) as c:
            k, v = _rows(rng, 21, 2, 128, "float16"), _rows(rng, 21, 2, 128, "float16")
            q = _rows(rng, 1, 4, 128, "float16")
            if dirty:
                bad = torch.full((48, 2, 128), float("inf"), dtype=torch.float16, device="cuda")
                bad[::3], bad[1::3] = float("nan"), -60000.0
                c.B.cs_plan_set(c.plan, [0], [48])
                c.B.cs_kv_append(c.plan, 0, bad, bad, rotate=False)
            c.B.cs_plan_set(c.plan, [0], [21])
            c.B.cs_kv_append(c.plan, 0, k, v)
            c.set([20, 0])
            c.B.cs_plan_set(c.plan, [0], [1])
            out = torch.full((3, 4, 128), 5.0, dtype=torch.float16, device="cuda")
            c.B.cs_attention_4bit(c.plan, 0, q, out[:1])
            torch.cuda.synchronize()
            assert bool((out[1:] == 5.0).all()) and bool(torch.isfinite(out).all())
            outs.append(out.clone())
    assert torch.equal(*outs)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n", [6, 40])                                  # 12 and 120 query rows: the 4-bit and the expanded form
def test_a_token_does_not_meet_what_later_tokens_hold(n, dtype):
    """Given keys and values of the later tokens of a step are NaN and infinite: the earlier tokens' outputs are the same bits as
    with finite ones, and the later tokens' are what the saturated values give."""
    import torch
    rng = np.random.default_rng(11)
    with K.Cache(6, 2, 128, n_seqs=1) as c:
        c.B.cs_plan_set(c.plan, [0], [33])
        c.B.cs_kv_append(c.plan, 0, *(_rows(rng, 33, 2, 128, dtype) for _ in range(2)))
        c.B.cs_kv_commit(c.plan)
        q, k, v = _rows(rng, n, 6, 128, dtype), _rows(rng, n, 2, 128, dtype), _rows(rng, n, 2, 128, dtype)
        c.B.cs_plan_set(c.plan, [0], [n], given=True)
        clean, out = torch.empty_like(q), torch.empty_like(q)
        c.B.cs_attention_4bit(c.plan, 0, q, clean, k, v)
        most = 65504.0 if dtype == "float16" else 65280.0
        bad_v, held_v, bad_k = v.clone(), v.clone(), k.clone()
        for at, value, held in (((3, 0, 5), float("nan"), 0.0), ((4, 1, 6), float("inf"), most), ((5, 0, 7), float("-inf"), -most)):
            bad_v[at], held_v[at] = value, held
        bad_k[4, 0, 0] = float("nan")
        c.B.cs_attention_4bit(c.plan, 0, q, out, bad_k, bad_v)
        torch.cuda.synchronize()
        assert torch.equal(out[:3], clean[:3]) and bool(torch.isfinite(out).all())
        held_k = k.clone()
        held_k[4, 0, 0] = 0.0
        c.B.cs_attention_4bit(c.plan, 0, q, clean, held_k, held_v)
        torch.cuda.synchronize()
        # bf16 has no 65504: an infinity saturates at fp16's largest value, 0.35% above the 65280 compared with
        assert float((out.double() - clean.double()).abs().max()) <= (0.0 if dtype == "float16" else 0.02 * most)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n1", [5, 60])                                 # 15 and 180 query rows: the 4-bit and the expanded form
def test_attention_on_slices_and_in_place(n1, dtype):
    import torch
    rng = np.random.default_rng(10)
    hq, hkv, hd, n = 6, 2, 128, 4 + n1
    with K.Cache(hq, hkv, hd, n_seqs=2) as c:
        fused = _rows(rng, n, hq + 2 * hkv, hd, dtype)
        q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        c.B.cs_plan_set(c.plan, [0, 1], [30, 50])
        c.B.cs_kv_append(c.plan, 0, *(_rows(rng, 80, hkv, hd, "float16") for _ in range(2)))
        c.set([30, 50])
        c.B.cs_plan_set(c.plan, [0, 1], [4, n1], given=True)
        plain = torch.empty(n, hq, hd, dtype=fused.dtype, device="cuda")
        # given keys of the fused matrix share one row stride
        c.B.cs_attention_4bit(c.plan, 0, q.contiguous(), plain, k.contiguous(), v.contiguous())
        c.B.cs_attention_4bit(c.plan, 0, q, q, k, v)
        torch.cuda.synchronize()
        assert torch.equal(q, plain)


def test_the_same_context_for_several_steps():
    """k candidates on one sequence (given keys): each equals the step on its own."""
    import torch
    rng = np.random.default_rng(12)
    with K.Cache(4, 2, 64, n_seqs=2) as c:
        c.B.cs_plan_set(c.plan, [1], [77])
        c.B.cs_kv_append(c.plan, 0, *(_rows(rng, 77, 2, 64, "float16") for _ in range(2)))
        c.B.cs_kv_commit(c.plan)
        q = _rows(rng, 9, 4, 64, "float16")
        k, v = _rows(rng, 9, 2, 64, "float16"), _rows(rng, 9, 2, 64, "float16")
        out, one = torch.empty_like(q), torch.empty_like(q)
        c.B.cs_plan_set(c.plan, [1, 1, 1], [2, 4, 3], given=True)
        with pytest.raises(c.B.ConfSpecError) as e:
            c.B.cs_kv_append(c.plan, 0, k, v)                            # two steps would write the same slots
        assert e.value.status == c.B.CS_EINVAL
        c.B.cs_attention_4bit(c.plan, 0, q, out, k, v)
        for a, b in ((0, 2), (2, 6), (6, 9)):
            c.B.cs_plan_set(c.plan, [1], [b - a], given=True)
            c.B.cs_attention_4bit(c.plan, 0, q[a:b], one[a:b], k[a:b], v[a:b])
        torch.cuda.synchronize()
        assert torch.equal(out, one)


def test_a_long_step_in_a_graph_and_a_plan_set_anew():
    """The expanded form captured and replayed, then the same plan for another batch (fewer rows, then more than before)."""
    import torch
    rng = np.random.default_rng(15)
    hq, hkv, hd = 8, 2, 64
    with K.Cache(hq, hkv, hd, n_seqs=3, pages_each=20) as c:
        c.B.cs_plan_set(c.plan, [0, 1, 2], [100, 37, 300])
        c.B.cs_kv_append(c.plan, 0, *(_rows(rng, 437, hkv, hd, "float16") for _ in range(2)))
        q = _rows(rng, 120, hq, hd, "float16")
        k, v = _rows(rng, 120, hkv, hd, "float16"), _rows(rng, 120, hkv, hd, "float16")
        c.set([100, 37, 300])

        def attend(lens, given):
            n = sum(lens)
            out = torch.full_like(q, 3.0)
            c.B.cs_plan_set(c.plan, [0, 1, 2], lens, given=given)
            new = (k[:n], v[:n]) if given else (None, None)
            c.B.cs_attention_4bit(c.plan, 0, q[:n], out[:n], *new)
            torch.cuda.synchronize()
            assert bool((out[n:] == 3.0).all())                          # rows behind the last token stay
            graph, again = torch.cuda.CUDAGraph(), torch.full_like(q, 3.0)
            with torch.cuda.graph(graph):
                c.B.cs_attention_4bit(c.plan, 0, q[:n], again[:n], *new)
            for _ in range(2):
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, again)
            return out[:n]

        first = attend([30, 2, 40], True)
        attend([1, 1, 2], True)
        attend([50, 30, 40], True)
        assert torch.equal(attend([30, 2, 40], True), first)
        c.set([70, 35, 260])                                             # the new tokens' keys out of the cache
        attend([30, 2, 40], False)
        attend([1, 1, 1], False)


def test_decoding_step_by_step_eager_and_as_a_graph():
    """Append, attend, commit for 40 tokens over two layers: each step's output equals the one of a single plan over all tokens
    to the roundings of both, and a captured step replays to the same bits on another stream."""
    import torch
    rng = np.random.default_rng(13)
    hq, hkv, hd, n = 6, 2, 128, 40
    with K.Cache(hq, hkv, hd, n_seqs=2, layers=2) as c:
        q, k, v = _rows(rng, n, hq, hd, "float16"), _rows(rng, n, hkv, hd, "float16"), _rows(rng, n, hkv, hd, "float16")
        c.set([5, 5])
        whole, each = torch.empty_like(q), torch.empty_like(q)
        c.B.cs_plan_set(c.plan, [0], [n])
        c.B.cs_kv_append(c.plan, 1, k, v, rotate=False)
        c.B.cs_attention_4bit(c.plan, 1, q, whole)
        for t in range(n):
            c.B.cs_plan_set(c.plan, [1], [1])
            c.B.cs_kv_append(c.plan, 1, k[t:t + 1], v[t:t + 1], rotate=False)
            c.B.cs_attention_4bit(c.plan, 1, q[t:t + 1], each[t:t + 1])
            if t == 30:
                torch.cuda.synchronize()
                eager = each[t].clone()
                qs, ks, vs, out = q[t:t + 1].clone(), k[t:t + 1].clone(), v[t:t + 1].clone(), torch.zeros_like(q[:1])
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    c.B.cs_kv_append(c.plan, 1, ks, vs, rotate=False)
                    c.B.cs_attention_4bit(c.plan, 1, qs, out)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out[0], eager)
                qs.mul_(-1.0)                                            # a replay reads its inputs anew
                graph.replay()
                torch.cuda.synchronize()
                assert not torch.equal(out[0], eager)
                qs.copy_(q[t:t + 1])
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out[0], eager)
                c.B.cs_kv_set_seq(c.kv, 0, c.pages[0], 5)                # the page table is no longer on the device
                with pytest.raises(c.B.ConfSpecError) as e:
                    with torch.cuda.graph(torch.cuda.CUDAGraph()):
                        c.B.cs_kv_append(c.plan, 1, ks, vs, rotate=False)
                assert e.value.status == c.B.CS_ESTATE
                c.B.cs_plan_set(c.plan, [1], [1])
            c.B.cs_kv_commit(c.plan)
        torch.cuda.synchronize()
        # the two orders of summation differ by the roundings of P and V: 2 x (2^-11 + 2^-11) of sum p |v| <= max |v|,
        # where |c s| <= the range of a group <= 2 max |v|
        assert float((whole - each).abs().max()) <= 2 * 3 * 2.0 ** -11 * float(v.abs().max()) + 2.0 ** -10
        assert torch.isfinite(each).all()
        other, _ = c.read([0, 1], [6, 6], layer=0)
        assert not other.any()                                           # the other layer was not touched
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            c.set([5, 45])
            c.B.cs_plan_set(c.plan, [1], [1])
            c.B.cs_attention_4bit(c.plan, 1, q[:1], each[:1])
        side.synchronize()


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3"])
def test_a_plan_stands_only_while_its_sequences_do(fmt):
    """Pages that a sequence has given up, and tokens that another call has committed, are not written through an older plan."""
    import torch
    rng = np.random.default_rng(23)
    k, q = _rows(rng, 2, 2, 128, "float16"), _rows(rng, 2, 4, 128, "float16")
    out = torch.zeros_like(q)
    with K.Cache(4, 2, 128, n_seqs=2, pages_each=2, fmt=fmt) as c:
        B = c.B
        other = B.cs_plan_create(c.kv)

        def refused(fn, *a):
            B.cs_take_launch_count()
            with pytest.raises(B.ConfSpecError) as e:
                fn(*a)
            assert e.value.status == B.CS_ESTATE and B.cs_take_launch_count() == 0

        c.set([17, 0])
        B.cs_plan_set(c.plan, [0], [2])
        B.cs_kv_set_seq(c.kv, 0, c.pages[0][:1], 16)                      # its second page goes ...
        B.cs_kv_set_seq(c.kv, 1, c.pages[0][1:], 0)                       # ... to the other sequence
        B.cs_plan_set(other, [1], [2])
        B.cs_kv_append(other, 0, k, k, None, None, False)
        held = c.read([1, 1], [0, 1])
        refused(B.cs_kv_append, c.plan, 0, -k, -k, None, None, False)
        if fmt == "int4":
            refused(B.cs_attention_4bit, c.plan, 0, q, out)
        refused(B.cs_kv_commit, c.plan)
        assert all(np.array_equal(x, y) for x, y in zip(held, c.read([1, 1], [0, 1])))
        # a sequence that is not the plan's may change; the plan's own commit leaves it standing
        B.cs_kv_set_seq(c.kv, 0, c.pages[1], 3)
        B.cs_kv_append(other, 0, k, k, None, None, False)
        B.cs_kv_commit(other)
        B.cs_kv_append(other, 0, k, k, None, None, False)
        # another call has lengthened the context: nothing is written over its tokens, while reading goes on
        B.cs_plan_set(c.plan, [0], [2])
        B.cs_plan_set(other, [0], [2])
        B.cs_kv_append(other, 0, k, k, None, None, False)
        B.cs_kv_commit(other)
        refused(B.cs_kv_append, c.plan, 0, -k, -k, None, None, False)
        refused(B.cs_kv_commit, c.plan)
        if fmt == "int4":
            B.cs_attention_4bit(c.plan, 0, q, out)
        B.cs_plan_set(c.plan, [0], [2])
        B.cs_kv_append(c.plan, 0, k, k, None, None, False)
        B.cs_kv_commit(c.plan)
        torch.cuda.synchronize()
        B.cs_plan_free(other)


def test_what_the_calls_refuse():
    import torch
    rng = np.random.default_rng(14)
    q, k = _rows(rng, 2, 4, 128, "float16"), _rows(rng, 2, 2, 128, "float16")
    out = torch.zeros_like(q)

    def status(c, fn, *a, **kw):
        c.B.cs_take_launch_count()
        with pytest.raises(c.B.ConfSpecError) as e:
            fn(*a, **kw)
        assert c.B.cs_take_launch_count() == 0
        return e.value.status

    with K.Cache(4, 2, 128, n_seqs=3, pages_each=2, layers=2) as c:
        B, EINVAL, ESTATE = c.B, c.B.CS_EINVAL, c.B.CS_ESTATE
        assert status(c, B.cs_kv_append, c.plan, 0, k, k) == ESTATE                        # no batch yet
        assert status(c, B.cs_attention_4bit, c.plan, 0, q, out) == ESTATE
        assert status(c, B.cs_kv_commit, c.plan) == ESTATE
        for seqs, lens in (([0, 3], [1, 1]), ([-1], [1]), ([0], [0]), ([0], [33]), ([0], [-4])):
            assert status(c, B.cs_plan_set, c.plan, seqs, lens) == EINVAL
        c.set([32, 31, 0])
        assert status(c, B.cs_plan_set, c.plan, [0], [1]) == EINVAL                        # no page left for the new token
        B.cs_plan_set(c.plan, [0, 1], [1, 1], given=True)
        torch.cuda.synchronize()
        assert status(c, B.cs_kv_append, c.plan, 0, k, k) == EINVAL
        assert status(c, B.cs_kv_commit, c.plan) == EINVAL
        assert status(c, B.cs_attention_4bit, c.plan, 0, q, out) == EINVAL                 # its keys were to be given
        c.set([3, 5, 0])
        B.cs_plan_set(c.plan, [0, 1], [1, 1])
        torch.cuda.synchronize()
        assert status(c, B.cs_attention_4bit, c.plan, 0, q, out, k, k) == EINVAL
        for layer in (-1, 2):
            assert status(c, B.cs_kv_append, c.plan, layer, k, k) == EINVAL
            assert status(c, B.cs_attention_4bit, c.plan, layer, q, out) == EINVAL
            assert status(c, B.cs_kv_read, c.kv, layer, *([torch.zeros(2, dtype=torch.int32, device="cuda")] * 2), k, k) == EINVAL
        assert status(c, B.cs_attention_4bit, c.plan, 0, q, out, scale=-1.0) == EINVAL
        assert status(c, B.cs_attention_4bit, c.plan, 0, q, out, scale=float("nan")) == EINVAL
        assert status(c, B.cs_kv_append, c.plan, 0, k, k, q=q, q_out=out, rotate=False) == EINVAL
        assert status(c, B.cs_kv_append, c.plan, 0, k, k, q=q) == EINVAL
        narrow = k.new_zeros(2 * 2 * 128 + 8)[1:1 + 2 * 256].view(2, 2, 128)
        assert status(c, B.cs_kv_append, c.plan, 0, narrow, k) == EINVAL                   # not 16-byte aligned
        odd = k.new_zeros(2, 257)[:, :256]
        assert status(c, B.cs_kv_append, c.plan, 0, odd, k) == EINVAL                      # row stride not a multiple of 8
        lib = B.load_library()
        assert lib.cs_kv_append(c.plan, 0, k.data_ptr(), 256, k.data_ptr(), 256, None, 0, None, 0, 0, 2, None) == EINVAL
        assert lib.cs_kv_append(c.plan, 0, k.data_ptr(), 248, k.data_ptr(), 256, None, 0, None, 0, 0, 0, None) == EINVAL
        assert lib.cs_kv_append(c.plan, 0, None, 256, k.data_ptr(), 256, None, 0, None, 0, 0, 0, None) == EINVAL
        # shared pages: two sequences may not write one page
        B.cs_kv_set_seq(c.kv, 2, c.pages[1], 9)
        B.cs_plan_set(c.plan, [1, 2], [1, 1])
        torch.cuda.synchronize()
        assert status(c, B.cs_kv_append, c.plan, 0, k, k) == EINVAL
        B.cs_plan_set(c.plan, [0, 1], [1, 1])
        B.cs_kv_set_seq(c.kv, 1, c.pages[1], 7)
        assert status(c, B.cs_kv_commit, c.plan) == ESTATE                                 # the sequence has changed since
        B.cs_plan_set(c.plan, [], [])
        none = q[:0]
        B.cs_attention_4bit(c.plan, 0, none, none)
        B.cs_kv_append(c.plan, 0, k[:0], k[:0])
        with pytest.raises(ValueError):
            B.cs_kv_append(c.plan, 0, k.float(), k.float())
        with pytest.raises(ValueError):
            B.cs_kv_append(c.plan, 0, k, k.bfloat16())
    with K.Cache(4, 2, 128, n_seqs=2, fmt="e4m3") as c:
        c.B.cs_plan_set(c.plan, [0, 1], [1, 1])
        torch.cuda.synchronize()
        assert status(c, c.B.cs_attention_4bit, c.plan, 0, q, out) == c.B.CS_EINVAL
