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


def _relative_bound(q, k, v, kc, vc, seen, scale, dtype):
    """64-bit attention over rows k, v and how far an output may be off where no probability is subnormal, so that every term is off
    in proportion to p |v| and p s: p to fp16 (2^-11 of p |v|), p s to fp16 (2^-11 of p s |c - 8| <= 8 p s); under a larger scale S in
    the context p s may become subnormal, 2^-25 8 codes in units of 2^-k <= S 2^-7 of a sum of at least 2^2: 2^-31 S a key; the
    scores as in K.attend; the output's own rounding. kc, vc: the groups' (codes, scales, offsets)."""
    n, hq, hd = q.shape
    group = hq // k.shape[1]
    mag = (79 * kc[1] + np.abs(kc[2])).max(-1)
    step = np.repeat(vc[1], K.GROUP, axis=-1)
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(hq):
        j = h // group
        for t in range(n):
            m = seen[t]
            s = k[:m, j] @ q[t, h] * scale
            p = np.exp(s - s.max())
            assert p.min() > 2.0 ** -14                                   # 2^2 p is a normal number
            p /= p.sum()
            out[t, h] = p @ v[:m, j]
            delta = (hd + 8) * 2.0 ** -23 * scale * np.abs(q[t, h]).sum() * mag[:m, j].max() + 2.0 ** -18
            spread = p @ np.abs(v[:m, j])
            bound[t, h] = 2.0 ** -11 * (spread + 8 * p @ step[:m, j]) + m * 2.0 ** -31 * step[:m, j].max() + 2 * delta * (spread + np.abs(out[t, h]))
    return out, bound + _out_eps(dtype) * np.abs(out) + 2.0 ** -100


def _sinks(sigma, hq, hkv, hd, n, ctx, given, lift):
    """Every sixteenth key draws e^lift times the weight of the others and has no value; the others' values have size sigma
    (a number, or one for each position)."""
    import torch
    rng = np.random.default_rng(hd + hq)
    held = ctx + (0 if given else n)
    k, v = np.zeros((held, hkv, hd)), rng.standard_normal((held, hkv, hd)) * np.broadcast_to(sigma, held)[:, None, None]
    k[::16] = lift / np.sqrt(hd)
    v[::16] = 0.0
    q = np.ones((n, hq, hd))
    q[:, 1::2] = 0.5
    kn, vn = np.zeros((n, hkv, hd)), rng.standard_normal((n, hkv, hd)) * np.broadcast_to(sigma, held)[-1]
    q, k, v, kn, vn = (_dev(x, "bfloat16") for x in (q, k, v, kn, vn))
    with K.Cache(hq, hkv, hd, n_seqs=1, pages_each=(ctx + n) // 16 + 1) as c:
        c.B.cs_plan_set(c.plan, [0], [held])
        c.B.cs_kv_append(c.plan, 0, k, v, rotate=False)
        c.set([ctx])
        c.B.cs_plan_set(c.plan, [0], [n], given=given)
        out = torch.full_like(q, float("nan"))
        c.B.cs_attention_4bit(c.plan, 0, q, out, *((kn, vn) if given else (None, None)))
        torch.cuda.synchronize()
    kq, vq = K.quantise(_np(k)), K.quantise(_np(v))
    xk, xv = K.values(*kq), K.values(*vq)
    if given:
        own = (np.zeros((n, hkv, hd)), np.zeros((n, hkv, hd // 64)))
        xk, xv = np.concatenate([xk, _np(kn)]), np.concatenate([xv, _np(vn)])
        kq, vq = ([np.concatenate([a, b]) for a, b in zip(z, (own[0], own[1], own[1]))] for z in (kq, vq))
    want, bound = _relative_bound(_np(q), xk, xv, kq, vq, ctx + np.arange(n) + 1, hd ** -0.5, "bfloat16")
    err = np.abs(_np(out) - want)
    assert np.all(err <= bound), (float(np.nanmax(err / bound)), float(np.nanmedian(err / bound)))


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("sigma", [1e-6, 1e-4, 1e-3, 1e-2, 0.1, 1.0, 300.0])
@pytest.mark.parametrize("hd,hq,hkv,n,ctx", [(128, 2, 1, 1, 600), (64, 2, 1, 1, 600), (128, 6, 2, 5, 333), (64, 6, 2, 5, 333),
                                             (128, 2, 2, 1, 9000)])
def test_small_values_beside_keys_that_draw_the_weight(hd, hq, hkv, n, ctx, sigma, given):
    """Probabilities of 2^-12 of the largest times scales of any size: what is lost is in proportion to the values, not to fp16's
    smallest number."""
    _sinks(sigma, hq, hkv, hd, n, ctx, given, 12 * np.log(2.0))


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("order", ["growing", "shrinking", "jumping"])
@pytest.mark.parametrize("hd,hq,hkv,n,ctx", [(128, 2, 1, 1, 1500), (64, 6, 2, 5, 1500)])
def test_values_whose_size_changes_along_a_context(hd, hq, hkv, n, ctx, order, given):
    at = np.arange(ctx + (0 if given else n))
    power = {"growing": -6 + 9 * at / len(at), "shrinking": 3 - 9 * at / len(at), "jumping": np.where(at // 48 % 2, 3.0, -4.0)}[order]
    _sinks(10.0 ** power, hq, hkv, hd, n, ctx, given, 6 * np.log(2.0))


@pytest.mark.parametrize("n", [1, 3, 5, 40])
def test_rows_have_to_be_the_plans(n):
    """A plan of four tokens and rows of another number, or of other heads: refused before anything is launched."""
    import torch
    rows = lambda m, h, d=128: torch.zeros(m, h, d, dtype=torch.float16, device="cuda")  # noqa: E731
    with K.Cache(4, 2, 128, n_seqs=2) as c:
        B = c.B
        B.cs_plan_set(c.plan, [0, 1], [1, 3])
        torch.cuda.synchronize()
        B.cs_take_launch_count()
        for call in (lambda: B.cs_kv_append(c.plan, 0, rows(n, 2), rows(n, 2)),
                     lambda: B.cs_kv_append(c.plan, 0, rows(4, 2), rows(4, 2), q=rows(n, 4), q_out=rows(n, 4)),
                     lambda: B.cs_kv_append(c.plan, 0, rows(4, 1), rows(4, 1)),
                     lambda: B.cs_kv_append(c.plan, 0, rows(4, 4, 64), rows(4, 4, 64)),
                     lambda: B.cs_attention_4bit(c.plan, 0, rows(n, 4), rows(n, 4)),
                     lambda: B.cs_attention_4bit(c.plan, 0, rows(4, 4), rows(4, 3)),
                     lambda: B.cs_kv_read(c.kv, 0, *([torch.zeros(4, dtype=torch.int32, device="cuda")] * 2), rows(4, 1), rows(4, 1))):
            with pytest.raises(ValueError):
                call()
        assert B.cs_take_launch_count() == 0


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3"])
def test_rows_are_read_right_behind_their_append(fmt):
    """Appending and reading back (and, of 4-bit pages, attention by the expanded form) follow one another without a wait, eager and
    as a graph: every read sees the rows of the append in front of it."""
    import torch
    rng = np.random.default_rng(31)
    n, rounds = 40, 12
    rows = [_dev(rng.standard_normal((n, 2, 128)), "float16") for _ in range(rounds)]
    seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    q = _dev(rng.standard_normal((n, 8, 128)), "float16")
    with K.Cache(8, 2, 128, n_seqs=1, fmt=fmt) as c:
        c.B.cs_plan_set(c.plan, [0], [n])
        got = [[torch.empty_like(rows[0]) for _ in range(2)] + [torch.empty_like(q)] for _ in range(rounds)]

        def all_rounds(wait):
            for x, (k, v, out) in zip(rows, got):
                c.B.cs_kv_append(c.plan, 0, x, -x, rotate=False)
                c.B.cs_kv_read(c.kv, 0, seq, pos, k, v)
                if fmt == "int4":
                    c.B.cs_attention_4bit(c.plan, 0, q, out)
                if wait:
                    torch.cuda.synchronize()

        all_rounds(True)
        want = [[t.clone() for t in g] for g in got]
        for g in got:
            for t in g:
                t.zero_()
        all_rounds(False)
        graph = torch.cuda.CUDAGraph()
        for again in range(2):
            torch.cuda.synchronize()
            for g, w in zip(got, want):
                assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1]) and (fmt != "int4" or torch.equal(g[2], w[2]))
                for t in g:
                    t.zero_()
            if not again:
                with torch.cuda.graph(graph):
                    all_rounds(False)
                graph.replay()
        assert not torch.equal(want[0][0], want[1][0])


def _keys_at_the_top(n, hd, theta, rng):
    """bf16 keys whose turned rows hold more than 65504 (stored as that) and nothing below 50 K: where a group's smallest value rounds up
    as fp16, 15 scales above the offset is beyond what fp16 rounds to 65504."""
    half = hd // 2
    t = rng.uniform(51000.0, 60000.0, (n, hd))
    t[:, 3] = t[:, half + 3] = 70000.0
    pos = np.arange(n) % 40
    a = -pos[:, None] * theta ** (-np.arange(half) / half)[None]
    x, y = t[:, :half], t[:, half:]
    return np.concatenate([x * np.cos(a) - y * np.sin(a), y * np.cos(a) + x * np.sin(a)], 1), pos


@pytest.mark.parametrize("hd", [64, 128])
def test_values_at_the_top_of_fp16_are_read_as_finite_ones(hd):
    """A key of 15 scales above its offset may stand for more than fp16's largest number: it is read, and expanded for long steps, as
    65504 (bf16 rows get the value itself). Attention over such keys in both forms: the bound of K.attend with the values that
    the codes stand for, at most 2^-11 above what is expanded."""
    import torch
    rng = np.random.default_rng(hd)
    n, theta = 4000, 1.0e4
    k, _ = _keys_at_the_top(n, hd, theta, rng)
    v = rng.standard_normal((n, 1, hd))
    with K.Cache(2, 1, hd, n_seqs=100, pages_each=10, theta=theta) as c:
        kd, vd = _dev(k[:, None], "bfloat16"), _dev(v, "bfloat16")
        assert bool(torch.isfinite(kd).all())
        c.B.cs_plan_set(c.plan, np.arange(100), np.full(100, 40))
        c.B.cs_kv_append(c.plan, 0, kd, vd)
        c.B.cs_kv_commit(c.plan)
        seq, pos = torch.arange(n, dtype=torch.int32) // 40, torch.arange(n, dtype=torch.int32) % 40
        wide = torch.empty(n, 1, hd, dtype=torch.bfloat16, device="cuda")
        c.B.cs_kv_read(c.kv, 0, seq.cuda(), pos.cuda(), wide, torch.empty_like(wide))
        got, _ = c.read(seq.numpy(), pos.numpy())
        beyond = _np(wide) > 65504.0                     # 65536, the bf16 number next to what the codes stand for
        assert beyond.any() and np.all(np.isfinite(got)) and got.max() == 65504.0
        assert np.all(np.abs(got - _np(wide)) <= 2.0 ** -8 * 65536.0 * (1 + 2.0 ** -3))
        at = int(np.argwhere(beyond)[0][0]) // 40
        for steps in (2, 60):                            # 4 and 120 query rows
            q = _dev(np.ones((steps, 2, hd)) * 2.0 ** -10, "float16")
            new = _dev(np.zeros((steps, 1, hd)), "float16")
            out = torch.full_like(q, float("nan"))
            c.B.cs_plan_set(c.plan, [at], [steps], given=True)
            c.B.cs_attention_4bit(c.plan, 0, q, out, new, new, scale=1.0e-6)
            torch.cuda.synchronize()
            # scores below 128 x 2^-10 x 65536 x 1e-6 = 0.0082: weights are even to 1 %, of 40 cached values and the own zeros
            mean = _np(c.torch.tensor(v[40 * at:40 * at + 40].mean(0)))[None] * 40 / (41 + np.arange(steps))[:, None, None]
            assert np.all(np.abs(_np(out) - mean) <= 0.1)


@pytest.mark.parametrize("fmt", ["int4", "16bit"])
def test_the_page_table_reaches_every_stream(fmt):
    """Two sequences change pages; the call that uploads the table stands behind a long kernel of its stream. Calls on another
    stream, which has to wait for that upload, read and write the new pages."""
    import torch
    rng = np.random.default_rng(41)
    k = _dev(rng.standard_normal((60, 2, 128)), "float16")
    q, new = _dev(rng.standard_normal((1, 4, 128)), "float16"), _dev(rng.standard_normal((1, 2, 128)), "float16")
    results = []
    for delayed in (False, True):
        with K.Cache(4, 2, 128, n_seqs=2, fmt=fmt) as c:
            B = c.B
            other = B.cs_plan_create(c.kv, 8)
            B.cs_plan_set(c.plan, [0, 1], [30, 30])
            B.cs_kv_append(c.plan, 0, k, -k, rotate=False)
            B.cs_plan_set(other, [1], [1])                           # its buffers are made
            torch.cuda.synchronize()
            out, seen = torch.zeros_like(q), torch.zeros(21, 2, 128, dtype=torch.float16, device="cuda")
            unused = torch.empty_like(seen)
            place = (torch.full((21,), 1, dtype=torch.int32, device="cuda"), torch.arange(21, dtype=torch.int32, device="cuda"))
            one, two = torch.cuda.Stream(), torch.cuda.Stream()
            for s in (one, two):
                s.wait_stream(torch.cuda.current_stream())
            c.pages = c.pages[::-1].copy()
            c.set([20, 20])
            with torch.cuda.stream(one):
                if delayed:
                    torch.cuda._sleep(100_000_000)
                B.cs_plan_set(c.plan, [0], [1])                      # uploads the table
            with torch.cuda.stream(two):
                B.cs_plan_set(other, [1], [1])
                B.cs_kv_append(other, 0, new, -new, rotate=False)
                if fmt == "int4":
                    B.cs_attention_4bit(other, 0, q, out)
                B.cs_kv_read(c.kv, 0, *place, seen, unused)
            torch.cuda.synchronize()
            # a read by itself on another stream than the upload's
            c.pages = c.pages[::-1].copy()
            c.set([20, 20])
            alone = torch.zeros_like(seen)
            with torch.cuda.stream(one):
                if delayed:
                    torch.cuda._sleep(100_000_000)
                B.cs_plan_set(c.plan, [0], [1])
            with torch.cuda.stream(two):
                B.cs_kv_read(c.kv, 0, *place, alone, unused)
            torch.cuda.synchronize()
            results.append([t.clone() for t in (out, seen, alone)])
            B.cs_plan_free(other)
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert not torch.equal(results[0][1][:20], results[0][2][:20])


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("made", ["slice", "empty"])
def test_an_empty_plan_takes_rows_of_no_tokens(given, made):
    """Tensors without elements may have no address: nothing is done, and nothing refused."""
    import torch
    rows = lambda h: (torch.zeros(3, h, 128, dtype=torch.float16, device="cuda")[:0] if made == "slice"  # noqa: E731
                      else torch.empty(0, h, 128, dtype=torch.float16, device="cuda"))
    with K.Cache(4, 2, 128, n_seqs=2) as c:
        c.B.cs_plan_set(c.plan, [], [], given=given)
        torch.cuda.synchronize()
        c.B.cs_take_launch_count()
        c.B.cs_attention_4bit(c.plan, 0, rows(4), rows(4), *((rows(2), rows(2)) if given else (None, None)))
        c.B.cs_kv_append(c.plan, 0, rows(2), rows(2), q=rows(4), q_out=rows(4))
        c.B.cs_kv_commit(c.plan)
        none = torch.empty(0, dtype=torch.int32, device="cuda")
        c.B.cs_kv_read(c.kv, 0, none, none, rows(2), rows(2))
        assert c.B.cs_take_launch_count() == 0


_SHORT_OF_MEMORY = """
import ctypes, resource, sys
import numpy as np, torch
import kv4_common as K
assert ctypes.CDLL(None).mallopt(-3, 65536)          # lists from 64 KB on are mapped one by one, so that the limit meets each
pages, n = 32768, 2000
with K.Cache(2, 1, 64, n_seqs=1, pages_each=pages) as c:
    B = c.B
    bits = np.zeros((16 * pages, 1, 64), np.uint16)
    prompt = np.full(100000, 5, np.int32)
    steps, ones, toks = np.zeros(n, np.int32), np.ones(n, np.int32), np.full(n, 5, np.int32)
    conf, acc = torch.empty(n, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda")
    def fill():
        B.cs_kv_set_seq(c.kv, 0, c.pages[0], 16 * pages)
        B.cs_kv_fill(c.kv, 0, 0, bits, bits)
    def verify():
        B.cs_kv_set_seq(c.kv, 0, c.pages[0], 64)
        B.cs_verify_steps(c.model, c.kv, steps, toks, ones, [1, 2], 0.5, conf, acc)
    def plan():
        B.cs_kv_set_seq(c.kv, 0, c.pages[0], 64)
        B.cs_plan_set(c.plan, steps, ones, given=True)
    def prefill():
        B.cs_kv_set_seq(c.kv, 0, c.pages[0], 64)
        B.cs_prefill(c.model, c.kv, [0], prompt, [100000])
    for call in (fill, verify, plan, prefill):
        call()                                       # buffers are made
        call()
        torch.cuda.synchronize()
        now = resource.getrlimit(resource.RLIMIT_AS)
        got = None
        resource.setrlimit(resource.RLIMIT_AS, (int(open("/proc/self/statm").read().split()[0]) * 4096 + 16384, now[1]))
        try:
            call()
        except B.ConfSpecError as e:
            got = e.status
        finally:
            resource.setrlimit(resource.RLIMIT_AS, now)
        torch.cuda.synchronize()
        print(call.__name__, got, flush=True)
        assert got == B.CS_ENOMEM
        call()
    torch.cuda.synchronize()
print("done")
"""


def test_host_memory_that_runs_out_is_an_error_status():
    """The lists of work are made in host memory: where it is not to be had the call returns CS_ENOMEM, and works again later. A process
    of its own, under a limit on its address space."""
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here), os.environ.get("PYTHONPATH", "")]))
    r = subprocess.run([sys.executable, "-c", _SHORT_OF_MEMORY], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), (r.returncode, r.stdout[-500:], r.stderr[-1500:])


@pytest.mark.parametrize("n", [2, 60])                                  # 4 and 120 query rows
def test_the_largest_scale_and_the_refusal_of_larger_ones(n):
    """The best key takes all the weight, where every score is far below zero too: its value, off by the roundings of p s (2^-11 of
    8 s), of the output (2^-11) and, expanded, of the value (2^-11). A scale of 2^60 over the 4-bit pages; scores of 2^24 for long steps."""
    import torch
    rng = np.random.default_rng(51)
    k, v = np.abs(rng.standard_normal((40, 1, 128))) * 100.0, rng.standard_normal((40, 1, 128))
    q = _dev(-np.abs(rng.standard_normal((n, 2, 128))) * 10.0, "float16")
    k, v = _dev(k, "float16"), _dev(v, "float16")
    new = _dev(np.full((n, 1, 128), 400.0), "float16")                   # worse than every cached key
    with K.Cache(2, 1, 128, n_seqs=1) as c:
        c.B.cs_plan_set(c.plan, [0], [40])
        c.B.cs_kv_append(c.plan, 0, k, v, rotate=False)
        c.B.cs_kv_commit(c.plan)
        c.B.cs_plan_set(c.plan, [0], [n], given=True)
        out = torch.full_like(q, float("nan"))
        kq, vq = K.quantise(_np(k)), K.quantise(_np(v))
        xk, xv = K.values(*kq)[:, 0], K.values(*vq)[:, 0]
        scores = np.einsum("thd,kd->thk", _np(q), xk)
        c.B.cs_attention_4bit(c.plan, 0, q, out, new, new, scale=2.0 ** 60 if n == 2 else float(2.0 ** 24 / np.abs(scores).max()))
        torch.cuda.synchronize()
        two = np.sort(scores, -1)[..., -2:]
        clear = two[..., 1] - two[..., 0] > 2.0 ** -12 * np.abs(two[..., 0])
        assert clear.mean() > 0.9
        want = xv[scores.argmax(-1)]
        err = np.abs(_np(out) - want)[clear]
        assert np.all(err <= 2.0 ** -11 * (8 * vq[1].max() + 2 * np.abs(want[clear])) + 2.0 ** -24)
        c.B.cs_take_launch_count()
        for scale in (2.0 ** 61, 1e25, 3e38, float("inf"), float("nan"), -1.0):
            with pytest.raises(c.B.ConfSpecError) as e:
                c.B.cs_attention_4bit(c.plan, 0, q, out, new, new, scale=scale)
            assert e.value.status == c.B.CS_EINVAL
        assert c.B.cs_take_launch_count() == 0


def test_in_place_needs_one_stride():
    """Rows written from where they are read, but further apart or closer, would land on rows that are still to be read."""
    import torch
    buf = torch.zeros(8, 1024, dtype=torch.float16, device="cuda")
    near, far, k = buf.view(16, 512)[:4], buf[:4, :512], torch.zeros(4, 256, dtype=torch.float16, device="cuda")
    with K.Cache(4, 2, 128, n_seqs=1) as c:
        B = c.B
        B.cs_plan_set(c.plan, [0], [4])
        torch.cuda.synchronize()
        B.cs_take_launch_count()
        for q, out in ((near, far), (far, near)):
            for call in (lambda: B.cs_attention_4bit(c.plan, 0, q, out), lambda: B.cs_kv_append(c.plan, 0, k, k, q=q, q_out=out)):
                with pytest.raises(B.ConfSpecError) as e:
                    call()
                assert e.value.status == B.CS_EINVAL
        assert B.cs_take_launch_count() == 0
        for q in (near, far):
            B.cs_kv_append(c.plan, 0, k, k, q=q, q_out=q)
            B.cs_attention_4bit(c.plan, 0, q, q)
        B.cs_plan_set(c.plan, [0], [1])
        B.cs_attention_4bit(c.plan, 0, near[:1], far[:1])
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["int4", "16bit"])
def test_a_new_cache_is_zero_before_any_stream_writes_to_it(fmt):
    """The last pages of a large pool, written on a stream of its own right behind the allocation: the zero fill has ended."""
    import torch
    rng = np.random.default_rng(61)
    k = _dev(rng.standard_normal((20, 8, 128)), "float16")
    with K.Cache(8, 8, 128, n_seqs=1) as c:
        B, pages = c.B, 1 << (20 if fmt == "int4" else 18)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        alloc = B.cs_kv_alloc_4bit if fmt == "int4" else B.cs_kv_alloc
        for _ in range(2):
            kv = alloc(c.model, pages, 16, 1, 2)
            B.cs_kv_set_seq(kv, 0, [pages - 1, pages - 2], 0)
            with torch.cuda.stream(side):
                plan = B.cs_plan_create(kv)
                B.cs_plan_set(plan, [0], [20])
                B.cs_kv_append(plan, 0, k, -k, rotate=False)
            torch.cuda.synchronize()
            out_k, out_v = torch.zeros_like(k), torch.zeros_like(k)
            B.cs_kv_read(kv, 0, torch.zeros(20, dtype=torch.int32, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda"),
                         out_k, out_v)
            torch.cuda.synchronize()
            B.cs_plan_free(plan)
            B.cs_kv_free(kv)
            want = K.values(*K.quantise(_np(k))) if fmt == "int4" else _np(k.bfloat16())
            assert np.array_equal(_np(out_k), want.astype(np.float16).astype(np.float64))
            assert bool((out_v != 0).any())


@pytest.mark.parametrize("fmt", ["int4", "16bit", "e4m3"])
def test_reading_ends_with_a_sequences_own_pages(fmt):
    """A sequence that has given pages up, and one that was never set, have no rows there: zeros and a status, not what the table's
    entries last named."""
    rng = np.random.default_rng(71)
    k = _dev(np.abs(rng.standard_normal((48, 2, 64))) + 1.0, "float16")
    with K.Cache(2, 2, 64, n_seqs=2, pages_each=3, fmt=fmt) as c:
        B = c.B
        B.cs_plan_set(c.plan, [0], [48])
        B.cs_kv_append(c.plan, 0, k, k, rotate=False)
        B.cs_kv_set_seq(c.kv, 0, c.pages[0][:1], 10)
        B.cs_kv_set_seq(c.kv, 1, [], 0)
        got = c.read([0, 0, 0, 0, 1], [0, 15, 16, 47, 0])[0]
        assert got[:2].all() and not got[2:].any()
        with pytest.raises(B.ConfSpecError) as e:
            B.cs_last_status(c.model)
        assert e.value.status == B.CS_ERANGE
        B.cs_kv_set_seq(c.kv, 1, c.pages[0][1:], 0)                      # its new owner reads them
        assert c.read([1, 1], [0, 31])[0].all()
        B.cs_last_status(c.model)


def test_pages_far_into_a_large_pool():
    """Attention in both forms over pages 19 GB into a pool gives the bits that it gives over the same rows in a small one."""
    import torch
    rng = np.random.default_rng(81)
    hq, hkv, pages, ctx = 16, 8, 1 << 20, 75
    k, v = _dev(rng.standard_normal((ctx, hkv, 128)), "float16"), _dev(rng.standard_normal((ctx, hkv, 128)), "float16")
    with K.Cache(hq, hkv, 128, n_seqs=1) as c:
        B = c.B
        far = B.cs_kv_alloc_4bit(c.model, pages, 16, 1, 8)
        plan = B.cs_plan_create(far)
        B.cs_kv_set_seq(far, 0, pages - 1 - np.arange(8), 0)
        for p in (c.plan, plan):
            B.cs_plan_set(p, [0], [ctx])
            B.cs_kv_append(p, 0, k, v)
            B.cs_kv_commit(p)
        for n in (1, 5, 50):                                             # 2, 10 and 100 query rows
            q = _dev(rng.standard_normal((n, hq, 128)), "float16")
            new = _dev(rng.standard_normal((n, hkv, 128)), "float16")
            outs = []
            for p in (c.plan, plan):
                B.cs_plan_set(p, [0], [n], given=True)
                outs.append(torch.full_like(q, float("nan")))
                B.cs_attention_4bit(p, 0, q, outs[-1], new, new)
            torch.cuda.synchronize()
            assert bool(torch.isfinite(outs[0]).all()) and torch.equal(*outs)
        B.cs_plan_free(plan)
        B.cs_kv_free(far)


def test_a_capture_while_the_page_table_is_on_its_way():
    """A capture records nothing of the wait for an upload that another stream is still at, and is not spoiled by it."""
    import torch
    rng = np.random.default_rng(91)
    k = _dev(rng.standard_normal((20, 2, 128)), "float16")
    with K.Cache(4, 2, 128, n_seqs=2) as c:
        B = c.B
        other = B.cs_plan_create(c.kv, 8)
        B.cs_plan_set(c.plan, [0], [20])
        B.cs_kv_append(c.plan, 0, k, -k, rotate=False)
        B.cs_kv_commit(c.plan)
        place = (torch.zeros(20, dtype=torch.int32, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda"))
        want, unused = torch.empty_like(k), torch.empty_like(k)
        B.cs_kv_read(c.kv, 0, *place, want, unused)
        got, q = torch.zeros_like(k), torch.ones(1, 4, 128, dtype=torch.float16, device="cuda")
        out, again = torch.zeros_like(q), torch.zeros_like(q)
        B.cs_plan_set(c.plan, [0], [1], given=True)
        B.cs_attention_4bit(c.plan, 0, q, out, k[:1], k[:1])
        torch.cuda.synchronize()
        B.cs_kv_set_seq(c.kv, 1, c.pages[1], 0)
        one = torch.cuda.Stream()
        with torch.cuda.stream(one):
            torch.cuda._sleep(50_000_000)
            B.cs_plan_set(other, [1], [3])                               # uploads the table
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.cs_kv_read(c.kv, 0, *place, got, unused)
            B.cs_attention_4bit(c.plan, 0, q, again, k[:1], k[:1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(out, again) and bool(want.any()) and bool(out.any())
        B.cs_plan_free(other)


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("hd,n", [(128, 1), (128, 5), (64, 1), (64, 5)])
def test_small_values_do_not_meet_what_lies_behind_a_sequence(hd, n, given):
    """The last page's other slots held rows of the largest scale: the outputs are the bits over clean pages, for values of size 1e-6
    as for others, beside a key that draws 2^11 times the weight."""
    import torch
    outs = []
    for dirty in (False, True):
        rng = np.random.default_rng(101)
        ctx = 37
        k, v = np.zeros((ctx + n, 2, hd)), rng.standard_normal((ctx + n, 2, hd)) * 1e-6
        k[32], v[32] = 11 * np.log(2.0) / np.sqrt(hd), 0.0
        q, k, v = (_dev(x, "bfloat16") for x in (np.ones((n, 6, hd)), k, v))
        with K.Cache(6, 2, hd, n_seqs=1) as c:
            if dirty:
                bad = _dev(np.where(np.arange(64)[:, None, None] % 2, 1, -1) * rng.uniform(2e4, 6e4, (64, 2, hd)) * np.where(
                    np.arange(hd) % 2, 1, -1), "bfloat16")
                c.B.cs_plan_set(c.plan, [0], [64])
                c.B.cs_kv_append(c.plan, 0, bad, bad, rotate=False)
            m = ctx if given else ctx + n
            c.B.cs_plan_set(c.plan, [0], [m])
            c.B.cs_kv_append(c.plan, 0, k[:m], v[:m], rotate=False)
            c.set([ctx])
            c.B.cs_plan_set(c.plan, [0], [n], given=given)
            out = torch.full_like(q, float("nan"))
            c.B.cs_attention_4bit(c.plan, 0, q, out, *((k[ctx:], v[ctx:]) if given else (None, None)))
            torch.cuda.synchronize()
            outs.append(out)
    assert bool(torch.isfinite(outs[0]).all()) and bool(outs[0].any())
    assert torch.equal(*outs)
