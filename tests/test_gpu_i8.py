"""Projections in 8-bit integers against their plain statement in 64 bits."""
import numpy as np
import pytest

import i8_common as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2602_18447_b200 import binding
    return binding


def _dev(a, kind=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if kind is None else t.to(I.torch_type(kind))


def _np(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------------ rows to codes
def _rows(g, rows, d, kind):
    """Rows of the type, as float64: spread magnitudes, and rows of ties (127 times a power of two against odd halves of it)."""
    import torch
    x = g.standard_normal((rows, d)) * np.exp(g.normal(size=(1, d)) * 0.7) * np.exp(g.normal(size=(rows, 1)) * 3)
    for r in range(0, rows, 3):
        x[r] = (g.integers(-126, 126, size=d) + 0.5) * 2.0 ** (r % 7 - 3)
        x[r, g.integers(d)] = 127.0 * 2.0 ** (r % 7 - 3)
    return torch.from_numpy(x).to(I.torch_type(kind)).double().numpy()


DIMS = [16, 48, 512, 1040, 1536, 8960, 18944, 32784, 131056]


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("rows", [1, 2, 37])
def test_quantize_and_back(B, kind, d, rows):
    import torch
    g = np.random.default_rng(d + rows)
    x = _rows(g, rows, d, kind)
    codes = torch.full((rows, d), 77, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, device="cuda")
    B.cs_quantize_i8(_dev(x, kind), codes, scales)
    want, most = I.quantise(x)
    assert np.array_equal(_np(codes), want)
    scale, bound = I.scale_of(most)
    I.check(_np(scales), scale, bound)
    for to in ("f16", "bf16", "f32"):
        out = torch.empty(rows, d, dtype=I.torch_type(to), device="cuda")
        B.cs_dequantize_i8(codes, scales, out)
        value = want * _np(scales)[:, None]
        with np.errstate(over="ignore"):
            big = np.abs(value) >= 65520 if to == "f16" else np.zeros_like(value, bool)
        got = _np(out)
        assert np.isinf(got[big]).all()
        I.check(got[~big], value[~big], I.rounded(value, I.EPS["f32"] * np.abs(value) + I.LOW["f32"], to)[~big], to)


def test_every_border_of_a_code(B):
    """fp32 numbers on, just below and just above each half, under largest magnitudes whose inverse is rounded either way."""
    import torch
    rows = []
    for most in (127.0, 1.0, 3.0, 0.7, 126.99999, 1e-30, 1e-38, 3e-39, 1e30, 3.3e38):
        m = np.float32(most)
        y = [m]
        for c in range(127):
            h = np.float32((c + 0.5) * float(m) / 127.0)
            for v in (h, np.nextafter(h, np.float32(0)), np.nextafter(h, np.float32(np.inf))):
                y += [v, -v]
        rows.append(np.resize(np.asarray(y, np.float32), 768))
    x = np.minimum(np.stack(rows), np.asarray([r[0] for r in rows])[:, None])
    codes = torch.empty(len(rows), 768, dtype=torch.int8, device="cuda")
    scales = torch.empty(len(rows), device="cuda")
    B.cs_quantize_i8(_dev(x), codes, scales)
    want, most = I.quantise(x)
    assert np.array_equal(_np(codes), want)
    I.check(_np(scales), *I.scale_of(most))


@pytest.mark.parametrize("kind, exponents", [("f16", (0, 1, 15, 30)), ("bf16", (0, 1, 60, 127, 230, 254))])
def test_every_code_of_16_bits(B, kind, exponents):
    """Every number of the type, of both signs, in rows of every largest magnitude that an exponent has. The quotient of numbers of 11
    bits and less is rounded to 53 bits without reaching or leaving a half."""
    import torch
    t, bits = I.torch_type(kind), 10 if kind == "f16" else 7
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16)
    every = torch.where(torch.isfinite(every.view(t)), every, 0)
    for e in exponents:
        tops = (torch.arange(1 << bits, dtype=torch.int32, device="cuda") + (e << bits)).to(torch.int16)
        tops = tops[tops > 0]
        for i in range(0, len(tops), 128):
            top = tops[i:i + 128, None]
            x = torch.where((every & 0x7fff) <= top, every, 0).view(t)
            codes = torch.empty(x.shape, dtype=torch.int8, device="cuda")
            scales = torch.empty(len(top), device="cuda")
            B.cs_quantize_i8(x, codes, scales)
            assert torch.equal(codes.double(), torch.round(127.0 * x.double() / top.view(t).double()))


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
def test_rows_of_zeros_and_of_no_numbers(B, kind):
    import torch
    x = np.ones((7, 1040), np.float32)
    x[1] = 0.0
    x[2, 1039], x[3, 0], x[4, 517], x[5] = np.nan, np.inf, -np.inf, -0.0
    codes = torch.full((7, 1040), 3, dtype=torch.int8, device="cuda")
    scales, out = torch.empty(7, device="cuda"), torch.empty(7, 1040, device="cuda")
    dx, gain = _dev(x, kind), torch.ones(1040, device="cuda")
    for call in (lambda: B.cs_quantize_i8(dx, codes, scales), lambda: B.cs_rmsnorm_i8(dx, gain, codes, scales, 0.0)):
        codes.fill_(3)
        call()
        B.cs_dequantize_i8(codes, scales, out)
        c, s, v = _np(codes), _np(scales), _np(out)
        assert (c[[0, 6]] == 127).all() and not c[1:6].any()
        assert (s[[1, 5]] == 0).all() and np.isnan(s[2:5]).all() and np.isfinite(s[[0, 6]]).all()
        assert np.isnan(v[2:5]).all() and not v[[1, 5]].any()


def test_rows_that_lie_apart(B):
    """Slices of wider matrices, also from an odd 16-byte place; what lies between stays as it was."""
    import torch
    g = np.random.default_rng(5)
    for kind, at in (("f16", 8), ("bf16", 24), ("f32", 4)):
        wide = _dev(g.standard_normal((9, 200)), kind)
        x = wide[:, at:at + 144]
        codes, scales = torch.empty(9, 144, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
        B.cs_quantize_i8(x, codes, scales)
        assert np.array_equal(_np(codes), I.quantise(_np(x))[0])
        room = torch.full((9, 200), -7.0, dtype=wide.dtype, device="cuda")
        B.cs_dequantize_i8(codes, scales, room[:, at:at + 144])
        r = _np(room)
        assert (r[:, :at] == -7).all() and (r[:, at + 144:] == -7).all() and not (r[:, at:at + 144] == -7).all()


# --------------------------------------------------------------------------------------------------------------- norm
def _chain(d):
    """Additions in a row of a block's sum of squares: at most 8 for each piece a thread has, and two trees of 5."""
    return 8 * max(4, -(-d // 8 // 32)) + 10 if d < 1024 else 8 * (-(-d // 8 // 1024) + 8) + 10


@pytest.mark.parametrize("kinds", [("f32", None), ("f16", None), ("bf16", None), ("f32", "f16"), ("f32", "bf16"), ("f32", "f32"),
                                   ("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,d", [(1, 16), (3, 256), (37, 1536), (2, 3584), (1, 18944), (3, 32784), (2, 131056)])
def test_norm_to_codes(B, kinds, rows, d):
    import torch
    kind, dkind = kinds
    g = np.random.default_rng(rows * d)
    x = _rows(g, rows, d, kind)
    gain = np.exp(0.3 * g.standard_normal(d)).astype(np.float32)
    gain[:2] = [0.0, -1.5]
    dx, dg = _dev(x, kind), _dev(gain)
    codes, scales = torch.empty(rows, d, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    if dkind is None:
        B.cs_rmsnorm_i8(dx, dg, codes, scales, 1e-6)
        held = x
    else:
        delta = _rows(g, rows, d, dkind)
        dd, xo = _dev(delta, dkind), torch.zeros_like(dx)
        B.cs_rmsnorm_i8(dx, dg, codes, scales, 1e-6, delta=dd, x_out=xo)
        held = I.add_rows(x, delta, kind)
        assert np.array_equal(_np(xo), held) and np.array_equal(_np(dx), x)
        again, ac = codes.clone(), torch.empty_like(codes)
        B.cs_rmsnorm_i8(dx, dg, ac, scales, 1e-6, delta=dd)                       # x takes the sum
        assert np.array_equal(_np(dx), held) and torch.equal(ac, again)
        if dkind == kind:
            dx = _dev(x, kind)
            B.cs_rmsnorm_i8(dx, dg, ac, scales, 1e-6, delta=dd, x_out=dd)         # so may delta
            assert np.array_equal(_np(dd), held) and torch.equal(ac, again)
    want, scale, bound = I.norm(held, gain, 1e-6, _chain(d))
    assert np.array_equal(_np(codes), want)
    I.check(_np(scales), scale, bound)


def test_norm_of_extreme_rows(B):
    import torch
    x = np.ones((6, 64), np.float32)
    x[0] *= 1e-30          # the root is that of eps
    x[1] *= 1e25           # the squares overflow: no number
    x[2, 5] = 3e38         # so do these
    x[3] *= 1e18
    x[4, 0] = 0.0
    gain = np.full(64, 2.0, np.float32)
    gain[7] = 1e30
    codes, scales = torch.empty(6, 64, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    B.cs_rmsnorm_i8(_dev(x), _dev(gain), codes, scales, 1e-6)
    want, scale, bound = I.norm(x, gain, 1e-6, 64)
    good = [0, 4, 5]
    assert np.array_equal(_np(codes)[good], want[good])
    I.check(_np(scales)[good], scale[good], bound[good])
    assert np.isnan(_np(scales)[[1, 2, 3]]).all() and not _np(codes)[[1, 2, 3]].any()      # 1e18 * 1e30 is none either
    B.cs_rmsnorm_i8(_dev(x), _dev(gain), codes, scales, 0.0)                               # the squares of 1e-30 vanish
    want, scale, bound = I.norm(x, gain, 0.0, 64)
    good = [4, 5]
    assert np.array_equal(_np(codes)[good], want[good])
    I.check(_np(scales)[good], scale[good], bound[good])
    assert np.isnan(_np(scales)[:4]).all() and not _np(codes)[:4].any()


# ----------------------------------------------------------------------------------------------------------- products
SHAPES = [  # M, N, K
    (1, 1, 16), (1, 2048, 1536), (2, 129, 144), (15, 264, 112), (16, 3584, 18944), (17, 127, 4096), (31, 300, 272), (33, 128, 128),
    (64, 1000, 2048), (65, 63, 640), (100, 1536, 1536), (128, 256, 8960), (129, 7, 1024), (200, 777, 256), (255, 512, 48),
    (256, 130, 2064), (257, 2048, 384), (300, 264, 1552), (421, 2048, 2048), (513, 1030, 896), (1163, 1536, 8960), (1, 5, 131056),
    (300, 640, 32768), (3001, 96, 64), (2050, 2500, 160),
    (260, 100, 4096), (512, 520, 2048), (5377, 1536, 1536), (270, 20001, 80),
]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("how", ["f16", "bf16", "f32", "add", "gated f16", "gated bf16"])
def test_product(B, M, N, K, how):
    import torch
    g = np.random.default_rng(M + N + K)
    a, sa = I.codes_of(g, M, K)
    w, sw = I.codes_of(g, N, K)
    sw /= np.float32(10 * np.sqrt(K))
    args = [_dev(v) for v in (a, sa, w, sw)]
    y, b = I.product(a, sa, w, sw)
    kind = "f32" if how == "add" else how.split()[-1]
    out = torch.full((M, N), -777.0, dtype=I.torch_type(kind), device="cuda")
    if how == "add":
        x = g.standard_normal((M, N)).astype(np.float32)
        dx = _dev(x)
        B.cs_gemm_i8(*args, out, add=dx)
        y = y + x
        assert np.array_equal(_np(dx), x)
        B.cs_gemm_i8(*args, dx, add=dx)                  # in place: the same bits
        assert torch.equal(dx, out)
    elif how.startswith("gated"):
        sw *= np.float32(500)                            # gates of ordinary size
        args[3] = _dev(sw)
        y, b = I.product(a, sa, w, sw)
        w2, sw2 = I.codes_of(g, N, K)
        y2, b2 = I.product(a, sa, w2, sw2)
        B.cs_gemm_i8(*args, out, w2=_dev(w2), w2_scales=_dev(sw2))
        y, b = I.gated(y, b, y2, b2)
    else:
        B.cs_gemm_i8(*args, out)
    big = np.abs(y) > 65000 if kind == "f16" else np.zeros(y.shape, bool)
    I.check(_np(out)[~big], y[~big], I.rounded(y, b, kind)[~big])
    B.cs_i8_status()


@pytest.mark.parametrize("N,K", [(264, 1552), (2048, 1536), (520, 8960)])
@pytest.mark.parametrize("how", ["f16", "add", "gated"])
def test_a_token_has_the_same_bits_in_every_batch(B, N, K, how):
    """Every form of the product applies the scales in one order to an exact sum."""
    import torch
    g = np.random.default_rng(N)
    a, sa = (_dev(v) for v in I.codes_of(g, 1200, K))
    w, sw = (_dev(v) for v in I.codes_of(g, N, K))
    sw /= 10.0
    more = dict(w2=w.flip(0).contiguous(), w2_scales=sw) if how == "gated" else {}
    x = torch.randn(1200, N, device="cuda") if how == "add" else None
    kind = torch.float32 if how == "add" else torch.float16
    whole = torch.empty(1200, N, dtype=kind, device="cuda")
    B.cs_gemm_i8(a, sa, w, sw, whole, add=x, **more)
    for m in (1, 16, 29, 60, 128, 250, 300, 512, 700):
        out = torch.empty(m, N, dtype=kind, device="cuda")
        B.cs_gemm_i8(a[7:7 + m], sa[7:7 + m], w, sw, out, add=None if x is None else x[7:7 + m], **more)
        assert torch.equal(out, whole[7:7 + m]), m


@pytest.mark.parametrize("M,N", [(1, 130), (40, 130), (130, 130), (300, 300), (600, 520)])
def test_the_largest_sums_are_exact(B, M, N):
    """All codes at their ends over the longest rows: sums next to 2^31 of either sign, and single differences in the last place."""
    import torch
    K = 131056
    a, w = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
    w[1::2] = 127
    a[0, 5] += 1
    w[0, K - 1] += 1
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    out = torch.empty(M, N, device="cuda")
    B.cs_gemm_i8(_dev(a), one(M), _dev(w), one(N), out)
    want = a.astype(np.float64) @ w.astype(np.float64).T
    assert np.array_equal(_np(out), want.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("M", [1, 20, 64, 129, 300, 700])
@pytest.mark.parametrize("gated", [False, True])
def test_rows_apart_odd_places_and_what_lies_around(B, M, gated):
    import torch
    g = np.random.default_rng(M)
    K, N = 208, 333
    a, sa = I.codes_of(g, M, K)
    w, sw = I.codes_of(g, N, K)
    wide = torch.full((M + 2, 512), 99, dtype=torch.int8, device="cuda")
    wide[1:M + 1, 16:16 + K] = _dev(a)
    more = dict(w2=_dev(w[::-1]), w2_scales=_dev(sw)) if gated else {}
    plain, room = torch.empty(M, N, dtype=torch.float16, device="cuda"), torch.full((M + 2, 401), 5.0, dtype=torch.float16, device="cuda")
    B.cs_gemm_i8(_dev(a), _dev(sa), _dev(w), _dev(sw), plain, **more)
    B.cs_gemm_i8(wide[1:M + 1, 16:16 + K], _dev(sa), _dev(w), _dev(sw), room[1:M + 1, 3:3 + N], **more)
    assert torch.equal(room[1:M + 1, 3:3 + N], plain)
    room[1:M + 1, 3:3 + N] = 5.0
    assert (room == 5.0).all()


def test_scales_of_no_number_and_results_beyond_the_type(B):
    import torch
    g = np.random.default_rng(1)
    for M in (3, 300):
        a, sa = I.codes_of(g, M, 64)
        w, sw = I.codes_of(g, 40, 64)
        sa[1], sw[7], sa[2], w[9], sw[9] = np.nan, np.nan, 1e30, 1, 1.0
        a[2] = 1
        out = torch.empty(M, 40, dtype=torch.float16, device="cuda")
        B.cs_gemm_i8(_dev(a), _dev(sa), _dev(w), _dev(sw), out)
        o = _np(out)
        assert np.isnan(o[1]).all() and np.isnan(o[:, 7]).all() and np.isposinf(o[2, 9])
        rest = np.ones(o.shape, bool)
        rest[[1, 2]], rest[:, 7] = False, False
        assert np.isfinite(o[rest]).all()


@pytest.mark.parametrize("M,N,K", [(1, 1536, 8960), (16, 256, 16384), (100, 520, 2064), (200, 300, 4096), (1163, 1536, 8960), (300, 130, 131056)])
def test_the_same_bits_every_time_and_beside_other_work(B, M, N, K):
    import torch
    g = np.random.default_rng(K)
    a, sa = I.codes_of(g, M, K)
    w, sw = I.codes_of(g, N, K)
    args = [_dev(v) for v in (a, sa, w, sw)]
    first = torch.empty(M, N, device="cuda")
    B.cs_gemm_i8(*args, first)
    outs = [torch.empty_like(first) for _ in range(8)]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):                                     # overlapping calls share nothing
        with torch.cuda.stream(streams[i % 4]):
            B.cs_gemm_i8(*args, o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    B.cs_i8_status()


@pytest.mark.parametrize("M", [1, 50, 421])
def test_a_block_as_it_is_used_and_replayed(B, M):
    """x += delta, norm to codes, gate and up, hidden rows to codes, down onto the residual: each stage against the plain statement on
    what the stage before it left, then all of it from a graph with other inputs."""
    import torch
    g = np.random.default_rng(M)
    d, f = 512, 1360
    mats = {}
    for name, n, k in (("g", f, d), ("u", f, d), ("d", d, f)):
        t = _dev(0.05 * g.standard_normal((n, k)), "bf16")
        mats[name] = (torch.empty(n, k, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"))
        B.cs_quantize_i8(t, *mats[name])
        assert np.array_equal(_np(mats[name][0]), I.quantise(_np(t))[0])
    gain = np.exp(0.2 * g.standard_normal(d)).astype(np.float32)
    x, delta, dg = torch.empty(M, d, device="cuda"), torch.empty(M, d, dtype=torch.float16, device="cuda"), _dev(gain)
    xs, c1, s1 = torch.empty_like(x), torch.empty(M, d, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    h, c2, s2 = torch.empty(M, f, dtype=torch.float16, device="cuda"), torch.empty(M, f, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    out = torch.empty_like(x)

    def block():
        B.cs_rmsnorm_i8(x, dg, c1, s1, 1e-6, delta=delta, x_out=xs)
        B.cs_gemm_i8(c1, s1, *mats["g"], h, w2=mats["u"][0], w2_scales=mats["u"][1])
        B.cs_quantize_i8(h, c2, s2)
        B.cs_gemm_i8(c2, s2, *mats["d"], out, add=xs)

    def put(seed):
        k = np.random.default_rng(seed)
        x.copy_(_dev(k.standard_normal((M, d)), "f32"))
        delta.copy_(_dev(0.3 * k.standard_normal((M, d)), "f16"))

    def hold():
        held = I.add_rows(_np(x), _np(delta), "f32")
        assert np.array_equal(_np(xs), held)
        codes, scale, bound = I.norm(held, gain, 1e-6, 64)
        assert np.array_equal(_np(c1), codes)
        I.check(_np(s1), scale, bound)
        y, b = I.gated(*I.product(codes, _np(s1), _np(mats["g"][0]), _np(mats["g"][1])), *I.product(codes, _np(s1), _np(mats["u"][0]), _np(mats["u"][1])))
        I.check(_np(h), y, I.rounded(y, b, "f16"))
        assert np.array_equal(_np(c2), I.quantise(_np(h))[0])
        y, b = I.product(_np(c2), _np(s2), _np(mats["d"][0]), _np(mats["d"][1]))
        I.check(_np(out), y + held, I.rounded(y + held, b, "f32"))

    put(1)
    block()
    hold()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        block()
    for seed in (2, 3):
        put(seed)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        hold()
    B.cs_i8_status()


def test_first_calls_inside_a_capture():
    """Nothing has to be prepared outside: a process whose first call of every form is captured."""
    import subprocess
    import sys
    import os
    code = """
import torch
from paper_2602_18447_b200 import binding as B
B.load_library()
w, sw = torch.ones(300, 256, dtype=torch.int8, device="cuda"), torch.ones(300, device="cuda")
x = torch.ones(700, 256, device="cuda")
c, s, y = torch.zeros(700, 256, dtype=torch.int8, device="cuda"), torch.zeros(700, device="cuda"), torch.zeros(700, 256, device="cuda")
outs = [torch.zeros(m, 300, device="cuda") for m in (1, 20, 700)]
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    B.cs_rmsnorm_i8(x, x[0].contiguous(), c, s, 0.0)
    B.cs_quantize_i8(x, c, s)
    for o in outs:
        B.cs_gemm_i8(c[:len(o)], s[:len(o)], w, sw, o)
    B.cs_dequantize_i8(c, s, y)
g.replay()
torch.cuda.synchronize()
assert all((o - 256).abs().max() < 1e-3 for o in outs) and (y - 1).abs().max() < 1e-6, [o[0, 0] for o in outs]
B.cs_i8_status()
print("fine")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_values_read_back_are_a_product_s_weights(B):
    """The fp16 product asks for its weights before anything else: they have to be there when the call in front of it writes them."""
    import torch
    g = np.random.default_rng(3)
    c, s = I.codes_of(g, 4096, 512)
    dc, ds = _dev(c), _dev(s)
    a = _dev(g.standard_normal((64, 512)), "f16")
    w = [torch.zeros(4096, 512, dtype=torch.float16, device="cuda") for _ in range(2)]
    ref, out = (torch.empty(64, 4096, dtype=torch.float16, device="cuda") for _ in range(2))
    B.cs_dequantize_i8(dc, ds, w[0])
    torch.cuda.synchronize()
    B.cs_gemm_f16(a, w[0], None, ref, 64, 4096, 512, 0)
    for _ in range(20):
        w[1].zero_()
        B.cs_dequantize_i8(dc, ds, w[1])
        B.cs_gemm_f16(a, w[1], None, out, 64, 4096, 512, 0)
        assert torch.equal(out, ref)
