"""Refusals of the 8-bit integer calls, at the C entries and in the binding: nothing here needs a device."""
import ctypes as C
import itertools

import numpy as np
import pytest
import torch

from test_host_kv4_rows import Rows as _Rows


class Rows(_Rows):
    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def data_ptr(self):
        return self.at

    at = 4096


@pytest.fixture(scope="module")
def lib():
    from paper_2602_18447_b200 import binding, build
    build.build()
    return binding.load_library()


P = 1 << 20          # stands for an address; nothing is launched


def _quant(lib, x=P, stride=64, kind=0, codes=P, scales=P, rows=3, d=64):
    return lib.cs_quantize_i8(x, stride, kind, codes, scales, rows, d, None)


def _read(lib, codes=P, scales=P, rows=3, d=64, out=P, stride=64, kind=0):
    return lib.cs_dequantize_i8(codes, scales, rows, d, out, stride, kind, None)


def _norm(lib, x=P, stride=64, kind=2, delta=None, ds=64, dkind=0, xo=None, xos=64, gain=P, codes=P, scales=P, rows=3, d=64, eps=1e-6):
    return lib.cs_rmsnorm_i8(x, stride, kind, delta, ds, dkind, xo, xos, gain, codes, scales, rows, d, eps, None)


def _gemm(lib, a=P, stride=64, sa=P, w=P, sw=P, w2=None, sw2=None, add=None, adds=8, out=P, outs=8, M=3, N=8, K=64, kind=0):
    return lib.cs_gemm_i8(a, stride, sa, w, sw, w2, sw2, add, adds, out, outs, M, N, K, kind, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=P + 8), dict(codes=None), dict(codes=P + 4), dict(scales=None), dict(scales=P + 2),
                                 dict(rows=-1), dict(d=0), dict(d=24), dict(d=-16), dict(stride=63), dict(stride=68), dict(kind=3),
                                 dict(kind=-1), dict(kind=2, stride=66)])
def test_quantize_refuses(lib, bad):
    assert _quant(lib, **bad) == 1
    if "stride" not in bad or bad["stride"] == 63:
        assert _read(lib, **{("out" if k == "x" else k): v for k, v in bad.items()}) == 1


@pytest.mark.parametrize("bad", [dict(x=None), dict(gain=None), dict(gain=P + 4), dict(delta=P), dict(xo=P), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(eps=float("inf")), dict(d=40), dict(rows=-2), dict(kind=7), dict(codes=P + 8), dict(scales=None),
                                 dict(delta=P, xo=P, dkind=5), dict(delta=P, xo=P, kind=0, dkind=1), dict(delta=P, xo=P, kind=1, dkind=2),
                                 dict(delta=P, xo=P, xos=128), dict(delta=P + 64, xo=P + 64, kind=0, ds=64, xos=72),
                                 dict(delta=P + 64, xo=P + 64, kind=2, dkind=0), dict(delta=P, xo=P, ds=60), dict(delta=P + 2, xo=P)])
def test_norm_refuses(lib, bad):
    assert _norm(lib, **bad) == 1


@pytest.mark.parametrize("bad", [dict(a=None), dict(a=P + 8), dict(w=None), dict(w=P + 1), dict(sa=None), dict(sw=None), dict(sw=P + 1),
                                 dict(out=None), dict(out=P + 1), dict(M=-1), dict(N=0), dict(K=0), dict(K=8), dict(K=72),
                                 dict(K=131072, stride=131072), dict(stride=48), dict(stride=72), dict(outs=7), dict(kind=3),
                                 dict(w2=P), dict(sw2=P), dict(w2=P + 8, sw2=P), dict(w2=P, sw2=P, kind=2), dict(add=P),
                                 dict(add=P, kind=2, adds=7), dict(add=P + 2, kind=2), dict(add=P, kind=2, adds=16),
                                 dict(add=P, kind=2, w2=P, sw2=P)])
def test_product_refuses(lib, bad):
    assert _gemm(lib, **bad) == 1


def test_no_rows_are_no_work(lib):
    assert _quant(lib, x=None, codes=None, scales=None, rows=0) == 0
    assert _read(lib, codes=None, scales=None, out=None, rows=0) == 0
    assert _norm(lib, x=None, gain=None, codes=None, scales=None, rows=0) == 0
    assert _gemm(lib, a=None, sa=None, out=None, M=0) == 0
    assert _quant(lib, rows=0, d=24) == 1 and _gemm(lib, M=0, K=24) == 1 and _norm(lib, rows=0, eps=-1.0) == 1


@pytest.fixture
def calls(monkeypatch):
    from paper_2602_18447_b200 import binding as B
    seen = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append((name, args))
                return B.CS_OK
            return call

    monkeypatch.setattr(B, "load_library", lambda path=None: Library())
    monkeypatch.setattr(B, "_stream_on", lambda dev, stream: 0)
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return B, seen


def _i8(*shape, **kw):
    return Rows(*shape, dtype=torch.int8, **kw)


def _f32(*shape, **kw):
    return Rows(*shape, dtype=torch.float32, **kw)


def test_strides_of_slices_and_of_single_rows(calls):
    B, seen = calls
    B.cs_quantize_i8(Rows(3, 64, strides=(640, 1)), _i8(3, 64), _f32(3))
    B.cs_quantize_i8(Rows(1, 64, strides=(7, 1)), _i8(1, 64), _f32(1))
    B.cs_gemm_i8(_i8(3, 64, strides=(128, 1)), _f32(3), _i8(5, 64), _f32(5), Rows(3, 5, strides=(11, 1)))
    B.cs_gemm_i8(_i8(1, 64, strides=(3, 1)), _f32(1), _i8(5, 64), _f32(5), Rows(1, 5, strides=(2, 1)))
    assert [c[1][1] for c in seen] == [640, 64, 128, 64] and [c[1][10] for c in seen[2:]] == [11, 5]
    B.cs_rmsnorm_i8(_f32(3, 64), _f32(64), _i8(3, 64), _f32(3), 1e-6, delta=Rows(3, 64))
    assert seen[-1][1][6] == 4096 and seen[-1][1][2] == 2 and seen[-1][1][5] == 0          # x itself takes the sum
    B.cs_gemm_i8(_i8(0, 64), _f32(0), _i8(5, 64), _f32(5), Rows(0, 5))
    assert seen[-1][1][0] is None


def test_shapes_types_and_places(calls):
    B, seen = calls
    x, c, s, g = Rows(3, 64), _i8(3, 64), _f32(3), _f32(64)
    bad_calls = [
        lambda: B.cs_quantize_i8(Rows(3, 64, dtype=torch.int32), c, s), lambda: B.cs_quantize_i8(x, _i8(3, 80), s),
        lambda: B.cs_quantize_i8(x, c, _f32(4)), lambda: B.cs_quantize_i8(x, Rows(3, 64), s),
        lambda: B.cs_quantize_i8(x, c, Rows(3)), lambda: B.cs_quantize_i8(Rows(3, 64, strides=(1, 3)), c, s),
        lambda: B.cs_quantize_i8(Rows(3, 64, strides=(32, 1)), c, s), lambda: B.cs_quantize_i8(x, _i8(3, 64, strides=(128, 1)), s),
        lambda: B.cs_quantize_i8(Rows(3, 64, device=1), c, s), lambda: B.cs_quantize_i8(x, _i8(3, 64, device=1), s),
        lambda: B.cs_quantize_i8(Rows(192), c, s), lambda: B.cs_dequantize_i8(c, s, Rows(3, 48)),
        lambda: B.cs_rmsnorm_i8(x, Rows(64), c, s, 1e-6), lambda: B.cs_rmsnorm_i8(x, _f32(63), c, s, 1e-6),
        lambda: B.cs_rmsnorm_i8(x, g, c, s, 1e-6, delta=Rows(3, 64, dtype=torch.bfloat16)),
        lambda: B.cs_rmsnorm_i8(x, g, c, s, 1e-6, x_out=x), lambda: B.cs_rmsnorm_i8(x, g, c, s, 1e-6, delta=x, x_out=_f32(3, 64)),
        lambda: B.cs_rmsnorm_i8(x, g, c, s, 1e-6, delta=Rows(2, 64)),
    ]
    a, sa, w, sw, o = _i8(3, 64), _f32(3), _i8(8, 64), _f32(8), Rows(3, 8)
    bad_calls += [
        lambda: B.cs_gemm_i8(a, _f32(8), w, sw, o), lambda: B.cs_gemm_i8(a, sa, _i8(8, 80), sw, o), lambda: B.cs_gemm_i8(a, sa, w, sa, o),
        lambda: B.cs_gemm_i8(a, sa, w, sw, Rows(3, 9)), lambda: B.cs_gemm_i8(a, sa, w, sw, _i8(3, 8)),
        lambda: B.cs_gemm_i8(a, sa, _i8(8, 64, strides=(128, 1)), sw, o), lambda: B.cs_gemm_i8(a, sa, w, sw, o, w2=_i8(9, 64), w2_scales=sw),
        lambda: B.cs_gemm_i8(a, sa, w, sw, o, w2_scales=sw), lambda: B.cs_gemm_i8(a, sa, w, sw, o, w2=w), lambda: B.cs_gemm_i8(a, sa, w, sw, _f32(3, 8), w2=w, w2_scales=sw),
        lambda: B.cs_gemm_i8(a, sa, w, sw, o, add=_f32(3, 8)), lambda: B.cs_gemm_i8(a, sa, w, sw, _f32(3, 8), add=o),
        lambda: B.cs_gemm_i8(a, sa, w, sw, _f32(3, 8), add=_f32(3, 8), w2=w, w2_scales=sw), lambda: B.cs_gemm_i8(a, sa, w, sw, Rows(3, 8, device=1)),
    ]
    for i, call in enumerate(bad_calls):
        with pytest.raises(ValueError):
            call()
            print(i)
    assert not seen


def test_the_plain_statement_on_ties_and_odd_rows():
    """The oracle itself: halves go to even codes, rows of zeros have a scale of 0, rows with something else than numbers NaN."""
    from i8_common import quantise
    y = np.zeros((4, 16))
    y[0, :6] = [127.0, 0.5, 1.5, -2.5, -126.5, 126.5]
    y[2, 3], y[3, 0] = np.inf, np.nan
    codes, most = quantise(y)
    assert codes[0, :6].tolist() == [127, 0, 2, -2, -126, 126] and most[:2].tolist() == [127, 0]
    assert np.isnan(most[2:]).all() and not codes[1:].any()
    assert list(itertools.chain(*codes[1:]))[:2] == [0, 0] and C.sizeof(C.c_int8) == 1
