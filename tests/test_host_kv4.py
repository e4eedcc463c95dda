"""What the calls on a plan answer without a device: arguments are checked before anything touches one."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2602_18447_b200 import binding, build
    binding.load_library(build.build())
    return binding


def test_null_handles_are_refused(B):
    lib, out = B.load_library(), ctypes.c_void_p(5)
    assert lib.cs_kv_alloc_4bit(None, 4, 16, 1, 4, ctypes.byref(out)) == B.CS_EINVAL and not out.value
    out = ctypes.c_void_p(5)
    assert lib.cs_plan_create(None, 0, ctypes.byref(out)) == B.CS_EINVAL and not out.value
    assert lib.cs_plan_set(None, None, None, 0, 0, None) == B.CS_EINVAL
    assert lib.cs_plan_free(None) == B.CS_OK
    assert lib.cs_kv_commit(None) == B.CS_EINVAL
    assert lib.cs_kv_append(None, 0, None, 0, None, 0, None, 0, None, 0, 0, 0, None) == B.CS_EINVAL
    assert lib.cs_attention_4bit(None, 0, None, 0, None, None, 0, None, 0, 0, 0.0, None) == B.CS_EINVAL
    assert lib.cs_kv_read(None, 0, None, None, 1, None, None, 0, None) == B.CS_EINVAL


def test_rows_have_to_be_contiguous_heads(B):
    import torch
    cpu = torch.zeros(2, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        B._rows(cpu)                                      # not on a device
    with pytest.raises(ValueError):
        B._dtype_code(cpu.float())
    assert B._dtype_code(cpu) == B.CS_F16 and B._dtype_code(cpu.bfloat16()) == B.CS_BF16


def test_the_plain_format_keeps_half_a_step():
    """The statement of the format that the GPU tests compare with: off by at most half a step, and at the ends of the range by
    the roundings of the scale (15 s 2^-11) and of the offset (2^-11 of the smallest value)."""
    import numpy as np
    import kv4_common as K
    rng = np.random.default_rng(0)
    for scale in (1e-3, 1.0, 300.0):
        x = (rng.standard_normal((40, 2, 128)) * scale).astype(np.float16).astype(np.float64)
        c, s, o = K.quantise(x)
        assert c.min() == 0 and c.max() == 15
        low = np.abs(x.reshape(40, 2, 2, 64).min(-1))
        off = np.abs(K.values(c, s, o) - x).reshape(40, 2, 2, 64).max(-1)
        assert np.all(off <= s / 2 + 15 * s * 2.0 ** -11 + 2.0 ** -11 * low + 2.0 ** -24)
    c, s, o = K.quantise(np.full((1, 64), 1.5))
    assert not c.any() and not s.any() and np.all(o == 1.5)
