"""The binding holds row arguments to the plan's tokens and the cache's heads before the library is called (with a stand-in for the
library and for device tensors: nothing here needs a device)."""
import pytest
import torch


class Rows:
    """What the binding looks at of a device tensor."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float16, strides=None, device=0):
        self.shape, self.dtype, self._device = torch.Size(shape), dtype, device
        self._strides = strides or torch.empty(shape, device="meta").stride()

    def stride(self):
        return self._strides

    def is_contiguous(self):
        return self._strides == torch.empty(self.shape, device="meta").stride()

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 4096


@pytest.fixture
def calls(monkeypatch):
    from paper_2602_18447_b200 import binding as B
    seen, handles = [], iter(range(1000, 2000))

    class Library:
        def __getattr__(self, name):
            def call(*args):
                seen.append(name)
                out = args[-1]
                if name.endswith(("alloc", "alloc_4bit", "alloc_8bit", "create", "load")):
                    out._obj.value = next(handles)
                return B.CS_OK
            return call

    monkeypatch.setattr(B, "load_library", lambda path=None: Library())
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_heads", {7: (4, 2, 128)})             # the model
    monkeypatch.setattr(B, "_plan_rows", {})
    kv = B.cs_kv_alloc_4bit(7, 8, 16, 2, 4)
    plan = B.cs_plan_create(kv)
    return B, kv, plan, seen


def _q(n=3, h=4, d=128, **kw):
    return Rows(n, h, d, **kw)


def _kv(n=3, h=2, d=128, **kw):
    return Rows(n, h, d, **kw)


def test_rows_of_the_plan_pass(calls):
    B, kv, plan, seen = calls
    B.cs_plan_set(plan, [0, 1], [1, 2])
    B.cs_kv_append(plan, 0, _kv(), _kv(), q=_q(), q_out=_q())
    B.cs_attention_4bit(plan, 0, Rows(3, 512), Rows(3, 512), Rows(3, 256), Rows(3, 256))
    fused = dict(strides=(8 * 128, 128, 1))
    B.cs_kv_append(plan, 0, _kv(**fused), _kv(**fused), q=_q(**fused), q_out=_q(**fused))
    B.cs_kv_read(kv, 0, Rows(5, dtype=torch.int32), Rows(5, dtype=torch.int32), _kv(5), _kv(5))
    B.cs_plan_set(plan, [], [])
    B.cs_kv_append(plan, 0, _kv(0), _kv(0))
    assert seen[-6:] == ["cs_kv_append", "cs_attention_4bit", "cs_kv_append", "cs_kv_read", "cs_plan_set", "cs_kv_append"]


@pytest.mark.parametrize("n", [1, 2, 4, 40])
def test_a_row_for_every_token_of_the_plan(calls, n):
    B, kv, plan, seen = calls
    B.cs_plan_set(plan, [0, 1], [1, 2])
    del seen[:]
    for call in (lambda: B.cs_kv_append(plan, 0, _kv(n), _kv(n)), lambda: B.cs_attention_4bit(plan, 0, _q(n), _q(n)),
                 lambda: B.cs_attention_4bit(plan, 0, _q(n), _q(n), _kv(n), _kv(n)),
                 lambda: B.cs_kv_append(plan, 0, _kv(), _kv(), q=_q(n), q_out=_q(n)),
                 lambda: B.cs_kv_read(kv, 0, Rows(3, dtype=torch.int32), Rows(3, dtype=torch.int32), _kv(n), _kv(n))):
        with pytest.raises(ValueError):
            call()
    assert not seen
    B.cs_plan_set(plan, [0], [n])                       # the last batch counts
    B.cs_kv_append(plan, 0, _kv(n), _kv(n))
    with pytest.raises(ValueError):
        B.cs_kv_append(plan, 0, _kv(), _kv())


@pytest.mark.parametrize("rows", [(2, 64), (1, 128), (3, 128), (4, 128), (2, 256)])
@pytest.mark.parametrize("n", [1, 3])
def test_the_heads_of_the_cache(calls, n, rows):
    """A single row that is a slice of a wider matrix is no exception."""
    B, kv, plan, seen = calls
    B.cs_plan_set(plan, [0], [n])
    del seen[:]
    h, d = rows
    wide = dict(strides=(4096, d, 1))
    for bad in (_kv(n, h, d), _kv(n, h, d, **wide), Rows(n, h * d, strides=(4096, 1))):
        if h * d == 256 and len(bad.shape) == 2:
            continue
        for call in (lambda: B.cs_kv_append(plan, 0, bad, bad), lambda: B.cs_kv_append(plan, 0, _kv(n), bad),
                     lambda: B.cs_attention_4bit(plan, 0, _q(n), _q(n), bad, bad),
                     lambda: B.cs_kv_read(kv, 0, Rows(n, dtype=torch.int32), Rows(n, dtype=torch.int32), bad, bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (_q(n, 2), _q(n, 4, 64), _q(n, 6)):
        for call in (lambda: B.cs_attention_4bit(plan, 0, bad, bad), lambda: B.cs_attention_4bit(plan, 0, _q(n), bad),
                     lambda: B.cs_kv_append(plan, 0, _kv(n), _kv(n), q=bad, q_out=bad)):
            with pytest.raises(ValueError):
                call()
    assert not seen


def test_places_and_rows_of_another_device(calls):
    B, kv, plan, seen = calls
    B.cs_plan_set(plan, [0], [3])
    del seen[:]
    here, there = Rows(3, dtype=torch.int32), Rows(3, dtype=torch.int32, device=1)
    for args in ((there, there, _kv(), _kv()), (here, there, _kv(), _kv()), (here, here, _kv(device=1), _kv(device=1)),
                 (here, here, _kv(), _kv(device=1))):
        with pytest.raises(ValueError):
            B.cs_kv_read(kv, 0, *args)
    with pytest.raises(ValueError):
        B.cs_kv_append(plan, 0, _kv(device=1), _kv(device=1))
    assert not seen


def test_handles_that_are_gone(calls):
    B, kv, plan, seen = calls
    B.cs_plan_set(plan, [0], [3])
    B.cs_plan_free(plan)
    with pytest.raises(ValueError):
        B.cs_kv_append(plan, 0, _kv(), _kv())
    B.cs_kv_free(kv)
    with pytest.raises(ValueError):
        B.cs_kv_read(kv, 0, Rows(3, dtype=torch.int32), Rows(3, dtype=torch.int32), _kv(), _kv())


def test_rows_that_a_kernel_may_have_written_are_read_by_ordinary_loads():
    """The kernels on cache rows start beside their predecessor: read-only loads are for what copies have brought."""
    import os
    import re
    from paper_2602_18447_b200 import build
    text = open(os.path.join(build.CSRC, "kv_rows.cu")).read()
    code = re.sub(r"//.*", "", text)
    assert all(re.match(r"(p\.)?(table|pages|n_pages)\b|static_cast", arg) for arg in re.findall(r"__ldg\(([^,;]*)", code)), re.findall(r"__ldg\(([^,;]*)", code)
    assert not re.findall(r"const uint8_t\s*\*\s*__restrict__|const uint16_t\s*\*\s*__restrict__|const float2\s*\*\s*__restrict__", code)
