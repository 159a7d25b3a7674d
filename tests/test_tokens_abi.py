"""Projections, attention and dropout without a GPU: their structs match the header, NULL
handles and parameters are refused, and so are tensors that are not on the handle's device
or do not fit each other, before anything reaches the library."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


@pytest.fixture(scope="module")
def ifvs():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs as mod
    return mod


def test_structs_match_the_header(ifvs, tmp_path):
    structs = {"ifvs_linear_params": ifvs.LinearParams, "ifvs_attend_params": ifvs.AttendParams}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ifvs.h"', "int main(void) {"]
    want = [ifvs.IFVS_ACT_NONE]
    lines.append('printf("%d\\n", (int)IFVS_ACT_NONE);')
    for name, cls in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, f))
            want.append(getattr(cls, f).offset)
    lines.append("return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c99", "-I", inc, "-o", str(exe), str(src)])
    assert [int(v) for v in subprocess.check_output([str(exe)], text=True).split()] == want


def test_null_handles_are_refused(ifvs):
    L, p, a = ifvs.lib(), ifvs.LinearParams(), ifvs.AttendParams()
    assert L.ifvs_linear(None, ctypes.byref(p), 16, None, 16) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_linear_grad(None, ctypes.byref(p), 16, 16, 16, 16, None) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_attend(None, ctypes.byref(a), 16, 16, 16, 16, None) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_attend_grad(None, ctypes.byref(a), *[16] * 9) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_dropout(None, 16, None, 4, 0, 0.5, 1, 2, None, 16, None) == ifvs.IFVS_ERR_ARG


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, at, shape, dtype=BF):
        self.at, self.shape, self.dtype = at, shape, dtype
        self.device = torch.device("cuda", at) if at >= 0 else torch.device("cpu")

    def get_device(self):
        return self.at

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for v in self.shape:
            n *= v
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


T, TK, I, O, H, HK, D, B = 6, 9, 16, 24, 4, 2, 8, 2
LINEAR = [("x", (T, I), BF), ("w", (O, I), BF), ("bias", (O,), BF)]
ATTEND = [("q", (T, H, D), BF), ("k", (TK, HK, D), BF), ("v", (TK, HK, D), BF), ("q_offsets", (B + 1,), I64), ("kv_offsets", (B + 1,), I64),
          ("kv_ids", (TK,), I32), ("out", (T, H, D), BF), ("lse", (T, H), F32)]
CALLS = {"linear": LINEAR + [("residual", (T, O), BF), ("y", (T, O), BF)],
         "linear_grad": LINEAR + [("dy", (T, O), BF), ("dx", (T, I), BF), ("d_w", (O, I), BF), ("d_bias", (O,), BF)],
         "attend": ATTEND,
         "attend_grad": ATTEND + [("d_out", (T, H, D), BF), ("dq", (T, H, D), BF), ("dk", (TK, HK, D), BF), ("dv", (TK, HK, D), BF)],
         "dropout": [("x", (T, I), F32), ("residual", (T, I), F32), ("out", (T, I), F32), ("step", (1,), I64)]}


def _call(ifvs, name, change=None):
    """The call with stand-ins on device 1, one of them changed: (name, device, shape, type)"""
    h = ifvs._LayersHandle()        # NULL: the library answers IFVS_ERR_ARG
    h.device = 1
    kw = {n: Tensor(1, shape, dt) for n, shape, dt in CALLS[name]}
    if change:
        kw[change[0]] = Tensor(*change[1:])
    if name == "dropout":
        kw.update(p=0.5, seed=1)
    return getattr(ifvs, "ifvs_" + name)(h, stream=1, **kw)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_of_another_device_are_refused(ifvs, name):
    with pytest.raises(ifvs.IfvsError):
        _call(ifvs, name)
    for n, shape, dt in CALLS[name]:
        for at in (0, -1):
            with pytest.raises(ValueError, match=n):
                _call(ifvs, name, (n, at, shape, dt))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_that_do_not_fit_are_refused(ifvs, name):
    for n, shape, dt in CALLS[name]:
        with pytest.raises((TypeError, ValueError)):
            _call(ifvs, name, (n, 1, shape, torch.float64))
        for i in range(len(shape)):
            wrong = tuple(v + 1 if i == j else v for j, v in enumerate(shape))
            with pytest.raises(ValueError):
                _call(ifvs, name, (n, 1, wrong, dt))
