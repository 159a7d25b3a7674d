"""The encoder's layers without a GPU: their structs match the header, and
creating a handle says that there is no device."""
import ctypes
import os
import subprocess

import pytest


@pytest.fixture(scope="module")
def ifvs():
    from paper_2607_22922_gb300 import build
    build.build()
    from paper_2607_22922_gb300 import ifvs as mod
    return mod


def test_layer_structs_match_the_header(ifvs, tmp_path):
    structs = {"ifvs_join_params": ifvs.JoinParams, "ifvs_ffn_params": ifvs.FfnParams}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ifvs.h"', "int main(void) {"]
    want = []
    for name, cls in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, f))
            want.append(getattr(cls, f).offset)
    for c in ("IFVS_T_F32", "IFVS_T_F16", "IFVS_T_BF16", "IFVS_ACT_SILU", "IFVS_ACT_GELU", "IFVS_ACT_RELU"):
        lines.append('printf("%%d\\n", (int)%s);' % c)
        want.append(getattr(ifvs, c))
    lines.append("return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c99", "-I", inc, "-o", str(exe), str(src)])
    assert [int(v) for v in subprocess.check_output([str(exe)], text=True).split()] == want


def test_null_handles_are_refused(ifvs):
    L = ifvs.lib()
    assert L.ifvs_layers_create(None, 0) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_embed(None, 16, 4, 8, 0, 16, 1, 1.0, 16, None) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_embed_grad(None, 16, 16, 1, 4, 8, 0, 1.0, 16, None) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_norm_join(None, None, 16, 16, 16, 16) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_norm_join_grad(*[None] * 11) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_ffn(None, None, 16, 16) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_ffn_grad(*[None] * 7) == ifvs.IFVS_ERR_ARG
    assert L.ifvs_layers_status(None) == ifvs.IFVS_ERR_ARG
    L.ifvs_layers_free(None)


@pytest.mark.skipif(os.path.exists("/dev/nvidia0"), reason="only meaningful without a GPU")
def test_no_device_is_reported(ifvs):
    with pytest.raises(ifvs.IfvsError) as e:
        ifvs.Layers()
    assert e.value.code == ifvs.IFVS_ERR_CUDA
