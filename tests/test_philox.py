"""The random words of dropout without a GPU: csrc/philox.h, compiled for the host,
against the generator's published answers and against Python's whole numbers."""
import os
import subprocess

import pytest

pytest.importorskip("torch")
import tokens_util as ref  # noqa: E402

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22922_gb300", "csrc")
# counter (block, step), key, words: the known answers that the generator's authors give
KNOWN = [(0, 0, 0, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
         (2**64 - 1, 2**64 - 1, 2**64 - 1, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
         (0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822, "d16cfe09 94fdcceb 5001e420 24126ea1")]


def test_words(tmp_path):
    src, exe = tmp_path / "w.cpp", tmp_path / "w"
    src.write_text('#include <stdio.h>\n#include <stdlib.h>\n#include "philox.h"\nint main(int n, char** a) {\n'
                   "  for (int i = 1; i + 2 < n; i += 3) {\n"
                   "    unsigned long long b = strtoull(a[i], 0, 10), s = strtoull(a[i + 1], 0, 10);\n"
                   "    ifvs::Words w = ifvs::philox((uint32_t)b, (uint32_t)(b >> 32), s, ifvs::round_keys(strtoull(a[i + 2], 0, 10)));\n"
                   '    printf("%08x %08x %08x %08x\\n", w.w[0], w.w[1], w.w[2], w.w[3]);\n  }\n  return 0;\n}\n')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)])
    asked = [k[:3] for k in KNOWN] + [(i * 0x9E3779B97F4A7C15 % 2**64, i, 2**63 + i) for i in range(50)]
    got = subprocess.check_output([str(exe)] + [str(v) for a in asked for v in a], text=True).splitlines()
    assert got[:3] == [k[3] for k in KNOWN]
    for (block, step, seed), line in zip(asked, got):
        assert line == "%08x %08x %08x %08x" % tuple(ref.philox(block, step, seed))
    assert ref.words(6, 7, 5, 4).tolist() == (ref.philox(1, 5, 4) + ref.philox(2, 5, 4) + ref.philox(3, 5, 4))[2:9]
