"""Tiles that leave shared memory by TMA are read there after the instruction that stores
them: a kernel's last stores have to be waited for before its CTA may end, or the memory's
next owner can overwrite them.  Read from the sources, since no run on a GPU shows it for
certain."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22922_gb300", "csrc")
STORE = re.compile(r"\btma_store(_heads)?\(|\bo\.store\(lane")       # the second: OutTile's


def _kernels(text):
    """name, body of every __global__ function that has one"""
    for m in re.finditer(r"__global__[^;{]*?\b(k_\w+)\s*\(", text):
        at = text.find("{", m.end())
        if ";" in text[m.end():at]:
            continue
        depth, end = 1, at + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield m.group(1), text[at:end]


def test_last_stores_are_waited_for():
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        with open(path) as f:
            text = f.read()
        for name, body in _kernels(text):
            stores = [m.start() for m in STORE.finditer(body)]
            if not stores:
                continue
            found.append(name)
            assert body.find("tma_wait_all()", stores[-1]) > 0, "%s in %s" % (name, os.path.basename(path))
    assert {"k_linear", "k_products", "k_attend_short", "k_grad_short"} <= set(found)


def test_every_store_is_looked_at():
    """Bulk stores are written out in two functions, which the kernels above call."""
    places = []
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        with open(path) as f:
            places += [os.path.basename(path)] * len(re.findall(r"global\.shared::cta[.\w]*bulk_group", f.read()))
    assert sorted(places) == ["attend_tc.cuh", "umma.cuh"]
