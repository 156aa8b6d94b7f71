"""How pced_attend divides its work when the workspace does not hold it at once: the library's host code over
stand-ins that record what every launch uses (tests/layer_room.cpp). Device addresses are never read."""
import ctypes
import os
import subprocess

import pytest

from paper_2601_08670_amd import _lib
from tests.test_host_path import CSRC, ROOT
from tests.test_layer_path import OK, Layers

# What is divided: (name, dtype, heads, layers, lengths, new tokens, (pages, first, last) or None, pages wanted; how many
# first layers and first token groups the launches have, at least). tests/test_gpu_layer_room.py runs them.
SPLITS = [
    ("one_token_in_one_launch", "f32", (2, 2, 4), 8, [6400] + [5] * 149, 1, (200, 1, 1), False, 2, 1),
    ("one_token_in_parts", "f32", (2, 2, 4), 8, [6400] + [5] * 199, 1, (300, 1, 1), False, 2, 1),
    ("one_token_long", "f32", (2, 2, 4), 12, [9000] + [5] * 149, 1, (300, 1, 1), False, 2, 1),
    ("tokens", "f32", (2, 2, 4), 3, [400, 300, 7], 150, (20, 1, 1), False, 3, 4),
    ("tokens_pages", "f32", (4, 2, 4), 1, [700, 90], 400, (30, 1, 2), True, 1, 2),
    ("tokens_long", "f32", (2, 1, 8), 1, [9000, 8500], 203, (40, 2, 3), False, 1, 2),
    ("tokens_all_pages", "f32", (16, 1, 128), 1, [4000, 3000], 130, None, False, 1, 2),
    ("bf16_layers", "bf16", (4, 4, 64), 12, [2000] + [40] * 9, 60, (100, 1, 1), False, 2, 1),
    ("bf16_tokens", "bf16", (4, 4, 64), 2, [2000] + [40] * 3, 300, (100, 1, 1), False, 2, 2),
    ("bf16_tokens_pages", "bf16", (4, 4, 64), 2, [2000] + [40] * 3, 300, (100, 1, 1), True, 2, 1),
]


@pytest.fixture(scope="session")
def room_host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("layer_room") / "layer_room.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    os.path.join(ROOT, "tests", "layer_room.cpp"), os.path.join(CSRC, "pced_api.cpp"),
                    os.path.join(CSRC, "pced_layer_api.cpp"), "-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", out],
                   check=True)
    lib = ctypes.CDLL(out)
    lib.rec_name.restype = ctypes.c_char_p
    lib.rec_value.restype = lib.room_begin.restype = lib.room_end.restype = lib.next_region.restype = ctypes.c_long
    lib.pced_workspace_bytes.restype = lib.pced_summary_bytes.restype = ctypes.c_size_t
    lib.pced_last_error.restype = ctypes.c_char_p
    return lib


def _plan(lib, dtype, heads, layers, lens, n, sel, pages):
    """(context, attend launches, regions that each launch's choice and attention use)"""
    b = Layers(lib, lens, n, dtype=dtype, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2], n_layers=layers)
    assert b.status == OK and b.bind() == OK and b.summarize() == OK and b.append(n, rope=None) == OK
    assert b.attend(n, sel, pages=1 << 47 if pages else None) == OK, b.error()
    launches, uses, choice = [], [], []
    for i in range(lib.rec_count()):
        name, v = lib.rec_name(i).decode(), [lib.rec_value(i, j) for j in range(8)]
        if name == "choice":
            where, choice = v[:4], []
        elif name in ("scores", "list"):
            choice.append((name, v[0], v[1]))
        elif name == "attend":
            assert not choice or where == v[:4]
            launches.append(v)
            uses.append(choice)
            choice = []
        else:
            assert name in ("acc", "ml")
            uses[-1].append((name, v[0], v[1]))
    return b, launches, uses


def _check(lib, case):
    name, dtype, heads, layers, lens, n, sel, pages, by_layer, by_group = case
    b, launches, uses = _plan(lib, dtype, heads, layers, lens, n, sel, pages)
    begin, end = lib.room_begin(b.ctx), lib.room_end(b.ctx)
    assert begin < end <= lib.next_region(b.ctx)
    seen = set()
    longest = -(-(max(lens) + n) // 16)
    for v, used in zip(launches, uses):
        l, nl, g, ng, parts, part_pages, pick, gt = v
        assert nl >= 1 and ng >= 1 and part_pages <= 256
        cells = {(i, j) for i in range(l, l + nl) for j in range(g, g + ng)}
        assert not cells & seen
        seen |= cells
        assert parts * part_pages >= min(longest, sel[0] if sel else longest)
        assert not pick or (n == 1 and parts == 1)
        for _, x, y in used:
            assert begin <= x < y <= end, (name, x - begin, y - begin, end - begin)
        spans = sorted((x, y) for _, x, y in used)
        assert all(a[1] <= c[0] for a, c in zip(spans, spans[1:])), (name, used)
        want = ({"list"} if sel and sel[0] < longest and not pages and not pick else set()) | ({"acc", "ml"} if parts > 1 else set())
        assert want <= {u for u, _, _ in used}, (name, used)
    groups = len(lens) * -(-n // 8)
    assert seen == {(i, j) for i in range(layers) for j in range(groups)}
    return launches


@pytest.mark.parametrize("case", SPLITS, ids=lambda c: c[0])
def test_split_launches(room_host, case):
    """Several launches, each within the region, no region twice in one launch, every row once."""
    launches = _check(room_host, case)
    assert len({v[0] for v in launches}) >= case[8] and len({v[2] for v in launches}) >= case[9], launches
    assert len(launches) > 1


@pytest.mark.parametrize("dtype,heads", [("f32", (1, 1, 4)), ("f32", (3, 3, 8)), ("f32", (16, 1, 20)), ("bf16", (4, 4, 64)),
                                         ("bf16", (32, 8, 128)), ("bf16", (16, 1, 128))])
@pytest.mark.parametrize("layers", [1, 7])
@pytest.mark.parametrize("lens,n", [([1, 1], 1), ([16, 15], 33), ([500] + [1] * 70, 1), ([3000, 20], 9), ([40000, 1], 64),
                                    ([200] * 40, 100)])
def test_every_size_fits(room_host, dtype, heads, layers, lens, n):
    longest = -(-(max(lens) + n) // 16)
    for sel in (None, (1, 0, 1), (2, 0, 1), (max(2, longest // 2), 1, 1), (max(2, longest - 1), 0, 1), (longest + 5, 3, 2)):
        for pages in (False, True) if sel else (False,):
            _check(room_host, ("", dtype, heads, layers, lens, n, sel, pages, 1, 1))
