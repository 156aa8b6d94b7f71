"""Refusals, states and plans of the layer-wise calls and of the adjusted logits,
checked without a GPU: the library's own host code over recording stand-ins
(tests/layer_path.cpp). Device addresses are never read."""
import ctypes
import os
import subprocess

import pytest

from paper_2601_08670_amd import _lib
from tests.test_host_path import CSRC, DEVICE, ROOT, Batch

OK, INVALID, CAPACITY, HIPERR, UNSUPPORTED, STATE = 0, 1, 2, 3, 4, 5
P = ctypes.c_void_p
Q, K, V, X = (DEVICE + (i << 34) for i in range(1, 5))  # far apart


@pytest.fixture(scope="session")
def layer_host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("layer_path") / "layer_path.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    os.path.join(ROOT, "tests", "layer_path.cpp"), os.path.join(CSRC, "pced_api.cpp"),
                    os.path.join(CSRC, "pced_layer_api.cpp"), "-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", out],
                   check=True)
    lib = ctypes.CDLL(out)
    lib.rec_name.restype = ctypes.c_char_p
    lib.rec_value.restype = ctypes.c_long
    lib.pced_workspace_bytes.restype = lib.pced_summary_bytes.restype = ctypes.c_size_t
    lib.pced_last_error.restype = ctypes.c_char_p
    return lib


class Layers(Batch):
    def append(self, n=1, layer=0, layers=None, rows=None, rope=(10000.0, 128, 0), q_out=X):
        self.lib.rec_clear()
        rows = _lib.pced_rows(**(rows if rows is not None else dict(q=Q, k=K, v=V)))
        rope = None if rope is None else ctypes.byref(_lib.pced_rope(*rope))
        return self.lib.pced_append(self.ctx, layer, self.layers if layers is None else layers, n, ctypes.byref(rows),
                                    rope, P(q_out), None)

    def attend(self, n=1, sel=(4, 1, 1), layer=0, layers=None, q=Q, x=X, pages=None):
        self.lib.rec_clear()
        sel = None if sel is None else ctypes.byref(_lib.pced_select(*sel))
        return self.lib.pced_attend(self.ctx, layer, self.layers if layers is None else layers, n, P(q), sel, P(x),
                                    P(pages), None)

    def bind(self, at=DEVICE):
        return self.lib.pced_bind_summary(self.ctx, P(at))

    def summarize(self):
        self.lib.rec_clear()
        return self.lib.pced_summarize(self.ctx, None)

    def advance(self, n=1):
        return self.lib.pced_advance(self.ctx, n)

    def lengths(self):
        out = (ctypes.c_int32 * len(self.lens))()
        assert self.lib.pced_get_lengths(self.ctx, out, len(self.lens)) == OK
        return list(out)

    def nothing_launched(self):
        return self.lib.rec_count() == 0


def test_before_load(layer_host):
    b = Layers(layer_host, [16, 40], 64)
    fresh = ctypes.c_void_p()
    ws = layer_host.pced_workspace_bytes(ctypes.byref(b.cfg))
    assert layer_host.pced_create(ctypes.byref(b.cfg), P(DEVICE), ctypes.c_size_t(ws), ctypes.byref(fresh)) == OK
    b.ctx, old = fresh, b.ctx
    adj, out = _lib.pced_adjust(), P(X)
    assert b.append() == b.attend() == b.summarize() == b.advance() == STATE
    assert layer_host.pced_adjust_logits(b.ctx, P(Q), ctypes.byref(adj), out, None) == STATE
    assert layer_host.pced_fuse_adjusted(b.ctx, P(Q), 1, ctypes.byref(adj), out, None, None) == STATE
    assert b.bind() == OK
    layer_host.pced_destroy(old)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), INVALID), (dict(n=-3), INVALID), (dict(layer=-1), INVALID), (dict(layer=1, layers=2), INVALID),
    (dict(layers=0), INVALID), (dict(n=10 ** 6), CAPACITY), (dict(n=2 ** 31 - 1), CAPACITY), (dict(n=100), CAPACITY),
    (dict(rows=dict(q=Q, v=V)), INVALID), (dict(rows=dict(q=Q, k=K)), INVALID), (dict(rows=dict(k=K, v=V)), INVALID),
    (dict(q_out=None), INVALID), (dict(rows=dict(q=Q + 2, k=K, v=V)), INVALID), (dict(rows=dict(q=Q, k=K + 8, v=V)), INVALID),
    (dict(q_out=X + 4), INVALID), (dict(rows=dict(q=Q, k=K, v=V, v_row=2 * 8 * 128 + 4)), INVALID),
    (dict(rows=dict(q=Q, k=K, v=V, k_row=8 * 128)), INVALID), (dict(rows=dict(q=Q, k=K, v=V, q_row=-8192)), INVALID),
    (dict(rope=(1.0, 128, 0)), INVALID), (dict(rope=(float("nan"), 128, 0)), INVALID),
    (dict(rope=(float("inf"), 128, 0)), INVALID), (dict(rope=(1e4, 129, 0)), INVALID), (dict(rope=(1e4, 130, 0)), INVALID),
    (dict(rope=(1e4, -2, 0)), INVALID), (dict(rope=(1e4, 24, 1)), INVALID), (dict(rope=(1e4, 32, 2)), INVALID),
    (dict(q_out=Q + 8192), INVALID), (dict(q_out=K), INVALID),
    (dict(q_out=Q, rows=dict(q=Q, k=K, v=V, q_row=3 * 8192)), INVALID),
])
def test_append_refusals(layer_host, kw, status):
    b = Layers(layer_host, [16, 40], 64, n_layers=2)
    assert b.append(**kw) == status, b.error()
    assert b.error() and b.nothing_launched()
    assert b.advance() == STATE and b.lengths() == [16, 40]


def test_append_takes(layer_host):
    b = Layers(layer_host, [16, 40], 64, n_layers=2)
    assert b.append() == OK and b.calls("append_rows")[0][:7] == [0, 2, 1, 1, 0, 0, 2 * 32 * 128]
    assert b.append(q_out=Q) == OK                                   # in place
    assert b.append(rope=None) == OK and b.append(rope=(1e4, 0, 1)) == OK and b.append(rope=(1e4, 22, 0)) == OK
    assert b.append(rows=dict(k=K, v=V, q_row=-5), q_out=None) == OK  # (no q rows: no distance)
    assert b.append(rows=dict(k=K, v=V), q_out=None, n=40) == OK and b.calls("append_rows")[0][3] == 3  # tokens 16 .. 55 and 40 .. 79
    fused = dict(q=Q, k=Q + 4096 * 2, v=Q + 5120 * 2, q_row=6144, k_row=6144, v_row=6144)
    assert b.append(layers=1, rows=fused) == OK
    assert b.lengths() == [16, 40]


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), INVALID), (dict(layer=2), INVALID), (dict(layers=3), INVALID), (dict(q=None), INVALID), (dict(x=None), INVALID),
    (dict(q=Q + 8), INVALID), (dict(x=X + 2), INVALID), (dict(sel=None, pages=K), INVALID), (dict(sel=(4, -1, 1)), INVALID),
    (dict(sel=(4, 0, 0)), INVALID), (dict(sel=(4, 2, 3)), INVALID), (dict(sel=(0, 0, 1)), INVALID),
    (dict(sel=(2 ** 30 + 1, 0, 1)), INVALID), (dict(sel=(-5, 0, 1)), INVALID),
    (dict(sel=(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)), INVALID), (dict(x=Q), INVALID),
    (dict(x=Q + 1024), INVALID), (dict(n=2), STATE), (dict(sel=(2, 0, 1)), STATE), (dict(n=1000), CAPACITY),
])
def test_attend_refusals(layer_host, kw, status):
    b = Layers(layer_host, [16, 40], 64, n_layers=2)
    assert b.append() == OK
    assert b.attend(**kw) == status, b.error()
    assert b.error() and b.nothing_launched()


def test_layer_by_layer(layer_host):
    b = Layers(layer_host, [16, 40], 64, n_layers=2)
    assert b.attend(layers=1) == STATE                # nothing appended
    assert b.append(layers=1, n=3) == OK
    assert b.attend(layers=1, n=3) == OK and b.attend(layers=1, n=2) == OK
    assert b.attend(layer=1, layers=1) == STATE and b.attend(n=3) == STATE and b.advance(1) == STATE
    assert b.append(layer=1, layers=1, n=3) == OK and b.attend(n=3) == OK
    assert b.advance(4) == STATE and b.advance(0) == INVALID and b.advance(2) == OK and b.lengths() == [18, 42]
    assert b.attend() == STATE and b.advance() == STATE
    assert b.append() == OK and b.calls("append_rows")[0][5] == 2    # positions from the new lengths


def test_summaries_follow_the_calls(layer_host):
    b = Layers(layer_host, [30, 200], 200, n_layers=2)
    few = (3, 1, 1)
    assert b.append() == OK and b.attend(sel=few) == STATE and b.summarize() == STATE
    assert b.bind(DEVICE + 16) == INVALID and b.bind() == OK
    assert b.append() == OK and b.calls("append_rows")[0][4] == 0 and b.attend(sel=few) == STATE
    assert b.summarize() == OK and b.calls("summarize")[0][0] == 200 // 16
    assert b.attend(sel=few) == STATE                 # (appended before the summaries were up to date)
    assert b.append(n=20) == OK and b.calls("append_rows")[0][4] == 1 and b.attend(sel=few, n=20) == OK
    assert [r[4] for r in b.calls("select")] == [1]
    assert b.attend(sel=(14, 1, 1), n=20) == OK and not b.calls("select")     # every page: nothing to choose
    assert b.attend(sel=(14, 1, 1), n=20, pages=V) == OK and b.calls("select")[0][4] == 0
    assert b.advance(6) == OK and b.append() == OK and b.calls("append_rows")[0][4] == 1 and b.advance() == OK
    assert b.step() == OK                             # a token that the summaries do not know of
    assert b.append() == OK and b.calls("append_rows")[0][4] == 0 and b.attend(sel=few) == STATE
    assert b.summarize() == OK and b.calls("summarize")[0][:2] == [1, 1]   # 208 tokens: a page is full
    assert b.append(layers=1) == OK and b.append(layer=1, layers=1) == OK and b.attend(sel=few) == OK
    assert b.load(200) == OK and b.append() == OK and b.attend(sel=few) == STATE
    assert b.summarize() == OK and b.append() == OK and b.attend(sel=few) == OK
    assert b.bind(None) == OK and b.attend(sel=few) == STATE and b.summarize() == STATE


@pytest.mark.parametrize("lens,n,sel,kw", [
    ([16, 40], 1, (2, 0, 1), {}), ([1, 100000], 1, (64, 1, 1), {}), ([1] * 60 + [30000], 40, None, {}),
    ([5000] * 4, 200, (3, 1, 1), dict(n_layers=3)), ([20, 17], 17, (1, 0, 1), dict(n_q_heads=1, n_kv_heads=1, head_dim=4, dtype="f32")),
    ([2000, 70], 30, (50, 2, 3), dict(n_q_heads=16, n_kv_heads=16, head_dim=64)),
    ([160, 70], 9, (5, 1, 1), dict(n_q_heads=5, n_kv_heads=5, head_dim=80, dtype="f32", n_layers=7)),
])
def test_launches_cover_every_row_once_within_the_workspace(layer_host, lens, n, sel, kw):
    b = Layers(layer_host, lens, n, **kw)
    assert b.status == OK and b.bind() == OK and b.summarize() == OK and b.append(n, rope=None) == OK
    assert b.attend(n, sel) == OK, b.error()
    layers = b.layers
    seen = set()
    start = DEVICE
    end = DEVICE + layer_host.pced_workspace_bytes(ctypes.byref(b.cfg))
    for l, nl, g, ng, parts, part_pages, last, first in b.calls("attend"):
        for i in range(l, l + nl):
            for j in range(g, g + ng):
                assert (i, j) not in seen
                seen.add((i, j))
        assert start <= first <= last <= end
        want = -(-(max(lens) + n) // 16)
        assert parts * part_pages >= min(want, sel[0] if sel else want)
    groups = len({j for _, j in seen})   # of up to some number of tokens of a sequence
    assert seen == {(i, j) for i in range(layers) for j in range(groups)}
    assert groups % len(lens) == 0 and groups // len(lens) <= n


def test_adjust_refusals(layer_host):
    b = Layers(layer_host, [16, 40, 7], 64)
    lib = layer_host
    logits, out, dev = P(Q), P(X), DEVICE
    run = lambda a, x=logits, y=out: lib.pced_adjust_logits(b.ctx, x, a and ctypes.byref(a), y, None)  # noqa: E731
    fuse = lambda a, x=logits, y=out, fresh=1: lib.pced_fuse_adjusted(  # noqa: E731
        b.ctx, x, fresh, a and ctypes.byref(a), y, None, None)
    lib.rec_clear()
    good = _lib.pced_adjust()
    for call in (run, fuse):
        assert call(None) == INVALID and call(good, None) == INVALID and call(good, logits, None) == INVALID
        for bad in (dict(n_history=-1), dict(n_bias=-1), dict(history=dev, history_off=dev, n_history=2 ** 31 - 1),
                    dict(n_bias=2 ** 30 + 1), dict(history=dev, n_history=3), dict(mask=dev, mask_row=31),
                    dict(bias_token=dev, bias_value=dev), dict(bias_token=dev, bias_off=dev), dict(mask=dev, mask_row=-32)):
            assert call(_lib.pced_adjust(**bad)) == INVALID, bad
    assert run(good, logits, P(Q + 4000)) == INVALID           # partly itself
    assert fuse(good, fresh=0) == STATE                        # dynamic beta, not known yet
    assert lib.rec_count() == 0
    assert run(good) == run(good, logits, logits) == OK        # in place
    assert run(_lib.pced_adjust(mask=dev)) == OK and b.calls("adjust")[-1][:2] == [3, 32]
    assert fuse(good) == fuse(good, fresh=0) == OK and len(b.calls("beta")) == 1
    moe = Layers(layer_host, [16, 40, 7], 64, aggregation="moe")
    assert lib.pced_fuse_adjusted(moe.ctx, logits, 1, ctypes.byref(good), out, None, None) == UNSUPPORTED
    assert lib.pced_adjust_logits(moe.ctx, logits, ctypes.byref(good), out, None) == OK


def test_launch_failures_are_reported(layer_host):
    b = Layers(layer_host, [16, 40], 64)
    layer_host.rec_fail(b"append_rows", 1)
    assert b.append() == HIPERR and b.advance() == STATE
    assert b.append() == OK
    layer_host.rec_fail(b"attend", 1)
    assert b.attend() == HIPERR and b.attend() == OK


def test_summary_bytes():
    c = _lib.make_config(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=100, dtype="bf16", max_queries=1,
                         max_seqs=4, max_pages=33, max_pages_per_seq=8)
    assert _lib.pced_summary_bytes(c) == -(-2 * 2 * 33 * 128 // 256) * 256 + -(-2 * 2 * 33 * 4 // 256) * 256
    c.n_layers = 0
    assert _lib.pced_summary_bytes(c) == 0


@pytest.mark.parametrize("struct,names", [
    (_lib.pced_rope, ("theta", "rot_dim", "halves")), (_lib.pced_rows, ("q", "k", "v", "q_row", "k_row", "v_row")),
    (_lib.pced_select, ("n_pages", "n_first", "n_last")),
    (_lib.pced_adjust, ("history", "history_off", "repetition", "presence", "frequency", "bias_token", "bias_value",
                        "bias_off", "mask", "mask_row", "n_history", "n_bias"))])
def test_structs_match_the_header(tmp_path, struct, names):
    name = struct.__name__
    src = tmp_path / "s.cpp"
    src.write_text('#include "pced.h"\n#include <cstdio>\nint main() { printf("%zu", sizeof(' + name + "));\n" + "".join(
        f'printf(" %zu", offsetof({name}, {n}));\n' for n in names) + "}\n")
    exe = str(tmp_path / "s")
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), str(src),
                    "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(struct)] + [getattr(struct, n).offset for n in names]


def test_calls_from_another_device_are_refused(monkeypatch):
    import torch

    from paper_2601_08670_amd.session import PcedSession
    s = object.__new__(PcedSession)
    s._device_index, s.k_pool = 0, torch.empty(0)
    monkeypatch.setattr(_lib, "current_device", lambda: 1)
    for call in (lambda: s.append(None, None, None), lambda: s.attend(None), lambda: s.summarize(),
                 lambda: s.adjust_logits(None, None), lambda: s.fuse_adjusted(None, None)):
        with pytest.raises(ValueError, match="current device"):
            call()
