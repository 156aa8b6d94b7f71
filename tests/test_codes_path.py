"""Refusals, states and plans of the calls on caches in 8 bits, checked without a GPU: the library's own host code over
recording stand-ins (tests/codes_path.cpp). Device addresses are never read."""
import ctypes
import os
import subprocess

import pytest

from paper_2601_08670_amd import _lib
from tests.test_host_path import CSRC, DEVICE, ROOT
from tests.test_layer_path import CAPACITY, HIPERR, INVALID, K, OK, P, Q, STATE, UNSUPPORTED, V, X, Layers

BUFFERS = ("k_codes", "v_codes", "scales", "k_open", "v_open")


@pytest.fixture(scope="session")
def codes_host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("codes_path") / "codes_path.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    os.path.join(ROOT, "tests", "codes_path.cpp")] +
                   [os.path.join(CSRC, f) for f in ("pced_api.cpp", "pced_layer_api.cpp", "pced_cache8_api.cpp")] +
                   ["-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.rec_name.restype = ctypes.c_char_p
    lib.rec_value.restype = lib.room_begin.restype = lib.room_end.restype = ctypes.c_long
    for f in ("pced_workspace_bytes", "pced_summary_bytes", "pced_codes_bytes", "pced_scales_bytes", "pced_open_bytes"):
        getattr(lib, f).restype = ctypes.c_size_t
    lib.pced_last_error.restype = ctypes.c_char_p
    return lib


class Codes(Layers):
    """A batch whose caches are in 8 bits (max_new = 64 unless given)."""

    def __init__(self, lib, lens, reserve, code=1, max_new=64, **kw):
        self.cache = dict(code=code, max_new=max_new, **{n: DEVICE + (40 + i << 40) for i, n in enumerate(BUFFERS)})
        super().__init__(lib, lens, reserve, **kw)

    def load(self, reserve, src=DEVICE, cache=(), struct=True):
        S = len(self.lens)
        ptrs = (ctypes.c_void_p * S)(*[src] * S)
        self.lib.rec_clear()
        c = ctypes.byref(_lib.pced_cache8(**dict(self.cache, **dict(cache)))) if struct else None
        return self.lib.pced_load_codes(self.ctx, 1, (ctypes.c_int32 * 1)(S - 1), (ctypes.c_int32 * S)(*self.lens), ptrs,
                                        ptrs, c, None, reserve, (ctypes.c_float * (S - 1))(*[0.5] * (S - 1)),
                                        ctypes.c_float(2.5), None, None)

    def pooled(self, reserve):
        return super().load(reserve)

    def append(self, n=1, layer=0, layers=None, rows=None, rope=(10000.0, 128, 0), q_out=X):
        self.lib.rec_clear()
        rows = _lib.pced_rows(**(rows if rows is not None else dict(q=Q, k=K, v=V)))
        rope = None if rope is None else ctypes.byref(_lib.pced_rope(*rope))
        return self.lib.pced_append_codes(self.ctx, layer, self.layers if layers is None else layers, n,
                                          ctypes.byref(rows), rope, P(q_out), None)

    def attend(self, n=1, layer=0, layers=None, q=Q, x=X):
        self.lib.rec_clear()
        return self.lib.pced_attend_codes(self.ctx, layer, self.layers if layers is None else layers, n, P(q), P(x), None)

    def read(self, seq=0, layer=0, start=0, count=1, k=K, v=V):
        self.lib.rec_clear()
        return self.lib.pced_read_codes(self.ctx, seq, layer, start, count, P(k), P(v), None)


def test_sizes():
    cfg = _lib.make_config(n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=100, dtype="bf16", max_queries=1,
                           max_seqs=5, max_pages=33, max_pages_per_seq=8)
    assert _lib.pced_codes_bytes(cfg) == 3 * 33 * 2 * 16 * 64 == _lib.pced_pool_bytes(cfg) // 2
    assert _lib.pced_scales_bytes(cfg) == 3 * 2 * 33 * 4
    tile = 2 * 16 * 64 * 2
    for n, ring in ((1, 1), (2, 2), (17, 2), (18, 3), (33, 3), (34, 4)):  # 16 k + 15 tokens, n more
        assert _lib.pced_open_bytes(cfg, n) == 3 * 5 * ring * tile, n
    assert _lib.pced_open_bytes(cfg, 0) == _lib.pced_open_bytes(cfg, -5) == 0
    f32 = _lib.make_config(n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=100, dtype="f32", max_queries=1,
                           max_seqs=5, max_pages=33, max_pages_per_seq=8)
    cfg.n_layers = 0
    for c in (cfg, f32):
        assert _lib.pced_codes_bytes(c) == _lib.pced_scales_bytes(c) == _lib.pced_open_bytes(c, 1) == 0


@pytest.mark.parametrize("cache,status", [
    (dict(code=0), INVALID), (dict(code=3), INVALID), (dict(code=-1), INVALID), (dict(max_new=0), INVALID),
    (dict(max_new=-7), INVALID), (dict(max_new=2 ** 31 - 1), INVALID), (dict(v_open=0), INVALID),
    (dict(scales=DEVICE + (50 << 40) + 128), INVALID), (dict(v_codes=DEVICE + (40 << 40)), INVALID),
    (dict(k_open=DEVICE + (42 << 40)), INVALID), (dict(scales=DEVICE + (40 << 40) + 256), INVALID),
] + [({n: 0}, INVALID) for n in BUFFERS])
def test_load_refusals(codes_host, cache, status):
    b = Codes(codes_host, [16, 40], 64)
    assert b.status == OK and b.append() == OK and b.advance() == OK
    assert b.load(64, cache=cache) == status, b.error()
    assert b.error() and b.nothing_launched()
    assert b.lengths() == [17, 41]


def test_load(codes_host):
    b = Codes(codes_host, [16, 40], 64, code=2, max_new=18)
    assert b.status == OK, b.error()
    assert b.calls("load_codes") == [[1 + 3, 1, 0, 1, 0, 0, 2, 3]] and not b.calls("load")
    assert b.load(64, struct=False) == INVALID and b.load(10 ** 6) == CAPACITY
    assert b.load(64, src=4096) == OK                      # host memory: sequence by sequence
    assert [c[:2] for c in b.calls("load_codes")] == [[1, 0], [3, 0]] and b.calls("synchronize")
    assert Codes(codes_host, [16, 40], 64, dtype="f32").status == UNSUPPORTED
    ctx = b.ctx
    assert codes_host.pced_load_codes(None, 1, None, None, None, None, None, None, 0, None, ctypes.c_float(1), None, None) == INVALID
    b.ctx = ctx
    codes_host.rec_fail(b"load_codes", 1)
    assert b.load(64) == HIPERR


def test_each_kind_of_batch_has_its_calls(codes_host):
    b = Codes(codes_host, [16, 40], 64, ffn_dim=512)
    pooled = lambda name, *a: getattr(codes_host, name)(b.ctx, *a)  # noqa: E731
    p, rows = P(DEVICE), ctypes.byref(_lib.pced_rows(q=Q, k=K, v=V))
    calls = [("pced_step", p, p, p, p, p, None, None), ("pced_generate", 1, ctypes.byref(_lib.pced_synth(1, 1)), p, p, None, None),
             ("pced_model_prefill", p, 1, p, None), ("pced_model_step", p, p, p, p, None, None),
             ("pced_model_generate", p, p, 1, p, p, None, None), ("pced_read_cache", 0, 0, 0, 1, p, p, None),
             ("pced_append", 0, 1, 1, rows, None, P(X), None), ("pced_attend", 0, 1, 1, P(Q), None, P(X), None),
             ("pced_summarize", None)]
    assert b.bind() == OK
    codes_host.rec_clear()
    for name, *a in calls:
        assert pooled(name, *a) == UNSUPPORTED, name
        assert "8 bits" in b.error() and b.nothing_launched()
    # those on logits and hidden states serve both
    assert codes_host.pced_fuse(b.ctx, P(Q), 1, P(X), None, None) == OK
    assert codes_host.pced_lmhead(b.ctx, P(Q), 2, P(K), P(X), None) == OK
    assert b.append() == OK and b.attend() == OK and b.advance() == OK and b.read() == OK
    # a batch in the pools again
    assert b.pooled(64) == OK and b.calls("load") and not b.calls("load_codes")
    assert b.append() == b.attend() == b.read() == STATE and b.nothing_launched()
    for name, *a in calls[5:7]:
        assert pooled(name, *a) == OK, (name, b.error())
    assert b.load(64) == OK and b.append() == OK


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), INVALID), (dict(n=-3), INVALID), (dict(layer=-1), INVALID), (dict(layer=1, layers=2), INVALID),
    (dict(n=10 ** 6), CAPACITY), (dict(n=65), CAPACITY), (dict(rows=dict(q=Q, v=V)), INVALID), (dict(q_out=None), INVALID),
    (dict(rows=dict(q=Q + 2, k=K, v=V)), INVALID), (dict(rows=dict(q=Q, k=K, v=V, k_row=8)), INVALID),
    (dict(rope=(1e4, 130, 0)), INVALID), (dict(rope=(1e4, 24, 1)), INVALID), (dict(q_out=Q + 8192), INVALID),
    (dict(q_out=K), INVALID),
])
def test_append_refusals(codes_host, kw, status):
    b = Codes(codes_host, [16, 40], 100, n_layers=2)
    assert b.append(**kw) == status, b.error()
    assert b.error() and b.nothing_launched()
    assert b.advance() == STATE and b.lengths() == [16, 40]


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), INVALID), (dict(layer=2), INVALID), (dict(layers=3), INVALID), (dict(q=None), INVALID), (dict(x=None), INVALID),
    (dict(q=Q + 8), INVALID), (dict(x=X + 2), INVALID), (dict(x=Q), INVALID), (dict(x=Q + 1024), INVALID), (dict(n=2), STATE),
    (dict(n=65), CAPACITY), (dict(n=1000), CAPACITY),
])
def test_attend_refusals(codes_host, kw, status):
    b = Codes(codes_host, [16, 40], 100, n_layers=2)
    assert b.attend() == STATE and b.append() == OK
    assert b.attend(**kw) == status, b.error()
    assert b.error() and b.nothing_launched()


@pytest.mark.parametrize("kw,status", [
    (dict(seq=2), INVALID), (dict(seq=-1), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID),
    (dict(start=-1), INVALID), (dict(count=-1), INVALID), (dict(count=17), INVALID), (dict(start=2 ** 31 - 1, count=2 ** 31 - 1), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(count=0), OK), (dict(count=0, k=None, v=None), OK),
])
def test_read_refusals(codes_host, kw, status):
    b = Codes(codes_host, [16, 40], 64, n_layers=2)
    assert b.read(**kw) == status, b.error()
    assert b.nothing_launched()
    assert b.read(1, 1, 3, 37) == OK and b.calls("read_codes")[0][:5] == [1, 1, 3, 37, 40]


def test_layer_by_layer(codes_host):
    b = Codes(codes_host, [16, 40], 64, n_layers=2, max_new=18)
    assert b.append(layers=1, n=3) == OK
    assert b.calls("append_codes") == [[0, 1, 3, 1, 3, 0, 2 * 3, 1]]
    assert b.attend(layers=1, n=3) == OK and b.attend(layers=1, n=2) == OK
    assert b.attend(layer=1, layers=1) == STATE and b.attend(n=3) == STATE and b.advance(1) == STATE
    assert b.append(layer=1, layers=1, n=3) == OK and b.attend(n=3) == OK
    assert b.advance(4) == STATE and b.advance(2) == OK and b.lengths() == [18, 42]
    assert b.attend() == STATE and b.advance() == STATE
    assert b.append() == OK and b.calls("append_codes")[0][5] == 2     # positions from the new lengths
    codes_host.rec_fail(b"append_codes", 1)
    b2 = Codes(codes_host, [16, 40], 64)
    codes_host.rec_fail(b"append_codes", 1)
    assert b2.append() == HIPERR and b2.advance() == STATE and b2.append() == OK
    codes_host.rec_fail(b"attend_codes", 1)
    assert b2.attend() == HIPERR and b2.attend() == OK


@pytest.mark.parametrize("heads", [(4, 4, 64), (32, 8, 128), (16, 1, 128), (28, 4, 128), (8, 4, 64)])
@pytest.mark.parametrize("layers", [1, 7])
@pytest.mark.parametrize("lens,n", [([1, 1], 1), ([16, 15], 33), ([500] + [1] * 70, 1), ([3000, 20], 9), ([40000, 1], 64),
                                    ([200] * 40, 60), ([100000, 17], 2)])
def test_every_size_fits(codes_host, heads, layers, lens, n):
    """Launches cover every token, layer and page once, within the workspace's region."""
    b = Codes(codes_host, lens, n, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2], n_layers=layers)
    assert b.status == OK and b.append(n, rope=None) == OK and b.attend(n) == OK, b.error()
    begin, end, seen, G = codes_host.room_begin(b.ctx), codes_host.room_end(b.ctx), set(), heads[0] // heads[1]
    splits = b.calls("attend_split")
    for (l, nl, s, ns, g, ng, *_), (parts, part_pages, gt, tiles, seq_parts, *_) in zip(b.calls("attend_codes"), splits):
        cells = {(i, j, k) for i in range(l, l + nl) for j in range(s, s + ns) for k in range(g, g + ng)}
        assert cells and not cells & seen
        seen |= cells
        pages = [(x + n - 1) // 16 + 1 for x in lens]
        assert parts == -(-max(pages) // part_pages) and part_pages % 8 == 0 and part_pages <= 256
        assert seq_parts == sum(-(-x // part_pages) for x in pages[s:s + ns])
        assert 1 <= gt and gt * G <= 16 * tiles and tiles in (1, 2)
        groups = -(-n // gt)
    spans = sorted((c[0], c[1]) for name in ("acc", "ml") for c in b.calls(name))
    for x, y in spans:
        assert begin <= x < y <= end
    assert seen == {(i, j, k) for i in range(layers) for j in range(len(lens)) for k in range(groups)}


def test_struct_matches_the_header(tmp_path):
    from tests.test_layer_path import test_structs_match_the_header
    test_structs_match_the_header(tmp_path, _lib.pced_cache8, ("code", "max_new") + BUFFERS)
