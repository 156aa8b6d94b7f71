"""Refusals and launches of sampling, checked without a GPU: the library's own host code over recording stand-ins
(tests/sample_path.cpp). Device addresses are never read."""
import ctypes
import os
import subprocess

import pytest

from paper_2601_08670_amd import _lib
from tests.test_host_path import CSRC, DEVICE, ROOT
from tests.test_layer_path import HIPERR, INVALID, OK, P, Q, STATE, UNSUPPORTED, X, Layers


@pytest.fixture(scope="session")
def sample_host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("sample_path") / "sample_path.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    os.path.join(ROOT, "tests", "sample_path.cpp")] +
                   [os.path.join(CSRC, f) for f in ("pced_api.cpp", "pced_layer_api.cpp", "pced_sample_api.cpp")] +
                   ["-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.rec_name.restype = ctypes.c_char_p
    lib.rec_value.restype = ctypes.c_long
    lib.pced_workspace_bytes.restype = ctypes.c_size_t
    lib.pced_last_error.restype = ctypes.c_char_p
    return lib


class Sampler(Layers):
    def sample(self, logits=Q, fresh=1, adjust=None, cut={}, u=DEVICE, out=X, extra=None):
        self.lib.rec_clear()
        self.lib.watch(self.ctx)
        cut = None if cut is None else ctypes.byref(_lib.pced_sampling(**dict(dict(temperature=DEVICE), **cut)))
        return self.lib.pced_sample(self.ctx, P(logits), fresh, adjust and ctypes.byref(adjust), cut, P(u), P(out),
                                    extra and ctypes.byref(extra), None)


def test_refusals(sample_host):
    b = Sampler(sample_host, [16, 40, 7], 64)
    for kw in (dict(logits=None), dict(cut=None), dict(cut=dict(temperature=None)), dict(u=None), dict(out=None),
               dict(adjust=_lib.pced_adjust(n_history=-1)), dict(adjust=_lib.pced_adjust(history=DEVICE, n_history=3)),
               dict(adjust=_lib.pced_adjust(mask=DEVICE, mask_row=31))):
        assert b.sample(**kw) == INVALID and b.error() and b.nothing_launched(), kw
    assert b.sample(fresh=0) == STATE and b.nothing_launched()      # dynamic beta, not known yet
    assert b.sample() == OK and len(b.calls("beta")) == 1
    assert b.sample(fresh=0) == OK and not b.calls("beta")
    moe = Sampler(sample_host, [16, 40, 7], 64, aggregation="poe")
    assert moe.sample() == UNSUPPORTED and moe.nothing_launched()
    assert sample_host.pced_sample(None, P(Q), 1, None, None, None, None, None, None) == INVALID
    fresh = ctypes.c_void_p()
    ws = sample_host.pced_workspace_bytes(ctypes.byref(b.cfg))
    assert sample_host.pced_create(ctypes.byref(b.cfg), P(DEVICE), ctypes.c_size_t(ws), ctypes.byref(fresh)) == OK
    b.ctx, old = fresh, b.ctx
    assert b.sample() == STATE and b.nothing_launched()
    sample_host.pced_destroy(old)


@pytest.mark.parametrize("vocab", [2, 3, 100, 1000, 4096, 50257, 128256, 151936, 1 << 20])
def test_launches(sample_host, vocab):
    """Everything the launches use lies in the workspace's own places; the weights' sums fit 62 bits."""
    b = Sampler(sample_host, [16, 40], 64, vocab=vocab)
    assert b.sample(adjust=_lib.pced_adjust(mask=DEVICE), cut=dict(top_k=DEVICE), extra=_lib.pced_sample_out(kept=DEVICE)) == OK
    (nblk, masked, *fits), = b.calls("fuse_scores")
    assert fits == [1] * 6 and masked == 1 and nblk == -(-vocab // 256)
    (queries, shift, parts, top_k, kept, *_), = b.calls("sample")
    assert queries == 1 and parts == nblk and top_k == kept == 1
    assert vocab << shift <= 1 << 62 < vocab << (shift + 1) or vocab & (vocab - 1) == 0
    assert b.sample() == OK and b.calls("fuse_scores")[0][1] == 0


def test_launch_failures_are_reported(sample_host):
    b = Sampler(sample_host, [16, 40], 64)
    for name in (b"fuse_scores", b"sample"):
        sample_host.rec_fail(name, 1)
        assert b.sample() == HIPERR and b.sample() == OK


@pytest.mark.parametrize("struct,names", [
    (_lib.pced_sampling, ("temperature", "top_k", "top_p", "min_p")),
    (_lib.pced_sample_out, ("winner", "score", "logprob", "kept", "beta_used"))])
def test_structs_match_the_header(tmp_path, struct, names):
    from tests.test_layer_path import test_structs_match_the_header as check
    check(tmp_path, struct, names)
