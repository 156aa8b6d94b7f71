"""Sampling on the GPU against the oracle (oracle/sample.py): scores are fp32 and equal bit for bit, tokens, experts
and counts are equal, log-probabilities are off by their rounding."""
import math

import numpy as np
import pytest

from oracle import sample as O
from tests.test_gpu_adjust import DEV, Limits, _logits, _session

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
SETTINGS = ("temperature", "top_k", "top_p", "min_p")


def _dev(x, dt):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=dt))).to(DEV)


class Case:
    """A batch's logits and settings; run() samples and compares every output with the oracle's."""

    def __init__(self, vocab, experts, seed=0, beta=0.5, lim=None, logits=None, spread=3.0):
        self.V, self.experts, self.B = vocab, experts, len(experts)
        self.s, self.beta, self.prior = _session(vocab, experts, beta=beta)
        self.x = _logits(self.s.S, vocab, seed, spread) if logits is None else logits
        self.t = _dev(self.x, np.float32)
        self.lim = lim
        self.adj = None if lim is None else self.s.adjust(**lim.tensors)
        self.scores, at, e = [], 0, 0
        for b, n in enumerate(experts):
            rows = self.x[at:at + n + 1]
            if lim is not None:
                rows = np.stack([lim.row(r, b) for r in rows])
            ok = lim.mask[b] if lim is not None and lim.has("mask") else None
            self.scores.append(O.scores(rows, self.beta[e:e + n], self.prior[e:e + n], ok))
            at, e = at + n + 1, e + n

    def settings(self, **kw):
        types = dict(temperature=np.float32, top_k=np.int32, top_p=np.float32, min_p=np.float32)
        return {k: np.broadcast_to(np.asarray(v, types[k]), (self.B,)).copy() for k, v in kw.items()}

    def run(self, u, **kw):
        kw = self.settings(**kw)
        u = np.broadcast_to(np.asarray(u, np.float32), (self.B,)).copy()
        out = self.s.sample(self.t, self.s.sampling(**{k: _dev(v, v.dtype) for k, v in kw.items()}), _dev(u, np.float32),
                            adjust=self.adj)
        self.check(out, u, kw)
        return out

    def check(self, out, u, kw):
        got = {k: v.cpu().numpy() for k, v in out.items()}
        assert np.array_equal(got["beta_used"], self.beta)
        # an fp64 sum's terms are rounded to multiples of 2^-shift of the highest weight, which is 1: the sum of V of
        # them is off by at most V 2^-(shift + 1) of itself; fp64's own errors are far below; then one fp32 rounding
        shift = 62 - math.ceil(math.log2(self.V))
        for b in range(self.B):
            S, who = self.scores[b]
            one = {k: v[b].item() for k, v in kw.items()}
            token, lp, n = O.sample(S, one.pop("temperature"), float(u[b]), **one)
            where = (b, {k: v[b] for k, v in kw.items()}, u[b])
            assert got["tokens"][b] == token, where + (token, got["tokens"][b])
            assert got["kept"][b] == n, where + (n, got["kept"][b])
            if token < 0:
                assert got["winner"][b] == 0 and got["score"][b] == got["logprob"][b] == -np.inf
                continue
            assert got["winner"][b] == who[token] and got["score"][b] == S[token], where
            tol = 2.0 ** -24 * abs(lp) + self.V * 2.0 ** -(shift + 1) + 1e-12
            assert abs(float(got["logprob"][b]) - lp) <= tol, where + (lp, got["logprob"][b])


CUTS = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=100000), dict(top_p=0.3), dict(top_p=0.95), dict(top_p=0.999999),
        dict(min_p=0.05), dict(min_p=1e-6), dict(top_k=40, top_p=0.9), dict(top_k=300, top_p=0.99, min_p=0.002),
        dict(top_p=0.5, min_p=0.3), dict(top_k=3, min_p=0.0001)]
SHAPES = [(2, [1]), (3, [2]), (33, [4, 1]), (255, [2, 1]), (257, [3]), (1025, [5, 1, 2]), (4098, [17]), (32000, [1, 2]),
          (50257, [3])]


@pytest.mark.parametrize("vocab,experts", SHAPES)
@pytest.mark.parametrize("cut", CUTS, ids=str)
def test_cuts(vocab, experts, cut):
    c = Case(vocab, experts, seed=vocab)
    r = np.random.RandomState(1)
    for T in (0.0, 0.3, 1.0, 3.0):
        for _ in range(2):
            c.run(r.rand(c.B), temperature=T, **cut)


@pytest.mark.parametrize("vocab,experts", [(1000, [8]), (4097, [2, 5]), (128256, [32]), (151936, [3, 1, 2])])
@pytest.mark.parametrize("allowed", [None, 0.5, 0.01])
def test_adjusted(vocab, experts, allowed):
    lim = Limits(vocab, len(experts), seed=3, history=200, biases=40, allowed=allowed)
    c = Case(vocab, experts, seed=4, lim=lim)
    r = np.random.RandomState(2)
    for cut in (dict(), dict(top_k=50, top_p=0.9), dict(top_p=0.98, min_p=0.001)):
        c.run(r.rand(c.B), temperature=0.8, **cut)


@pytest.mark.parametrize("kind", ["equal", "halves", "two", "far", "near", "ramp"])
@pytest.mark.parametrize("vocab", [900, 1025, 20000, 131072])
def test_crowded_scores(kind, vocab):
    """Scores that fall into few places of their range: long lists, ties at every cut."""
    x = np.zeros((2, vocab), np.float32)
    r = np.random.RandomState(5)
    if kind == "halves":
        x[1] = np.round(r.randn(vocab) * 2) / 2
    elif kind == "two":
        x[1] = (r.rand(vocab) < 0.3) * np.float32(0.1)
    elif kind == "far":  # one token far above, the others close together
        x[1] = r.randn(vocab) * 1e-3
        x[1, vocab // 2] = 20.0
    elif kind == "near":  # differences of single steps of fp32
        x[1] = np.float32(1000) + r.randint(0, 4, vocab) * np.float32(2.0 ** -14)
    elif kind == "ramp":
        x[1] = np.arange(vocab) * np.float32(1e-6)
    c = Case(vocab, [1], logits=x)
    for cut in CUTS:
        for u in (0.0, 0.37, 0.999999):
            c.run(u, temperature=1.0, **cut)
    c.run(0.7, temperature=100.0, top_p=0.5)
    c.run(0.7, temperature=0.01, top_k=vocab // 2, top_p=0.7)


def test_extreme_settings():
    c = Case(5000, [2], seed=6)
    inf, nan = math.inf, math.nan
    for T in (1e-3, 1e-30, 1e-38, 1e-44, 50.0, 1e30, inf, nan, -1.0, -inf):
        for u in (0.0, 0.5, 1.0 - 2.0 ** -24):
            c.run(u, temperature=T)
            c.run(u, temperature=T, top_k=10, top_p=0.9, min_p=0.01)
    for u in (-1.0, -0.0, 1.0, 7.0, nan, inf, -inf, 1e-30):
        c.run(u, temperature=1.0)
    for cut in (dict(top_k=0), dict(top_k=-5), dict(top_k=2 ** 31 - 1), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=1.0),
                dict(top_p=2.0), dict(top_p=nan), dict(top_p=1e-30), dict(min_p=-1.0), dict(min_p=nan), dict(min_p=1.0),
                dict(min_p=1.5), dict(min_p=inf), dict(min_p=1e-38)):
        for u in (0.0, 0.6):
            c.run(u, temperature=1.0, **cut)


def test_infinite_temperature():
    """With min_p = 1 the tokens of the highest score stay: their weight alone reaches it."""
    x = _logits(2, 3000, 30)
    x[1] = np.round(x[1])
    c = Case(3000, [1], beta=0.0, logits=x)
    for T in (math.inf, float(np.finfo(np.float32).max)):
        for min_p in (1e-30, 1.0, 2.0, math.inf):
            for u in (0.0, 0.5, 0.99):
                c.run(u, temperature=T, min_p=min_p)
                c.run(u, temperature=T, min_p=min_p, top_k=2, top_p=0.9)


@pytest.mark.parametrize("vocab", [700, 4096, 40000])
def test_infinities_and_nan(vocab):
    """NaN and -inf are no candidates, +inf is above all; rows of nothing else; the largest numbers."""
    x = _logits(4, vocab, 7)
    x[:, 10:200:3] = np.nan
    x[0, 300] = np.nan
    x[1:, 301:400] = -np.inf
    c = Case(vocab, [3], logits=x)
    for u in (0.0, 0.4, 0.99):
        c.run(u, temperature=1.0, top_p=0.9)
    y = x.copy()
    y[2, [5, 350, 650]] = np.inf
    c = Case(vocab, [3], logits=y)
    for u in (0.0, 0.4, 0.99):
        for cut in CUTS:
            c.run(u, temperature=1.0, **cut)
    for bad in (np.nan, -np.inf):
        z = x.copy()
        z[1:] = bad
        Case(vocab, [3], logits=z).run(0.5, temperature=1.0, top_k=5, top_p=0.5, min_p=0.1)
        Case(vocab, [3], logits=z).run(0.5, temperature=0.0)
        z[3, vocab - 1] = 1.0
        Case(vocab, [3], logits=z).run(0.5, temperature=1.0, top_k=5, top_p=0.5, min_p=0.1)
    w = np.zeros((2, vocab), np.float32)
    w[1] = np.random.RandomState(8).uniform(-3e38, 3e38, vocab)
    Case(vocab, [1], beta=0.0, logits=w).run(0.5, temperature=1e37)
    Case(vocab, [1], beta=0.0, logits=w).run(0.5, temperature=1.0, top_k=5)


def test_closed_masks():
    lim = Limits(3000, 3, seed=9, allowed=0.5)
    lim.mask[1] = False
    lim.mask[2] = False
    lim.mask[2, 2999] = True
    bits = np.zeros((3, 94 * 32), bool)
    bits[:, :3000] = lim.mask
    lim.tensors["mask"] = _dev(np.packbits(bits, axis=1, bitorder="little").view(np.int32), np.int32)
    c = Case(3000, [2, 2, 1], seed=10, lim=lim)
    for T in (0.0, 1.0):
        out = c.run(0.5, temperature=T, top_p=0.9)
        assert out["tokens"][1] == -1 and out["tokens"][2] == 2999


def test_many_queries_with_settings_of_their_own():
    B = 70
    r = np.random.RandomState(11)
    c = Case(3001, [1 + b % 3 for b in range(B)], seed=12)
    for _ in range(3):
        c.run(r.rand(B), temperature=r.choice([0, 0.2, 0.7, 1, 2], B), top_k=r.choice([0, 1, 5, 100, 3000], B),
              top_p=r.choice([0.1, 0.5, 0.9, 0.99, 1], B), min_p=r.choice([0, 0.001, 0.1, 1], B))


def test_shares():
    """Evenly spaced random numbers give every token its share: n p draws, one more or less."""
    B, n = 50, 4000
    x = _logits(2, 40, 13, spread=1.0)
    c = Case(40, [1] * B, logits=np.tile(x, (B, 1)))
    S = O.scores(x, c.beta[:1], c.prior[:1])[0].astype(np.float64)
    c.s.load([1] * B, [1] * (2 * B), *[[torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16, device=DEV)] * (2 * B)] * 2,
             [0.5] * B, beta=[float(c.beta[0])] * B)  # (equal priors: they move all scores alike)
    sampling = c.s.sampling(temperature=torch.full((B,), 0.7, device=DEV))
    count = np.zeros(40)
    for i in range(0, n, B):
        u = (np.arange(i, i + B) + 0.5) / n
        got = c.s.sample(c.t, sampling, _dev(u, np.float32), want=())
        assert set(got) == {"tokens"}
        np.add.at(count, got["tokens"].cpu().numpy(), 1)
    p = np.exp((S - S.max()) / np.float32(0.7))
    assert (np.abs(count - n * p / p.sum()) <= 1.01).all()


def test_greedy_is_the_choice():
    lim = Limits(50257, 3, seed=14, history=100, biases=20, allowed=0.5)
    c = Case(50257, [4, 2, 1], seed=15, lim=lim)
    out = c.run(0.9, temperature=0.0, top_p=0.5, min_p=0.5, top_k=9)
    want = c.s.fuse_adjusted(c.t, c.adj)
    assert torch.equal(out["tokens"], want["tokens"]) and torch.equal(out["winner"], want["winner"])
    assert torch.equal(out["score"], want["top1"]) and (out["logprob"] == 0).all() and (out["kept"] == 1).all()


def test_dynamic_beta():
    s, _, prior = _session(2000, [3, 2], beta=None)
    t = _dev(_logits(s.S, 2000, 16), np.float32)
    sampling, u = s.sampling(temperature=torch.zeros(2, device=DEV)), torch.zeros(2, device=DEV)
    from paper_2601_08670_amd import _lib
    with pytest.raises(_lib.PcedError, match="STATE"):
        s.sample(t, sampling, u)
    a = s.sample(t, sampling, u, refresh_beta=True)
    b = s.fuse_adjusted(t, s.adjust())
    for x, y in (("tokens", "tokens"), ("winner", "winner"), ("score", "top1"), ("beta_used", "beta_used")):
        assert torch.equal(a[x], b[y]), x
    assert (a["beta_used"] > 0).all()
    again = s.sample(t + 1, sampling, u)
    assert torch.equal(again["beta_used"], a["beta_used"])


def test_streams_and_graphs():
    """A captured draw replays with new logits, numbers, settings and histories; repeated calls give the same bits."""
    lim = Limits(20000, 4, seed=17, history=50, allowed=0.7)
    c = Case(20000, [2, 1, 3, 1], seed=18, lim=lim)
    kw = c.settings(temperature=0.9, top_k=400, top_p=0.95, min_p=0.0001)
    dev = {k: _dev(v, v.dtype) for k, v in kw.items()}
    sampling, u = c.s.sampling(**dev), _dev(np.full(4, 0.5), np.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.s.sample(c.t, sampling, u, adjust=c.adj)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = c.s.sample(c.t, sampling, u, adjust=c.adj)
    for i in range(4):
        d = Case(20000, [2, 1, 3, 1], seed=20 + i, lim=lim)
        c.t.copy_(d.t)
        un = np.random.RandomState(i).rand(4).astype(np.float32)
        u.copy_(_dev(un, np.float32))
        kw["temperature"][:] = 0.5 + 0.3 * i
        dev["temperature"].copy_(_dev(kw["temperature"], np.float32))
        for t in out.values():
            t.fill_(77)
        g.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        d.check(got, un, kw)
        for _ in range(2):
            eager = c.s.sample(c.t, sampling, u, adjust=c.adj)
            torch.cuda.synchronize()
            assert all(torch.equal(eager[k], got[k]) for k in got)


def test_refusals():
    from paper_2601_08670_amd import _lib
    c = Case(500, [2, 1], seed=21)
    s, good = c.s, dict(temperature=torch.ones(2, device=DEV))
    for bad in (dict(), dict(good, top_k=torch.ones(2, device=DEV)), dict(temperature=torch.ones(3, device=DEV)),
                dict(temperature=torch.ones(2)), dict(good, top_q=torch.ones(2, device=DEV)),
                dict(good, top_p=torch.ones(4, device=DEV)[::2])):
        with pytest.raises(ValueError):
            s.sampling(**bad)
    cut, u = s.sampling(**good), torch.zeros(2, device=DEV)
    for args in ((c.t[:4], cut, u), (c.t.double(), cut, u), (c.t, cut, u[:1]), (c.t, cut, u.double()), (c.t, cut, u.cpu()),
                 (c.t.cpu(), cut, u)):
        with pytest.raises(ValueError):
            s.sample(*args)
    with pytest.raises(ValueError):
        s.sample(c.t, cut, u, want=("top1",))
    other = Case(500, [1], seed=22)
    with pytest.raises(ValueError, match="batch"):
        s.sample(c.t, other.s.sampling(temperature=torch.ones(1, device=DEV)), u)
    moe, _, _ = _session(500, [2, 1], aggregation="moe")
    with pytest.raises(_lib.PcedError, match="UNSUPPORTED"):
        moe.sample(c.t, moe.sampling(**good), u)
