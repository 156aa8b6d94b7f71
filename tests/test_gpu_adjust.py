"""Adjusted logits and the choice over them on the GPU against the oracle
(oracle/layer.py): every adjustment is one fp32 operation, so the fp32 oracle gives the
same bits."""
import numpy as np
import pytest

from oracle import layer as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _session(vocab, experts, beta=0.5, seed=0, **kw):
    from paper_2601_08670_amd.session import PcedSession
    S = sum(experts) + len(experts)
    s = PcedSession(n_layers=1, n_q_heads=4, n_kv_heads=1, head_dim=64, vocab=vocab, dtype="bf16",
                    max_queries=len(experts), max_seqs=S, max_pages=S, max_pages_per_seq=1, device=DEV, poison=True, **kw)
    cache = [torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16, device=DEV)] * S
    r = np.random.RandomState(seed)
    rel = r.uniform(0.05, 0.95, sum(experts)).astype(np.float32)
    b = None if beta is None else (r.uniform(0, 1, sum(experts)) * 2 * beta).astype(np.float32)
    s.load(experts, [1] * S, cache, cache, rel.tolist(), gamma=2.5, beta=None if b is None else b.tolist())
    prior = (2.5 * np.log(np.clip(rel.astype(np.float64), 1e-8, 1 - 1e-8))).astype(np.float32)
    return s, b, prior


class Limits:
    """Random adjustments of a batch, as host lists per query and as device tensors."""

    def __init__(self, vocab, B, seed=0, history=20, biases=6, allowed=0.6, only=None, words=None):
        r = np.random.RandomState(seed)
        self.V, self.B = vocab, B
        self.history = [r.randint(-2, vocab + 2, r.randint(0, history + 1)) if b % 3 != 2 else
                        np.full(history, vocab - 1) for b in range(B)]
        self.biases = [[(int(t), np.float32(x)) for t, x in zip(r.randint(-1, vocab + 1, biases), r.randn(biases) * 3)]
                       for b in range(B)]
        for b in self.biases:  # the same token twice: the last entry counts
            if len(b) > 2:
                b[2] = (b[0][0], np.float32(1.25))
        self.rep, self.pres, self.freq = (r.uniform(*x, B).astype(np.float32) for x in ((0.7, 1.6), (-0.5, 1), (-0.2, 0.5)))
        self.mask = None if allowed is None else r.rand(B, vocab) < allowed
        self.only = only
        t = lambda x, dt: torch.from_numpy(np.ascontiguousarray(x, dtype=dt)).to(DEV)  # noqa: E731
        off = lambda xs: t(np.cumsum([0] + [len(x) for x in xs]), np.int32)  # noqa: E731
        flat = [e for b in self.biases for e in b]
        self.tensors = dict(
            history=t(np.concatenate(self.history), np.int32), history_off=off(self.history), repetition=t(self.rep, np.float32),
            presence=t(self.pres, np.float32), frequency=t(self.freq, np.float32), bias_token=t([e[0] for e in flat], np.int32),
            bias_value=t([e[1] for e in flat], np.float32), bias_off=off(self.biases))
        if self.mask is not None:
            words = words or -(-vocab // 32)
            bits = np.ones((B, words * 32), bool)  # bits past the vocabulary are set
            bits[:, :vocab] = self.mask
            self.tensors["mask"] = t(np.packbits(bits, axis=1, bitorder="little").view(np.int32), np.int32)
        if only is not None:
            self.tensors = {k: x for k, x in self.tensors.items() if k in only}

    def has(self, name):
        return name in self.tensors

    def row(self, s, b, real=np.float32):
        return L.adjust_row(s, history=self.history[b] if self.has("history") else (),
                            repetition=self.rep[b] if self.has("repetition") else 1.0,
                            presence=self.pres[b] if self.has("presence") else 0.0,
                            frequency=self.freq[b] if self.has("frequency") else 0.0,
                            biases=self.biases[b] if self.has("bias_token") else (),
                            allowed=self.mask[b] if self.has("mask") else None, real=real)


def _logits(S, V, seed, spread=3.0):
    return (np.random.RandomState(seed).randn(S, V) * spread).astype(np.float32)


def _same(got, want):
    """Equal values: NaN where NaN is wanted, and zeros of either sign."""
    got, want = np.asarray(got), np.asarray(want)
    assert got.shape == want.shape
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


SHAPES = [(2, [1]), (3, [2]), (31, [1, 3]), (32, [2]), (33, [4]), (255, [2, 1]), (256, [1]), (257, [3]), (1000, [8]),
          (1024, [2]), (1025, [5, 1, 2]), (4098, [17]), (8192, [40])]


@pytest.mark.parametrize("vocab,experts", SHAPES)
@pytest.mark.parametrize("allowed", [None, 0.6, 0.02])
def test_adjust_logits(vocab, experts, allowed):
    s, _, _ = _session(vocab, experts)
    lim = Limits(vocab, len(experts), seed=vocab, allowed=allowed)
    x = _logits(s.S, vocab, 1)
    x.reshape(-1)[::7] = 0
    x.reshape(-1)[::11] *= -0.0
    t = torch.from_numpy(x).to(DEV)
    adj = s.adjust(**lim.tensors)
    out = s.adjust_logits(t, adj)
    assert torch.equal(t.cpu(), torch.from_numpy(x))
    query = np.repeat(np.arange(len(experts)), [n + 1 for n in experts])
    want = np.stack([lim.row(x[r], query[r]) for r in range(s.S)])
    _same(out.cpu().numpy(), want)
    assert s.adjust_logits(t, adj, out=t) is t       # in place
    _same(t.cpu().numpy(), want)
    exact = np.stack([lim.row(x[r].astype(np.float64), query[r], np.float64) for r in range(s.S)])
    fin = np.isfinite(exact)
    # four fp32 operations, each off by at most half a step of a value below 2^5 (20 tokens at most, |x| < 16)
    assert (np.abs(want[fin] - exact[fin]) <= 4 * 2.0 ** -24 * 64).all()


@pytest.mark.parametrize("only", [(), ("history", "history_off"), ("history", "history_off", "repetition"),
                                  ("history", "history_off", "frequency", "presence"), ("repetition", "presence"),
                                  ("bias_token", "bias_value", "bias_off"), ("mask",)])
@pytest.mark.parametrize("vocab", [999, 1000])
def test_parts_of_the_adjustments(only, vocab):
    s, beta, prior = _session(vocab, [3, 2])
    lim = Limits(vocab, 2, seed=5, only=only, words=40)
    x = _logits(s.S, vocab, 2)
    t, adj = torch.from_numpy(x).to(DEV), s.adjust(**lim.tensors)
    rows = np.stack([lim.row(x[r], 0 if r < 4 else 1) for r in range(7)])
    _same(s.adjust_logits(t, adj).cpu().numpy(), rows)
    _check_choice(s, t, adj, rows, lim, beta, prior, [3, 2])


def _check_choice(s, t, adj, rows, lim, beta, prior, experts):
    out = {k: v.cpu().numpy() for k, v in s.fuse_adjusted(t, adj).items()}
    e0 = r0 = 0
    for b, n in enumerate(experts):
        want = L.choose(rows[r0:r0 + n + 1], beta[e0:e0 + n], prior[e0:e0 + n],
                        lim.mask[b] if lim.has("mask") else None, np.float32)
        got = (int(out["tokens"][b]), int(out["winner"][b]), float(out["top1"][b]), float(out["top2"][b]))
        assert got == want, (b, got, want)
        e0, r0 = e0 + n, r0 + n + 1
    assert np.array_equal(out["beta_used"], beta)


@pytest.mark.parametrize("vocab,experts", SHAPES + [(640, [1] * 40), (5000, [3] * 33)])
@pytest.mark.parametrize("allowed", [None, 0.5, 0.01])
def test_fuse_adjusted(vocab, experts, allowed):
    s, beta, prior = _session(vocab, experts, seed=vocab)
    lim = Limits(vocab, len(experts), seed=vocab + 1, allowed=allowed)
    x = _logits(s.S, vocab, 3)
    query = np.repeat(np.arange(len(experts)), [n + 1 for n in experts])
    rows = np.stack([lim.row(x[r], query[r]) for r in range(s.S)])
    _check_choice(s, torch.from_numpy(x).to(DEV), s.adjust(**lim.tensors), rows, lim, beta, prior, experts)


def test_nothing_allowed_one_allowed_and_bad_values():
    """Empty masks, a single open token, NaN and infinities in closed and open places, ties."""
    V, experts = 700, [3] * 6
    s, beta, prior = _session(V, experts)
    lim = Limits(V, 6, seed=6, allowed=0.5, only=("mask",))
    x = _logits(s.S, V, 4)
    lim.mask[0] = False
    lim.mask[1] = False
    lim.mask[1, 699] = True
    x[8:12][:, ~lim.mask[2]] = np.nan
    x[8:12, np.argmax(lim.mask[2])] = np.nan
    x[9, ~lim.mask[2]] = np.inf
    x[12:16] = np.float32(np.finfo(np.float32).min)     # the type's lowest value everywhere
    x[16:20] = -np.inf
    x[17:20, np.flatnonzero(lim.mask[4])[5]] = 1.0        # (the amateur's -inf: +inf against it)
    x[20:24] = 2.0                                        # ties
    bits = np.zeros((6, 22 * 32), bool)
    bits[:, :V] = lim.mask
    lim.tensors["mask"] = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)
    rows = np.stack([lim.row(x[r], r // 4) for r in range(s.S)])
    t, adj = torch.from_numpy(x).to(DEV), s.adjust(**lim.tensors)
    _same(s.adjust_logits(t, adj).cpu().numpy(), rows)
    _check_choice(s, t, adj, rows, lim, beta, prior, experts)
    out = s.fuse_adjusted(t, adj)
    assert out["tokens"].tolist()[:2] == [-1, 699] and out["winner"].tolist()[0] == 0
    assert out["top1"].tolist()[0] == out["top2"].tolist()[0] == -np.inf == out["top2"].tolist()[1]


def test_lists_are_cut_to_their_arrays():
    """Offsets before the start, past the end or falling, and padded batches, read nothing outside."""
    V = 300
    s, beta, prior = _session(V, [2, 1, 1, 2])
    history = torch.arange(12, dtype=torch.int32, device=DEV)
    adj = dict(history=history, history_off=torch.tensor([-7, 4, 2, 9, 1 << 30], dtype=torch.int32, device=DEV),
               presence=torch.ones(4, device=DEV))
    x = _logits(s.S, V, 5)
    out = s.adjust_logits(torch.from_numpy(x).to(DEV), s.adjust(**adj)).cpu().numpy()
    seen = [range(0, 4), (), range(2, 9), range(9, 12)]
    query = np.repeat(np.arange(4), [3, 2, 2, 3])
    _same(out, np.stack([L.adjust_row(x[r], seen[query[r]], presence=1.0, real=np.float32) for r in range(10)]))
    empty = s.adjust(history=history[:0], history_off=adj["history_off"], presence=adj["presence"])
    _same(s.adjust_logits(torch.from_numpy(x).to(DEV), empty).cpu().numpy(), x)


def test_long_history():
    """More tokens than any block holds, most of them the same few; counts stay exact."""
    V = 5000
    s, beta, prior = _session(V, [6])
    r = np.random.RandomState(7)
    h = np.concatenate([r.randint(0, 40, 60000), r.randint(0, V, 40000)]).astype(np.int32)
    lim = Limits(V, 1, seed=8, only=("frequency", "presence", "repetition"))
    lim.freq[0] = 1e-4
    lim.history = [h]
    lim.tensors.update(frequency=torch.from_numpy(lim.freq).to(DEV), history=torch.from_numpy(h).to(DEV),
                       history_off=torch.tensor([0, len(h)], dtype=torch.int32, device=DEV))
    x = _logits(s.S, V, 6)
    t, adj = torch.from_numpy(x).to(DEV), s.adjust(**lim.tensors)
    rows = np.stack([lim.row(x[i], 0) for i in range(7)])
    _same(s.adjust_logits(t, adj).cpu().numpy(), rows)
    _check_choice(s, t, adj, rows, lim, beta, prior, [6])


def test_fuse_adjusted_without_adjustments_is_pced_fuse():
    """Same tokens, experts, scores and beta, with dynamic beta (per expert or one per query) refreshed or kept."""
    V, experts = 4000, [5, 2, 9]
    for kw in (dict(), dict(beta_scalar=True)):
        a, _, _ = _session(V, experts, beta=None, **kw)
        b, _, _ = _session(V, experts, beta=None, **kw)
        for i, refresh in enumerate((True, False, True)):
            t = torch.from_numpy(_logits(a.S, V, 10 + i, 1.0)).to(DEV)
            tokens = torch.empty(3, dtype=torch.int32, device=DEV)
            want = a.out_buffers(("winner", "top1", "top2", "beta_used"))
            a.ctx.pced_fuse(t, int(refresh), tokens, want)
            got = b.fuse_adjusted(t, b.adjust(), refresh_beta=refresh)
            assert torch.equal(got["tokens"], tokens)
            for k, x in want.items():
                if k == "beta_used":  # (summed by another launch)
                    assert (got[k] - x).abs().max() <= 2.0 ** -20
                elif k == "winner":
                    assert torch.equal(got[k], x)
                else:  # scores move by at most |s_k - s_0| < 16 times beta's difference, and a rounding
                    assert (got[k] - x).abs().max() <= 16 * 2.0 ** -20 + 2.0 ** -20


def test_replayed_choice():
    """Captured once; the history, its bounds, the mask and the logits change between the replays."""
    V, experts = 3000, [4, 4]
    s, beta, prior = _session(V, experts)
    lims = [Limits(V, 2, seed=20 + i, history=30) for i in range(3)]
    room = {k: (torch.zeros(100, dtype=torch.int32, device=DEV) if k == "history" else x.clone())
            for k, x in lims[0].tensors.items()}
    t, tokens = torch.zeros((s.S, V), device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    adj, out = s.adjust(**room), s.out_buffers(("winner", "top1", "top2"))
    run = lambda: s.ctx.pced_fuse_adjusted(t, 0, adj.struct, tokens, out)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i, lim in enumerate(lims):
        x = _logits(s.S, V, 30 + i)
        t.copy_(torch.from_numpy(x))
        for k, v in lim.tensors.items():
            room[k][:v.shape[0]].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        rows = np.stack([lim.row(x[r], r // 5) for r in range(10)])
        for b in range(2):
            want = L.choose(rows[5 * b:5 * b + 5], beta[4 * b:4 * b + 4], prior[4 * b:4 * b + 4], lim.mask[b], np.float32)
            assert (int(tokens[b]), int(out["winner"][b]), float(out["top1"][b]), float(out["top2"][b])) == want


def test_session_refusals():
    s, _, _ = _session(500, [2, 2])
    i32 = dict(dtype=torch.int32, device=DEV)
    z = torch.zeros(3, **i32)
    for bad in (dict(history=z.long(), history_off=z), dict(history=z), dict(history=z, history_off=z[:2]),
                dict(presence=torch.zeros(1, device=DEV)), dict(presence=torch.zeros((2, 2), device=DEV)),
                dict(bias_token=z, bias_off=z), dict(bias_token=z, bias_off=z, bias_value=torch.zeros(2, device=DEV)),
                dict(mask=torch.zeros((2, 15), **i32)), dict(mask=torch.zeros((1, 16), **i32)),
                dict(mask=torch.zeros((16, 2), **i32).t()), dict(mask=torch.zeros((1, 16), **i32).expand(2, 16)), dict(temperature=z),
                dict(presence=torch.zeros(2)), dict(mask=torch.zeros((2, 16), dtype=torch.int32))):
        with pytest.raises(ValueError):
            s.adjust(**bad)
    adj, t = s.adjust(), torch.zeros((6, 500), device=DEV)
    for bad in (lambda: s.adjust_logits(t[:5], adj), lambda: s.adjust_logits(t.double(), adj),
                lambda: s.adjust_logits(t, adj, out=torch.zeros((6, 501), device=DEV)),
                lambda: s.fuse_adjusted(torch.zeros((500, 6), device=DEV).t(), adj), lambda: s.adjust_logits(t.cpu(), adj),
                lambda: s.adjust_logits(t, adj, out=t.cpu()), lambda: s.fuse_adjusted(t, adj, want=("logits",))):
        with pytest.raises(ValueError):
            bad()
    other, _, _ = _session(400, [2, 2])
    with pytest.raises(ValueError, match="another batch"):
        other.adjust_logits(torch.zeros((6, 400), device=DEV), adj)
