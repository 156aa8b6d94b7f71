"""Sampling where it is used: behind the decoder stack's steps, with dynamic beta, and in a captured step over caches in
8 bits whose attention uses the same part of the workspace."""
import numpy as np
import pytest

from oracle import sample as O
from pced_inputs import workloads as W
from pced_inputs.model import LAYER_TENSORS, ModelSpec
from tests.test_gpu_adjust import DEV, _logits, _session
from tests.test_gpu_codes import Coded
from tests.test_gpu_layer import _eq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _check(out, logits, experts, beta, prior, u, T, **cuts):
    """Every query's token, expert and count against the oracle, for the beta that the call used."""
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert np.array_equal(got["beta_used"], beta)
    at = e = 0
    for b, n in enumerate(experts):
        S, who = O.scores(logits[at:at + n + 1], beta[e:e + n], prior[e:e + n])
        token, _, kept = O.sample(S, float(np.float32(T)), float(u[b]), **cuts)
        assert (got["tokens"][b], got["winner"][b], got["kept"][b]) == (token, who[token], kept), b
        assert got["score"][b] == S[token]
        at, e = at + n + 1, e + n


@pytest.mark.parametrize("T", [0.0, 0.7, 1.5])
def test_decoder_stack_steps(T):
    """model_step -> sample -> the next model_step's tokens: two queries, beta from the first step's logits."""
    from paper_2601_08670_amd.session import session_for_workload
    geom, experts = W.Geometry(2, 8, 2, 64, 512, 3000, "bf16"), [3, 2]
    wl = W.custom(geom, experts, [40, 300, 17, 5, 129], amateur_len=16, steps=6, seed=41)
    spec = ModelSpec(geom, ffn_dim=1024, rope_theta=10000.0, seed=41)
    sess = session_for_workload(wl, device=DEV, extra_tokens=6, poison=True, ffn_dim=1024, rope_theta=10000)
    model = sess.pack_model(lambda l: [spec.device(n, l, DEV) for n in LAYER_TENSORS], spec.device("embed", 0, DEV),
                            spec.device("final_norm", 0, DEV))
    head = sess.pack_lm_head(wl.lm_head_device(DEV))
    rel = np.clip(np.asarray(wl.relevance, np.float64), 1e-8, 1 - 1e-8)
    prior = (wl.gamma * np.log(rel)).astype(np.float32)
    sampling = sess.sampling(temperature=torch.full((2,), T, device=DEV), top_k=torch.full((2,), 200, dtype=torch.int32, device=DEV))
    tokens, r, lens = torch.tensor([7, 11], dtype=torch.int32, device=DEV), np.random.RandomState(42), sess.lengths()
    drawn = []
    for i in range(5):
        step = sess.model_step(model, head, tokens)
        u = r.rand(2).astype(np.float32)
        out = sess.sample(step["logits"], sampling, torch.from_numpy(u).to(DEV))
        tokens = out["tokens"]
        torch.cuda.synchronize()
        _check(out, step["logits"].cpu().numpy(), experts, step["beta_used"].cpu().numpy(), prior, u, T, top_k=200)
        if T == 0:
            for x, y in (("tokens", "tokens"), ("winner", "winner"), ("score", "top1")):
                _eq(out[x], step[y], x)
        assert sess.lengths() == [n + i + 1 for n in lens]
        drawn.append(tokens.tolist())
    assert T == 0 or len(set(map(tuple, drawn))) > 1  # (random numbers of five steps)


@pytest.mark.parametrize("V,experts", [(2000, [3, 2]), (50257, [4]), (4099, [1, 5, 2])])
@pytest.mark.parametrize("T", [0.6, 3.0])
def test_dynamic_beta_at_temperatures(V, experts, T):
    """Beta from the logits of the call itself, kept for later calls; draws from scores by it."""
    s, _, prior = _session(V, experts, beta=None)
    B, r = len(experts), np.random.RandomState(43)
    sampling = s.sampling(temperature=torch.full((B,), T, device=DEV), top_p=torch.full((B,), 0.9, device=DEV))
    x = _logits(s.S, V, 44)
    t = torch.from_numpy(x).to(DEV)
    beta = s.fuse_adjusted(t, s.adjust(), refresh_beta=True)["beta_used"].cpu().numpy()
    s2, _, _ = _session(V, experts, beta=None)
    cuts = dict(top_p=float(np.float32(0.9)))
    for i in range(3):
        u = r.rand(B).astype(np.float32)
        out = s2.sample(t, sampling, torch.from_numpy(u).to(DEV), refresh_beta=i == 0)
        torch.cuda.synchronize()
        _check(out, x, experts, beta, prior, u, T, **cuts)


def test_a_captured_step():
    """append -> attend over divided sequences -> LM head -> sample in one graph, replayed on new rows between eager
    steps: attention's partial states and sampling's lists follow each other in one region."""
    m = Coded([6000, 40, 300], 4, "int8", (8, 2, 64), seed=45)
    V, r = 500, np.random.RandomState(46)
    w = (torch.randn(V, 512, generator=torch.Generator().manual_seed(1)) * 0.05).to(torch.bfloat16).to(DEV)
    head = m.sess.pack_lm_head(w)
    sampling = m.sess.sampling(temperature=torch.full((1,), 0.9, device=DEV), top_p=torch.full((1,), 0.95, device=DEV))
    q, k, v = m.rows(1)
    u, qr = torch.full((1,), 0.5, device=DEV), torch.empty_like(q)
    logits = torch.empty((m.S, V), device=DEV)
    x = torch.empty((m.S, 1, 512), dtype=torch.bfloat16, device=DEV)

    def step():
        m.sess.append(q, k, v, rope=(10000.0, 64, False), q_out=qr)
        m.sess.attend(qr, x_out=x)
        m.sess.ctx.pced_lmhead(x[:, 0], m.S, head, logits)
        return m.sess.sample(logits, sampling, u)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    seen = set()
    for i in range(5):
        for a, b in zip((q, k, v), m.rows(1)):
            a.copy_(b)
        u.fill_(float(r.rand()))
        x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in out.items()}, x.clone(), logits.clone()
        want = step()
        torch.cuda.synchronize()
        assert torch.isfinite(got[1]).all()
        _eq(got[1], x), _eq(got[2], logits)
        for n in want:
            _eq(got[0][n], want[n], (i, n))
        seen.add(int(want["tokens"]))
    assert len(seen) > 1
