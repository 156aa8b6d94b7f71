"""A serving loop over caches in 8 bits: a question's rows, then tokens one by one, each layer append -> attend, the last
layer's rows through the LM head, the token sampled from Eq. 2's scores; against the oracles throughout."""
import numpy as np
import pytest

from oracle import sample as O
from tests.test_gpu_adjust import Limits
from tests.test_gpu_codes import CODES, Coded, _check_attend
from tests.test_gpu_layer import Model

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("greedy", [False, True])
def test_decode_loop(code, greedy):
    lens, V, N, layers = [7, 100, 46, 31], 500, 3, 2
    m = Coded(lens, 64, code, (8, 2, 64), layers, max_new=20, seed=21)
    twin = Model(lens, 64, "bf16", (8, 2, 64), layers, seed=21)
    hidden = 8 * 64
    w = (torch.randn(V, hidden, generator=torch.Generator().manual_seed(1)) * 0.05).to(torch.bfloat16).to(DEV)
    head = m.sess.pack_lm_head(w)
    embed = torch.randn(V, layers, 12, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    lim = Limits(V, 1, seed=3, history=30, biases=4, allowed=0.8)
    adjust = m.sess.adjust(**lim.tensors)
    sampling = m.sess.sampling(temperature=torch.tensor([0.0 if greedy else 0.8], device=DEV),
                               top_k=torch.tensor([50], dtype=torch.int32, device=DEV),
                               top_p=torch.tensor([0.95], device=DEV))
    beta, prior = np.full(N, 0.5, np.float32), np.full(N, np.float32(2.5 * np.log(0.5)))
    r = np.random.RandomState(4)

    def step(tokens, lens):
        """The sequences' shared tokens through the layers, and their rows as the twin's pools store them."""
        T = len(tokens)
        rows = embed[torch.as_tensor(tokens, device=DEV)].repeat(m.S, 1, 1, 1)  # [S T][L][12][D]
        q, k, v = rows[:, :, :8], rows[:, :, 8:10], rows[:, :, 10:]
        rope = (10000.0, 64, True)
        for l in range(layers):
            one = lambda t: t[:, l:l + 1].contiguous()  # noqa: E731
            qr = m.sess.append(one(q), one(k), one(v), n_tokens=T, layer=l, n_layers=1, rope=rope)
            x = m.sess.attend(qr, n_tokens=T, layer=l, n_layers=1)["x"]
        m.sess.advance(T)
        twin.sess.append(None, k.contiguous(), v.contiguous(), n_tokens=T, rope=rope)
        twin.sess.advance(T)
        stored = [[twin.sess.read_cache(s, l, n, T) for l in range(layers)] for s, n in enumerate(lens)]
        for i, cache in enumerate((m.k, m.v)):
            for s in range(m.S):
                new = torch.stack([stored[s][l][i].view(torch.bfloat16) for l in range(layers)])
                cache[s] = torch.cat([cache[s], new], 1)
        return qr, x

    tokens = [int(t) for t in r.randint(0, V, 18)]
    for i in range(12):
        qr, x = step(tokens, lens)
        T = len(tokens)
        torch.cuda.synchronize()
        _check_attend(m, qr, x, T, lens, layers=[layers - 1])
        last = x[T - 1::T, 0].contiguous()
        logits = torch.empty((m.S, V), device=DEV)
        m.sess.ctx.pced_lmhead(last, m.S, head, logits)
        u = np.float32(r.rand())
        out = m.sess.sample(logits, sampling, torch.tensor([u], device=DEV), adjust=adjust)
        torch.cuda.synchronize()
        rows = np.stack([lim.row(z, 0) for z in logits.cpu().numpy()])
        S, who = O.scores(rows, beta, prior, lim.mask[0])
        token, _, kept = O.sample(S, 0.0 if greedy else np.float32(0.8).item(), float(u), top_k=50, top_p=np.float32(0.95).item())
        assert out["tokens"].item() == token and out["kept"].item() == kept and out["winner"].item() == who[token]
        if greedy:
            assert m.sess.fuse_adjusted(logits, adjust)["tokens"].item() == token
        lens = [n + T for n in lens]
        assert m.sess.lengths() == lens
        tokens = [token]
