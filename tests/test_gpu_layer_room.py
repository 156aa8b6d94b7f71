"""Calls of pced_attend that the workspace divides into several launches (tests/test_layer_room.py shows that
these are), and captured layers whose every output is cleared before a replay."""
import numpy as np
import pytest

from oracle import layer as L

torch = pytest.importorskip("torch")
from tests.test_gpu_layer import DEV, PAGE, Model, _eq, _f64, _tt  # noqa: E402
from tests.test_layer_room import SPLITS  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", SPLITS, ids=lambda c: c[0])
def test_divided_calls(case):
    """Rows of every launch against the oracle, and all of them against the layers one by one."""
    _, dtype, heads, layers, lens, T, sel, pages = case[:8]
    m = Model(lens, T, dtype, heads, layers, seed=50)
    G = m.hq // m.hkv
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(T)
    m.sess.append(None, kn, vn, n_tokens=T, rope=None)
    m.grow(kn, vn, T)
    out = m.sess.attend(q, n_tokens=T, select=sel, want=("pages",) if pages else ())
    torch.cuda.synchronize()
    x = _f64(out["x"]).reshape(m.S * T, layers, m.hq, m.d)
    half = torch.finfo(_tt(dtype)).eps / 2
    tokens = sorted({0, 1, 7, 8, T // 3, T // 2, T - 2, T - 1} & set(range(T)))
    for s in range(m.S):
        if s > 20 and s % 16 != 5 and s != m.S - 1:  # (short ones, all alike)
            continue
        ks, vs = _f64(m.k[s]), _f64(m.v[s])
        for i in tokens:
            n = m.lens[s] + i + 1
            for l in range(layers):
                for h in range(m.hkv):
                    qq, kk, vv = _f64(q[s * T + i, l, h * G:(h + 1) * G]), ks[l, :n, h], vs[l, :n, h]
                    pg = L.chosen_pages(qq, kk, *sel) if sel else list(range(-(-n // PAGE)))
                    want = L.attend(qq, kk, vv, pg)
                    # (as in test_gpu_layer: scores, weights, sums)
                    ds = (m.d + 4) * 2.0 ** -24 * (np.abs(qq) @ np.abs(kk).T).max() / np.sqrt(m.d)
                    rel = 2 * (2 * ds + 2.0 ** -17 + 2.0 ** -21) + 2 * len(pg) * PAGE * 2.0 ** -24
                    err = np.abs(x[s * T + i, l, h * G:(h + 1) * G] - want)
                    assert (err <= half * np.abs(want) + rel * np.abs(vv).max()).all(), (s, i, l, h, float(err.max()))
                    if pages:
                        assert out["pages"][s * T + i, l, h].tolist() == pg + [-1] * (sel[0] - len(pg)), (s, i, l, h)
    # the bound above for any row: |q| . |k| <= sum |q| max |k|
    top = lambda t: float(t.float().abs().max())  # noqa: E731
    ds = (m.d + 4) * 2.0 ** -24 * float(q.float().abs().sum(-1).max()) * max(map(top, m.k)) / np.sqrt(m.d)
    most = min(-(-(max(m.lens) + T) // PAGE), sel[0] if sel else 1 << 30)
    bound = (2 * (2 * ds + 2.0 ** -17 + 2.0 ** -21) + 2 * most * PAGE * 2.0 ** -24) * max(map(top, m.v))
    for l in range(layers):
        one = m.sess.attend(q[:, l:l + 1].contiguous(), n_tokens=T, select=sel, layer=l, n_layers=1,
                            want=("pages",) if pages else ())
        y = _f64(one["x"]).reshape(m.S * T, m.hq, m.d)
        if pages:
            assert torch.equal(one["pages"][:, 0], out["pages"][:, l])
        # (other parts: sums in another order, each result within the bound of the exact one, and rounded)
        assert (np.abs(y - x[:, l]) <= 2 * (half * (np.maximum(np.abs(y), np.abs(x[:, l])) + bound) + bound)).all()


@pytest.mark.parametrize("dtype,heads,sel", [("bf16", (8, 2, 128), (5, 1, 1)), ("f32", (4, 2, 64), (5, 1, 1)),
                                             ("bf16", (8, 2, 64), None)])
@pytest.mark.parametrize("T", [1, 5, 20])
def test_replayed_appends_write_everything(dtype, heads, sel, T):
    """append and attend captured, then replayed with other rows: the pools' new slots, the summaries of the pages
    that the rows fill, q and x are all cleared before a replay, and equal an eager call's after it."""
    m = Model([211, 47], T, dtype, heads, layers=2, seed=51)  # (the second's page fills)
    m.sess.bind_summary()
    m.sess.summarize()
    q, k, v = m.rows(T)
    q_out, x = torch.empty_like(q), torch.empty((2 * T, 2, m.hq * m.d), dtype=q.dtype, device=DEV)
    rope = (10000.0, m.d, False)

    def layer():
        m.sess.append(q, k, v, n_tokens=T, rope=rope, q_out=q_out)
        m.sess.attend(q_out, n_tokens=T, select=sel, x_out=x)

    torch.cuda.synchronize()
    empty = [p.clone() for p in (m.sess.k_pool, m.sess.v_pool, m.sess.summary)]

    def clear():
        for p, e in zip((m.sess.k_pool, m.sess.v_pool, m.sess.summary), empty):
            p.copy_(e)
        q_out.fill_(0)
        x.fill_(0)

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(3):
        for t, new in zip((q, k, v), m.rows(T)):
            t.copy_(new)
        clear()
        layer()
        torch.cuda.synchronize()
        want = [t.clone() for t in (q_out, x, m.sess.k_pool, m.sess.v_pool, m.sess.summary)]
        assert all(not torch.equal(a, b) for a, b in zip(want[2:], empty))
        clear()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, a, b in zip(("q", "x", "K", "V", "summaries"), (q_out, x, m.sess.k_pool, m.sess.v_pool, m.sess.summary), want):
            _eq(a, b, name)
