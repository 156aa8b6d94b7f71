"""Attention over caches in 8 bits where pages' scales lie far apart and where single weights show: each output against
64 bits, within what the roundings of its own tokens' weights allow."""
import numpy as np
import pytest

from oracle import codes as C
from tests.test_gpu_codes import CODES, Coded, _append_rows
from tests.test_gpu_layer import _f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def _check_weighted(m, q, x, T, lens, products=None):
    """x [S * T][1][Hq * D]: each element is the bf16 of a number as near to the oracle's as the roundings before it allow.

    With w the softmax's weights (largest 1) over a row's n tokens and v the dimension's values, numerator and sum are off by
    * the scores': an fp32 sum of `products` products (D unless the others are zero), its scale and the difference of
      scores: (products + 6) 2^-24 of the products' sizes, relative, twice with the reference's; exp2: 2^-22;
    * in the numerator: the product with V's scale 2^-24, the sum of two bf16 in its place 2^-17;
    * the fp32 sums over n tokens and the parts' states: (n + 64) 2^-24 of the summands' sizes;
    * weights below 2^-126 may count as 0, as may products with V's scale below 2^-126 (2^-108 where a scale is 2^100 or more),
      which meet codes up to 448.
    """
    G = m.hq // m.hkv
    ks, vs = m.values(lens)
    got = _f64(x).reshape(m.S * T, m.hq, m.d)
    for s in range(m.S):
        for i in range(T):
            n = lens[s] + i + 1
            for h in range(m.hkv):
                qq = _f64(q[s * T + i, 0, h * G:(h + 1) * G])
                kk, vv = ks[s][0, :n, h], vs[s][0, :n, h]
                z = qq @ kk.T / np.sqrt(m.d)
                w = np.exp(z - z.max(1, keepdims=True))
                total, size = w.sum(1, keepdims=True), w @ np.abs(vv)
                ds = ((m.d if products is None else products) + 6) * 2.0 ** -24 * (np.abs(qq) @ np.abs(kk).T).max() / np.sqrt(m.d)
                rel = 2 * (2 * ds + 2.0 ** -22) + 2.0 ** -24 + 2.0 ** -17 + 2 * (n + 64) * 2.0 ** -24
                least = 448 * n * 2.0 ** (-108 if np.abs(vv).max() >= 2.0 ** 106 else -126)
                off = (rel * size + np.where(w < 2.0 ** -125, w, 0) @ np.abs(vv)) / total + least
                want, y = C.attend(qq, kk, vv), got[s * T + i, h * G:(h + 1) * G]
                bad = ~((_bf16(want - off) <= y) & (y <= _bf16(want + off)))
                assert not bad.any(), (s, i, h, int(bad.sum()), want[bad][:4], y[bad][:4], off[bad][:4])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("T", [1, 9, 40])
@pytest.mark.parametrize("large,nats", [(2.0 ** 24, 40), (2.0 ** 33, 40), (2.0 ** 60, 90), (float("inf"), 200)])
def test_large_values_that_nothing_looks_at(code, T, large, nats):
    """Pages of values of size 1 next to pages of far larger ones whose scores are `nats` below; some columns look at
    those instead (where they are finite)."""
    lens = [4200, 700, 300]
    m = Coded(lens, T, code, (8, 2, 64), seed=31)
    a = np.sqrt(nats / 2 * 8.0)  # scores of +-nats / 2 from one dimension
    for s, n in enumerate(lens):
        far = np.arange(n) // 16 % 7 == 2
        m.k[s][:, :, :, 0] = torch.from_numpy(np.where(far, -a, a)).to(m.k[s])[:, None]
        at = torch.from_numpy(far).to(m.v[s].device)
        if np.isfinite(large):
            m.v[s][:, at] *= large
        else:  # a single one per page
            m.v[s][:, at.nonzero()[::16, 0], :, 5] = large
    m.load()
    q, k, v = m.rows(T)
    k[..., 0] = a
    q[..., 0] = a
    if np.isfinite(large):
        q[:, :, 2::4, 0] = -a
    m.sess.append(None, k, v, n_tokens=T, rope=None)
    x = m.sess.attend(q, n_tokens=T)["x"]
    m.grow(k, v, T)
    torch.cuda.synchronize()
    _check_weighted(m, q, x, T, lens)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 128), (16, 1, 128)])
@pytest.mark.parametrize("T", [1, 9, 40])
def test_single_weights(code, heads, T):
    """Dimensions that are one token's weight each: the weights' own roundings show."""
    lens = [96, 50, 16]
    m = Coded(lens, T, code, heads, seed=32)
    for s, n in enumerate(lens):
        m.k[s][..., 1:] = 0
        m.v[s][:] = 0
        d = torch.arange(m.d, device=m.v[s].device)
        m.v[s][:, d * 37 % n, :, d] = 1
    m.load()
    q, k, v = m.rows(T)
    q[..., 1:], k[..., 1:], v[:] = 0, 0, 0
    m.sess.append(None, k, v, n_tokens=T, rope=None)
    x = m.sess.attend(q, n_tokens=T)["x"]
    m.grow(k, v, T)
    torch.cuda.synchronize()
    _check_weighted(m, q, x, T, lens, products=1)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("heads,layers,lens,T", [
    ((8, 2, 64), 1, [1, 300, 16, 47, 15], 1),
    ((28, 4, 128), 1, [1000, 20], 5),
    ((8, 2, 64), 1, [4500, 17], 20),
    ((16, 1, 128), 1, [400, 33], 2),   # 32 columns: one tile
    ((16, 1, 64), 1, [400, 33], 3),    # 48: two tiles, two groups of two and one token
    ((44, 4, 64), 1, [130, 5], 3),     # 33: two tiles, two tokens of 22 columns, then one
    ((12, 1, 128), 1, [129, 5], 7),    # groups of two tokens of 24 columns, the last of one
    ((4, 4, 64), 1, [257 * 16 - 3, 9], 33),
])
def test_weighted_bound(code, heads, layers, lens, T):
    m = Coded(lens, T, code, heads, layers, seed=33)
    q, k, v = _append_rows(m, T)
    x = m.sess.attend(q, n_tokens=T)["x"]
    m.grow(k, v, T)
    torch.cuda.synchronize()
    _check_weighted(m, q, x, T, lens)


@pytest.mark.parametrize("code", CODES)
def test_sharp_scores_and_uneven_blocks_weighted(code):
    """Scores far apart and blocks whose scales differ by twenty orders, each row held to the tokens it looks at."""
    m = Coded([400, 333], 2, code, (8, 2, 64), seed=8)
    m.v[0][:, 32:64] *= 1e10
    m.v[0][:, 64:96] *= 1e-10
    m.k[1][:, 48:64] = 0
    m.load()
    q, k, v = _append_rows(m, 2, spread=30.0)
    q[2] = 0
    x = m.sess.attend(q, n_tokens=2)["x"]
    m.grow(k, v, 2)
    torch.cuda.synchronize()
    _check_weighted(m, q, x, 2, [400, 333])


@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 4, 128), (16, 1, 64)])
@pytest.mark.parametrize("T", [1, 5, 21])
def test_infinite_values_behind_the_complete_pages(heads, T):
    """Infinities and NaN in some dimensions of rows that columns see: the weighted sum's own, and its other dimensions as
    if they were 0."""
    lens = [37, 127, 11]
    m = Coded(lens, T, "int8", heads, seed=34)
    q, k, v = m.rows(T)
    r = np.random.RandomState(35)

    def bad(x):
        """x with one in forty values replaced."""
        what = torch.from_numpy(r.choice([np.inf, -np.inf, np.nan], tuple(x.shape), p=[0.45, 0.45, 0.1])).to(x)
        return torch.where(torch.from_numpy(r.rand(*x.shape) < 1 / 40).to(x.device), what, x)

    v = bad(v)
    for s, n in enumerate(lens):
        m.v[s][:, n // 16 * 16:] = bad(m.v[s][:, n // 16 * 16:])
    rows, new = m.v, v
    out = []
    for clean in (False, True):
        zero = (lambda x: torch.where(torch.isfinite(x), x, 0)) if clean else (lambda x: x)
        m.v, v = [zero(x) for x in rows], zero(new)
        m.load()
        m.sess.append(None, k, v, n_tokens=T, rope=None)
        out.append(_f64(m.sess.attend(q, n_tokens=T)["x"]).reshape(m.S * T, m.hq, m.d))
    m.v, v, G = rows, new, m.hq // m.hkv
    m.grow(k, v, T)
    ks, vs = m.values(lens)
    seen = set()
    for s in range(m.S):
        for i in range(T):
            n = lens[s] + i + 1
            for h in range(m.hkv):
                at = (s * T + i, slice(h * G, (h + 1) * G))
                with np.errstate(invalid="ignore"):
                    want = C.attend(_f64(q[s * T + i, 0, h * G:(h + 1) * G]), ks[s][0, :n, h], vs[s][0, :n, h])
                odd = ~np.isfinite(want)
                assert np.array_equal(out[0][at][odd], want[odd], equal_nan=True), (s, i, h)
                assert np.array_equal(out[0][at][~odd], out[1][at][~odd]), (s, i, h)
                seen |= set(map(str, want[odd]))
    assert seen == {"inf", "-inf", "nan"}
