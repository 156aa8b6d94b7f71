"""pced_attend where scores are -infinity, the type's lowest value or far from zero: weights follow from the
differences of scores alone, whatever batch, wave or part a page falls into."""
import numpy as np
import pytest

from oracle import layer as L

torch = pytest.importorskip("torch")
from tests.test_gpu_layer import DEV, PAGE, Model, _f64, _tt  # noqa: E402

pytestmark = pytest.mark.gpu


def _model(lens, T, dtype, heads, low, value, seed):
    """A session whose sequence 0 has `value` in every key of the pages `low`, and the rows of T appended tokens."""
    m = Model(lens, T, dtype, heads, 1, seed=seed)
    for p in low:
        m.k[0][:, PAGE * p:PAGE * (p + 1)] = value
    m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(T)
    m.sess.append(None, kn, vn, n_tokens=T, rope=None)
    m.grow(kn, vn, T)
    return m, q.abs() + 0.5


def _check(m, q, T, sel, value):
    """Tokens whose keys are `value` weigh nothing; the rest as a softmax without them."""
    out = m.sess.attend(q, n_tokens=T, select=sel)["x"]
    torch.cuda.synchronize()
    got, G = _f64(out).reshape(m.S * T, m.hq, m.d), m.hq // m.hkv
    half = torch.finfo(_tt(m.dtype)).eps / 2
    for s in range(m.S):
        for i in range(T):
            n = m.lens[s] + i + 1
            for h in range(m.hkv):
                qq, kk, vv = _f64(q[s * T + i, 0, h * G:(h + 1) * G]), _f64(m.k[s][0, :n, h]), _f64(m.v[s][0, :n, h])
                pages = L.chosen_pages(qq, kk, *sel) if sel else list(range(-(-n // PAGE)))
                want = L.attend(qq, kk, vv, pages)
                kept = kk[(kk != float(torch.tensor(value, dtype=_tt(m.dtype)).double())).any(axis=1)]
                # scores: fp32 sums of D products; weights: scores, exp2, two bf16 parts, in numerator and sum; sums
                # over the tokens
                ds = (m.d + 4) * 2.0 ** -24 * (np.abs(qq) @ np.abs(kept).T).max() / np.sqrt(m.d)
                rel = 2 * (2 * ds + 2.0 ** -17 + 2.0 ** -21) + 2 * len(pages) * PAGE * 2.0 ** -24
                err = np.abs(got[s * T + i, h * G:(h + 1) * G] - want)
                assert (err <= half * np.abs(want) + rel * np.abs(vv).max()).all(), (s, i, h, float(err.max()))


# pages of sequence 0 (300 tokens: pages 0 .. 18) whose scores are all -inf: a first batch, a batch in the middle, a
# wave's batches, a part of 8 pages, all but the row's own page, and all but pages in the middle
LOW = [[0], [0, 1], [4, 5, 6], [2, 3, 10, 11], list(range(8)), list(range(8, 16)), list(range(18)),
       [p for p in range(18) if p not in (6, 13)]]


@pytest.mark.parametrize("low", LOW, ids=lambda x: "_".join(map(str, x[:4])) + ("_and_more" if len(x) > 4 else ""))
@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 64)), ("bf16", (4, 1, 128)), ("f32", (4, 2, 64)), ("f32", (5, 5, 80))])
@pytest.mark.parametrize("value", [float("-inf"), "lowest"])
def test_scores_of_minus_infinity_weigh_nothing(dtype, heads, low, value):
    """-inf keys, and finite ones whose products with q overflow."""
    value = torch.finfo(_tt(dtype)).min if value == "lowest" else value
    for T, sel in ((1, None), (3, None), (1, (6, 2, 1)), (3, (6, 2, 1)), (1, (19, 1, 1))):
        m, q = _model([300, 20], T, dtype, heads, low, value, seed=40)
        _check(m, q, T, sel, value)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_runs_of_minus_infinity(dtype):
    """Whole parts of a long cache, merged with others by k_attend_merge."""
    for low in (range(256), range(100, 561), range(562)):
        for sel in (None, (300, 280, 10)):
            m, q = _model([9000, 17], 1, dtype, (4, 2, 64), low, float("-inf"), seed=41)
            _check(m, q, 1, sel, float("-inf"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sel", [None, (5, 1, 1)])
def test_nothing_but_minus_infinity_is_nan(dtype, sel):
    """As the softmax of such a row is; the other sequence's rows are as ever."""
    m = Model([200, 50], 2, dtype, (4, 2, 64), 1, seed=42)
    m.k[0][:] = float("-inf")
    m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(2)
    kn[:2] = float("-inf")
    m.sess.append(None, kn, vn, n_tokens=2, rope=None)
    m.grow(kn, vn, 2)
    q = q.abs() + 0.5
    x = m.sess.attend(q, n_tokens=2, select=sel)["x"]
    torch.cuda.synchronize()
    assert torch.isnan(x[:2]).all() and torch.isfinite(x[2:]).all()


@pytest.mark.parametrize("low", [-2.0 ** 127, -2.0 ** 120])
def test_finite_scores_far_below_zero(low):
    """Scores near the lowest number of fp32, all alike: the mean of V; and one higher page takes it all."""
    m = Model([80, 18], 1, "f32", (2, 1, 4), 1, seed=43)
    m.k[0][:] = 0
    m.k[0][..., 0] = low
    m.load()
    q, kn, vn = m.rows(1)
    q[:] = 1
    kn[:] = 0
    kn[..., 0] = low
    m.sess.append(None, kn, vn, rope=None)
    m.grow(kn, vn, 1)
    x = m.sess.attend(q)["x"]
    torch.cuda.synchronize()
    v = _f64(m.v[0][0, :, 0])
    # 81 equal weights: sums of 81 terms and a division in fp32
    assert np.abs(_f64(x[0, 0]).reshape(2, 4) - v.mean(0)).max() <= 84 * 2.0 ** -24 * np.abs(v).max()
    m.k[0] = m.k[0][:, :80].clone()
    m.v[0], m.k[1], m.v[1] = m.v[0][:, :80].contiguous(), m.k[1][:, :18].contiguous(), m.v[1][:, :18].contiguous()
    m.k[0][:, 32:48, :, 0] = low / 2
    m.load()
    m.sess.append(None, kn, vn, rope=None)
    x = m.sess.attend(q)["x"]
    torch.cuda.synchronize()
    want = v[32:48].mean(0)
    assert np.abs(_f64(x[0, 0]).reshape(2, 4) - want).max() <= 84 * 2.0 ** -24 * np.abs(v).max()


@pytest.mark.parametrize("heads", [(2, 1, 64), (2, 1, 36)])
@pytest.mark.parametrize("sel", [None, (6, 1, 1)])
@pytest.mark.parametrize("far", [0.0, 20000.0, -300000.0])
def test_scores_far_from_zero(heads, sel, far):
    """Whole-number q and K, whose products are exact, all scores around far / sqrt(D): only differences count."""
    d = heads[2]
    m = Model([250, 20], 1, "f32", heads, 1, seed=44)
    for s in range(2):
        m.k[s] = m.k[s].clamp(-3, 3).round()
        m.k[s][..., 0] = far
    m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(1)
    q, kn = q.clamp(-3, 3).round(), kn.clamp(-3, 3).round()
    q[..., 0], kn[..., 0] = 1, far
    m.sess.append(None, kn, vn, rope=None)
    m.grow(kn, vn, 1)
    x = m.sess.attend(q, select=sel)["x"]
    torch.cuda.synchronize()
    for s in range(2):
        qq, kk, vv = _f64(q[s, 0]), _f64(m.k[s][0, :, 0]), _f64(m.v[s][0, :, 0])
        pages = L.chosen_pages(qq, kk, *sel) if sel else list(range(-(-len(kk) // PAGE)))
        at = np.concatenate([np.arange(PAGE * p, min(PAGE * (p + 1), len(kk))) for p in pages])
        sc = (qq @ kk[at].T) * np.log2(np.e) / np.sqrt(d)
        # exponents: a difference of whole numbers (exact), times a constant rounded to fp32 and a rounding, twice
        # (to the wave's reference and to the block's); exp2 and its uses 2^-21; sums over the tokens; a division
        rel = 2 * (np.log(2) * np.ptp(sc, axis=1).max() * 4 * 2.0 ** -24 + 2.0 ** -21) + 2 * (len(at) + 4) * 2.0 ** -24
        err = np.abs(_f64(x[s, 0]).reshape(-1, d) - L.attend(qq, kk, vv, pages))
        assert err.max() <= rel * np.abs(vv).max(), (s, float(err.max()), rel)


def _one_chain(q, k):
    """q k^T as one fp32 chain per score, products added one after the other (fused): what a single accumulator gives."""
    s = np.zeros((len(q), len(k)), np.float32)
    for d in range(q.shape[1]):
        s = (s.astype(np.float64) + q[:, d:d + 1] * k[None, :, d]).astype(np.float32)
    return s.astype(np.float64)


@pytest.mark.parametrize("heads", [(4, 4, 64), (4, 4, 80), (4, 4, 128)])
def test_fp32_scores_are_summed_in_more_than_one_chain(heads):
    """Wide q, so that the scores' sums make most of the error. A chain's rounding errors add up like its length (each
    is of the partial sum's size, which grows like the root): two halves, added, have 1/sqrt(2) = 0.71 of its error."""
    d = heads[2]
    m = Model([700, 900, 1100, 1300, 800], 1, "f32", heads, 2, seed=45)
    q, kn, vn = m.rows(1)
    q = q * 4
    m.sess.append(None, kn, vn, rope=None)
    m.grow(kn, vn, 1)
    x = m.sess.attend(q)["x"]
    torch.cuda.synchronize()
    mine = chain = 0.0
    for s in range(m.S):
        for l in range(2):
            for h in range(m.hkv):
                qq, kk, vv = _f64(q[s, l, h:h + 1]), _f64(m.k[s][l, :, h]), _f64(m.v[s][l, :, h])
                want = L.attend(qq, kk, vv, range(-(-len(kk) // PAGE)))
                w = _one_chain(qq, kk) / np.sqrt(d)
                w = np.exp(w - w.max())
                mine += ((_f64(x[s, l]).reshape(-1, d)[h] - want) ** 2).sum() / (want ** 2).sum()
                chain += (((w / w.sum()) @ vv - want) ** 2).sum() / (want ** 2).sum()
    assert mine <= 0.85 ** 2 * chain, (mine ** 0.5, chain ** 0.5)
