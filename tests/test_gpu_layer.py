"""The layer-wise calls on the GPU (append with rotation, page summaries, attention over
chosen pages) against the float64 oracle (oracle/layer.py), at sizes where they can go
wrong. Summaries and chosen pages are exact; other tolerances follow from the roundings."""
import numpy as np
import pytest

from oracle import layer as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 16


def _tt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _eq(a, b, msg=""):
    """Equal bits."""
    v = {2: torch.int16, 4: torch.int32, 1: torch.uint8}[a.element_size()]
    assert a.shape == b.shape and torch.equal(a.contiguous().view(v), b.contiguous().view(v)), msg


class Model:
    """A session over random caches (poisoned pools, pages in random order) and the caches' rows, which grow
    with every append."""

    def __init__(self, lens, room, dtype="bf16", heads=(8, 2, 64), layers=1, seed=0, scale=1.0, order=True, **kw):
        from paper_2601_08670_amd.session import PcedSession
        self.hq, self.hkv, self.d = heads
        self.dtype, self.lens, self.layers, self.S = dtype, list(lens), layers, len(lens)
        self.r = np.random.RandomState(seed)
        need = [-(-(n + room) // PAGE) for n in lens]
        self.sess = PcedSession(n_layers=layers, n_q_heads=self.hq, n_kv_heads=self.hkv, head_dim=self.d, vocab=500,
                                dtype=dtype, max_queries=1, max_seqs=max(2, self.S), max_pages=sum(need) + 3,
                                max_pages_per_seq=max(need), device=DEV, poison=True, **kw)
        ids = self.r.permutation(sum(need) + 3) if order else np.arange(sum(need))
        self.table, at = np.full((self.S, max(need)), -1, np.int32), 0
        for s, n in enumerate(need):
            self.table[s, :n] = ids[at:at + n]
            at += n
        shape = lambda n: (layers, n, self.hkv, self.d)  # noqa: E731
        self.k = [self.rand(shape(n), scale) for n in lens]
        self.v = [self.rand(shape(n)) for n in lens]
        self.load()

    def load(self):
        self.sess.load([self.S - 1], self.lens, self.k, self.v, [0.5] * (self.S - 1), beta=[0.5] * (self.S - 1),
                       page_table=self.table)

    def rand(self, shape, scale=1.0):
        return torch.from_numpy(self.r.randn(*shape) * scale).to(_tt(self.dtype)).to(DEV)

    def rows(self, T, layers=None, scale=1.0):
        n = self.layers if layers is None else layers
        return tuple(self.rand((self.S * T, n, h, self.d), scale) for h in (self.hq, self.hkv, self.hkv))

    def grow(self, k, v, T):
        """The caches with the rows as they were stored (taken from the pool by the caller)."""
        for s in range(self.S):
            self.k[s] = torch.cat([self.k[s], k[s * T:(s + 1) * T].transpose(0, 1)], 1)
            self.v[s] = torch.cat([self.v[s], v[s * T:(s + 1) * T].transpose(0, 1)], 1)

    def tile_offsets(self):
        t, d = np.arange(PAGE)[:, None], np.arange(self.d)[None, :]
        if self.dtype == "f32":
            return [torch.from_numpy(t * self.d + d).to(DEV)] * 2
        j = d // 16
        k = ((d // 32) * 64 + t + 16 * ((d % 32) // 8)) * 8 + d % 8
        v = ((j // 2 * 64 + d % 16 + 16 * (t // 4)) * 2 + j % 2) * 4 + t % 4
        return [torch.from_numpy(x).to(DEV) for x in (k, v)]

    def pools(self):
        """[K, V] pools as [L][pages][Hkv][16][D] copies, tokens in order."""
        out = []
        for p, at in zip((self.sess.k_pool, self.sess.v_pool), self.tile_offsets()):
            x = p.view(_tt(self.dtype)).view(self.layers, -1, self.hkv, PAGE * self.d)
            out.append(x[..., at.reshape(-1)].view(self.layers, -1, self.hkv, PAGE, self.d).clone())
        return out

    def summaries(self):
        """Codes [L][Hkv][pages][2D] and scales [L][Hkv][pages]."""
        n = self.layers * self.hkv * self.sess.cfg.max_pages
        row = -(-2 * self.d // 64) * 64
        codes = self.sess.summary[:n * row].view(torch.int8).view(self.layers, self.hkv, -1, row)
        at = -(-n * row // 256) * 256
        scale = self.sess.summary[at:at + 4 * n].view(torch.float32).view(self.layers, self.hkv, -1)
        return codes.cpu().numpy(), scale.cpu().numpy()


# (dtype, (Hq, Hkv, D), layers, lengths, new tokens)
APPENDS = [
    ("bf16", (8, 2, 64), 1, [5, 40, 16, 31, 1], 1),
    ("bf16", (4, 4, 64), 2, [15, 32], 1),
    ("bf16", (32, 8, 128), 3, [2, 47, 17], 1),
    ("bf16", (8, 8, 128), 1, [13, 30, 64], 7),
    ("bf16", (28, 4, 128), 1, [1, 100], 33),
    ("bf16", (16, 1, 128), 2, [14, 3], 50),
    ("f32", (4, 2, 64), 1, [5, 40, 16], 1),
    ("f32", (5, 5, 80), 2, [15, 31], 18),
    ("f32", (6, 2, 32), 1, [9, 12], 5),
    ("f32", (4, 1, 4), 1, [16, 7], 3),
]


@pytest.mark.parametrize("dtype,heads,layers,lens,T", APPENDS)
@pytest.mark.parametrize("rot,halves", [(1.0, False), (1.0, True), (0.5, True), (0.25, False), (0.0, True), (None, False)])
def test_append(dtype, heads, layers, lens, T, rot, halves):
    m = Model(lens, T, dtype, heads, layers)
    d, theta = heads[2], 10000.0
    unit = 16 if dtype == "bf16" else 8
    n_rot = 0 if rot is None else int(d * rot) // (unit if halves else 2) * (unit if halves else 2)
    q, k, v = m.rows(T)
    before = m.pools()
    got = m.sess.append(q, k, v, n_tokens=T, rope=None if rot is None else (theta, n_rot, halves))
    torch.cuda.synchronize()
    after = m.pools()
    assert m.sess.lengths() == lens
    new = torch.zeros(before[0].shape[1:4:2], dtype=torch.bool, device=DEV)  # [pages][16]
    half = torch.finfo(_tt(dtype)).eps / 2
    for s, n in enumerate(lens):
        for i in range(T):
            page, t, r = int(m.table[s, (n + i) // PAGE]), (n + i) % PAGE, s * T + i
            new[page, t] = True
            _eq(after[1][:, page, :, t], v[r], (s, i))
            for x, y in ((k[r], after[0][:, page, :, t]), (q[r], got[r])):
                _eq(x[..., n_rot:], y[..., n_rot:], (s, i))
                if n_rot:
                    x64 = _f64(x)
                    want = L.rotate(x64, n + i, theta, n_rot, halves)[..., :n_rot]
                    # rounded once to the type; before that cos, sin (half a step of 1, twice), two products and
                    # their sum in fp32, of values at most |a| + |b| <= 2 max |x|
                    tol = half * np.abs(want) + 5 * 2.0 ** -24 * 2 * np.abs(x64).max() * (1 + half)
                    assert (np.abs(_f64(y)[..., :n_rot] - want) <= tol).all(), (s, i)
    for a, b in zip(before, after):  # everything else is as it was
        keep = ~new[None, :, None, :, None].expand(a.shape)
        _eq(torch.where(keep, a, 0), torch.where(keep, b, 0))


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 128)), ("f32", (5, 5, 80))])
def test_append_of_strided_rows_in_place_and_of_layers(dtype, heads):
    """Views of one projection's output, q in place, and one layer at a time: as whole contiguous calls."""
    hq, hkv, d = heads
    T, lens, rope = 5, [14, 40], (500000.0, d, True)
    a, b, c = (Model(lens, T, dtype, heads, 2, seed=3) for _ in range(3))
    q, k, v = a.rows(T)
    want = a.sess.append(q, k, v, n_tokens=T, rope=rope)
    for l in range(2):
        fused = torch.cat([x[:, l].reshape(len(lens) * T, -1) for x in (q, k, v)] + [a.rand((len(lens) * T, 16))], 1)
        parts = [x.unflatten(1, (1, h, d)) for x, h in zip(fused.split([hq * d, hkv * d, hkv * d, 16], 1), (hq, hkv, hkv))]
        _eq(b.sess.append(*parts, n_tokens=T, rope=rope, layer=l, n_layers=1)[:, 0], want[:, l])
    mine = q.clone()
    assert c.sess.append(mine, k, v, n_tokens=T, rope=rope, q_out=mine) is mine
    _eq(mine, want)
    for x, y, z in zip(a.pools(), b.pools(), c.pools()):
        _eq(x, y)
        _eq(x, z)
    assert c.sess.append(None, k, v, n_tokens=T, rope=rope) is None
    for x, z in zip(a.pools(), c.pools()):
        _eq(x, z)


def test_far_positions():
    """Angles of positions beyond 2^17, where fp32 angles would be off by more than 2^-8."""
    m = Model([140000, 1], 2, "f32", (2, 1, 64), order=False)
    q, k, v = m.rows(1)
    got = m.sess.append(q, k, v, rope=(500000.0, 64, False))
    want = L.rotate(_f64(q[0]), 140000, 500000.0, 64, False)
    assert np.abs(_f64(got[0]) - want).max() <= 2.0 ** -23 * 2 * np.abs(_f64(q[0])).max() * 3


def _check_summaries(m, upto):
    codes, scale = m.summaries()
    for s in range(m.S):
        for p in range(upto[s] // PAGE):
            phys = int(m.table[s, p])
            for l in range(m.layers):
                for h in range(m.hkv):
                    k = _f64(m.k[s][l, PAGE * p:PAGE * (p + 1), h])
                    mx, mn, e = L.summarize(k)
                    assert np.array_equal(codes[l, h, phys, :m.d], mx), (s, p, l, h)
                    assert np.array_equal(codes[l, h, phys, m.d:2 * m.d], mn), (s, p, l, h)
                    assert scale[l, h, phys] == 2.0 ** e


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 64)), ("bf16", (8, 2, 128)), ("f32", (5, 5, 80)), ("f32", (4, 2, 4))])
def test_summaries(dtype, heads):
    """Exact, of caches with zeros, infinities, NaN and extreme scales, and kept by appends that fill pages."""
    m = Model([5, 16, 95, 33], 70, dtype, heads, layers=2, seed=4)
    k = m.k[2]
    k[0, 0:16] = 0
    k[0, 16:32] *= 1e-30
    k[0, 32:48] *= 1e25
    k[0, 50] = float("inf")
    k[1, 3, :, 1] = float("nan")
    k[1, 16:32, :, 2] = float("nan")
    k[1, 32:48] = float("nan")
    k[1, 64:80] = 1.0
    k[1, 64, :, 0] = 127.5
    k[1, 80:90] = -1e-40 if dtype == "f32" else -1e-39
    m.load()
    m.sess.bind_summary()
    m.sess.summary.fill_(85)
    m.sess.summarize()
    torch.cuda.synchronize()
    _check_summaries(m, [n for n in m.lens])
    upto = list(m.lens)
    for T in (11, 1, 1, 40):
        q, kn, vn = m.rows(T)
        m.sess.append(None, kn * 3, vn, n_tokens=T, rope=None)      # (rows that are replaced)
        m.sess.append(None, kn, vn, n_tokens=T, rope=None)
        m.sess.advance(T)
        m.grow(kn, vn, T)
        upto = [n + T for n in upto]
        torch.cuda.synchronize()
        _check_summaries(m, upto)
    assert m.sess.lengths() == upto


def _attend_ref(m, q, T, sel, pages_of=None):
    """(x [R][L][Hq][D], pages [R][L][Hkv] lists, error bound of x before rounding)"""
    R, G = m.S * T, m.hq // m.hkv
    x, bound = np.zeros((R, m.layers, m.hq, m.d)), np.zeros((R, m.layers, m.hq, 1))
    pages = {}
    for s in range(m.S):
        ks, vs = _f64(m.k[s]), _f64(m.v[s])
        for i in range(T):
            n = m.lens[s] + i + 1
            for l in range(m.layers):
                for h in range(m.hkv):
                    qq, kk, vv = _f64(q[s * T + i, l, h * G:(h + 1) * G]), ks[l, :n, h], vs[l, :n, h]
                    pg = L.chosen_pages(qq, kk, *sel) if sel else list(range(-(-n // PAGE)))
                    pages[s * T + i, l, h] = pg
                    x[s * T + i, l, h * G:(h + 1) * G] = L.attend(qq, kk, vv, pg)
                    # a score's fp32 sum of D products (and its scaling) is off by at most (D + 4) 2^-24 times the
                    # sum of their sizes; a weight's relative error is at most that of scores, of exp2 and of its two
                    # bf16 parts (2^-17), twice (numerator and sum), and the sums over n tokens add n 2^-24
                    ds = (m.d + 4) * 2.0 ** -24 * (np.abs(qq) @ np.abs(kk).T).max() / np.sqrt(m.d)
                    rel = 2 * (2 * ds + 2.0 ** -17 + 2.0 ** -21) + 2 * len(pg) * PAGE * 2.0 ** -24
                    bound[s * T + i, l, h * G:(h + 1) * G] = rel * np.abs(vv).max()
    return x, pages, bound


def _run_attend(m, T, sel, q=None, spread=1.0):
    qr, kn, vn = m.rows(T)
    q = qr * spread if q is None else q
    m.sess.append(None, kn, vn, n_tokens=T, rope=None)
    m.grow(kn, vn, T)
    out = m.sess.attend(q, n_tokens=T, select=sel, want=("pages",) if sel else ())
    torch.cuda.synchronize()
    return q, out


def _check_attend(m, q, out, T, sel):
    x, pages, bound = _attend_ref(m, q, T, sel)
    got = _f64(out["x"]).reshape(x.shape)
    half = torch.finfo(_tt(m.dtype)).eps / 2
    if sel:
        lists = out["pages"].cpu().numpy()
        for (r, l, h), pg in pages.items():
            assert lists[r, l, h].tolist() == pg + [-1] * (sel[0] - len(pg)), (r, l, h)
    err = np.abs(got - x) - (half * np.abs(x) + bound)
    assert (err <= 0).all(), float(err.max())


# (dtype, heads, layers, lengths, new tokens, (pages, first, last) or None)
ATTENDS = [
    ("bf16", (8, 2, 64), 1, [1, 300, 16, 47], 1, (4, 1, 1)),
    ("bf16", (8, 2, 64), 2, [500, 15], 1, (5, 0, 1)),
    ("bf16", (32, 8, 128), 1, [64, 700, 431], 1, (8, 1, 2)),
    ("bf16", (28, 4, 128), 1, [1000, 20], 5, (9, 2, 3)),
    ("bf16", (16, 1, 128), 1, [400, 33], 19, (6, 1, 1)),
    ("bf16", (4, 4, 64), 3, [250, 60, 7], 17, (3, 1, 1)),
    ("bf16", (8, 2, 128), 1, [300, 40], 33, (3, 1, 2)),
    ("bf16", (8, 2, 128), 1, [300, 40], 2, (1, 0, 1)),
    ("bf16", (8, 2, 128), 1, [300, 40], 1, None),
    ("bf16", (8, 2, 64), 2, [6000, 1], 1, None),
    ("bf16", (8, 2, 64), 1, [4500, 1], 1, (200, 1, 5)),
    ("bf16", (8, 2, 64), 1, [100, 17], 16, (100, 1, 5)),
    ("f32", (4, 2, 64), 1, [128, 300, 16, 1], 1, (4, 1, 1)),
    ("f32", (5, 5, 80), 2, [200, 31], 3, (5, 1, 2)),
    ("f32", (6, 2, 32), 1, [2000, 15], 1, (60, 0, 1)),
    ("f32", (16, 1, 128), 1, [300, 2], 18, (7, 1, 1)),
    ("f32", (4, 2, 4), 1, [90, 33], 2, (3, 1, 1)),
    ("f32", (3, 3, 100), 1, [90, 33], 2, None),
]


@pytest.mark.parametrize("dtype,heads,layers,lens,T,sel", ATTENDS)
def test_attend(dtype, heads, layers, lens, T, sel):
    m = Model(lens, T, dtype, heads, layers, seed=7)
    m.sess.bind_summary()
    m.sess.summarize()
    q, out = _run_attend(m, T, sel)
    _check_attend(m, q, out, T, sel)


@pytest.mark.parametrize("dtype,lens,T,sel", [
    ("f32", [9000, 100], 1, (40, 2, 3)),        # bounds and choice in two launches, from here on
    ("bf16", [20000, 8300], 2, (600, 1, 1)),
    ("f32", [131500, 40], 1, (300, 0, 1)),
    ("f32", [270000, 500], 1, (100, 1, 1)),     # keys in rounds
])
def test_attend_over_long_caches(dtype, lens, T, sel):
    m = Model(lens, T, dtype, (4, 2, 64) if dtype == "bf16" else (2, 1, 8), seed=30)
    m.sess.bind_summary()
    m.sess.summarize()
    q, out = _run_attend(m, T, sel)
    _check_attend(m, q, out, T, sel)


@pytest.mark.parametrize("kind", ["equal", "outlier", "steps", "many_steps"])
def test_long_choices_among_crowded_bounds(kind):
    """Bounds that fall into few places of their range: all equal, all but one close together, a few values."""
    m = Model([300000 if kind == "many_steps" else 12000, 20], 1, "f32", (2, 1, 8), seed=31)
    k, n = m.k[0], m.lens[0]
    if kind == "equal":
        k[:] = 0.5
    elif kind == "outlier":
        k *= 1e-4
        k[:, 5000] = 1e4
    else:
        k[:] = torch.arange(n, device=DEV).div(16, rounding_mode="floor").remainder(5).float().view(1, -1, 1, 1) + 1
    m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    for sel in ((100, 1, 1), (3, 1, 1), (700, 0, 2)):
        q = m.rows(1)[0].abs()
        kn, vn = m.rows(1)[1:]
        m.sess.append(None, kn, vn)
        out = m.sess.attend(q, select=sel, want=("pages",))
        torch.cuda.synchronize()
        pages = L.chosen_pages(_f64(q[0, 0]), np.concatenate([_f64(m.k[0][0, :, 0]), _f64(kn[0, 0])]), *sel)
        assert out["pages"][0, 0, 0].tolist() == pages


@pytest.mark.parametrize("n", [12000, 40000, 70000])
@pytest.mark.parametrize("kind", ["random", "equal"])
def test_long_choices_of_many_rows(n, kind):
    """Rows beyond the compute units (all layers together) and within them (layer by layer) choose the same pages."""
    m = Model([n, 20], 1, "f32", (64, 64, 4), layers=3, seed=32)
    if kind == "equal":
        m.k[0][1:] = 0.5
        m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(1)
    if kind == "equal":
        q = q.abs()
    m.sess.append(None, kn, vn)
    for sel in ((200, 1, 1), (7, 0, 2)):
        a = m.sess.attend(q, select=sel, want=("pages",))["pages"]
        for l in range(3):
            b = m.sess.attend(q[:, l:l + 1].contiguous(), select=sel, layer=l, n_layers=1, want=("pages",))["pages"]
            assert torch.equal(b[:, 0], a[:, l])
            for h in (0, 63):
                keys = np.concatenate([_f64(m.k[0][l, :, h]), _f64(kn[0, l, h:h + 1])])
                assert a[0, l, h].tolist() == L.chosen_pages(_f64(q[0, l, h:h + 1]), keys, *sel)


def test_attend_sharp_and_equal_scores():
    """Scores far apart (one token takes it all), and pages that measure the same: the lower ones are chosen."""
    m = Model([400, 333], 1, "bf16", (8, 2, 64), seed=8)
    m.k[0][:, 64:208] = m.k[0][:, 48:64].repeat(1, 9, 1, 1)      # pages 4 .. 12 are page 3 again
    m.k[1][:] = 0.25
    m.load()
    m.sess.bind_summary()
    m.sess.summarize()
    q, out = _run_attend(m, 1, (7, 1, 1), spread=30.0)
    _check_attend(m, q, out, 1, (7, 1, 1))


def test_attend_zero_and_extreme_queries():
    m = Model([200, 100], 1, "f32", (4, 2, 64), seed=9)
    m.sess.bind_summary()
    m.sess.summarize()
    q = m.rows(1)[0]
    q[0] = 0
    q[1, :, :2] *= 1e-38
    q, out = _run_attend(m, 1, (4, 1, 1), q=q)
    _check_attend(m, q, out, 1, (4, 1, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_with_unwritten_rows_and_bad_values_behind(dtype):
    """NaN and infinities behind a row's position (in its own page) leave it alone; within its reach they show."""
    m = Model([37, 100], 4, dtype, (4, 2, 64), seed=10)
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(4)
    bad_k, bad_v = kn.clone(), vn.clone()
    bad_k[2::4] = float("nan")          # token 2 of each sequence
    bad_v[2::4] = float("inf")
    m.sess.append(None, kn, vn, n_tokens=4, rope=None)
    good = m.sess.attend(q, n_tokens=4, select=(3, 1, 1))["x"]
    m.sess.append(None, bad_k, bad_v, n_tokens=4, rope=None)
    out = m.sess.attend(q, n_tokens=4, select=(3, 1, 1))["x"]
    torch.cuda.synchronize()
    for s in range(2):
        _eq(out[4 * s:4 * s + 2], good[4 * s:4 * s + 2])
        assert torch.isnan(out[4 * s + 2:4 * s + 4]).all()
    # fewer tokens than were appended: the first ones
    two = torch.cat([q[0:2], q[4:6]])
    _eq(m.sess.attend(two, n_tokens=2, select=(3, 1, 1))["x"], torch.cat([good[0:2], good[4:6]]))


def test_attend_is_the_same_however_it_is_launched():
    """Layers together or one by one, and repeated calls: the same bits."""
    m = Model([700, 33, 512], 3, "bf16", (8, 2, 128), layers=5, seed=11)
    m.sess.bind_summary()
    m.sess.summarize()
    q, kn, vn = m.rows(3)
    m.sess.append(None, kn, vn, n_tokens=3, rope=None)
    sel = (12, 1, 2)
    a = m.sess.attend(q, n_tokens=3, select=sel, want=("pages",))
    b = m.sess.attend(q, n_tokens=3, select=sel)      # lists kept in the workspace
    _eq(a["x"], b["x"])
    for l in range(5):
        c = m.sess.attend(q[:, l:l + 1].contiguous(), n_tokens=3, select=sel, layer=l, n_layers=1, want=("pages",))
        _eq(c["pages"][:, 0], a["pages"][:, l])
        # (another number of parts sums in another order)
        diff = (c["x"][:, 0].float() - a["x"][:, l].float()).abs().max()
        assert float(diff) <= 2.0 ** -8 * float(a["x"].float().abs().max())


def test_pages_beyond_the_workspace_go_in_several_launches():
    """One long sequence and many rows: the page lists and partial states of all rows do not fit at once."""
    m = Model([3000, 1], 48, "f32", (4, 4, 8), layers=3, seed=12)
    m.sess.bind_summary()
    m.sess.summarize()
    q, out = _run_attend(m, 48, (20, 1, 1))
    _check_attend(m, q, out, 48, (20, 1, 1))


def test_attention_of_a_step_agrees_with_pced_step():
    """append + attend over all pages against pced_step's own append and attention, and the lengths after both."""
    a = Model([70, 300, 16], 3, "bf16", (8, 2, 64), layers=2, seed=13)
    b = Model([70, 300, 16], 3, "bf16", (8, 2, 64), layers=2, seed=13)
    w = a.sess.pack_lm_head(a.rand((500, 512), 0.02))
    for _ in range(3):
        q, k, v = a.rows(1)
        ref = a.sess.step(q, k, v, w, want=("attn_out", "hidden"))
        b.sess.append(None, k, v)
        x = b.sess.attend(q)["x"]
        b.sess.advance()
        torch.cuda.synchronize()
        want = ref["attn_out"].view(3, 2, 512)
        # the step rounds its weights and its partial outputs to bf16 (2^-8 each), both round the output
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -8 * 3) * float(max(t.float().abs().max() for t in a.v))
        assert ((x.float() - want).abs() <= tol).all()
        for p, r in zip(a.pools(), b.pools()):
            _eq(torch.nan_to_num(p), torch.nan_to_num(r))
    assert a.sess.lengths() == b.sess.lengths() == [73, 303, 19]


def test_summaries_after_steps_and_generated_text():
    """Tokens that other calls append are summarised by pced_summarize, which appends then keep up to date."""
    from paper_2601_08670_amd._lib import PcedError
    m = Model([30, 100], 60, "bf16", (8, 2, 64), layers=2, seed=14)
    m.sess.bind_summary()
    m.sess.summarize()
    w = m.sess.pack_lm_head(m.rand((500, 512), 0.02))
    m.sess.generate(20, 5, 1, w)
    q, kn, vn = m.rows(1)
    m.sess.append(None, kn, vn)
    with pytest.raises(PcedError, match="STATE.*up to date"):
        m.sess.attend(q, select=(3, 1, 1))
    m.sess.summarize()
    m.sess.append(None, kn, vn)
    out = m.sess.attend(q, select=(3, 1, 1), want=("pages",))
    torch.cuda.synchronize()
    for s, n in enumerate(m.sess.lengths()):
        rows = [m.sess.read_cache(s, l, 0, n) for l in range(2)]
        m.k[s], m.v[s] = (torch.stack([x[i].view(torch.bfloat16) for x in rows]) for i in (0, 1))
    m.lens = m.sess.lengths()
    m.grow(kn, vn, 1)
    _check_summaries(m, m.lens)
    _check_attend(m, q, out, 1, (3, 1, 1))


def test_replayed_layer():
    """append and attend captured into a graph and replayed with other rows, eager work between the replays."""
    m = Model([200, 47], 3, "bf16", (8, 2, 128), layers=2, seed=15)
    m.sess.bind_summary()
    m.sess.summarize()
    q, k, v = m.rows(3)
    q_out, x = torch.empty_like(q), torch.empty((6, 2, 1024), dtype=q.dtype, device=DEV)
    rope, sel = (10000.0, 128, False), (5, 1, 1)

    def layer():
        m.sess.append(q, k, v, n_tokens=3, rope=rope, q_out=q_out)
        m.sess.attend(q_out, n_tokens=3, select=sel, x_out=x)

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(3):
        for t, new in zip((q, k, v), m.rows(3)):
            t.copy_(new)
        layer()
        want = (q_out.clone(), x.clone(), m.pools())
        torch.cuda.synchronize()
        x.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        _eq(q_out, want[0])
        _eq(x, want[1])
        for a, b in zip(m.pools(), want[2]):
            _eq(a, b)


def test_other_stream_and_two_sessions():
    a = Model([600, 33], 1, "bf16", (8, 2, 64), seed=16)
    b = Model([90, 410], 1, "bf16", (8, 2, 64), seed=17)
    sel, want = (6, 1, 1), []
    rows = [m.rows(1) for m in (a, b)]
    for m in (a, b):
        m.sess.bind_summary()
        m.sess.summarize()
    for m, (q, k, v) in zip((a, b), rows):
        m.sess.append(None, k, v)
        want.append(m.sess.attend(q, select=sel)["x"].clone())
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for m, (q, k, v), st in zip((a, b), rows, streams):
        with torch.cuda.stream(st):
            m.sess.append(None, k, v)
            got.append(m.sess.attend(q, select=sel)["x"])
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        _eq(x, y)


def test_session_refusals():
    m = Model([40, 20], 4, "bf16", (8, 2, 64), layers=2)
    q, k, v = m.rows(2)
    s = m.sess
    for bad in (lambda: s.append(q.float(), k, v, n_tokens=2), lambda: s.append(q, k[:2], v, n_tokens=2),
                lambda: s.append(q, k, v, n_tokens=1), lambda: s.append(q, k, v.transpose(0, 1), n_tokens=2),
                lambda: s.append(q, k, v, n_tokens=2, q_out=q[:2]), lambda: s.append(q, k, v, n_tokens=2, layer=1),
                lambda: s.append(q, k[..., ::2], v, n_tokens=2), lambda: s.attend(q, n_tokens=1),
                lambda: s.attend(q[:, :1], n_tokens=2, n_layers=1), lambda: s.attend(q, n_tokens=2, want=("pages",)),
                lambda: s.attend(q, n_tokens=2, want=("scores",), select=(2, 0, 1)),
                lambda: s.attend(q, n_tokens=2, x_out=q), lambda: s.append(q.cpu(), k, v, n_tokens=2),
                lambda: s.append(None, k, v.cpu(), n_tokens=2), lambda: s.attend(q.cpu(), n_tokens=2),
                lambda: s.append(q, k, v, n_tokens=2, q_out=q.cpu())):
        with pytest.raises(ValueError):
            bad()
    assert s.lengths() == [40, 20]


def test_steps_of_a_model_layer_by_layer_under_constraints():
    """Decode steps as a program with its own projections runs them: per layer append, attention over chosen pages
    and an output product, then the LM head and the choice under penalties and a mask, with the history growing.
    Every stage is checked from the GPU's own inputs to it."""
    m = Model([900, 40, 333], 8, "bf16", (8, 2, 64), layers=2, seed=20)
    s, H, V, T = m.sess, 512, 500, 2
    s.bind_summary()
    s.summarize()
    wq, wk, wv, wo = (m.rand((2, H, n), 0.05) for n in (512, 128, 128, 512))
    embed, head = m.rand((V, H)), s.pack_lm_head(m.rand((V, H), 0.2))
    history = torch.full((16,), -1, dtype=torch.int32, device=DEV)
    allowed = m.r.rand(V) < 0.3
    bits = np.zeros(512, bool)
    bits[:V] = allowed
    adj = s.adjust(history=history, history_off=torch.tensor([0, 16], dtype=torch.int32, device=DEV),
                   presence=torch.full((1,), 100.0, device=DEV),
                   mask=torch.from_numpy(np.packbits(bits, bitorder="little").view(np.int32)[None].copy()).to(DEV))
    prior = np.float32(2.5 * np.log(np.float64(np.float32(0.5))))
    sel, rope = (10, 1, 2), (10000.0, 64, True)
    tokens = [3, 4]
    for step in range(4):
        T = len(tokens)
        h = embed[torch.tensor(tokens, device=DEV)].repeat(3, 1)
        k_all, v_all = [], []
        for l in range(2):
            q, k, v = ((h @ w[l]).view(3 * T, 1, -1, 64) for w in (wq, wk, wv))
            qr = s.append(q, k, v, n_tokens=T, rope=rope, layer=l, n_layers=1)
            x = s.attend(qr, n_tokens=T, select=sel, layer=l, n_layers=1, want=("pages",))
            h = h + x["x"].view(3 * T, H) @ wo[l]
            if step in (0, 3):
                one = Model.__new__(Model)
                one.__dict__.update(m.__dict__, layers=1)
                pool = m.pools()
                one.k, one.v, one.lens = [], [], s.lengths()
                for i, n in enumerate(one.lens):
                    at = torch.from_numpy(m.table[i, :-(-(n + T) // PAGE)].astype(np.int64)).to(DEV)
                    for dst, p in ((one.k, pool[0]), (one.v, pool[1])):
                        dst.append(p[l, at].transpose(1, 2).reshape(1, -1, m.hkv, m.d)[:, :n + T])
                _check_attend(one, qr, x, T, sel)
        s.advance(T)
        last = h.view(3, T, H)[:, -1].contiguous()
        logits = torch.empty((3, V), device=DEV)
        s.ctx.pced_lmhead(last, 3, head, logits)
        out = s.fuse_adjusted(logits, adj)
        torch.cuda.synchronize()
        seen = [t for t in history.tolist() if t >= 0]
        rows = [L.adjust_row(r, history=seen, presence=100.0, allowed=allowed, real=np.float32) for r in logits.cpu().numpy()]
        want = L.choose(rows, [np.float32(0.5)] * 2, [prior] * 2, allowed, np.float32)
        assert (int(out["tokens"][0]), int(out["winner"][0]), float(out["top1"][0]), float(out["top2"][0])) == want
        assert allowed[want[0]] and want[0] not in seen
        history[step:step + 1] = out["tokens"]
        tokens = [want[0]]
    assert s.lengths() == [905, 45, 338]


def test_tokens_of_the_decoder_stack_under_penalties():
    """pced_model_step's logits, adjusted and chosen, feed the next step: no token comes twice."""
    from paper_2601_08670_amd.session import PcedSession
    r = np.random.RandomState(21)
    rand = lambda *n, scale=0.05: torch.from_numpy(r.randn(*n) * scale).to(torch.bfloat16).to(DEV)  # noqa: E731
    V, H, F = 300, 512, 256
    s = PcedSession(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=V, dtype="bf16", max_queries=1, max_seqs=3,
                    max_pages=30, max_pages_per_seq=10, ffn_dim=F, device=DEV, poison=True)
    model = s.pack_model(lambda l: [1 + rand(H), rand(512, H), rand(128, H), rand(128, H), rand(H, 512), 1 + rand(H),
                                    rand(F, H), rand(F, H), rand(H, F)], rand(V, H, scale=1.0), 1 + rand(H))
    head = s.pack_lm_head(rand(V, H))
    lens = [20, 50, 33]
    cache = [rand(1, n, 2, 64, scale=1.0) for n in lens]
    s.load([2], lens, cache, cache, [0.3, 0.8], reserve_tokens=40)
    history = torch.full((8,), -1, dtype=torch.int32, device=DEV)
    adj = s.adjust(history=history, history_off=torch.tensor([0, 8], dtype=torch.int32, device=DEV),
                   presence=torch.full((1,), 1e4, device=DEV))
    tok = torch.tensor([7], dtype=torch.int32, device=DEV)
    for i in range(8):
        out = s.model_step(model, head, tok, want=("logits", "beta_used"))
        got = s.fuse_adjusted(out["logits"], adj)
        assert torch.equal(got["beta_used"], out["beta_used"])
        tok = got["tokens"]
        history[i:i + 1] = tok
    torch.cuda.synchronize()
    assert len(set(history.tolist())) == 8 and min(history.tolist()) >= 0
