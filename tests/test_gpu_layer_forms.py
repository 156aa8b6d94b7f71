"""Forms of the layer-wise calls that their other tests leave out: fp32 heads of every size, kernel timing."""
import pytest

torch = pytest.importorskip("torch")
from tests.test_gpu_layer import Model, _check_attend, _check_summaries, _eq, _run_attend  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [8, 12, 20, 28, 36, 48, 52, 68, 76, 84, 96, 108, 112, 116, 124])
@pytest.mark.parametrize("T,sel", [(1, (5, 1, 1)), (1, None), (3, (5, 2, 1))])
def test_fp32_heads(d, T, sel):
    m = Model([130, 300, 15], T, "f32", (6, 2, d), 2, seed=d)
    m.sess.bind_summary()
    m.sess.summarize()
    q, out = _run_attend(m, T, sel)
    _check_attend(m, q, out, T, sel)
    if sel:
        _check_summaries(m, [n + T for n in m.lens])


@pytest.mark.parametrize("lens,T,sel", [([300, 40], 1, (5, 1, 1)), ([300, 40], 1, None), ([9000, 40], 1, (300, 1, 1)),
                                        ([9000, 40], 3, (300, 1, 1))])
def test_timed_launches(lens, T, sel):
    """With kernel timing on: the same bits, and every launch counted with a time."""
    m = Model(lens, T, "bf16", (8, 2, 64), 2, seed=71)
    m.sess.bind_summary()
    m.sess.summarize()
    q, k, v = m.rows(T)
    rope = (10000.0, 64, False)
    qr = m.sess.append(q, k, v, n_tokens=T, rope=rope)
    x = m.sess.attend(qr, n_tokens=T, select=sel)["x"]
    ctx = m.sess.ctx
    ctx.pced_profile_enable(True)
    for _ in range(3):
        _eq(m.sess.append(q, k, v, n_tokens=T, rope=rope), qr)
        _eq(m.sess.attend(qr, n_tokens=T, select=sel)["x"], x)
    torch.cuda.synchronize()
    p = ctx.pced_profile_read()
    ctx.pced_profile_enable(False)
    for name in ("append", "attn"):
        assert p[name]["launches"] >= 3 and p[name]["ms"] > 0 and p[name]["bytes"] > 0, p
