"""pced_summarize between pced_append and pced_attend on the GPU."""
import pytest

torch = pytest.importorskip("torch")
from tests.test_gpu_layer import Model, _check_attend, _check_summaries, _eq  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 64)), ("f32", (5, 5, 80))])
def test_summarize_between_append_and_attend(dtype, heads):
    """Pages that appended rows filled stay summarised, and are chosen from."""
    T, sel = 40, (4, 0, 1)
    m = Model([30, 200], 2 * T, dtype, heads, layers=2, seed=70)
    m.sess.bind_summary()
    m.sess.summarize()
    for _ in range(2):
        q, kn, vn = m.rows(T)
        m.sess.append(None, kn * 2, vn, n_tokens=T, rope=None)
        m.sess.append(None, kn, vn, n_tokens=T, rope=None)
        codes = m.sess.summary.clone()
        m.sess.summarize()
        torch.cuda.synchronize()
        _eq(m.sess.summary, codes)
        m.grow(kn, vn, T)
        out = m.sess.attend(q, n_tokens=T, select=sel, want=("pages",))
        torch.cuda.synchronize()
        _check_attend(m, q, out, T, sel)
        m.sess.advance(T)
        m.lens = [n + T for n in m.lens]
        _check_summaries(m, m.lens)
