"""Stored adjusted logits against the oracle in fp32, bit by bit: a token that no list names keeps its bits,
the sign of a zero among them, whatever the lists name around it."""
import numpy as np
import pytest

from oracle import layer as L

torch = pytest.importorskip("torch")
from tests.test_gpu_adjust import DEV, Limits, _logits, _session  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [3, 257, 1000, 1023, 4098])
@pytest.mark.parametrize("only", [None, ("history", "history_off"), ("history", "history_off", "repetition", "presence"),
                                  ("bias_token", "bias_value", "bias_off"), ("mask",), ()])
def test_zeros_keep_their_sign(vocab, only):
    s, _, _ = _session(vocab, [3, 2])
    lim = Limits(vocab, 2, seed=vocab, only=only)
    x = _logits(s.S, vocab, 1)
    x.reshape(-1)[::3] = -0.0
    x.reshape(-1)[1::5] = 0.0
    got = s.adjust_logits(torch.from_numpy(x).to(DEV), s.adjust(**lim.tensors)).cpu().numpy()
    want = np.stack([lim.row(x[r], 0 if r < 4 else 1) for r in range(s.S)])
    assert want.dtype == np.float32 and not np.isnan(want).any()
    bad = np.argwhere(got.view(np.int32) != want.view(np.int32))
    assert len(bad) == 0, (bad[:4], [(got[tuple(b)], want[tuple(b)]) for b in bad[:4]])


def test_a_bias_of_zero_is_an_addition():
    """-0 + 0 is 0 where a bias names the token, and -0 next to it."""
    s, _, _ = _session(64, [1])
    i32 = dict(dtype=torch.int32, device=DEV)
    adj = s.adjust(bias_token=torch.tensor([5], **i32), bias_value=torch.zeros(1, device=DEV), bias_off=torch.tensor([0, 1], **i32))
    got = s.adjust_logits(torch.full((2, 64), -0.0, device=DEV), adj).cpu().numpy()
    assert [v for v in range(64) if not np.signbit(got[0, v])] == [5] and not np.signbit(L.adjust_row([-0.0], biases=[(0, 0.0)])[0])
