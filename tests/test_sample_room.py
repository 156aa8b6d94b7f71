"""What sampling takes of the workspace, and the scale of its weights; without a GPU."""
import pytest

from paper_2601_08670_amd import _lib
from tests.test_layer_path import DEVICE, OK
from tests.test_sample_path import Sampler, sample_host  # noqa: F401  (the fixture)


def _workspace(vocab, aggregation="max", **kw):
    c = dict(n_layers=32, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype="bf16", max_queries=16, max_seqs=272,
             max_pages=272 * 64, max_pages_per_seq=64)
    c.update(kw)
    return _lib.pced_workspace_bytes(_lib.make_config(vocab=vocab, aggregation=aggregation, **c))


def _per_vocab(seqs, queries, V):
    """What the calls without sampling hold per vocabulary entry, at most: logits, beta's sums per 4096 entries, a candidate
    per 128; and the alignment of each."""
    return seqs * (4 * V + 12 * (-(-V // 4096))) + 20 * queries * -(-V // 128) + 16 * 256


@pytest.mark.parametrize("aggregation", ["max", "moe", "poe"])
def test_lists_take_no_workspace_of_their_own(aggregation):
    """16 queries of 151936 tokens: their lists (20 MB) lie where the attention's partial states do."""
    grow = _workspace(2 * 151936, aggregation) - _workspace(151936, aggregation)
    assert grow <= _per_vocab(272, 16, 151936)


def test_lists_beyond_the_partial_states():
    """A context whose attention needs next to nothing has room for the lists, if it may sample."""
    small = dict(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, max_queries=4, max_seqs=8, max_pages=8, max_pages_per_seq=1)
    V = 1 << 20
    grow = [_workspace(2 * V, a, **small) - _workspace(V, a, **small) for a in ("max", "moe", "poe")]
    assert grow[1] == grow[2] <= _per_vocab(8, 4, V)
    assert grow[1] < grow[0] <= _per_vocab(8, 4, V) + 4 * 8 * V


@pytest.mark.parametrize("vocab", [2, 3, 100, 1000, 4096, 50257, 65536, 128256, 151936, 1 << 20])
@pytest.mark.parametrize("kw", [{}, dict(n_layers=3, n_q_heads=32, n_kv_heads=8, head_dim=128)])
def test_launches(sample_host, vocab, kw):  # noqa: F811
    """Each region of a launch lies in its place; the weights of all tokens add up to 2^62 at most, and to more than half
    of it at the next scale."""
    b = Sampler(sample_host, [16, 40], 64, vocab=vocab, **kw)
    assert b.sample(extra=_lib.pced_sample_out(kept=DEVICE)) == OK
    (nblk, _, *fits), = b.calls("fuse_scores")
    assert fits == [1] * 6
    (_, shift, *_), = b.calls("sample")
    assert vocab << shift <= 1 << 62 < vocab << (shift + 1)
