"""What PcedSession hands to the layer-wise calls, checked without a GPU: tensors of the CPU, and a context that
records its calls instead of making them."""
import pytest
import torch

from paper_2601_08670_amd import _lib
from paper_2601_08670_amd.session import PcedSession

L, HQ, HKV, D, S = 2, 4, 2, 8, 3


class Calls:
    def __init__(self):
        self.rows = []

    def pced_append(self, layer, n_layers, n_tokens, rows, rope, q_out):
        self.rows.append((rows.q_row, rows.k_row, rows.v_row))


@pytest.fixture
def session(monkeypatch):
    s = object.__new__(PcedSession)
    s.geom = dict(n_layers=L, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, vocab=10)
    s.S, s.B, s._device_index, s.k_pool, s.dtype, s._dtypes = S, 1, -1, torch.empty(0), "f32", (torch.float32,)
    s.device = torch.device("cpu")
    s._rows, s._ropes, s.ctx = _lib.pced_rows(), {}, Calls()
    monkeypatch.setattr(_lib, "current_device", lambda: -1)
    return s


def _rows(n):
    return tuple(torch.zeros(n, L, h, D) for h in (HQ, HKV, HKV))


@pytest.mark.parametrize("which", [0, 1, 2])
def test_rows_that_share_memory_are_refused(session, which):
    """A distance of 0 means rows that follow each other to the library, which would read past a broadcast row."""
    rows = list(_rows(S))
    session.append(*rows)
    rows[which] = rows[which][:1].expand(S, -1, -1, -1)
    with pytest.raises(ValueError, match="overlap"):
        session.append(*rows)
    rows[which] = torch.zeros(1000).as_strided(rows[which].shape, (4,) + rows[which].stride()[1:])
    with pytest.raises(ValueError, match="overlap"):
        session.append(*rows)
    assert len(session.ctx.rows) == 1


def test_distances_of_rows(session):
    w = L * D
    session.append(*_rows(S))
    wide = torch.zeros(S, L, HQ + 2 * HKV, D)
    session.append(None, *(torch.zeros(S, 100).as_strided((S, L, HKV, D), (100, HKV * D, D, 1)) for _ in range(2)))
    one = wide[:, :1]
    session.append(one[:, :, :HQ], one[:, :, HQ:HQ + HKV], one[:, :, HQ + HKV:], n_layers=1)
    session.S = 1  # (one row: no distance)
    session.append(*(x[:1].expand(1, -1, -1, -1) for x in _rows(1)))
    assert session.ctx.rows == [(HQ * w, HKV * w, HKV * w), (0, 100, 100), (w * (HQ + 2 * HKV),) * 3, (HQ * w, HKV * w, HKV * w)]


def test_adjustments_of_another_device_are_refused(session):
    """Same number of queries and vocabulary, but their lists lie elsewhere."""
    from paper_2601_08670_amd.session import Adjust
    here, there = Adjust(1, 10, torch.device("cpu")), Adjust(1, 10, torch.device("cuda", 1))
    assert session._adjust(here) is here.struct
    with pytest.raises(ValueError, match="cuda:1"):
        session._adjust(there)


def test_a_session_names_its_device(monkeypatch):
    """"cuda" is the device that is current when the session is made; what it allocates later lies there too."""
    class Context:
        def __init__(self, cfg, device):
            self.workspace = torch.empty(1)

        def pced_bind_summary(self, summary):
            pass

    monkeypatch.setattr(_lib, "Context", Context)
    s = PcedSession(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=8, vocab=10, dtype="f32", max_queries=1, max_seqs=2,
                    max_pages=2, max_pages_per_seq=1, device="cpu")
    assert s.device == s.k_pool.device == torch.device("cpu")
    s.bind_summary()
    assert s.summary.device == s.k_pool.device
