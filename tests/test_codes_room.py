"""The two arrays of partial states that a launch of 8-bit attention uses do not meet; without a GPU."""
import pytest

from tests.test_codes_path import OK, Codes, codes_host  # noqa: F401  (the fixture)


@pytest.mark.parametrize("heads", [(4, 4, 64), (32, 8, 128), (16, 1, 128), (28, 4, 128), (5 * 4, 5, 64)])
@pytest.mark.parametrize("layers", [1, 7])
@pytest.mark.parametrize("lens,n", [([3000, 20], 9), ([40000, 1], 64), ([100000, 17], 2), ([5000] + [1] * 12, 1),
                                    ([4200, 4100, 4300], 31)])
def test_states_are_apart(codes_host, heads, layers, lens, n):  # noqa: F811
    b = Codes(codes_host, lens, n, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2], n_layers=layers)
    assert b.status == OK and b.append(n, rope=None) == OK and b.attend(n) == OK, b.error()
    acc, ml = b.calls("acc"), b.calls("ml")
    begin, end = codes_host.room_begin(b.ctx), codes_host.room_end(b.ctx)
    launches = [s for s in b.calls("attend_split") if s[0] > 1]
    assert len(acc) == len(ml) == len(launches)
    assert launches or max(lens) + n <= 4096  # (a part is 256 pages at most)
    for (a0, a1, *_), (m0, m1, *_) in zip(acc, ml):
        assert begin <= a0 < a1 <= m0 < m1 <= end
