"""The shapes of tests/test_gpu_attention_split.py reach what they are for: workers of several units that cross sequences."""
import pytest

from attention_checks import UNIT, stretches, workers
from paper_2412_08521_amd import binding as B
from test_gpu_attention_split import COMPACT, RINGS, SHARED

MODES = [B.EMS_BF16, B.EMS_F32]


def _row_bytes(d, mode):
    return d * (4 if mode == B.EMS_F32 else 2)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name", sorted(SHARED))
def test_shared_shapes(name, mode):
    b, hq, hkv, d, ps, lens, columns = SHARED[name]
    n = workers(b, hkv, hq // hkv, ps * columns, _row_bytes(d, mode))
    assert n > 0 and sum(-(-x // UNIT) for x in lens) > n
    assert max(lens) <= ps * columns
    got = stretches(lens, n)
    assert len({sum(u for _, _, u, _ in w) for w in got}) == (1 if name == "even" else 2)
    crossing = [w for w in got if len(w) > 1]
    partial = lambda part: part[2] < part[3]  # noqa: E731
    both = [w for w in crossing if partial(w[0]) and partial(w[-1])]
    if name == "even":                            # every sequence ends where a worker does
        assert not crossing
    else:
        assert crossing and both
    over = any(w[i + 1][0] > w[i][0] + 1 for w in crossing for i in range(len(w) - 1))
    assert over == (name in ("ragged", "many", "wide"))      # over an empty sequence
    assert any(u > 1 for w in got for _, _, u, _ in w)
    past = b * hkv * ps * columns * 2 * _row_bytes(d, mode) > 80 << 20
    assert past == (name != "caches")


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", COMPACT)
def test_compact_shapes(shape, mode):
    b, hq, hkv, d, budget, window, ratio = shape
    t = budget + int(ratio * budget) + 1
    n = workers(b, hkv, hq // hkv, t, _row_bytes(d, mode))
    assert 0 < n < b * -(-t // UNIT)
    assert any(len(w) > 1 for w in stretches([t] * b, n))


@pytest.mark.parametrize("name", sorted(RINGS))
def test_ring_shapes(name):
    """Live rows of a wave by the hundred: a ring of 128 wraps more than once."""
    (b, hq, hkv, d, ps, lens, columns), mode = RINGS[name]
    group = hq // hkv
    n = workers(b, hkv, group, ps * columns, _row_bytes(d, mode))
    blocks = b * hkv * (1 if group <= 16 else -(-group // 32))
    assert blocks * ps * columns * 2 * _row_bytes(d, mode) > 80 << 20 and -(-group // 32) == 1
    if name.startswith("whole"):
        assert n == 0 and blocks >= 512
        most = max(lens)
    else:
        most = UNIT * max(u for w in stretches(lens, n) for _, _, u, _ in w)
    assert most // 4 > 128 + 32, most
    assert max(lens) <= ps * columns
