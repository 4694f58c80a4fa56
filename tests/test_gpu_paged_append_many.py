"""Rotary positions and new tokens of long prompts, where a wave takes up to six pieces of a token: as for few tokens."""
import pytest

from tests import paged_util as pu
from tests.test_gpu_paged_append import run

pytestmark = pytest.mark.gpu

PROMPTS = [2100, 1, 0, 1500, 600]


def case(hq, hkv, d, scale=1, **kw):
    new = [n // scale for n in PROMPTS]
    return pu.Case([n + 7 * i for i, n in enumerate(new)], new, hq=hq, hkv=hkv, d=d, page=32, **kw)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rotary", [(12, 2, 64, 64), (5, 5, 128, 48), (40, 8, 64, 16)])
def test_types_and_layouts(dtype, cache, interleaved, hq, hkv, d, rotary):
    """One to four pieces a token, the last of them part of a wave."""
    assert run(case(hq, hkv, d, dtype=dtype, cache=cache, heads_first=interleaved, seed=hq), rotary, interleaved) == 0


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_more_pieces_than_a_wave_takes(interleaved, cache):
    """Nine pieces: a wave of six and one of three, the last of a few lanes."""
    assert run(case(128, 1, 64, scale=2, cache=cache, seed=1), 64, interleaved) == 0


@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_in_place_and_left_out(interleaved):
    assert run(case(12, 2, 64, seed=2), 64, interleaved, in_place=True) == 0
    assert run(case(12, 4, 64, seed=3), 64, interleaved, with_q=False) == 0


def test_far_positions_by_parts():
    n = sum(PROMPTS)
    assert run(case(6, 2, 64, dtype="f16", seed=4), 32, True, "parts", 8.0, positions=[(1 << 20) + 3 * i for i in range(n)]) == 0


def test_rows_of_no_sequence_and_sequences_too_short():
    new = [2100, 2000]
    c = pu.Case([2100, 1990], new, hq=4, hkv=2, d=64, page=32, extra_rows=50, seed=5)
    assert run(c, 64) == 2
