"""Eviction at lengths inside and at the edges of each way that a workgroup holds its keys (registers of 1, 2, 4 and 8 groups a thread, or none)."""
import pytest

from tests import paged_util as pu
from tests.test_gpu_paged_evict import fill, run

pytestmark = pytest.mark.gpu

LENGTHS = [4096, 8192, 8193, 12000, 16384, 16385, 20001, 32768, 32769]


def case(n, heads=1, **kw):
    return pu.Case([n, 60], [1, 1], hq=heads, hkv=heads, d=64, page=256, **kw)


@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("leave", [1, 4, 5, 300, 3000])
@pytest.mark.parametrize("in_place", [False, True])
def test_lengths(n, leave, in_place):
    """Up to four leaving tokens are found as the least keys; more than 256 are moved by a launch of their own."""
    c = case(n, seed=n % 97 + leave)
    fill(c, [n + 5, 60], seed=leave)
    assert run(c, [n + 5, 60], n - leave, 4, 32, in_place) == 0


@pytest.mark.parametrize("n", [4000, 8192, 12001, 16384, 20001, 32768, 33001])
@pytest.mark.parametrize("kind", ["ties", "equal", "odd"])
@pytest.mark.parametrize("in_place", [False, True])
def test_kinds_of_weights(n, kind, in_place):
    c = case(n, seed=7)
    fill(c, [n, 60], kind, seed=n % 89)
    assert run(c, [n, 60], n // 3, 2, 50, in_place) == 0


@pytest.mark.parametrize("n", [9001, 30000])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_heads_apart(n, cache):
    c = case(n, heads=3, cache=cache, seed=8)
    fill(c, [n + 1, 60], seed=9)
    assert run(c, [n + 1, 60], n - 700, 0, 3, True) == 0


@pytest.mark.parametrize("n", [12000, 20000])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_cache_under_the_budget_beside_one_over_it(n, in_place):
    c = pu.Case([n, n - 3000], [1, 1], hq=1, hkv=1, d=64, page=64, seed=10)
    fill(c, [n, n], seed=10)
    assert run(c, [n, n], n - 2000, 1, 1, in_place) == 0
