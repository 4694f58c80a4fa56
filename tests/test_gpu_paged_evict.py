"""Eviction by received weight: exactly the definition's tokens, in exactly its slots."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def fill(case, seen, kind="spread", seed=0):
    """ids: distinct tokens of each (sequence, head), in no order; weights of the kind."""
    rng = np.random.default_rng(seed)
    w, ids = np.full(case.weights.shape, 5.0, np.float32), np.full(case.ids.shape, -9, np.int32)
    for b, n in enumerate(case.lens):
        for h in range(case.hkv):
            tokens = rng.permutation(seen[b])[:n]
            for j in range(n):
                p = po.place(case.pool, b, j)
                if p is None:
                    continue
                ids[p[0], h, p[1]] = tokens[j]
                w[p[0], h, p[1]] = {"spread": np.exp(3 * rng.standard_normal()), "ties": rng.integers(0, 3), "equal": 1.0,
                                    "odd": rng.choice([np.nan, -np.inf, np.inf, 0.0, -0.0, -1.5, 1e-42, 2.0, rng.standard_normal()])}[kind]
    case.weights.copy_(torch.from_numpy(w))
    case.ids.copy_(torch.from_numpy(ids))
    case.pool["weights"], case.pool["ids"] = w, ids


def run(case, seen, budget, sinks=0, recent=0, in_place=False):
    h = case.handle()
    d_seen = torch.tensor(seen, dtype=torch.int32, device=case.device)
    pages, batch = case.pages(), case.batch(seen=d_seen)
    w, ids = (case.weights, case.ids) if in_place else (torch.full_like(case.weights, 77.0), torch.full_like(case.ids, 77))
    lens = case.d_lens if in_place else torch.full_like(case.d_lens, 77)
    raw = case.pool["weights"].copy(), case.pool["ids"].copy()
    h.evict(pages, batch, budget, sinks, recent, weights_out=w, ids_out=ids, lens_out=lens)
    torch.cuda.synchronize()
    k, v, rw, ri, rl, written = po.evict(case.pool, case.lens, seen, budget, sinks, recent)
    assert np.array_equal(case.wide(case.k), k, equal_nan=True) and np.array_equal(case.wide(case.v), v, equal_nan=True)
    assert lens.cpu().tolist() == rl.tolist()
    gw, gi = w.cpu().numpy(), ids.cpu().numpy()
    assert np.array_equal(gw[written].view(np.uint32), rw[written].view(np.uint32)) and np.array_equal(gi[written], ri[written])
    rest = (raw[0], raw[1]) if in_place else (np.float32(77), np.int32(77))
    assert np.array_equal(gw[~written], np.broadcast_to(rest[0], gw.shape)[~written], equal_nan=True)
    assert np.array_equal(gi[~written], np.broadcast_to(rest[1], gi.shape)[~written])
    status = h.status()
    h.close()
    return status


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (40, 0, 0), (64, 4, 30), (99, 2, 1), (100, 50, 50), (200, 0, 3)])
@pytest.mark.parametrize("in_place", [False, True])
def test_what_stays(kind, budget, sinks, recent, in_place):
    lens = [100, 230, 101, 0, 5, 64]
    case = pu.Case(lens, [1 if n else 0 for n in lens], hq=3, hkv=3, page=16, seed=budget)
    seen = [n + 7 for n in lens]
    fill(case, seen, kind, seed=budget)
    assert run(case, seen, budget, sinks, recent, in_place) == 0


@pytest.mark.parametrize("dtype,cache,d", [("f16", "f16", 64), ("bf16", "bf16", 128), ("bf16", "e4m3", 64), ("f16", "e4m3", 128)])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page", [8, 128])
def test_types_and_layouts(dtype, cache, d, heads_first, page):
    case = pu.Case([700, 1500], [1, 1], hq=2, hkv=2, d=d, dtype=dtype, cache=cache, heads_first=heads_first, page=page, seed=page)
    fill(case, [700, 1600], seed=1)
    assert run(case, [700, 1600], 600, 4, 16) == 0


@pytest.mark.parametrize("n,budget", [(4097, 4096), (5000, 1024), (33500, 33000), (40000, 3000)])
def test_long_caches(n, budget):
    """Up to and beyond the keys that a workgroup holds in LDS."""
    case = pu.Case([n, 60], [1, 1], hq=1, hkv=1, d=64, page=256, seed=2)
    fill(case, [n + 5, 60], seed=2)
    assert run(case, [n + 5, 60], budget, 4, 32) == 0


def test_more_protected_than_the_budget_and_none_seen():
    case = pu.Case([50, 40], [1, 1], hq=1, hkv=1, page=8, seed=3)
    fill(case, [50, 40], seed=3)
    case.pool["ids"][:] = 0                                  # every id below sinks
    case.ids.zero_()
    assert run(case, [50, 40], 20, 1, 2) == 0


def test_pages_outside_the_pool_go_first():
    case = pu.Case([100, 60], [1, 1], hq=1, hkv=1, page=8, seed=4)
    for b, e, bad in ((0, 2, -1), (0, 11, case.n_pages + 3), (1, 0, 1 << 30)):
        case.pool["table"][b, e] = bad
    case.table.copy_(torch.from_numpy(case.pool["table"]))
    fill(case, [100, 60], seed=4)
    assert run(case, [100, 60], 50, 0, 0) == 1


def test_one_token_a_step_moves_one_row():
    """A cache that gives up one token a step: everything but one slot of each head is where it was."""
    case = pu.Case([513], [1], hq=4, hkv=4, page=64, seed=5)
    fill(case, [513], seed=5)
    before = case.wide(case.k)
    assert run(case, [513], 512, 4, 32) == 0
    changed = (case.wide(case.k) != before).any(-1) & ~np.isnan(before).any(-1)
    assert (changed.sum((0, 1)) <= 1).all()


def test_the_workspace_is_shared_with_attention():
    """An eviction between two attention calls whose results are joined from partial ones, and again."""
    case = pu.Case([3000], [1], hq=2, hkv=2, page=64, seed=6)
    fill(case, [3000], seed=6)
    h, pages, batch = case.handle(), case.pages(), case.batch()
    q = case.rows(2)
    outs = [torch.empty_like(q) for _ in range(2)]
    scratch = torch.zeros_like(case.weights), torch.zeros_like(case.ids), torch.zeros_like(case.d_lens)
    k0, v0 = case.k.clone(), case.v.clone()
    for o in outs:
        h.attend(pages, batch, q, o)
        h.evict(pages, batch, 100, 0, 0, weights_out=scratch[0], ids_out=scratch[1], lens_out=scratch[2])
        torch.cuda.synchronize()
        case.k.copy_(k0)
        case.v.copy_(v0)
    assert torch.equal(*outs)
