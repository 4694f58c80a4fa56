"""Rotary positions and the cache's new tokens against their 64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2601_01204_amd as kvx
from oracle import paged_oracle as po
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

SCALINGS = {"plain": kvx.KV_ROPE_PLAIN, "linear": kvx.KV_ROPE_LINEAR, "base": kvx.KV_ROPE_BASE, "parts": kvx.KV_ROPE_PARTS}


def run(case, rotary=0, interleaved=False, scaling="plain", factor=1.0, base=10000.0, magnitude=1.0, freqs=None, positions=None, seen=None, in_place=False,
        with_q=True, original=256):
    h = case.handle(rotary_dim=rotary, rope_layout=int(interleaved), rope_scaling=SCALINGS[scaling], rope_factor=factor, rope_base=base,
                    rope_original_len=original, rope_magnitude=magnitude, rope_freqs=freqs)
    w = np.asarray(freqs, np.float64) if freqs is not None else po.rope_frequencies(rotary, scaling, base, factor, original)
    q, k, v = case.rows(case.hq), case.rows(case.hkv), case.rows(case.hkv, scale=3.0)
    q0 = q.clone()
    case.weights.fill_(3.0)
    case.ids.fill_(-5)
    before = case.wide(case.k), case.wide(case.v)
    seen = case.lens if seen is None else seen
    d_seen = torch.tensor(seen, dtype=torch.int32, device=case.device)
    q_out = (q if in_place else torch.full_like(q, 9.0)) if with_q else None
    p = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=case.device)
    h.append(case.pages(), case.batch(seen=d_seen), k, v, q=q if with_q else None, q_out=q_out, positions=p)
    torch.cuda.synchronize()
    status = h.status()
    h.close()

    u = pu.HALF_STEP[case.dtype]
    places, at, token = [], np.zeros(case.n_tokens, np.int64), np.zeros(case.n_tokens, np.int64)
    for b, n in enumerate(case.new):
        for i in range(n):
            t, j = case.start[b] + i, case.lens[b] - n + i
            token[t] = seen[b] - n + i
            at[t] = token[t] if positions is None else positions[t]
            places.append((t, po.place(case.pool, b, j) if j >= 0 else None))

    def turned(x):
        x = x.float().cpu().double().numpy()
        # fp32 sine and cosine, two products and a sum: 2^-21 of the two channels' magnitudes; then the rounding to the output's type
        ref = po.rotate(x, at, w, interleaved, magnitude)
        r, near = len(w), np.zeros_like(x)
        for i in range(r):
            a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
            near[:, :, a] = near[:, :, c] = magnitude * (np.abs(x[:, :, a]) + np.abs(x[:, :, c]))
        return ref, near * 2.0 ** -21

    if with_q:
        ref, fp32 = turned(q0)
        n = case.start[-1]
        got = q_out.float().cpu().double().numpy()
        pu.check(got[:n], ref[:n], u * np.abs(ref[:n]) + 2 * fp32[:n] + 2.0 ** -25, "q_out")
        assert in_place or (got[n:] == 9).all(), "rows of no sequence are left alone"
    k_ref, k_fp32 = turned(k)
    v_ref = v.float().cpu().double().numpy()
    got = case.wide(case.k), case.wide(case.v)
    touched = np.zeros(got[0].shape[:2], bool)
    for t, p in places:
        if p is None:
            continue
        touched[p] = True
        for x, ref, fp32, s, what in ((got[0], k_ref, k_fp32, case.k_scale, "k"), (got[1], v_ref, 0 * k_fp32, case.v_scale, "v")):
            y, e = ref[t], fp32[t]
            if case.cache == "e4m3":
                y, e = y / s.numpy()[:, None], e / s.numpy()[:, None] + 2.0 ** -23 * np.abs(y / s.numpy()[:, None])
                y = np.clip(y, -448, 448)
                pu.check(x[p], y, np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10) + 2 * e, what)      # (the least step is 2^-9)
            else:
                pu.check(x[p], y, (u * np.abs(y) + 2 * e + 2.0 ** -25) if what == "k" else 0.0, what)
        assert (case.ids.cpu().numpy()[p[0], :, p[1]] == token[t]).all() and (case.weights.cpu().numpy()[p[0], :, p[1]] == 0).all()
    for x, y in zip(got, before):
        assert np.array_equal(x[~touched], y[~touched], equal_nan=True), "other slots are left alone"
    rest = ~np.broadcast_to(touched[:, None, :], case.ids.shape)
    assert (case.ids.cpu().numpy()[rest] == -5).all() and (case.weights.cpu().numpy()[rest] == 3).all()
    return status


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d,rotary", [(64, 64), (64, 16), (128, 128), (128, 48), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_and_parts_of_the_head(dtype, cache, d, rotary, interleaved):
    case = pu.Case([40, 9, 70], [7, 9, 1], hq=6, hkv=2, d=d, dtype=dtype, cache=cache, seed=d + rotary, heads_first=interleaved)
    assert run(case, rotary, interleaved) == 0


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (12, 2), (40, 8), (128, 1)])
@pytest.mark.parametrize("page", [8, 128])
def test_heads(hq, hkv, page):
    assert run(pu.Case([100, 3], [30, 3], hq=hq, hkv=hkv, page=page, seed=hq), 64) == 0


@pytest.mark.parametrize("scaling,factor", [("plain", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 8.0)])
@pytest.mark.parametrize("far", [0, 131071, (1 << 24) + 1, (1 << 31) - 8])
def test_scalings_and_far_positions(scaling, factor, far):
    """The angle of position 2^31 is exact to 2^-33 turns; in 64 bits it is off by 2^-53 of itself, 3e-7 radians, inside the bound's fp32 part."""
    case = pu.Case([30], [6], hq=3, hkv=1, d=64, dtype="f16", seed=far & 255)
    assert run(case, 64, scaling=scaling, factor=factor, positions=[far + i for i in range(6)]) == 0


def test_negative_positions_given_frequencies_and_magnitude():
    case = pu.Case([30], [6], hq=3, hkv=1, d=64, dtype="f16", seed=1)
    freqs = list(np.linspace(-9.0, 9.0, 16))                 # more than a turn a position, and backwards
    assert run(case, 32, freqs=freqs, positions=[-3, -2, -1, 0, 1, 2], magnitude=1.25) == 0


def test_ids_go_by_what_was_seen():
    assert run(pu.Case([40, 8], [5, 1], seed=2), 32, seen=[1040, 8]) == 0


def test_queries_in_place_and_left_out():
    assert run(pu.Case([40, 8], [5, 1], seed=3), 64, in_place=True) == 0
    assert run(pu.Case([40, 8], [5, 1], seed=4), 64, with_q=False) == 0


def test_sequences_without_new_tokens_and_rows_of_none():
    assert run(pu.Case([40, 8, 0, 17, 3], [0, 1, 0, 17, 0], seed=5, extra_rows=6), 64) == 0


def test_more_sequences_than_lanes():
    assert run(pu.Case([5 + i % 11 for i in range(150)], [i % 4 for i in range(150)], hq=2, hkv=1, page=8, seed=6), 64) == 0


def test_pages_outside_the_pool_and_sequences_too_short():
    case = pu.Case([40, 30], [20, 5], page=8, seed=7)
    case.pool["table"][0, 4] = case.n_pages
    case.pool["table"][1, 3] = -1
    case.table.copy_(torch.from_numpy(case.pool["table"]))
    assert run(case, 64) == 1
    case = pu.Case([3, 30], [6, 5], page=8, seed=8)          # six new tokens, three places
    assert run(case, 64) == 2


def test_values_beyond_eight_bits():
    case = pu.Case([8], [2], hq=1, hkv=1, d=64, dtype="f16", cache="e4m3", seed=9)
    case.k_scale, case.v_scale = torch.tensor([0.5]), torch.tensor([0.25])
    h = case.handle()
    k, v = torch.zeros(2, 1, 64, dtype=torch.float16, device=case.device), torch.zeros(2, 1, 64, dtype=torch.float16, device=case.device)
    v[0, 0, :6] = torch.tensor([112.0, 113.0, 60000.0, -60000.0, float("inf"), float("nan")])
    h.append(case.pages(), case.batch(), k, v)
    page, slot = po.place(case.pool, 0, 6)
    got = case.wide(case.v)[page, slot, 0, :6]
    assert got[:5].tolist() == [448.0, 448.0, 448.0, -448.0, 448.0] and np.isnan(got[5])
