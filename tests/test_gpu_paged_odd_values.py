"""Infinities and NaN among values that rows see: a row has them in their channels however little weight they have there."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def put(case, b, j, channels, x):
    """The value of key j of sequence b in some channels of every head, in the pool and in its 64-bit copy."""
    page, slot = po.place(case.pool, b, j)
    case.pool["v"][page, slot][:, channels] = x
    bits = torch.uint8 if case.cache == "e4m3" else torch.int16
    raw = torch.full((case.hkv, len(channels)), x).to(pu.TYPES[case.cache]).view(bits).to(case.device)
    rows = case.v.view(bits)[page, :, slot] if case.heads_first else case.v.view(bits)[page, slot]
    rows[:, channels] = raw


def check_attend(case, q, window=0):
    h = case.handle()
    out, lse = torch.empty_like(q), torch.empty(case.n_tokens, case.hq, device=case.device)
    h.attend(case.pages(), case.batch(), q, out, lse=lse, window=window)
    torch.cuda.synchronize()
    h.close()
    scales = [None if x is None else x.numpy() for x in (case.k_scale, case.v_scale)]
    with np.errstate(invalid="ignore"):
        ref, rl, gained, absolute, reach = po.attend(case.pool, q.float().cpu().numpy(), case.start, case.lens, 1 / math.sqrt(case.d), True, window, *scales)
    finite = np.where(np.isfinite(absolute), absolute, 0.0)
    b_out, b_lse, _ = pu.attend_bounds(case, np.where(np.isfinite(ref), ref, 0.0), finite, rl, gained, reach, True)
    pu.check(out.float().cpu().numpy(), ref, b_out, "out")
    pu.check(lse.cpu().numpy(), rl, b_lse, "lse")
    return ref


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length,new", [(200, 1), (400, 1), (400, 9), (400, 60), (9000, 1), (9000, 9), (9000, 60)])
@pytest.mark.parametrize("scale", [1.0, 40.0])
def test_values_that_every_row_sees(dtype, cache, d, length, new, scale):
    """At a scale of 40 logits spread over hundreds, so that most weights are zero in fp32; 400 keys and more are joined from pieces in calls of few
    rows, 9000 from several ranges in others."""
    case = pu.Case([length, 40], [new, 1], hq=4, hkv=2, d=d, page=16, dtype=dtype, cache=cache, heads_first=d == 64, seed=length + new)
    inf, nan = (math.inf, math.nan) if cache != "e4m3" else (math.nan, math.nan)
    for j, channels, x in ((10, [0, 5], inf), (length // 2, [5, 9], -inf), (length // 2 + 1, [20, 63], inf), (length - new - 3, [33], nan), (length // 3, [63], inf)):
        put(case, 0, j, channels, x)
    ref = check_attend(case, case.rows(4, scale=scale))
    rows = ref[:new]
    assert np.isnan(rows[..., [5, 33]]).all() and np.isfinite(rows[..., [1, 62]]).all()
    if cache != "e4m3":
        assert (rows[..., [0, 20, 63]] == math.inf).all() and (rows[..., 9] == -math.inf).all()


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [9, 100])
@pytest.mark.parametrize("window", [0, 5000])
def test_values_that_some_rows_see_in_long_caches(dtype, cache, d, new, window):
    """Among the new tokens and at the window's beginning, where results are joined from partial ones and most weights are zero in fp32."""
    length, inf = 9000, math.inf if cache != "e4m3" else math.nan
    case = pu.Case([length], [new], hq=4, hkv=2, d=d, page=16, dtype=dtype, cache=cache, seed=new)
    first = length - new
    odd = [(first + new // 2, [3], inf), (first + 5, [3, 8], -inf), (first + 2, [40], math.nan)]
    if window:                                               # row i sees keys from first + i - window + 1 on
        odd += [(first - window + 3, [50, 8], inf), (first - window, [51], math.nan), (first - window + 6, [52], -inf)]
    for j, channels, x in odd:
        put(case, 0, j, channels, x)
    ref = check_attend(case, case.rows(4, scale=40.0), window)
    assert np.isfinite(ref[0, :, [3, 8, 40]] if not window else ref[0, :, [3, 40]]).all() and np.isnan(ref[-1, :, 40]).all()
    assert np.isfinite(ref[..., [1, 51]]).all()


@pytest.mark.parametrize("new", [1, 60])
def test_a_logit_that_is_not_a_number_makes_its_row_one(new):
    """Also where an infinite value is seen: its weight is not a number either."""
    case = pu.Case([500], [new], hq=2, hkv=1, d=64, seed=new)
    put(case, 0, 20, [3], math.inf)
    q = case.rows(2)
    q[0, 1] = math.nan
    h, out = case.handle(), torch.empty_like(q)
    h.attend(case.pages(), case.batch(), q, out)
    torch.cuda.synchronize()
    h.close()
    assert out[0, 1].isnan().all() and (out[0, 0, 3] == math.inf).item() and out[0, 0, 4:].isfinite().all()
