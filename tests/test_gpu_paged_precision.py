"""What attention over a paged cache holds in how many bits: bounds that leave room for fp32 arithmetic and for one rounding, the output's."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


def attend(case, q, causal=True):
    h = case.handle()
    out, lse = torch.empty_like(q), torch.empty(case.n_tokens, case.hq, device=case.device)
    h.attend(case.pages(), case.batch(), q, out, lse=lse, causal=causal)
    torch.cuda.synchronize()
    h.close()
    scales = [None if x is None else x.numpy() for x in (case.k_scale, case.v_scale)]
    ref, rl, _, absolute, reach = po.attend(case.pool, q.float().cpu().numpy(), case.start, case.lens, 1 / math.sqrt(case.d), causal, 0, *scales)
    return out.float().cpu().double().numpy(), lse.cpu().double().numpy(), ref, rl, absolute, reach


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new,hq,hkv", [([300, 97], [150, 97], 4, 2), ([4000], [60], 2, 2), ([33, 700], [33, 40], 6, 1)])
def test_chunks_round_the_output_alone(dtype, cache, d, lens, new, hq, hkv):
    """Probabilities rounded to 16 bits would be off by as much as the output's own rounding, u.  Left: logits, sums of d products in fp32 ((d + 4) 2^-24 of
    their magnitudes, counted for the row and for its reference); the exponential; fp32 sums over the keys; pairs of 16-bit values, 2 u^2 (a pair holds
    a probability to u^2, and its product with a value is exact); in fp16 what lies below half its least step, 2^-25 of a row's reference for every key.
    The reference's probability is 1, so the row's sum is at least that."""
    case = pu.Case(lens, new, hq=hq, hkv=hkv, d=d, page=32, dtype=dtype, cache=cache, seed=d + len(lens))
    q = case.rows(hq)
    got, _, ref, _, absolute, reach = attend(case, q)
    u, keys = pu.HALF_STEP[dtype], max(lens)
    relative = 2 * (d + 4) * 2.0 ** -24 * reach + pu.EXP_ERROR + keys * 2.0 ** -23 + 2 * u * u
    largest = max(np.nanmax(np.abs(case.pool["v"])) * (1.0 if case.v_scale is None else float(case.v_scale.max())), 1.0)
    floor = keys * 2.0 ** -25 * largest + 2.0 ** -25 if dtype == "f16" else 0.0
    pu.check(got, ref, u * np.abs(ref) + relative[..., None] * absolute * (1 + u) + floor, "out")
