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


@pytest.mark.parametrize("dtype,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("new", [1, 9, 20])
@pytest.mark.parametrize("below", [17.5, 22.0])
@pytest.mark.parametrize("top", [0, 18001])
def test_many_keys_of_little_weight(dtype, cache, new, below, top):
    """One key `below` nats above all others, whose weights lie under fp16's steps if the largest is 1; the values of its run of 32 keys are the output
    (of all keys in the second head: those far from it have references of their own where waves or ranges share the keys).  Bounds as above, with fp16's least
    step counted where the references lie: 2^-39 of the largest weight for a key in calls of up to 32 rows of a key head, 2^-35 in others.  Logits
    are exact here but for the scale's rounding, 2^-23 of them."""
    length = 20000
    case = pu.Case([length], [new], hq=4, hkv=2, d=64, page=64, dtype=dtype, cache=cache, seed=new)
    if cache == "e4m3":
        case.k_scale, case.v_scale = torch.tensor([0.5] * 2), torch.tensor([4.0] * 2)
    shape = case.k.shape
    k, v = torch.zeros(shape), torch.full(shape, 1000.0 if cache != "e4m3" else 256.0)
    v[:, :, 0] = 0.0
    for j in range(top // 32 * 32, top // 32 * 32 + 32):
        page, slot = po.place(case.pool, 0, j)
        v[page, slot, 0] = v[page, slot, 1]
    page, slot = po.place(case.pool, 0, top)
    k[page, slot, :, 0], v[page, slot] = below * (2 if cache == "e4m3" else 1), 0.0
    case.k.copy_(k.to(pu.TYPES[cache]))
    case.v.copy_(v.to(pu.TYPES[cache]))
    case.pool["k"], case.pool["v"] = case.wide(case.k), case.wide(case.v)
    q = torch.zeros(new, 4, 64)
    q[:, :, 0] = 8.0                                         # a logit is its key's first channel
    got, lse, ref, rl, absolute, _ = attend(case, q.to(pu.TYPES[dtype]).to(case.device))
    u = pu.HALF_STEP[dtype]
    relative = 2 * 2.0 ** -22 * below + pu.EXP_ERROR + length * 2.0 ** -23 + 2 * u * u
    keys = np.array([32, 32, length, length])[None, :, None]
    floor = keys * (2.0 ** -39 if new * 2 <= 32 else 2.0 ** -35) * 1024.0 if dtype == "f16" else 0.0
    assert ref.min() > 5e-6
    pu.check(got, ref, u * np.abs(ref) + relative * absolute * (1 + u) + floor + 2.0 ** -25, "out")
    pu.check(lse, rl, 2.0 ** -22 * below + pu.EXP_ERROR + length * 2.0 ** -24 + np.abs(rl) * 2.0 ** -23, "lse")
