"""Calls whose bounds are far above what their sequences hold."""
import numpy as np
import pytest
import torch

import paper_2601_01204_amd as kvx
from tests import paged_util as pu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 5])
@pytest.mark.parametrize("seqs,hkv,hq,bound", [(256, 8, 32, 1 << 20), (65536, 1, 1, 8)])
def test_weights_under_generous_bounds(seqs, hkv, hq, bound, new):
    """256 sequences of up to a million tokens (2^24 workgroups form weights again), and as many sequences as there may be: as with the bounds that fit."""
    rng = np.random.default_rng(seqs + new)
    page = 1024 if bound > 1024 else 8
    lens = rng.integers(new, 40, seqs) if bound > 40 else rng.integers(new, bound + 1, seqs)
    per = bound // page
    table = torch.zeros(seqs, per, dtype=torch.int32)
    table[:, 0] = torch.from_numpy(rng.permutation(seqs).astype(np.int32))
    g = torch.Generator().manual_seed(seqs)
    dev = "cuda:0"
    k, v = (torch.randn(seqs, page, hkv, 64, generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
    weights = torch.rand(seqs, hkv, page, generator=g).to(dev)
    q = torch.randn(seqs * new, hq, 64, generator=g).to(torch.bfloat16).to(dev)
    start = torch.arange(0, seqs * new + 1, new, dtype=torch.int32, device=dev)
    d_lens = torch.from_numpy(lens.astype(np.int32)).to(dev)
    got = []
    for most in (bound, int(lens.max())):
        h = kvx.KvPaged(n_q_heads=hq, n_kv_heads=hkv, head_dim=64, page_size=page, max_seqs=seqs, max_tokens=seqs * new, max_len=most, max_evicted=1)
        pages = kvx.KvPages(k, v, table.to(dev), weights=weights)
        out, w = torch.empty_like(q), torch.zeros_like(weights)
        h.attend(pages, kvx.KvPagedBatch(start, d_lens, n_tokens=seqs * new, max_new=new, max_len=most), q, out, weights_out=w)
        torch.cuda.synchronize()
        assert h.status() == 0
        h.close()
        got.append((out.float().cpu(), w.double().cpu()))
    # the other bound may join other pieces: half a step of each output, fp32 sums of up to 40 keys and their exponentials
    u = pu.HALF_STEP["bf16"]
    a, b = got[0][0], got[1][0]
    assert ((a - b).abs() <= 2 * u * b.abs() + 8 * (2 * pu.EXP_ERROR + 40 * 2.0 ** -23)).all()
    assert ((got[0][1] - got[1][1]).abs() <= new * (hq // hkv) * (2 * pu.EXP_ERROR + 40 * 2.0 ** -23)).all()
    gained = got[0][1].sum() - sum(float(weights[table[b, 0], :, :int(lens[b])].double().sum()) for b in range(seqs)) if seqs < 1000 else None
    assert gained is None or abs(float(gained) - seqs * new * hq) < seqs * new * hq * 2.0 ** -16
