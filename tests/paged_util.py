"""Pools, batches and error bounds shared by the tests of the paged cache."""
import numpy as np
import torch

import paper_2601_01204_amd as kvx

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
NAMES = {"bf16": kvx.KV_BF16, "f16": kvx.KV_F16, "e4m3": kvx.KV_E4M3}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "e4m3": 2.0 ** -4}      # largest relative rounding error (eps / 2)
EXP_ERROR = 2.0 ** -20          # of a probability: hardware 2^x and the fp32 argument's own rounding (|argument| below 16)


class Case:
    """A pool with everything a call needs, on the host (64-bit values of what is stored) and on the GPU."""

    def __init__(self, lens, new, hq=4, hkv=2, d=64, page=16, dtype="bf16", cache=None, heads_first=False, seed=0, junk=True, spare=3, max_len=None,
                 device="cuda:0", extra_rows=0, gap=0):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.new, self.hq, self.hkv, self.d, self.page = list(lens), list(new), hq, hkv, d, page
        self.dtype, self.cache, self.heads_first = dtype, cache or dtype, heads_first
        self.device, B = device, len(self.lens)
        counts = [-(-n // page) for n in self.lens]
        width = max(1, max(counts))
        n_pages = sum(counts) + spare
        order = rng.permutation(n_pages)
        table = np.full((B, width), -1, np.int32)            # unused entries name no page
        at = 0
        for b, n in enumerate(counts):
            table[b, :n] = order[at:at + n]
            at += n
        self.n_pages, self.n_tokens = n_pages, sum(self.new) + extra_rows
        self.max_len = max(1, max(self.lens)) if max_len is None else max_len
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        shape = (n_pages, hkv, page, d) if heads_first else (n_pages, page, hkv, d)
        k, v = (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) for _ in range(2))
        if self.cache == "e4m3":
            k, v = (20 * k).clamp(-448, 448), (30 * v).clamp(-448, 448)
        k, v = k.to(TYPES[self.cache]), v.to(TYPES[self.cache])
        if junk:                                             # what no token holds: NaN
            used = torch.zeros(n_pages, page, dtype=torch.bool)
            for b, n in enumerate(self.lens):
                j = np.arange(n)
                used[table[b, j // page], j % page] = True
            where = ~(used[:, None, :, None] if heads_first else used[:, :, None, None]).expand(shape)
            nan = torch.tensor(float("nan")).to(TYPES[self.cache])
            bits = torch.int16 if self.cache != "e4m3" else torch.uint8
            for x in (k, v):
                x.view(bits)[where] = nan.view(bits)
        self.k_scale = (0.01 + 0.05 * torch.rand(hkv, generator=torch.Generator().manual_seed(seed))) if self.cache == "e4m3" else None
        self.v_scale = (0.01 + 0.05 * torch.rand(hkv, generator=torch.Generator().manual_seed(seed + 1))) if self.cache == "e4m3" else None
        self.pool = dict(k=self.wide(k), v=self.wide(v), table=table)
        to = lambda x: x.to(device) if x is not None else None  # noqa: E731
        self.k, self.v, self.table = to(k), to(v), to(torch.from_numpy(table))
        self.weights = torch.zeros(n_pages, hkv, page, device=device)
        self.ids = torch.zeros(n_pages, hkv, page, dtype=torch.int32, device=device)
        self.d_start, self.d_lens = to(torch.from_numpy(self.start)), to(torch.tensor(self.lens, dtype=torch.int32))

    def wide(self, x):
        """[pages, slots, heads, d] of 64-bit values."""
        x = x.detach().cpu().float().double().numpy()
        return np.ascontiguousarray(x.transpose(0, 2, 1, 3)) if self.heads_first else x

    def rows(self, heads, scale=1.0):
        return torch.from_numpy((scale * self.rng.standard_normal((self.n_tokens, heads, self.d))).astype(np.float32)).to(TYPES[self.dtype]).to(self.device)

    def handle(self, **kw):
        cfg = dict(n_q_heads=self.hq, n_kv_heads=self.hkv, head_dim=self.d, page_size=self.page, dtype=NAMES[self.dtype], cache_dtype=NAMES[self.cache],
                   max_seqs=len(self.lens), max_tokens=max(1, self.n_tokens), max_len=self.max_len)
        cfg.update(kw)
        return kvx.KvPaged(**cfg)

    def pages(self, **kw):
        args = dict(heads_first=self.heads_first, k_scale=self.k_scale.to(self.device) if self.k_scale is not None else None,
                    v_scale=self.v_scale.to(self.device) if self.v_scale is not None else None, weights=self.weights, ids=self.ids)
        args.update(kw)
        return kvx.KvPages(self.k, self.v, self.table, **args)

    def batch(self, seen=None, max_new=None):
        return kvx.KvPagedBatch(self.d_start, self.d_lens, n_tokens=self.n_tokens, max_new=max([0] + self.new) if max_new is None else max_new,
                                max_len=self.max_len, seen=seen)


def attend_bounds(case, ref, absolute, lse, gained, reach, few):
    """Largest errors of out, lse and gained weights.  u: half a step of the 16-bit type.
    A logit is an fp32 sum of d exact products, scaled: its error is at most (d + 4) 2^-24 of the sum of magnitudes (`reach`).  That, the
    exponential and fp32 sums over the keys (2^-24 a key) perturb a probability; in launches of more than 32 rows of a key head the
    probabilities are also rounded to 16 bits (u each).  The output is rounded once more."""
    u = HALF_STEP[case.dtype]
    keys = max(1, max(case.lens))
    logit = (case.d + 4) * 2.0 ** -24 * reach
    relative = 2 * logit + EXP_ERROR + keys * 2.0 ** -23 + (0.0 if few else 2 * u)
    if few:
        relative = relative + 2 * u * u                      # probabilities as pairs of 16-bit values
    tiny = {"bf16": 0.0, "f16": 2.0 ** -24}[case.dtype]      # fp16 probabilities and outputs below 2^-14 are rounded to multiples of 2^-24
    out = u * np.abs(ref) + relative[..., None] * absolute * (1 + u) + tiny * (1 + absolute) * (1 if few else keys)
    l_err = logit + EXP_ERROR + keys * 2.0 ** -24 + np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -23
    rows = max([1] + case.new) * case.hq // case.hkv
    # (a weight's own rounding in the sum of what was there, up to 1 here, and what is gained)
    w_err = gained * (2 * logit.max(initial=0) + 2 * EXP_ERROR + l_err.max(initial=0) + rows * 2.0 ** -24) + 2.0 ** -24 * (1 + gained)
    return out, l_err, w_err


def check(got, ref, bound, what):
    got = np.asarray(got, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities differ"
    fine = np.isfinite(ref)
    over = np.abs(got[fine] - ref[fine]) - np.broadcast_to(bound, ref.shape)[fine]
    assert np.isfinite(got[fine]).all() and (over.size == 0 or over.max() <= 0), f"{what}: {over.max():.3g} over its bound, at {np.unravel_index(np.argmax(np.where(fine, np.abs(got - ref) - bound, -1)), ref.shape)}"
