"""Measured cases of the operators on a paged cache: append (rotary positions, then keys and values into the pages), attend
(attention of the new tokens of every sequence over its pages, with the weights that the cached tokens received) and evict
(a cache brought back to its budget by those weights).

A case is one call in the middle of a serving loop over one layer: `prepare` makes the pool of pages, the page tables, the
lengths and the call's tensors, and `run` makes the call.  Lengths are a function of the case, contents and the order of the
pages one of the seed.  Page 0 is nobody's: unused entries of the page tables name it.

`own` False: the operators in elementary torch operations, in 32 bits (angles in 64), rounded once at the end.  `own` True: the
framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BASE = dict(dtype="bf16", cache="bf16", hq=32, hkv=8, d=128, page=16, heads_first=False, seqs=1, new=1, len=1, ragged=False)
APPEND = dict(BASE, op="append", rotary=128, layout="half", scaling="plain", factor=1.0, far=0)
ATTEND = dict(BASE, op="attend", causal=True, window=0, weights=False, lse=False)
EVICT = dict(BASE, op="evict", budget=0, sinks=4, recent=32)


def listed():
    return [
        # decoding one stream: one token of 32 heads of queries and 8 of keys, nothing but latency
        dict(APPEND, name="append_one_token", len=700),
        # a serving step that mixes prompts of uneven length, half of each head rotated, positions far beyond the length that the
        # frequencies were made for, 8-bit cache
        dict(APPEND, name="append_prompts_e4m3", cache="e4m3", rotary=64, layout="interleaved", scaling="parts", factor=8.0, seqs=7, new=2311,
             len=9000, ragged=True, far=1 << 20),
        # one token of one short sequence
        dict(ATTEND, name="attend_one_token", dtype="f16", cache="f16", hq=16, hkv=16, d=64, len=517),
        # a decoding batch whose sequences differ in length
        dict(ATTEND, name="attend_decode_ragged", seqs=64, len=8192, ragged=True),
        # a few very long sequences, 8-bit cache, eight query heads to a key head
        dict(ATTEND, name="attend_decode_long_e4m3", cache="e4m3", hq=64, hkv=8, page=64, heads_first=True, seqs=4, len=131072),
        # one frame of 1041 tokens over the tokens of a stream and itself, all of its tokens visible to each other
        dict(ATTEND, name="attend_frame", hq=16, hkv=16, d=64, page=64, new=1041, len=16384 + 1041, causal=False),
        # a long prompt in pieces: the pieces' statistics are kept for a later merge
        dict(ATTEND, name="attend_chunk", seqs=2, new=4096, len=20480, lse=True),
        # decoding and prompt pieces of uneven length in one call, sliding window, six query heads to a key head
        dict(ATTEND, name="attend_mixed_window", dtype="f16", cache="f16", hq=12, hkv=2, page=32, seqs=13, new=700, len=6000, ragged=True, window=1000),
        # a decoding batch that collects the weights its cached tokens receive
        dict(ATTEND, name="attend_decode_weights", seqs=32, len=4097, weights=True, lse=True),
        # a prompt piece that collects them
        dict(ATTEND, name="attend_chunk_weights", hq=16, hkv=16, d=64, new=1024, len=9216, weights=True, lse=True),
        # a decoding batch of full caches: one token of each leaves
        dict(EVICT, name="evict_step", seqs=32, len=4097, budget=4096),
        # two caches brought down after a long prompt
        dict(EVICT, name="evict_prompt", seqs=2, len=18432, budget=8192, new=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(8, 8), (16, 16), (32, 8), (12, 2), (24, 3), (64, 8), (6, 1), (5, 5)])
    d, dtype = rng.choice([64, 128]), rng.choice(["bf16", "f16"])
    both = dict(dtype=dtype, cache=rng.choice([dtype, dtype, "e4m3"]), hq=heads[0], hkv=heads[1], d=d, page=rng.choice([8, 16, 32, 64, 128]),
                heads_first=rng.random() < 0.5, ragged=rng.random() < 0.6)
    op = rng.choice(["append", "append", "attend", "attend", "attend", "evict", "evict"])
    if op == "append":
        seqs, new = _log(rng, 1, 64), _log(rng, 1, 2048)
        new = max(1, min(new, 12000 // seqs))
        scaling = rng.choice(["plain", "linear", "base", "parts"])
        return dict(APPEND, **both, op=op, seqs=seqs, new=new, len=new + _log(rng, 1, 3000), rotary=rng.choice([d, d // 2, d // 4]),
                    layout=rng.choice(["half", "interleaved"]), scaling=scaling, factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0]),
                    far=rng.choice([0, 0, 1 << 20]))
    if op == "attend":
        kind = rng.choice(["one", "few", "chunk"])
        weights = rng.random() < 0.35
        if kind == "one":
            seqs, new, n = _log(rng, 1, 96), 1, _log(rng, 1, 40000)
            n = max(1, min(n, (300000 if heads[1] <= 8 else 150000) // seqs))
        elif kind == "few":
            seqs, new, n = _log(rng, 1, 24), _log(rng, 2, 40), _log(rng, 40, 12000)
        else:
            seqs, new = _log(rng, 1, 6), _log(rng, 41, 2048)
            n = new + _log(rng, 1, 10000 // seqs)
        return dict(ATTEND, **both, op=op, seqs=seqs, new=new, len=max(n, new), causal=rng.random() < 0.8, window=rng.choice([0, 0, _log(rng, 16, 4000)]),
                    weights=weights, lse=weights or rng.random() < 0.5)
    seqs, n = _log(rng, 1, 40), _log(rng, 130, 16000)
    n = max(130, min(n, 80000 // seqs))
    new = max(1, min(_log(rng, 1, 1024), n // 2))
    return dict(EVICT, **both, op=op, seqs=seqs, len=n, new=new, budget=n - _log(rng, 1, n - 64), sinks=rng.choice([0, 1, 4]), recent=_log(rng, 1, 59))


# ---- what a case holds -----------------------------------------------------------------------------------------------------
def _lengths(case):
    """(new tokens, cached tokens with the new ones) of every sequence; the first has the most of both."""
    new, total = [], []
    for i in range(case["seqs"]):
        u, w = ((i * 0.6180339887498949) % 1.0, (i * 0.7548776662466927) % 1.0) if case["ragged"] and i else (1.0, 1.0)
        n = max(1, round(case["new"] * u ** 2)) if u else 1
        t = n + round((case["len"] - case["new"]) * w)
        new.append(n)
        total.append(t)
    return new, total


def _visible(case):
    """Per sequence: (pairs of a row and a key that it sees, keys that at least one row sees)."""
    got = []
    for n, t in zip(*_lengths(case)):
        pairs = n * t - n * (n - 1) // 2 if case["causal"] else n * t
        low = 0
        if case["window"]:
            first = t - n + 1 - case["window"]                # the first key of row 0, row i begins i further on
            i = max(0, -first)                                # rows that begin at key 0
            low = max(0, first)
            pairs -= max(0, n - i) * (first + i + first + n - 1) // 2
        got.append((pairs, t - low))
    return got


def work(case):
    new, total = _lengths(case)
    N, T, B = sum(new), sum(total), case["seqs"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    elt = 1 if case["cache"] == "e4m3" else 2
    if case["op"] == "append":
        return {"bytes": N * d * (2 * 2 * hq + 2 * (2 + elt) * hkv) + N * (4 + hkv * 8) + 4 * B, "flops": 3.0 * N * case["rotary"] * (hq + hkv)}
    if case["op"] == "attend":
        seen = _visible(case)
        pairs, keys = sum(p for p, _ in seen), sum(k for _, k in seen)
        return {"bytes": 2 * 2 * N * hq * d + 2 * keys * hkv * d * elt + (4 * N * hq if case["lse"] else 0) + (8 * T * hkv if case["weights"] else 0),
                "flops": 4.0 * pairs * hq * d}
    budget, moved = case["budget"], 0.0
    for n, t in zip(new, total):
        if t > budget:      # the last ones stay, of the others behind the budget as many as of all that are not protected
            protected = case["sinks"] + case["recent"]
            behind = t - budget
            moved += min(behind, case["recent"]) + max(0, behind - case["recent"]) * max(0, budget - protected) / max(1, t - protected)
    kept = sum(min(t, budget) for t in total)
    return {"bytes": 8.0 * (T + kept) * hkv + moved * hkv * 4 * d * elt, "flops": float(T * hkv)}


def _frequencies(case):
    """Radians per position of every pair, 64 bits: plain, positions divided by the factor, a larger base, or by parts (long
    wavelengths divided by the factor, short ones as they are, a linear ramp between)."""
    r, f = case["rotary"], case["factor"]
    i = torch.arange(0, r, 2, dtype=torch.float64)
    base = 10000.0 * (f ** (r / (r - 2)) if case["scaling"] == "base" else 1.0)
    w = base ** (-i / r)
    if case["scaling"] == "linear":
        return w / f
    if case["scaling"] == "parts":
        turns = 8192 * w / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return w / f * (1 - keep) + w * keep
    return w


def _pages(case, total, g, dev):
    """Page table (in an order of the seed) and the pool's two tensors, filled with what was there before the call."""
    P, hkv, d = case["page"], case["hkv"], case["d"]
    counts = [-(-t // P) for t in total]
    n_pages = 1 + sum(counts) + 3
    order = 1 + torch.randperm(n_pages - 1, generator=g, device=dev)
    width = max(counts)
    slot = torch.arange(width, device=dev)[None, :]
    count = torch.tensor(counts, device=dev)
    first = (count.cumsum(0) - count)[:, None]
    table = torch.where(slot < count[:, None], order[(first + slot).clamp(max=n_pages - 2)], 0).to(torch.int32)
    shape = (n_pages, hkv, P, d) if case["heads_first"] else (n_pages, P, hkv, d)
    dt, scale = DTYPES[case["cache"]], case["cache"] == "e4m3"
    spread = torch.exp(0.5 * torch.randn(hkv, d, generator=g, device=dev))
    spread = spread[:, None, :] if case["heads_first"] else spread
    k = torch.randn(shape, generator=g, device=dev) * spread
    v = torch.randn(shape, generator=g, device=dev)
    k_scale = 0.02 + 0.01 * torch.rand(hkv, generator=g, device=dev) if scale else None
    v_scale = 0.01 + 0.01 * torch.rand(hkv, generator=g, device=dev) if scale else None
    if scale:
        by = (1, hkv, 1, 1) if case["heads_first"] else (1, 1, hkv, 1)
        k, v = (k / k_scale.view(by)).clamp(-448, 448), (v / v_scale.view(by)).clamp(-448, 448)
    return table, k.to(dt), v.to(dt), k_scale, v_scale


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    new, total = _lengths(case)
    B, N, hq, hkv, d, P, op = case["seqs"], sum(new), case["hq"], case["hkv"], case["d"], case["page"], case["op"]
    dt = DTYPES[case["dtype"]]
    s = dict(case=case, n_new=new, n_len=total)
    s["table"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"] = _pages(case, total, g, dev)
    n_pages = s["k_pages"].shape[0]
    s["start"] = torch.tensor([sum(new[:i]) for i in range(B + 1)], dtype=torch.int32, device=dev)
    s["lens"] = torch.tensor(total, dtype=torch.int32, device=dev)
    s["seen"] = s["lens"] + (11 if op == "evict" else 0)
    s["ids"] = torch.zeros(n_pages, hkv, P, dtype=torch.int32, device=dev)
    s["weights"] = torch.zeros(n_pages, hkv, P, device=dev)
    if op == "append":
        qkv = torch.randn(N, hq + 2 * hkv, d, generator=g, device=dev).to(dt)      # one projection's rows: q, k and v are parts of them
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty(N, hq, d, dtype=dt, device=dev)
        s["positions"] = torch.cat([torch.arange(t - n, t, device=dev) for n, t in zip(new, total)]).to(torch.int32) + case["far"]
        s["frequencies"] = _frequencies(case)
    elif op == "attend":
        s["q"] = torch.randn(N, hq, d, generator=g, device=dev).to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(N, hq, device=dev) if case["lse"] else None
        if case["weights"]:
            s["weights"] = torch.rand(n_pages, hkv, P, generator=g, device=dev)
            s["weights_out"] = torch.zeros_like(s["weights"])
    else:
        # what a cache that has pruned before holds: its slots are not in the order of arrival, some tokens were never attended to
        for b, (n, t) in enumerate(zip(new, total)):
            j = torch.arange(t, device=dev)
            page, slot = s["table"][b, j // P].long(), j % P
            old = torch.rand(hkv, t + 11 - n, generator=g, device=dev).argsort(1)[:, :t - n]
            ids = torch.cat([old, torch.arange(t + 11 - n, t + 11, device=dev).expand(hkv, n)], 1)
            w = torch.exp(2 * torch.randn(hkv, t, generator=g, device=dev)) * (torch.rand(hkv, t, generator=g, device=dev) > 0.05)
            s["ids"][page, :, slot] = ids.T.to(torch.int32)
            s["weights"][page, :, slot] = w.T
        s["ids_out"], s["weights_out"] = s["ids"].clone(), s["weights"].clone()
        s["lens_out"] = torch.empty_like(s["lens"])
    if own:
        import paper_2601_01204_amd as kvx
        names = {"bf16": kvx.KV_BF16, "f16": kvx.KV_F16, "e4m3": kvx.KV_E4M3}
        rope = {}
        if op == "append":
            rope = dict(rotary_dim=case["rotary"], rope_layout=kvx.KV_ROPE_HALF if case["layout"] == "half" else kvx.KV_ROPE_INTERLEAVED,
                        rope_scaling={"plain": kvx.KV_ROPE_PLAIN, "linear": kvx.KV_ROPE_LINEAR, "base": kvx.KV_ROPE_BASE, "parts": kvx.KV_ROPE_PARTS}[case["scaling"]],
                        rope_base=10000.0, rope_factor=case["factor"], rope_original_len=8192)
        s["handle"] = kvx.KvPaged(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=P, dtype=names[case["dtype"]], cache_dtype=names[case["cache"]],
                                  max_seqs=B, max_tokens=N, max_len=max(total), **rope)
        s["pages"] = kvx.KvPages(s["k_pages"], s["v_pages"], s["table"], heads_first=case["heads_first"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                 weights=s["weights"], ids=s["ids"])
        s["batch"] = kvx.KvPagedBatch(s["start"], s["lens"], n_tokens=N, max_new=max(new), max_len=max(total), seen=s["seen"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        c, stream = s["case"], torch.cuda.current_stream().cuda_stream
        h, pages, batch = s["handle"], s["pages"], s["batch"]
        if op == "append":
            h.append(pages, batch, s["k"], s["v"], q=s["q"], q_out=s["q_out"], positions=s["positions"], hip_stream=stream)
        elif op == "attend":
            h.attend(pages, batch, s["q"], s["out"], lse=s["lse"], causal=c["causal"], window=c["window"],
                     weights_out=s["weights_out"] if c["weights"] else None, hip_stream=stream)
        else:
            h.evict(pages, batch, budget=c["budget"], sinks=c["sinks"], recent=c["recent"], weights_out=s["weights_out"], ids_out=s["ids_out"],
                    lens_out=s["lens_out"], hip_stream=stream)
    elif op == "append":
        _append(s)
    elif op == "attend":
        _attend(s)
    else:
        _evict(s)
    if op == "append":
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "ids": s["ids"], "weights": s["weights"]}
    if op == "attend":
        got = {"out": s["out"]}
        if s["lse"] is not None:
            got["lse"] = s["lse"]
        if s["case"]["weights"]:
            got["weights"] = s["weights_out"]
        return got
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "ids": s["ids_out"], "weights": s["weights_out"], "lens": s["lens_out"]}


def _token_major(s, name):
    """The pool as [pages, slots, heads, d]."""
    return s[name].transpose(1, 2) if s["case"]["heads_first"] else s[name]


def _places(s):
    """Of every new token: its sequence, its row in it, its page and its slot there."""
    start, lens = s["start"].long(), s["lens"].long()
    t = torch.arange(sum(s["n_new"]), device=start.device)
    b = torch.searchsorted(start[1:], t, right=True)
    row = t - start[b]
    at = lens[b] - (start[1:] - start[:-1])[b] + row
    P = s["case"]["page"]
    return b, row, s["table"][b, at // P].long(), at % P


def _append(s):
    c = s["case"]
    r, scaled = c["rotary"], c["cache"] == "e4m3"
    angle = s["positions"].double()[:, None] * s["frequencies"].to(s["positions"].device)
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def rotated(x):
        x = x.float()
        y = x.clone()
        first, second = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        return y

    b, row, page, slot = _places(s)
    k, v = rotated(s["k"]), s["v"].float()
    if scaled:
        k, v = (k / s["k_scale"][:, None]).clamp(-448, 448), (v / s["v_scale"][:, None]).clamp(-448, 448)
    s["q_out"].copy_(rotated(s["q"]))
    kp, vp = _token_major(s, "k_pages"), _token_major(s, "v_pages")
    if scaled:      # (torch indexes bytes, not 8-bit floats)
        kp.view(torch.uint8)[page, slot] = k.to(kp.dtype).view(torch.uint8)
        vp.view(torch.uint8)[page, slot] = v.to(vp.dtype).view(torch.uint8)
    else:
        kp[page, slot], vp[page, slot] = k.to(kp.dtype), v.to(vp.dtype)
    new = (s["start"][1:] - s["start"][:-1]).long()
    s["ids"][page, :, slot] = (s["seen"].long()[b] - new[b] + row).to(torch.int32)[:, None].expand(-1, c["hkv"])
    s["weights"][page, :, slot] = 0.0


def _gathered(s, name, scale, width):
    """[sequences, heads, width, d] in 32 bits; zero behind each sequence's end."""
    c = s["case"]
    j = torch.arange(width, device=s["table"].device)
    page = s["table"][:, j // c["page"]].long()
    pool = _token_major(s, name)
    x = (pool.view(torch.uint8)[page, j % c["page"]].view(pool.dtype) if c["cache"] == "e4m3" else pool[page, j % c["page"]]).float()
    if scale is not None:
        x = x * scale[:, None]
    x = torch.where((j[None, :] < s["lens"][:, None])[:, :, None, None], x, 0.0)
    return x.permute(0, 2, 1, 3).contiguous()


def _attend(s):
    c = s["case"]
    hq, hkv, d, B, G = c["hq"], c["hkv"], c["d"], c["seqs"], c["hq"] // c["hkv"]
    n, width = max(s["n_new"]), max(s["n_len"])
    b, row, _, _ = _places(s)
    q = torch.zeros(B, n, hq, d, device=s["q"].device)
    q[b, row] = s["q"].float() / math.sqrt(d)
    q = q.view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B * hkv, n * G, d)
    k, v = _gathered(s, "k_pages", s["k_scale"], width), _gathered(s, "v_pages", s["v_scale"], width)
    x = torch.bmm(q, k.view(B * hkv, width, d).transpose(1, 2).contiguous()).view(B, hkv, n, G, width)
    del k
    j = torch.arange(width, device=q.device)
    new, lens = (s["start"][1:] - s["start"][:-1]).long()[:, None], s["lens"].long()[:, None]
    own_key = lens - new + torch.arange(n, device=q.device)[None, :]      # a row's own place among the keys
    hide = (j >= lens)[:, None, :]
    if c["causal"]:
        hide = hide | (j > own_key[:, :, None])
    if c["window"]:
        hide = hide | (j <= own_key[:, :, None] - c["window"])
    x.masked_fill_(hide[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    x.div_(torch.where(total == 0, 1.0, total))
    out = torch.bmm(x.view(B * hkv, n * G, width), v.view(B * hkv, width, d)).view(B, hkv, n, G, d)
    s["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(B, n, hq, d)[b, row])
    if s["lse"] is not None:
        lse = (top + total.log()).view(B, hkv, n, G).permute(0, 2, 1, 3).reshape(B, n, hq)
        s["lse"].copy_(lse[b, row])
    if c["weights"]:
        real = (torch.arange(n, device=q.device)[None, :] < new)[:, None, :, None, None]
        got = torch.where(real, x, 0.0).sum((2, 3))                       # [B, hkv, width]
        page, slot = s["table"][:, j // c["page"]].long(), (j % c["page"]).expand(B, width)
        before = s["weights"][page, :, slot]                              # [B, width, hkv]
        live = (j[None, :] < s["lens"][:, None])[:, :, None]
        s["weights_out"][page, :, slot] = torch.where(live, before + got.transpose(1, 2), s["weights_out"][page, :, slot])


def _evict(s):
    c = s["case"]
    B, width, budget = c["seqs"], max(s["n_len"]), c["budget"]
    j = torch.arange(width, device=s["table"].device)
    page, slot = s["table"][:, j // c["page"]].long(), (j % c["page"]).expand(B, width)
    w, ids = s["weights"][page, :, slot].transpose(1, 2), s["ids"][page, :, slot].transpose(1, 2)      # [B, hkv, width]
    live = (j < s["lens"][:, None])[:, None, :]
    key = torch.where((ids < c["sinks"]) | (ids >= s["seen"][:, None, None] - c["recent"]), math.inf, w)
    order = torch.where(live, key, -1.0).sort(dim=-1, descending=True, stable=True).indices              # weights are never negative
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order).contiguous())
    keep = live & (rank < budget)
    mover, hole = keep & (j >= budget), live & ~keep & (j < budget)
    m = min(budget, width)
    movers = torch.where(mover, j, width).sort(dim=-1).values                                              # ascending, then nothing
    nth = hole.long().cumsum(-1) - 1
    src = torch.where(hole, movers.gather(-1, nth.clamp(min=0)).clamp(max=width - 1), j)[..., :m]      # [B, hkv, m]
    head = torch.arange(c["hkv"], device=j.device)[None, :, None]
    from_page, from_slot = page[:, None, :].expand(-1, c["hkv"], -1).gather(-1, src), src % c["page"]
    to_page, to_slot = page[:, None, :m], slot[:, None, :m]
    for name in ("k_pages", "v_pages"):
        pool = _token_major(s, name)
        pool = pool.view(torch.uint8) if c["cache"] == "e4m3" else pool
        pool[to_page, to_slot, head] = pool[from_page, from_slot, head]
    new_w, new_ids = w.gather(-1, src), ids.gather(-1, src)
    left = torch.where(live[..., :m], torch.ones_like(src, dtype=torch.bool), False)
    s["weights_out"][to_page, head, to_slot] = torch.where(left, new_w, s["weights_out"][to_page, head, to_slot])
    s["ids_out"][to_page, head, to_slot] = torch.where(left, new_ids, s["ids_out"][to_page, head, to_slot])
    s["lens_out"].copy_(s["lens"].clamp(max=budget))


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------
def exact(case, seed):
    """Sequence by sequence and head by head, in 64 bits."""
    s = prepare(case, seed)
    new, total, P, hkv = s["n_new"], s["n_len"], case["page"], case["hkv"]
    start = [sum(new[:i]) for i in range(case["seqs"])]
    kp, vp = (x.transpose(1, 2) if case["heads_first"] else x for x in (s["k_pages"], s["v_pages"]))
    if case["op"] == "append":
        r, f = case["rotary"], _frequencies(case).to(s["q"].device)
        a = s["positions"].double().view(-1, 1, 1) * f

        def turn(x):
            x = x.double()
            part, rest = x[..., :r], x[..., r:]
            p = part.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (r // 2, 2))
            z = torch.view_as_complex(p.contiguous()) * torch.polar(torch.ones_like(a), a)
            z = torch.view_as_real(z)
            return torch.cat([z.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else z.flatten(-2), rest], -1)

        k_all, v_all = kp.double(), vp.double()
        k, v = turn(s["k"]), s["v"].double()
        if case["cache"] == "e4m3":
            k, v = (k / s["k_scale"].double()[:, None]).clamp(-448, 448), (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
        for b in range(case["seqs"]):
            j = torch.arange(total[b] - new[b], total[b], device=k.device)
            page = s["table"][b, j // P].long()
            k_all[page, j % P], v_all[page, j % P] = k[start[b]:start[b] + new[b]], v[start[b]:start[b] + new[b]]
        if case["heads_first"]:
            k_all, v_all = k_all.transpose(1, 2), v_all.transpose(1, 2)
        return {"q": turn(s["q"]), "k_pages": k_all, "v_pages": v_all, "ids": None, "weights": None}
    if case["op"] == "evict":
        return None      # nothing is computed: rows are kept or moved
    if sum(p for p, _ in _visible(case)) * case["hq"] * case["d"] > 1e13:
        return None
    G = case["hq"] // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=out.device)
    weights = s["weights_out"].double() if case["weights"] else None
    for b in range(case["seqs"]):
        j = torch.arange(total[b], device=out.device)
        page, slot = s["table"][b, j // P].long(), j % P
        at = total[b] - new[b] + torch.arange(new[b], device=out.device)
        see = torch.ones(new[b], total[b], dtype=torch.bool, device=out.device)
        if case["causal"]:
            see &= j[None, :] <= at[:, None]
        if case["window"]:
            see &= j[None, :] > at[:, None] - case["window"]
        rows = slice(start[b], start[b] + new[b])
        for h in range(hkv):
            if case["cache"] == "e4m3":
                k, v = (x.view(torch.uint8)[page, slot, h].view(x.dtype).double() * y[h].double() for x, y in ((kp, s["k_scale"]), (vp, s["v_scale"])))
            else:
                k, v = kp[page, slot, h].double(), vp[page, slot, h].double()
            got = torch.zeros(total[b], dtype=torch.float64, device=out.device)
            for g in range(h * G, h * G + G):
                z = (s["q"][rows, g].double() @ k.T.contiguous()) / math.sqrt(case["d"])
                z = torch.where(see, z, -math.inf)
                lse[rows, g] = torch.logsumexp(z, 1)
                p = torch.where(see, torch.exp(z - lse[rows, g][:, None]), 0.0)
                out[rows, g] = p @ v
                got += p.sum(0)
            if weights is not None:
                weights[page, h, slot] = s["weights"][page, h, slot].double() + got
    found = {"out": out}
    if case["lse"]:
        found["lse"] = lse
    if case["weights"]:
        found["weights"] = weights
    return found
