"""The paged cache's operators together, as a serving loop uses them: prompts, then single tokens, each step append, attend with
weights, evict; captured into a graph and replayed; on other streams; in pools of more than 4 GB."""
import math

import numpy as np
import pytest
import torch

import paper_2601_01204_amd as kvx
from oracle import paged_oracle as po
from tests import paged_util as pu

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Loop:
    """Sequences of up to `room` tokens in a pool of their own, with everything on the device that a step reads and moves on."""

    def __init__(self, seqs, room, budget, hq=4, hkv=2, d=64, page=16, dtype="bf16", cache=None, rotary=64, max_new=1, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.budget, self.hq, self.hkv, self.d, self.page, self.dtype, self.cache = seqs, budget, hq, hkv, d, page, dtype, cache or dtype
        per = -(-room // page)
        n = seqs * per + 2
        self.table = (torch.randperm(n, generator=g)[:seqs * per].view(seqs, per)).to(torch.int32).to(DEV)
        dt = pu.TYPES[self.cache]
        self.k, self.v = (torch.full((n, page, hkv, d), float("nan")).to(dt).to(DEV) for _ in range(2))
        self.weights = torch.zeros(n, hkv, page, device=DEV)
        self.ids = torch.zeros(n, hkv, page, dtype=torch.int32, device=DEV)
        self.lens, self.seen = (torch.zeros(seqs, dtype=torch.int32, device=DEV) for _ in range(2))
        self.scales = (torch.full((hkv,), 0.02), torch.full((hkv,), 0.03)) if self.cache == "e4m3" else (None, None)
        to = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        self.pages = kvx.KvPages(self.k, self.v, self.table, k_scale=to(self.scales[0]), v_scale=to(self.scales[1]), weights=self.weights, ids=self.ids)
        self.room, self.rotary = room, rotary
        self.h = kvx.KvPaged(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=page, dtype=pu.NAMES[dtype], cache_dtype=pu.NAMES[self.cache], max_seqs=seqs,
                             max_tokens=seqs * max_new, max_len=room, rotary_dim=rotary)

    def tensors(self, new, seed):
        """A step's rows: q, k, v, out, lse, and where each sequence's rows begin."""
        g = torch.Generator().manual_seed(seed)
        n = sum(new)
        q, k, v = (torch.randn(n, h, self.d, generator=g).to(pu.TYPES[self.dtype]).to(DEV) for h in (self.hq, self.hkv, self.hkv))
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        return dict(q=q, k=k, v=v, q_out=torch.empty_like(q), out=torch.empty_like(q), lse=torch.empty(n, self.hq, device=DEV), start=start, new=list(new),
                    d_new=(start[1:] - start[:-1]).contiguous())

    def append(self, t, stream=0):
        self.lens += t["d_new"]
        self.seen += t["d_new"]
        self.batch = kvx.KvPagedBatch(t["start"], self.lens, n_tokens=sum(t["new"]), max_new=max(t["new"]), max_len=self.room, seen=self.seen)
        self.h.append(self.pages, self.batch, t["k"], t["v"], q=t["q"], q_out=t["q_out"], hip_stream=stream)

    def attend(self, t, stream=0):
        self.h.attend(self.pages, self.batch, t["q_out"], t["out"], lse=t["lse"], weights_out=self.weights, hip_stream=stream)

    def evict(self, stream=0):
        self.h.evict(self.pages, self.batch, self.budget, sinks=2, recent=8, weights_out=self.weights, ids_out=self.ids, lens_out=self.lens, hip_stream=stream)

    def step(self, t, stream=0):
        self.append(t, stream)
        self.attend(t, stream)
        self.evict(stream)

    def pool(self):
        wide = lambda x: x.cpu().float().double().numpy()  # noqa: E731
        return dict(k=wide(self.k), v=wide(self.v), table=self.table.cpu().numpy(), weights=self.weights.cpu().numpy().copy(), ids=self.ids.cpu().numpy().copy())

    def state(self):
        return [x.clone() for x in (self.k.view(torch.uint8), self.v.view(torch.uint8), self.weights, self.ids, self.lens, self.seen)]


def check_step(loop, t):
    """One step, each operator against the definition on the state that it found."""
    loop.append(t)
    torch.cuda.synchronize()
    pool, lens, seen = loop.pool(), loop.lens.tolist(), loop.seen.tolist()
    start = t["start"].tolist()
    at = np.concatenate([np.arange(seen[b] - n, seen[b]) for b, n in enumerate(t["new"])])
    u = pu.HALF_STEP[loop.dtype]
    ref = po.rotate(t["q"].float().cpu().numpy(), at, po.rope_frequencies(loop.rotary), False)
    pu.check(t["q_out"].float().cpu().numpy(), ref, u * np.abs(ref) + 2.0 ** -20 * np.abs(t["q"].float().cpu().numpy()).max(), "turned queries")
    for b, n in enumerate(t["new"]):
        for i in range(n):
            page, slot = po.place(pool, b, lens[b] - n + i)
            assert (pool["ids"][page, :, slot] == seen[b] - n + i).all() and (pool["weights"][page, :, slot] == 0).all()

    loop.attend(t)
    torch.cuda.synchronize()
    scales = [None if x is None else x.numpy() for x in loop.scales]
    out, lse, gained, absolute, reach = po.attend(pool, t["q_out"].float().cpu().numpy(), start, lens, 1 / math.sqrt(loop.d), True, 0, *scales)
    case = type("Case", (), dict(dtype=loop.dtype, d=loop.d, lens=lens, new=t["new"], hq=loop.hq, hkv=loop.hkv))
    b_out, b_lse, b_w = pu.attend_bounds(case, out, absolute, lse, gained, reach, max(t["new"]) * loop.hq // loop.hkv <= 32)
    pu.check(t["out"].float().cpu().numpy(), out, b_out, "out")
    pu.check(t["lse"].cpu().numpy(), lse, b_lse, "lse")
    before = pool["weights"].astype(np.float64)
    pu.check(loop.weights.cpu().numpy(), before + gained, b_w + 2.0 ** -24 * before, "weights")

    pool = loop.pool()
    loop.evict()
    torch.cuda.synchronize()
    k, v, w, ids, new_lens, written = po.evict(pool, lens, seen, loop.budget, 2, 8)
    got = loop.pool()
    assert np.array_equal(got["k"], k, equal_nan=True) and np.array_equal(got["v"], v, equal_nan=True)
    assert np.array_equal(got["weights"][written], w[written]) and np.array_equal(got["ids"][written], ids[written])
    assert loop.lens.tolist() == new_lens.tolist() and loop.h.status() == 0


@pytest.mark.parametrize("dtype,cache,d,hq,hkv", [("bf16", "bf16", 64, 4, 2), ("f16", "f16", 128, 6, 2), ("bf16", "e4m3", 128, 8, 1)])
def test_prompts_then_single_tokens_under_a_budget(dtype, cache, d, hq, hkv):
    loop = Loop(3, 200, 60, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, max_new=100, seed=d)
    for i, new in enumerate([[50, 90, 1], [1, 40, 100], [7, 1, 1]] + [[1, 1, 1]] * 6):
        check_step(loop, loop.tensors(new, i))
    assert loop.lens.tolist() == [60, 60, 60] and loop.seen.tolist() == [64, 137, 108]


def test_captured_steps_replay_on_what_the_device_holds():
    """A decoding step in a graph: lengths, page tables and weights move on between replays; an eager twin does the same steps."""
    eager, graphed = Loop(4, 80, 64, seed=1, max_new=70), Loop(4, 80, 64, seed=1, max_new=70)
    prompt = eager.tensors([60, 30, 70, 1], 1)
    for x in (eager, graphed):
        x.step(prompt)
    t = graphed.tensors([1] * 4, 2)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        graphed.step(t, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(graphed.lens, eager.lens), "nothing has run yet"
    for i in range(8):
        fresh = eager.tensors([1] * 4, 100 + i)
        for name in ("q", "k", "v"):
            t[name].copy_(fresh[name])
        graph.replay()
        noise = torch.randn(1 << 20, device=DEV).sum().item()        # the program's own work between the replays
        eager.step(fresh)
        torch.cuda.synchronize()
        assert torch.equal(t["out"], fresh["out"]) and torch.equal(t["lse"], fresh["lse"]), (i, noise)
        for a, b in zip(graphed.state(), eager.state()):
            assert torch.equal(a, b), i
    assert eager.lens.tolist() == [64, 38, 64, 9]


def test_another_stream_and_two_handles_at_once():
    loops = [Loop(2, 600, 500, seed=5 + i, max_new=300) for i in range(2)]
    twins = [Loop(2, 600, 500, seed=5 + i, max_new=300) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in loops]
    steps = [[x.tensors([300, 20], 9), x.tensors([250, 1], 10), x.tensors([1, 1], 11)] for x in loops]
    apart = [[x.tensors([300, 20], 9), x.tensors([250, 1], 10), x.tensors([1, 1], 11)] for x in twins]
    torch.cuda.synchronize()
    for i in range(3):
        for x, s, t in zip(loops, streams, steps):
            with torch.cuda.stream(s):
                t[i]["q"].mul_(1.0)                                  # the inputs come from the call's own stream
                x.step(t[i], stream=s.cuda_stream)
    torch.cuda.synchronize()
    for x, t in zip(twins, apart):
        for i in range(3):
            x.step(t[i])
    torch.cuda.synchronize()
    for x, y, s, t in zip(loops, twins, steps, apart):
        assert all(torch.equal(a["out"], b["out"]) for a, b in zip(s, t))
        assert all(torch.equal(a, b) for a, b in zip(x.state(), y.state()))


@pytest.mark.parametrize("heads_first", [False, True])
def test_pools_of_more_than_four_gigabytes(heads_first):
    """The same sequences in a small pool and in pages beyond 2^32 bytes (and 2^31 elements) of a large one."""
    d, hkv, hq, page, n_small, n_large = 128, 4, 8, 64, 16, 70000
    far = n_large - n_small
    lens, new = [300, 129, 64], [40, 1, 64]
    small = pu.Case(lens, new, hq=hq, hkv=hkv, d=d, page=page, heads_first=heads_first, seed=7, junk=False, spare=n_small - 9)
    assert small.n_pages == n_small
    shape = (n_large,) + tuple(small.k.shape[1:])
    big = [torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    assert big[0].numel() * 2 > 1 << 32
    big[0][far:], big[1][far:] = small.k, small.v
    meta = [torch.zeros(n_large, hkv, page, dtype=dt, device=DEV) for dt in (torch.float32, torch.int32)]
    h = small.handle(rotary_dim=128)
    q, k, v = small.rows(hq), small.rows(hkv), small.rows(hkv)
    got = []
    for kp, vp, table, w, ids, first in ((small.k, small.v, small.table, small.weights, small.ids, 0),
                                         (big[0], big[1], torch.where(small.table < 0, -1, small.table + far), meta[0], meta[1], far)):
        pages = kvx.KvPages(kp, vp, table, heads_first=heads_first, weights=w, ids=ids)
        q_out, out, lens_out = torch.empty_like(q), torch.empty_like(q), torch.empty_like(small.d_lens)
        h.append(pages, small.batch(), k, v, q=q, q_out=q_out)
        h.attend(pages, small.batch(), q_out, out, weights_out=w)
        h.evict(pages, small.batch(), 100, 2, 8, weights_out=w, ids_out=ids, lens_out=lens_out)
        torch.cuda.synchronize()
        got.append([q_out, out, kp[first:].clone(), vp[first:].clone(), w[first:].clone(), ids[first:].clone(), lens_out])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][6].tolist() == [100, 100, 64]


def test_refusals_of_a_live_handle():
    case = pu.Case([40], [2], seed=1)
    h, q, k = case.handle(), case.rows(4), case.rows(2)
    pages, batch = case.pages(), case.batch()
    with pytest.raises(kvx.KvError) as e:
        h.attend(pages, kvx.KvPagedBatch(case.d_start, case.d_lens, n_tokens=2, max_new=2, max_len=41), q, q)
    assert e.value.code == -3 and "max_len" in str(e.value)
    with pytest.raises(kvx.KvError) as e:
        h.evict(pages, batch, 0, weights_out=case.weights, ids_out=case.ids, lens_out=case.d_lens)
    assert e.value.code == -1
    for bad in (q[:1], q[:, :2], q.float(), q.transpose(1, 2).contiguous().transpose(1, 2)[..., :63], q.cpu()):
        with pytest.raises(AssertionError):
            h.attend(pages, batch, bad, q)
    with pytest.raises(AssertionError):
        h.append(pages, batch, k, k, positions=torch.zeros(3, dtype=torch.int32, device=case.device))
    with pytest.raises(AssertionError):
        h.attend(pages, batch, q, torch.empty_like(q), weights_out=case.weights[:, :, ::2])
    other = pu.Case([40], [2], page=32, seed=1)
    with pytest.raises(AssertionError):
        h.attend(other.pages(), batch, q, q)
    h.attend(pages, batch, q, torch.empty_like(q))
    h.close()
