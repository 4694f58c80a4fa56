"""The paged cache's binding without a GPU: a stand-in for the library that keeps what it is called with."""
import ctypes as C
import threading

import pytest
import torch

import paper_2601_01204_amd as kvx
from paper_2601_01204_amd import paged


class Library:
    """kv_paged_* as far as the binding calls them."""

    def __init__(self):
        self.calls, self.inside = [], lambda q: None

    def kv_paged_init(self, cfg, out):
        C.cast(out, C.POINTER(C.c_void_p))[0] = 1
        return 0

    def kv_paged_append(self, h, pages, batch, positions, q, q_out, k, v, stream):
        self.calls.append("append")
        return 0

    def kv_paged_attend(self, h, pages, batch, q, out, lse, causal, window, weights_out, stream):
        self.calls.append("attend")
        before = q._obj.data
        self.inside(q._obj)
        self.calls.append((before, q._obj.data, out._obj.data))
        return 0

    def kv_paged_evict(self, h, *args):
        self.calls.append("evict")
        return 0

    def kv_paged_destroy(self, h):
        pass

    def kv_paged_last_error(self, h):
        return b"stand-in"


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(paged, "_library", lambda: lib)
    return lib


def make(monkeypatch, device):
    """A handle made while `device` was current, with a pool, a batch and rows in host memory."""
    monkeypatch.setattr(paged, "_current_device", lambda: device)
    h = kvx.KvPaged(n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, max_seqs=2, max_tokens=3, max_len=32)
    pages = kvx.KvPages(torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32),
                        weights=torch.zeros(4, 2, 16), ids=torch.zeros(4, 2, 16, dtype=torch.int32))
    batch = kvx.KvPagedBatch(torch.tensor([0, 2, 3], dtype=torch.int32), torch.tensor([9, 9], dtype=torch.int32), n_tokens=3, max_new=2, max_len=32)
    return h, pages, batch, torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)


def test_tensors_that_are_not_on_the_handles_device_are_refused(library, monkeypatch):
    """Everything in host memory, which agrees with itself: no call reaches the library."""
    h, pages, batch, q, k = make(monkeypatch, torch.device("cuda", 0))
    for call in (lambda: h.append(pages, batch, k, k), lambda: h.attend(pages, batch, q, torch.empty_like(q)),
                 lambda: h.evict(pages, batch, 8, weights_out=pages.weights, ids_out=pages.ids, lens_out=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(AssertionError, match="cuda:0"):
            call()
    assert library.calls == []


def test_two_threads_on_one_handle_do_not_swap_their_rows(library, monkeypatch):
    """While one thread is in the library, which runs without the interpreter's lock, another one makes its call."""
    h, pages, batch, _, _ = make(monkeypatch, torch.device("cpu"))
    qs, outs = ([torch.zeros(3, 4, 64, dtype=torch.bfloat16) for _ in range(2)] for _ in range(2))
    entered, second_done = threading.Event(), threading.Event()

    def inside(q):
        if not entered.is_set():
            entered.set()
            second_done.wait(1.0)                            # the other call, if nothing holds it back

    library.inside = inside
    first = threading.Thread(target=h.attend, args=(pages, batch, qs[0], outs[0]))
    first.start()
    assert entered.wait(10.0)

    def other():
        h.attend(pages, batch, qs[1], outs[1])
        second_done.set()

    second = threading.Thread(target=other)
    second.start()
    first.join(10.0)
    second.join(10.0)
    seen = [c for c in library.calls if c != "attend"]
    assert sorted(seen) == sorted((q.data_ptr(), q.data_ptr(), o.data_ptr()) for q, o in zip(qs, outs))
