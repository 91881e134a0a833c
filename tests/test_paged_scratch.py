"""The binding's scratch for the paged cache's calls, without a GPU: the library's calls are stand-ins."""
import threading
import time

import pytest
import torch

import paper_2311_04951_amd as sv


class Library:
    """Calls that note what scratch they were given, and take a while."""

    def __init__(self, need=1 << 21):
        self.under_way, self.clashes, self.calls, self.need = {}, [], [], need

    def ss_paged_attention_workspace_bytes(self, *args):
        return self.need

    ss_paged_evict_workspace_bytes = ss_paged_attention_workspace_bytes

    def note(self, ws, size):
        if self.under_way.get(ws):
            self.clashes.append(ws)
        self.under_way[ws] = True
        self.calls.append((ws, size))
        time.sleep(0.002)
        self.under_way[ws] = False
        return 0

    def ss_paged_attention(self, kv, layer, q, ldq, hq, heads, M, pending, scale, out, ldo, ho, w, max_len, ws, size, stream):
        return self.note(ws, size)

    def ss_paged_evict(self, kv, budget, first, recent, w, p, l, max_len, ws, size, stream):
        return self.note(ws, size)


def cache():
    kv = object.__new__(sv.PagedKV)
    kv.k = torch.zeros(1, 4, 2, 16, 64)
    kv.batch, kv.head_dim, kv.n_kv_heads, kv._p = 1, 64, 2, 0
    kv._dtype, kv._device, kv._index, kv._ws = torch.float32, torch.device("cpu"), kv.k.get_device(), {}
    kv.weight = kv.position = kv.length = None
    return kv


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    monkeypatch.setattr(sv, "lib", lambda: fake)
    monkeypatch.setattr(sv, "_stream", lambda stream: 0 if stream is None else stream)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    monkeypatch.setattr(sv, "_captures", lambda handle: False)
    # scratch that is there already: one for each of two streams
    monkeypatch.setattr(sv, "_paged_workspaces", {(torch.device("cpu"), h): torch.empty(1 << 22, dtype=torch.uint8) for h in (0, 1)})
    return fake


def in_threads(*calls):
    threads = [threading.Thread(target=lambda f=f: [f() for _ in range(10)]) for f in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()


def test_calls_of_two_threads_on_one_stream_do_not_share_scratch_at_a_time(library):
    """A call is several launches that pass on what is in the scratch: those of another thread must not come between."""
    one, two, three, q = cache(), cache(), cache(), torch.zeros(1, 1, 2, 64)
    in_threads(lambda: sv.ss_paged_attention(one, 0, q), lambda: sv.ss_paged_attention(two, 0, q), lambda: sv.ss_paged_evict(three, 8))
    assert len(library.calls) == 30 and not library.clashes


def test_calls_on_two_streams_do_not_wait_for_each_other(library):
    one, two, q = cache(), cache(), torch.zeros(1, 1, 2, 64)
    both = threading.Barrier(2, timeout=20)
    library.note = lambda ws, size: 0 * both.wait()           # returns when both calls are under way
    in_threads(lambda: sv.ss_paged_attention(one, 0, q, stream=0), lambda: sv.ss_paged_attention(two, 0, q, stream=1))
    assert not both.broken


def test_a_call_that_fails_leaves_the_scratch_to_others(library):
    kv, q = cache(), torch.zeros(1, 1, 2, 64)
    library.ss_last_error = lambda: b"no"
    library.note = lambda ws, size: -1
    for _ in range(2):
        with pytest.raises(sv.SpecVerifyError):
            sv.ss_paged_attention(kv, 0, q)


def test_what_a_cache_remembers_of_workspaces_is_bounded(library):
    """A decoding loop passes another bound with every token."""
    kv, q = cache(), torch.zeros(1, 1, 2, 64)
    library.note = lambda ws, size: 0
    for n in range(1, 1000):
        sv.ss_paged_attention(kv, 0, q, max_len=n)
        sv.ss_paged_evict(kv, 8, max_len=n)
    assert len(kv._ws) <= 256
    library.need = 1 << 20
    sv.ss_paged_attention(kv, 0, q, max_len=999)             # (remembered)
    assert max(kv._ws.values()) == 1 << 21


def test_arguments_that_do_not_fit_are_refused_as_such(library):
    kv, w = cache(), torch.zeros(1, 4, 2, 16)
    with pytest.raises(ValueError, match="weights"):
        sv.ss_paged_evict(kv, 8, weight_out=w)               # a cache without weights
    with pytest.raises(ValueError, match="positions"):
        sv.ss_paged_evict(kv, 8, position_out=w.int())
    for shape in ((64,), (2, 64), (1, 2, 64)):
        with pytest.raises(ValueError, match="queries"):
            sv.ss_paged_attention(kv, 0, torch.zeros(shape))
