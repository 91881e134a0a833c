"""Paged calls of several threads, and of streams that are captured while another one is current."""
import threading

import pytest
import torch

import paper_2311_04951_amd as sv
from paged_util import Cache

pytestmark = pytest.mark.gpu


def case(seed, n):
    c = Cache(seed, "bf16", 2, 2, 64, 32, [n, 300], room=1)
    q = torch.randn((2, 1, 8, 64), generator=c.generator).to(c.dtype).cuda()
    return c.device(), q


def test_two_threads_on_one_stream_get_what_one_gets():
    cases = [case(1, 6000), case(2, 5000)]
    want = [(sv.ss_paged_attention(kv, 0, q, weight_out=(w := torch.zeros_like(kv.weight))), w) for kv, q in cases]
    got, torch_stream = [None, None], torch.cuda.current_stream()
    torch.cuda.synchronize()

    def work(i):
        kv, q = cases[i]
        with torch.cuda.stream(torch_stream):
            got[i] = [(sv.ss_paged_attention(kv, 0, q, weight_out=(w := torch.zeros_like(kv.weight))), w) for _ in range(40)]
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (out, w), all_ in zip(want, got):
        assert all(torch.equal(a, out) and torch.equal(b, w) for a, b in all_)


def test_a_captured_stream_that_is_not_the_current_one():
    """The call's stream counts: its scratch would be the graph's to keep."""
    kv, q = case(3, 900)
    out, want = torch.empty_like(q), sv.ss_paged_attention(kv, 0, q)
    ws = torch.empty(sv.ss_paged_attention_workspace_bytes(kv, 8, 1), dtype=torch.uint8, device="cuda")
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        with torch.cuda.stream(other):
            with pytest.raises(ValueError, match="workspace"):
                sv.ss_paged_attention(kv, 0, q, out=out, stream=side)
            sv.ss_paged_attention(kv, 0, q, out=out, stream=side, ws=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert (kv.k.device, side.cuda_stream) not in sv._paged_workspaces
