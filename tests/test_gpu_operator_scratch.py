"""What the operators for many requests keep on the device between calls, and for whom."""
import ctypes as C
import gc

import pytest
import torch

from tests.test_gpu_adapters_paths import PATHS, Call
from tests.test_gpu_paged import DEV, LONG, _setup

pytestmark = pytest.mark.gpu


def _allocated():
    gc.collect()
    torch.cuda.synchronize()
    return torch.cuda.memory_allocated()


@pytest.mark.parametrize("path", list(PATHS))
def test_project_adapters_keeps_nothing(path):
    c = Call(path)
    c.run()
    stream = torch.cuda.Stream()
    before = _allocated()
    with torch.cuda.stream(stream):
        y = c.run()
        stream.synchronize()
    assert _allocated() == before + -(-y.numel() * y.element_size() // 512) * 512
    del y
    assert _allocated() == before


def test_project_adapters_keeps_nothing_of_a_capture():
    c = Call("pair_512")
    want = c.run()
    torch.cuda.synchronize()
    before = _allocated()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        y = [c.run() for _ in range(2)]
    gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in y)
    del y, gr
    assert _allocated() == before


def test_paged_attention_gives_a_capture_s_scratch_back():
    from paper_2406_13170_b200 import paged_attention
    s = _setup(71, lens=LONG[0])
    want = paged_attention(*s)                         # this stream's own
    before = _allocated()
    for _ in range(3):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            y = [paged_attention(*s) for _ in range(2)]
        eager = paged_attention(*s)
        for _ in range(3):                             # the graph has its scratch all the same
            gr.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, want) for o in y) and torch.equal(eager, want)
        del y, gr, eager
        assert _allocated() == before


@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_calls_outside_a_capture_that_goes_on(mode):
    """A capture on one stream, with calls outside it on another between its own."""
    from paper_2406_13170_b200 import paged_attention
    s = _setup(72, lens=LONG[1])
    want = paged_attention(*s)
    side, inside = torch.cuda.Stream(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = [torch.zeros_like(want) for _ in range(6)]
    with torch.cuda.stream(side):
        paged_attention(*s, out=eager[0])
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    y = []
    with torch.cuda.graph(gr, stream=inside, capture_error_mode=mode):
        for i in range(3):
            y.append(paged_attention(*s))
            with torch.cuda.stream(side):
                paged_attention(*s, out=eager[i])
    for i in range(3):
        gr.replay()
        with torch.cuda.stream(side):
            paged_attention(*s, out=eager[3 + i])
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in y + eager[: 4 + i])


def test_a_stream_with_another_s_handle_gets_scratch_of_its_own():
    """A stream is destroyed and the next one has its handle: work of the first may still run, so nothing of its scratch is taken over."""
    from paper_2406_13170_b200 import paged_attention
    s = _setup(73, lens=LONG[0])
    want = paged_attention(*s)
    out = torch.zeros_like(want)
    rt = torch.cuda.cudart()
    seen, came_back = set(), 0
    for _ in range(4):
        handles = []
        for _ in range(20):
            h = C.c_void_p()
            assert int(rt.cudaStreamCreate(C.addressof(h))) == 0
            handles.append(h.value)
        made = []
        for h in handles:
            stream = torch.cuda.ExternalStream(h)
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                counts = [torch.cuda.memory_stats()["allocation.all.allocated"]]
                for _ in range(2):
                    paged_attention(*s, out=out)
                    counts.append(torch.cuda.memory_stats()["allocation.all.allocated"])
            stream.synchronize()
            assert torch.equal(out, want)
            made.append([b - a for a, b in zip(counts, counts[1:])])
        came_back += len(seen & set(handles))
        seen |= set(handles)
        for h in handles:
            assert int(rt.cudaStreamDestroy(h)) == 0
        assert made == [[1, 0]] * len(handles)         # a new stream's first call makes scratch, its next one finds it
    if not came_back:
        pytest.skip("no handle came back")
