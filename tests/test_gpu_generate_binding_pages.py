"""Both ways of the binding, and each of several streams, write the cache's pages themselves: from pages that hold nothing, the same bytes."""
import pytest
import torch

from paper_2105_00053_amd import binding, generate
from test_gpu_generate_binding import Step, same

pytestmark = pytest.mark.gpu


def cleared(step):
    for pages in step.pages.values():
        for t in pages:
            t.zero_()
    return step.run()


def pages_of(step):
    return [t for pages in step.pages.values() for t in pages]


@pytest.mark.parametrize("long", [40, 3000])
def test_both_ways_write_the_pages(monkeypatch, long):
    generate._load()
    if binding._native is None:
        pytest.skip("the extension module is not built")
    step = Step(long=long)
    a, pages = cleared(step), [t.clone() for t in pages_of(step)]
    assert all(t.any() for t in pages)
    monkeypatch.setattr(binding, "_native", None)
    same(a, cleared(step))
    same(pages, pages_of(step))


def test_two_streams_write_their_pages():
    steps = [Step(3, long=2000), Step(4, long=1500)]
    want = [cleared(s) for s in steps]
    pages = [[t.clone() for t in pages_of(s)] for s in steps]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in steps], [[], []]
    for _ in range(3):
        for s, stream, g in zip(steps, streams, got):
            with torch.cuda.stream(stream):
                g.append(cleared(s))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for one in g:
            same(w, one)
    for s, p in zip(steps, pages):
        same(p, pages_of(s))


def test_a_replayed_graph_writes_the_pages():
    step = Step(5, long=700)
    want = cleared(step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step.run()
    for _ in range(3):
        for t in pages_of(step):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        same(want, [None if t is None else t.clone() for t in out])
