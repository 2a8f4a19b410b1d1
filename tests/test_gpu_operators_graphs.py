"""A list's calls captured into CUDA graphs: on a stream that the list has not been used on, and replayed beside its other calls with no order
between them.  (Every call on the same tensors gives the same bits, so equality is what is asked.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2008_11343_b200 import operators as O
from test_gpu_operators import gen

# lists whose norm is formed by the tiles' last CTA, by one CTA, and by the groups' CTAs
LISTS = {"short": [70_000, 33, 9000], "middling": [2_000_003] * 4 + [9000] * 80, "long": [9000] * 40 + [8200 * 8192]}


def made(name, scale=1.0):
    return [torch.empty(n, device="cuda").normal_(0.0, scale, generator=gen(41 + k % 7)) for k, n in enumerate(LISTS[name])]


@pytest.mark.parametrize("name", LISTS)
def test_capture_on_a_stream_of_its_own(name):
    ts = made(name)
    tl = O.TensorList(ts)
    flat, flat2 = torch.empty(tl.numel, device="cuda"), torch.empty(tl.numel, device="cuda")
    norm, norms = tl.grad_norm(ts)                                           # the list's last call is on this stream
    tl.clip_grads(ts, 1.0, out=flat)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                                            # on another
        norm2, norms2 = tl.grad_norm(ts)
        norm3 = tl.clip_grads(ts, 1.0, out=flat2)
    for _ in range(3):
        for t in (norm2, norms2, norm3, flat2):
            t.fill_(-1.0)
        graph.replay()
        assert torch.equal(norm2, norm) and torch.equal(norms2, norms) and torch.equal(norm3, norm) and torch.equal(flat2, flat)
    assert torch.equal(tl.grad_norm(ts)[0], norm)                            # and the list goes on
    for t in ts:
        t.mul_(4.0)
    graph.replay()
    assert torch.equal(norm2, norm * 4.0) and torch.equal(norm3, norm * 4.0)


@pytest.mark.parametrize("name", LISTS)
def test_replays_and_calls_with_no_order_between_them(name):
    """Two graphs and plain calls of one list, on three streams, on tensors whose norms differ."""
    ts, others, third = made(name), made(name, 8.0), made(name, 0.25)
    tl = O.TensorList(ts)
    wants = [tl.grad_norm(g)[0] for g in (ts, others, third)]
    flats = [torch.empty(tl.numel, device="cuda") for _ in range(3)]
    kept = []
    for g, f in zip((ts, others, third), flats):
        tl.clip_grads(g, 1.0, out=f)
        kept.append(f.clone())
    graphs, norms = [], []
    for g, f in ((ts, flats[0]), (others, flats[1])):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            norms.append(tl.clip_grads(g, 1.0, out=f))
    streams = [torch.cuda.Stream() for _ in range(3)]
    plain = []
    torch.cuda.synchronize()
    for _ in range(20):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        with torch.cuda.stream(streams[2]):
            plain.append(tl.clip_grads(third, 1.0, out=flats[2]))
    torch.cuda.synchronize()
    assert torch.equal(norms[0], wants[0]) and torch.equal(norms[1], wants[1]) and all(torch.equal(n, wants[2]) for n in plain)
    assert all(torch.equal(a, b) for a, b in zip(flats, kept))


def test_a_list_is_built_outside():
    ts = made("short")
    tl = O.TensorList(ts)
    want = tl.grad_norm(ts)[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="before a graph's capture"):
            O.TensorList(ts)
        norm = tl.grad_norm(ts)[0]                                           # the capture is still sound
    graph.replay()
    assert torch.equal(norm, want)


def test_more_captured_calls_than_a_list_has_tickets():
    """1100 calls in graphs of 100, replayed on two streams at once: each call clips its own tensors to its own norm."""
    sets = [[torch.full((n,), float(k + 1), device="cuda") for n in (900, 5)] for k in range(2)]
    tl = O.TensorList(sets[0])
    wants = [tl.grad_norm(ts)[0] for ts in sets]
    graphs, norms = [], []
    for k in range(11):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            norms.append([tl.grad_norm(sets[(k + j) % 2])[0] for j in range(100)])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for k, graph in enumerate(graphs):
            with torch.cuda.stream(streams[k % 2]):
                graph.replay()
    torch.cuda.synchronize()
    for k, got in enumerate(norms):
        assert all(torch.equal(n, wants[(k + j) % 2]) for j, n in enumerate(got))
    assert torch.equal(tl.grad_norm(sets[1])[0], wants[1])
