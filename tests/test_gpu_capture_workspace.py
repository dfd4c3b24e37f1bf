"""Workspaces of the quantised and the prefix attention under capture: each graph has its own, whatever stream it was captured on."""
import numpy as np
import pytest
import torch

import quant_util as qu
from gpu_util import rapid
from test_gpu_prefix import Batch, i32

pytestmark = pytest.mark.gpu


class Spy:
    """The library, with a note of the workspaces that the attention calls were given."""

    def __init__(self, lib):
        self.lib, self.seen = lib, []

    def __getattr__(self, name):
        f = getattr(self.lib, name)
        if name not in ("rapid_verify_attn_quant", "rapid_verify_attn_prefix"):
            return f

        def call(*args):
            rc = f(*args)
            if rc == 0:
                self.seen.append(args[-3:-1])
            return rc
        return call


def calls(rng, r):
    """Two of each kind that use partials, of different sizes."""
    got = []
    for lens, Q in (([20000], 9), ([3000, 900], 4)):
        cache = qu.QuantCache(rng, lens, 2, 128)
        args = (qu.bf16(rng, (len(lens), Q, 8, 128)).cuda(), *cache.dev()[:4], i32(lens))
        got.append(lambda args=args, **kw: r.rapid_verify_attn_quant(*args, **kw))
    for P, B in ((5000, 3), (900, 2)):
        args, kw = Batch(rng, P, [40, 300, 7][:B], 2, 128).args("token")
        q = qu.bf16(rng, (B, 4, 8, 128)).cuda()
        got.append(lambda q=q, args=args, more=kw, **kw: r.rapid_verify_attn_prefix(q, *args, **more, **kw))
    return got


def capture(call, out):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out)
    return graph


@pytest.mark.parametrize("warm", [False, True])
def test_no_two_graphs_and_no_eager_call_share_memory(warm):
    from paper_2502_20330_amd import binding
    r = binding.Rapid(0)
    some = calls(np.random.default_rng(1), r)
    want = [call() for call in some]
    side = torch.cuda.Stream()
    if warm:
        with torch.cuda.stream(side):
            for call in some:
                call()
    torch.cuda.synchronize()
    r.lib = Spy(r.lib)
    outs = [torch.empty_like(w) for w in want]
    graphs = [capture(call, out) for call, out in zip(some, outs)]
    stream = torch.cuda.graph.default_capture_stream
    with torch.cuda.stream(stream):                       # an eager call on the stream that they were captured on
        some[0]()
    some[1]()
    torch.cuda.synchronize()
    seen = sorted(r.lib.seen)
    assert len(seen) == 6
    assert all(a + n <= b for (a, n), (b, _) in zip(seen, seen[1:])), "workspaces overlap"
    for graph, out, w in zip(graphs, outs, want):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)


def test_graphs_replayed_on_two_streams_at_once():
    """Captured the usual way, on torch's one capture stream; eager calls on that stream beside them."""
    r = rapid()
    some = calls(np.random.default_rng(2), r)
    want = [call() for call in some]
    outs = [torch.empty_like(w) for w in want]
    graphs = [capture(call, out) for call, out in zip(some, outs)]
    streams = [torch.cuda.Stream() for _ in graphs]
    own = torch.cuda.graph.default_capture_stream
    torch.cuda.synchronize()
    for _ in range(3):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
            with torch.cuda.stream(own):
                eager = some[0]()
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0])
        assert all(torch.equal(out, w) for out, w in zip(outs, want))


def test_layers_of_one_graph_take_turns():
    """Calls one after another in a graph, of different sizes, replayed several times with eager calls between."""
    r = rapid()
    some = calls(np.random.default_rng(3), r)
    want = [call() for call in some]
    outs = [torch.empty_like(w) for w in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call, out in zip(some, outs):
            call(out=out)
    for turn in range(4):
        for out in outs:
            out.zero_()
        graph.replay()
        eager = some[turn]()
        torch.cuda.synchronize()
        assert torch.equal(eager, want[turn]) and all(torch.equal(out, w) for out, w in zip(outs, want))
