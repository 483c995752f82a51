"""Calls that a CUDA graph holds, the first ones of their handle among them: what they report, and what later calls may take for
granted."""
import pytest
import torch

import paper_2510_11236_b200 as xq
from tests.test_shared_cache import DEV, _config, _filled, _queries, _tokens


def _reports(cache):
    try:
        cache.check_device()
    except xq.XQError as e:
        assert e.code == xq.XQ_ERR_DEVICE
        return True
    return False


def _gather_then_decode(index):
    """A handle whose first calls are captured: a gather, then a decode of both layers and a cross attention."""
    cfg = _config(batch=4, max_seq=300)
    src, dst = _filled(cfg, *_tokens(cfg, 1, 200)), xq.Cache(cfg, DEV)
    dst.workspace.fill_(0xff)
    q = _queries(cfg, 2, 1).to(DEV)
    outs = [torch.empty_like(q[0]), torch.empty_like(q[0]), torch.empty_like(q)]
    space = torch.empty(xq.xq_cross_workspace_bytes(dst.handle, 1), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dst.gather_sequences(src, index)
        for layer in (0, 1):
            dst.decode_attention(layer, q[0], out=outs[layer])
        dst.cross_attention(1, q, out=outs[2], workspace=space)
    want = [src.decode_attention(0, q[0]), src.decode_attention(1, q[0]), src.cross_attention(1, q)]
    return src, dst, q, outs, want, graph


@pytest.mark.gpu
def test_a_later_call_of_the_graph_does_not_hide_a_report():
    index = torch.tensor([0, 1, -1, 3], dtype=torch.int32, device=DEV)
    src, dst, q, outs, want, graph = _gather_then_decode(index)
    assert not _reports(dst)  # the graph has not run
    graph.replay()
    assert _reports(dst)
    # nor does the next run of the graph, until the handle is reset
    index.copy_(torch.arange(4, dtype=torch.int32))
    graph.replay()
    assert _reports(dst)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    xq.xq_reset(dst.handle)
    assert not _reports(dst)
    dst.gather_sequences(src, index)
    assert not _reports(dst) and torch.equal(dst.decode_attention(1, q[0]), want[1])


@pytest.mark.gpu
def test_an_eager_call_does_not_hide_what_a_graph_reported():
    index = torch.tensor([0, 9, 2, 3], dtype=torch.int32, device=DEV)
    src, dst, q, outs, want, graph = _gather_then_decode(index)
    graph.replay()
    dst.cross_attention(0, q)  # the handle's first call outside of a graph
    assert _reports(dst)


@pytest.mark.gpu
def test_graph_of_first_calls_gives_the_results_of_the_others():
    index = torch.arange(4, dtype=torch.int32, device=DEV)
    src, dst, q, outs, want, graph = _gather_then_decode(index)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert not _reports(dst)


def _nodes(calls):
    runtime = pytest.importorskip("cuda.bindings.runtime")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        calls()
    err, _, n = runtime.cudaGraphGetNodes(runtime.cudaGraph_t(graph.raw_cuda_graph()), 0)
    assert int(err) == 0
    return n


@pytest.mark.gpu
def test_a_graph_clears_the_counters_once():
    # what clears them stands between launches that overlap: at most two nodes before the first call, none before the others
    cfg = _config(batch=2, max_seq=600)
    q = _queries(cfg, 2, 3).to(DEV)
    out = torch.empty_like(q)

    def calls(cache):
        for _ in range(3):
            for layer in (0, 1):
                cache.decode_attention(layer, q[0], out=out[0])
                cache.attention_chunk(layer, q, out=out)
    fresh, used = (_filled(cfg, *_tokens(cfg, 1, 500)) for _ in range(2))
    calls(used)
    torch.cuda.synchronize()
    n = _nodes(lambda: calls(used))
    assert n >= 12 and _nodes(lambda: calls(fresh)) <= n + 2


@pytest.mark.gpu
def test_code_differences_after_a_capture_that_never_runs():
    # the counters of xq_delta_histogram start at zero, whatever the first append that counts was captured into
    cfg = _config(batch=2, max_seq=300, delta_stats=1)
    K, V = _tokens(cfg, 1, 200)
    want, fresh = xq.Cache(cfg, DEV), xq.Cache(cfg, DEV)
    fresh.workspace.fill_(0xff)
    torch.cuda.synchronize()
    k, v = ([x.to(DEV) for x in y] for y in (K, V))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in (0, 1):
            fresh.append_kv(layer, k[layer], v[layer])
    stream = torch.cuda.current_stream().cuda_stream
    assert xq.xq_delta_histogram(fresh.handle, 1, 0, stream) == (0, [0, 0, 0, 0])
    xq.xq_reset(fresh.handle)
    for cache in (want, fresh):
        for layer in (0, 1):
            cache.append_kv(layer, k[layer], v[layer])
    for kind in (0, 1):
        rc, counts = xq.xq_delta_histogram(want.handle, 1, kind, stream)
        assert rc == 0 and sum(counts) == 2 * 2 * 192 * 128
        assert xq.xq_delta_histogram(fresh.handle, 1, kind, stream) == (0, counts)


@pytest.mark.gpu
def test_code_differences_that_a_graph_counts():
    cfg = _config(batch=2, max_seq=300, delta_stats=1)
    K, V = _tokens(cfg, 1, 200)
    k, v = ([x.to(DEV) for x in y] for y in (K, V))
    want = _filled(cfg, K, V)
    fresh = xq.Cache(cfg, DEV)
    fresh.workspace.fill_(0xff)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in (0, 1):
            fresh.append_kv(layer, k[layer], v[layer])
    graph.replay()
    stream = torch.cuda.current_stream().cuda_stream
    once = xq.xq_delta_histogram(want.handle, 1, 0, stream)
    assert xq.xq_delta_histogram(fresh.handle, 1, 0, stream) == once
    graph.replay()  # counts once more
    assert xq.xq_delta_histogram(fresh.handle, 1, 0, stream) == (0, [2 * n for n in once[1]])


@pytest.mark.gpu
@pytest.mark.parametrize("writer", ["gather", "append"])
def test_a_captured_decode_says_nothing_about_calls_outside(writer):
    # a decode fetches packed data early when it has waited for the launch that wrote them before; one that was only captured
    # has not.  The writer is held back by other work, and the decode launched right behind it.
    S = 1500
    cfg = _config(batch=4, max_seq=4000)
    src = _filled(cfg, *_tokens(cfg, 1, S))
    other = _filled(cfg, *_tokens(cfg, 2, S))
    more = [[x.to(DEV) for x in y] for y in _tokens(cfg, 3, S)]
    q = _queries(cfg, 4, 1)[0].to(DEV)
    index = torch.tensor([3, 1, 0, 2], dtype=torch.int32, device=DEV)
    dst, want = xq.Cache(cfg, DEV), xq.Cache(cfg, DEV)
    out, side, graphs = torch.empty_like(q), torch.cuda.Stream(), []
    for k in range(6):
        for cache in (want, dst):
            xq.xq_reset(cache.handle)
            cache.gather_sequences(other, index)  # what an early fetch would find
            cache.decode_attention(0, q, out=out), cache.decode_attention(1, q, out=out)
        layer = k % 2
        for cache in (want, dst):
            torch.cuda.synchronize()
            if cache is dst:
                torch.cuda._sleep(20_000_000)
            if writer == "gather":
                cache.gather_sequences(src, index)
            else:
                for l in (0, 1):
                    cache.append_kv(l, more[0][l], more[1][l])
            if cache is dst:
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.stream(side):
                    graphs[-1].capture_begin()
                    cache.decode_attention(layer, q, out=out)
                    graphs[-1].capture_end()
            result = cache.decode_attention(layer, q)
            if cache is want:
                expected = result
        assert torch.equal(result, expected)
    dst.check_device()


@pytest.mark.gpu
@pytest.mark.parametrize("each,T", [(1, 1), (2, 1), (12, 1), (3, 30)])  # decode, rows and chunk kernels
def test_caches_that_use_one_prefix_at_once(each, T):
    # two handles on two streams, eager and in two graphs: a prefix is only read, each handle has its own scratch and workspace
    P, Sp = 3, 900
    prefix = _filled(_config(batch=P, max_seq=Sp), *_tokens(_config(batch=P, max_seq=Sp), 1, Sp))
    cfg = _config(batch=P * each, max_seq=400)
    caches = [_filled(cfg, *_tokens(cfg, 2 + k, 250)) for k in range(2)]
    qs = [_queries(cfg, 5 + k, T).to(DEV) for k in range(2)]
    spaces = [torch.empty(xq.xq_prefix_workspace_bytes(c.handle, prefix.handle, T), dtype=torch.uint8, device=DEV) for c in caches]
    want = [[c.prefix_attention(prefix, layer, q, f32=True) for layer in (0, 1)] for c, q in zip(caches, qs)]
    outs = [[torch.empty_like(x) for x in w] for w in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]

    def calls(k):
        for layer in (0, 1):
            caches[k].prefix_attention(prefix, layer, qs[k], out=outs[k][layer], f32=True, workspace=spaces[k])
    graphs = []
    for k in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            calls(k)
    for run in (calls, lambda k: graphs[k].replay()):
        for x in outs[0] + outs[1]:
            x.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for k in (0, 1):
                with torch.cuda.stream(streams[k]):
                    run(k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for k in (0, 1) for a, b in zip(outs[k], want[k]))
    for c in caches:
        c.check_device()
