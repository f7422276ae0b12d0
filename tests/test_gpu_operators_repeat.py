"""Tree and weighted attention, kv_select and kv_compact on the GPU: what a call leaves behind for the calls and captured graphs after it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2603_13358_amd as ppd  # noqa: E402
from test_gpu_operators import Batch, dev, random_mask  # noqa: E402


@pytest.mark.parametrize("kind", ["tree", "weighted", "select"])
def test_first_call_under_capture_is_refused_and_the_capture_stays_valid(kind):
    b = Batch([300, 20], [3, 40], 8, 2, 64, seed=50)
    mask = dev(random_mask(b, 1, seed=51).view(np.int64))
    out = torch.zeros((43, 8, 64), dtype=torch.bfloat16, device="cuda")
    w0 = torch.rand((2, 2, 20000), device="cuda")
    w, keep = w0.clone(), torch.full((2, 2, 50), -1, dtype=torch.int32, device="cuda")

    def call(stream=None):
        if kind == "tree":
            b.ctx.tree_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, mask, b.scale, out, stream=stream)
        elif kind == "weighted":
            b.ctx.weighted_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, out, w, stream=stream)
        else:
            b.ctx.kv_select(w, np.array([20000, 70], np.int32), 50, 2, 3, keep, stream=stream)

    refused = torch.cuda.CUDAGraph()
    mark = torch.zeros(1, device="cuda")
    with torch.cuda.graph(refused):
        with pytest.raises(ppd.PPDError) as e:
            call(torch.cuda.current_stream().cuda_stream)
        assert e.value.status == -3 and "capture" in str(e.value)
        mark.add_(1)
    refused.replay()
    torch.cuda.synchronize()
    assert mark.item() == 1 and not out.any() and (keep == -1).all() and torch.equal(w, w0)
    call()
    ref = (out.clone(), w.clone(), keep.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.zero_()
        w.copy_(w0)
        keep.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((out, w, keep), ref))
    assert b.flags() == 0


def test_graphs_of_one_kind_outlive_calls_of_the_other():
    """Tree and weighted attention of the same lengths, together in one graph and eagerly between its replays."""
    b = Batch([900, 30, 4000], [12, 5, 2], 32, 8, 128, seed=52)
    mask = dev(random_mask(b, 1, seed=53).view(np.int64))
    w0 = torch.rand((3, 8, 4100), device="cuda")

    def tree(out, stream=None):
        b.ctx.tree_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, mask, b.scale, out, stream=stream)

    t_ref, w_ref = torch.empty((19, 32, 128), dtype=torch.bfloat16, device="cuda"), w0.clone()
    o_ref = b.weighted(w_ref)
    tree(t_ref)
    t_out, o_out, w = torch.zeros_like(t_ref), torch.zeros_like(o_ref), w0.clone()
    graph, alone = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        tree(t_out, s)
        b.weighted(w, out=o_out, stream=s)
    with torch.cuda.graph(alone):
        b.weighted(w, out=o_out, stream=torch.cuda.current_stream().cuda_stream)
    for replayed, between in [(graph, None), (graph, "tree"), (alone, "tree"), (alone, "weighted"), (graph, "weighted"), (alone, None)]:
        if between == "tree":
            tree(t_out)
            assert torch.equal(t_out, t_ref)
        elif between == "weighted":
            w.copy_(w0)
            b.weighted(w, out=o_out)
            assert torch.equal(w, w_ref) and torch.equal(o_out, o_ref)
        w.copy_(w0)
        for x in (o_out, t_out):
            x.zero_()
        torch.cuda.synchronize()
        replayed.replay()
        torch.cuda.synchronize()
        assert torch.equal(o_out, o_ref) and torch.equal(w, w_ref)
        assert replayed is alone or torch.equal(t_out, t_ref)
    assert b.flags() == 0
