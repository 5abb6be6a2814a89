"""Lists of tensors, laid out for later calls (-m gpu)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_lists_are_not_laid_out_while_a_graph_is_recorded():
    """What a recorded copy reads of the host's memory is something else when the graph is replayed; a list from before is as good within a graph."""
    import paper_1806_11248_amd as g
    side = torch.cuda.Stream()
    ctx = g.Context(0, stream=side)
    try:
        t = torch.randn(70, 100, generator=torch.Generator().manual_seed(1)).cuda()
        out, clipped = torch.zeros_like(t), torch.zeros_like(t)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            matrices, gradients = ctx.matrix_list([t], [out]), ctx.gradient_list([t], [clipped])
            ctx.orthogonalise(matrices), ctx.clip_gradients(gradients, 1.0)
            side.synchronize()
            want = out.clone(), clipped.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for call in (ctx.matrix_list, ctx.gradient_list):
                    with pytest.raises(g.GbtError) as e:
                        call([t], [out])
                    assert e.value.code == g.binding.EUNSUPPORTED
                ctx.orthogonalise(matrices), ctx.clip_gradients(gradients, 1.0)
            for _ in range(3):
                out.zero_(), clipped.zero_()
                graph.replay()
                side.synchronize()
                assert torch.equal(out, want[0]) and torch.equal(clipped, want[1])
                ctx.matrix_list([t], [out])                                           # and afterwards again
    finally:
        ctx.close()
