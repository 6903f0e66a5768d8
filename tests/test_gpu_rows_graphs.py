"""Dropout in a captured graph: seed and offset are those of the capture, as the header says."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2205_04702_amd import tokens as tk  # noqa: E402
from tests import rows_reference as ref  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_replays_draw_the_captured_mask_and_a_graph_per_offset_its_own():
    n, dim, p, seed = 30, 72, 0.4, 9
    x, tok = torch.ones((n, dim), device="cuda"), torch.arange(n, device="cuda")
    tk.dropout(x, p, seed, 0)
    graphs = []
    for offset in (5, 6):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = tk.dropout(x, p, seed, offset), tk.lookup(tok, x, 1.0, p, seed, offset), \
                tk.lookup_grad(tok, x, n, 1.0, p, seed, offset)
        graphs.append((offset, graph, outs))
    for round_ in range(3):
        for offset, graph, outs in graphs:
            want = ref.keep_mask(n, dim, p, seed, offset)
            x.fill_(1.0 + round_)
            graph.replay()
            torch.cuda.synchronize()
            for out in outs:
                assert torch.equal((out != 0).cpu(), want)
            assert torch.equal(outs[0], tk.dropout(x, p, seed, offset))
        assert not torch.equal(graphs[0][2][0], graphs[1][2][0])
