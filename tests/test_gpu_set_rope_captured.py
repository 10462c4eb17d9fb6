"""psv_set_rope recorded into a graph: nothing changes before the graph runs, and frequencies and magnitude change together when it does."""
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from paper_2501_08192_amd import synth
from paper_2501_08192_amd.harness import Session

pytestmark = pytest.mark.gpu


def recorded(s, rope):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s.main):
        psv.psv_set_rope(s.ctx, rope)
    return graph


def replay(s, graph):
    torch.cuda.synchronize()
    with torch.cuda.stream(s.main):
        graph.replay()


@pytest.mark.parametrize("theta", [500000.0, 0.0])
def test_a_recorded_call_takes_effect_when_its_graph_runs(theta):
    w = synth.Workload("rope_graph", 1, 512, 4, 2, 128, 512, 3, 200, False, (0.0, 0.0), rope_theta=theta)
    scaled = psv.psv_rope_plan(theta=10000.0, scaling="linear", factor=4.0, magnitude=1.25)
    other = psv.psv_rope_plan(theta=10000.0)
    with Session(w, seed=15) as s:
        plain = s.run().clone()
        want = {}
        for name, rope in (("scaled", scaled), ("other", other)):
            psv.psv_set_rope(s.ctx, rope)
            want[name] = s.run().clone()
        psv.psv_set_rope(s.ctx, None)
        assert torch.equal(s.run(), plain) and not torch.equal(want["scaled"], want["other"])
        graphs = {"scaled": recorded(s, scaled)}
        assert torch.equal(s.run(), plain)
        graphs["plain"] = recorded(s, None)
        assert torch.equal(s.run(), plain)
        want["plain"] = plain
        psv.psv_set_rope(s.ctx, other)
        assert torch.equal(s.run(), want["other"])
        for name in ("scaled", "plain", "scaled", "scaled", "plain"):
            replay(s, graphs[name])
            assert torch.equal(s.run(), want[name])
            psv.psv_set_rope(s.ctx, other)
            assert torch.equal(s.run(), want["other"])
