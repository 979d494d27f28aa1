"""The measured cases of the paged operators (perf/operators.py) on the stream that is current: between its fills and its reads, and
as part of what is captured there."""
import pytest
import torch

from perf import operators as P

pytestmark = pytest.mark.gpu
CASES = [c for c in P.listed() if c["name"] in ("append-64", "decode-8", "prompt-77")]


@pytest.fixture()
def own():
    P.own = True
    yield
    P.own = False


def _outputs(out):
    return [t.clone() for t in (out.values() if isinstance(out, dict) else [out])]


@pytest.mark.parametrize("case", CASES, ids=lambda c: c["name"])
def test_a_pass_lies_on_the_current_stream(own, case):
    """Behind long products on a side stream, with inputs that come only after them; the reads follow on that stream."""
    ready = P.prepare(case, 3)
    want = _outputs(P.run(ready))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s = P.prepare(case, 3)
        P.run(s)
        side.synchronize()
        source = s.qkv if case["kind"] == "append" else s.q
        late = source.clone()
        source.zero_()
        s.out.zero_()
        side.synchronize()
        b = a
        for _ in range(8):
            b = torch.mm(a, b) * 1e-2
        source.copy_(late)
        got = _outputs(P.run(s))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_a_pass_can_be_captured(own):
    """A graph of a pass on a side stream, replayed with the program's own work between: every replay gives the eager result."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = P.prepare(CASES[1], 5)
        P.run(s)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            P.run(s)
        for _ in range(4):
            s.q.normal_()
            want = _outputs(P.run(s))[0]
            s.out.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(s.out, want)
    new = torch.cuda.Stream()
    while new.cuda_stream == side.cuda_stream:
        new = torch.cuda.Stream()
    P._contexts.pop((0, new.cuda_stream), None)
    with pytest.raises(RuntimeError, match="first pass"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=new):
            P.run(s)
    torch.cuda.synchronize()
