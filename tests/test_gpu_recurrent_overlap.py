"""The recurrent block's operators beside other work: two calls at once on operands of their own, another stream, captured and replayed.  Before every call its workspace and its outputs are filled
with a pattern, on the stream it is made on, and every call has outputs of its own: what a call reads too early, or from another one, is then not by chance what it should have been."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_recurrent import NAMES, calls, leave_nothing, outputs  # noqa: E402, F401


def reference(call, need, shapes):
    outs = outputs(shapes)[1]
    call(torch.empty(need, dtype=torch.uint8, device="cuda"), outs)
    torch.cuda.synchronize()
    return outs


def soil(ws, outs, turn):
    """Patterns that are no residues: words of 2^63 and more."""
    ws.fill_(0xa0 + turn)
    for o in outs:
        o.fill_(-2 - turn)


def same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50), (12, 7, 3, 3, 56)])
@pytest.mark.parametrize("name", NAMES)
def test_two_calls_at_once_on_different_operands(name, ring):
    """One context, a stream, a workspace and keys for each call; the context's second stream serves both."""
    sides = []
    for seed in (3, 4):
        call, need, shapes = calls(ring, seed)[1][name]
        sides.append((call, need, shapes, reference(call, need, shapes), torch.empty(need, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), [outputs(shapes)[1] for _ in range(3)]))
    assert not any(torch.equal(a, b) for a, b in zip(sides[0][3], sides[1][3]))
    torch.cuda.synchronize()
    for turn in range(3):
        for call, _, _, _, ws, stream, outs in sides:
            with torch.cuda.stream(stream):
                soil(ws, outs[turn], turn)
            call(ws, outs[turn], stream.cuda_stream)
    torch.cuda.synchronize()
    for turn in range(3):
        for _, _, _, want, _, _, outs in sides:
            assert same(outs[turn], want), turn


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50)])
def test_different_calls_at_once(ring):
    """Every operator beside the next one, on streams in turn."""
    ops = calls(ring, 5)[1]
    want = {name: reference(*ops[name]) for name in NAMES}
    streams = [torch.cuda.Stream() for _ in range(2)]
    runs = []
    for turn in range(2):
        for i, name in enumerate(NAMES):
            call, need, shapes = ops[name]
            runs.append((name, call, torch.empty(need, dtype=torch.uint8, device="cuda"), outputs(shapes)[1], streams[(i + turn) % 2], turn))
    torch.cuda.synchronize()
    for _, call, ws, outs, stream, turn in runs:
        with torch.cuda.stream(stream):
            soil(ws, outs, turn)
        call(ws, outs, stream.cuda_stream)
    torch.cuda.synchronize()
    for name, _, _, outs, _, turn in runs:
        assert same(outs, want[name]), (name, turn)


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50)])
@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream_than_the_operands(name, ring):
    call, need, shapes = calls(ring, 6)[1][name]
    want, ws, side = reference(call, need, shapes), torch.empty(need, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    runs = [outputs(shapes)[1] for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        soil(ws, runs[0], 0)
    call(ws, runs[0], side.cuda_stream)
    with torch.cuda.stream(side):  # the current stream is taken where none is given
        soil(ws, runs[1], 1)
        call(ws, runs[1])
    side.synchronize()
    assert all(same(outs, want) for outs in runs)


@pytest.mark.parametrize("ring", [(12, 7, 3, 3, 50), (14, 7, 3, 3, 50)])
@pytest.mark.parametrize("name", NAMES)
def test_graphs_that_share_a_workspace_with_other_calls(name, ring):
    """Two graphs on operands of their own and one workspace, replayed in turn, an eager call between them."""
    ops = [calls(ring, seed)[1][name] for seed in (7, 8)]
    want = [reference(*op) for op in ops]
    ws = torch.empty(ops[0][1], dtype=torch.uint8, device="cuda")
    graphs = []
    for call, _, shapes in ops:
        outs, g = outputs(shapes)[1], torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(ws, outs)
        graphs.append((g, outs))
    for turn in range(3):
        for i, (g, outs) in enumerate(graphs):
            soil(ws, outs, turn)
            g.replay()
            torch.cuda.synchronize()
            assert same(outs, want[i]), (turn, i)
        eager = outputs(ops[1][2])[1]
        soil(ws, eager, turn)
        ops[1][0](ws, eager)
        torch.cuda.synchronize()
        assert same(eager, want[1]), turn
