"""TokenScorer and Orthogonalizer within programs that use autograd and several streams, on the GPU."""
import pytest
import torch

import paper_2406_03285_amd as rb

pytestmark = pytest.mark.gpu


def test_backward_raises_for_what_a_call_has_overwritten():
    z = torch.randn((6, 300), device="cuda", requires_grad=True)
    t = torch.randint(0, 300, (6, 1), device="cuda")
    scorer = rb.TokenScorer(300, top=2)
    w = torch.ones((6, 1), device="cuda")
    s = scorer(z, t)                                     # saves the logits, lse and entropy
    scorer.grad(z.detach(), t, s.lse, s.entropy.detach(), w, out=z.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        s.logp.sum().backward()
    out = scorer.outputs(6)
    scorer.score(z.detach(), t, out=out)
    x = torch.ones((6, 1), device="cuda", requires_grad=True)
    y = (x * out.logp).sum()                             # saves logp
    scorer.score(z.detach(), t, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    u = torch.randn((8, 9), device="cuda", requires_grad=True)
    y = (u * u).sum()
    rb.Orthogonalizer(8, 9).orthogonalize(u.detach(), out=u.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_calls_on_streams_in_turn_and_a_handle_that_is_dropped_behind_them():
    """The handle orders its own calls, and its workspace is not given away while they run.  (Inputs and results are ready before, and read behind,
    all of it.)"""
    u = [torch.randn((700, 900), generator=torch.Generator("cuda").manual_seed(k), device="cuda") for k in range(3)]
    z = [torch.randn((2, 200000), generator=torch.Generator("cuda").manual_seed(k), device="cuda") for k in range(3)]
    t = torch.zeros((2, 1), dtype=torch.int64, device="cuda")
    ortho, scorer = rb.Orthogonalizer(700, 900), rb.TokenScorer(200000, top=20)
    want = [ortho.orthogonalize(x) for x in u]
    wanted = [scorer.score(x, t) for x in z]
    out, outs = [torch.empty_like(x) for x in want], [scorer.outputs(2) for _ in z]
    size = ortho.workspace.numel()
    streams = [torch.cuda.Stream() for _ in range(2)] + [torch.cuda.current_stream()]
    torch.cuda.synchronize()
    for turn in range(3):
        for k in range(3):
            with torch.cuda.stream(streams[(k + turn) % 3]):
                ortho.orthogonalize(u[k], out=out[k])
                scorer.score(z[k], t, out=outs[k])
    with torch.cuda.stream(streams[0]):                  # the last calls, on a stream that is not the workspaces' own
        for k in range(3):
            ortho.orthogonalize(u[k], out=out[k])
            scorer.score(z[k], t, out=outs[k])
    del ortho, scorer
    for _ in range(4):
        torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for k in range(3):
        assert torch.equal(out[k], want[k])
        assert all(torch.equal(a, b) for a, b in zip(outs[k], wanted[k]))


def test_calls_on_streams_in_turn_behind_a_capture():
    """Calls on two streams in turn behind a capture, and replays between them."""
    o = rb.Orthogonalizer(700, 900)
    u = [torch.randn((700, 900), generator=torch.Generator("cuda").manual_seed(k), device="cuda") for k in range(2)]
    want = [o.orthogonalize(x) for x in u]
    out, captured = [torch.empty_like(x) for x in want], torch.empty_like(want[0])
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.orthogonalize(u[0], out=captured)
    for _ in range(3):
        with torch.cuda.stream(one):
            o.orthogonalize(u[0], out=out[0])
        with torch.cuda.stream(two):
            o.orthogonalize(u[1], out=out[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(captured, want[0])
