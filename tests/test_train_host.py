"""What TokenScorer and Orthogonalizer do on the host around a call, without a GPU: the calls themselves do nothing here."""
import pytest
import torch

import paper_2406_03285_amd as rb
from paper_2406_03285_amd import train

CALLED = []


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    """Handles of tensors in host memory whose calls are noted and end well."""
    CALLED.clear()
    for kind in (rb.TokenScorer, rb.Orthogonalizer):
        monkeypatch.setattr(kind, "_on_stream", lambda self, call, *args: CALLED.append(args) or rb.RB_OK)


def scorer_of(vocab, given, top, dtype=torch.float32):
    s = object.__new__(rb.TokenScorer)
    s.handle, s.vocab, s.dtype, s.given, s.top, s.device, s._index = None, vocab, dtype, given, top, torch.device("cpu"), -1
    return s


def ortho_of(m, n):
    o = object.__new__(rb.Orthogonalizer)
    o.handle, o.m, o.n, o.batch, o.dtype, o.out_dtype, o.device = None, m, n, 1, torch.float32, torch.float32, torch.device("cpu")
    return o


def versions(tensors):
    return [None if t is None else t._version for t in tensors]


@pytest.mark.parametrize("given,top", [(1, 0), (3, 2), (0, 4)])
def test_scores_written_into_given_tensors_are_new_versions_of_them(given, top):
    s = scorer_of(11, given, top)
    z, t = torch.zeros((5, 11)), torch.zeros((5, given), dtype=torch.int64)
    for out in (s.outputs(5), train.Scores(*s.outputs(5))):
        before = versions(out)
        s.score(z, t, out=out)
        assert versions(out) == [None if v is None else v + 1 for v in before] and len(CALLED) == 1
        assert z._version == 0 and t._version == 0
        CALLED.clear()


def test_a_gradient_written_into_a_given_tensor_is_a_new_version_of_it():
    s = scorer_of(11, 1, 0)
    z, t, row = torch.zeros((5, 11)), torch.zeros((5, 1), dtype=torch.int64), torch.zeros(5)
    w = torch.zeros((5, 1))
    s.grad(z, t, row, row, w, row, out=z)
    assert len(CALLED) == 1 and z._version == 1
    other = torch.zeros((5, 11))
    s.grad(z, t, row, row, w, row, out=other)
    s.grad(z, t, row, row, w, row)
    assert len(CALLED) == 3 and z._version == 1 and other._version == 1
    assert t._version == row._version == w._version == 0


def test_an_orthogonalised_update_written_into_a_given_tensor_is_a_new_version_of_it():
    o = ortho_of(4, 6)
    u, out = torch.zeros((4, 6)), torch.zeros((4, 6))
    o.orthogonalize(u)
    o.orthogonalize(u, out=out)
    assert u._version == 0 and out._version == 1
    o.orthogonalize(u, out=u)
    assert len(CALLED) == 3 and u._version == 1


def test_backward_refuses_logits_that_a_call_has_overwritten():
    """As for torch's own operators: what autograd has saved and a call has changed since ends backward."""
    s = scorer_of(11, 1, 0)
    z = torch.randn((5, 11), requires_grad=True)
    y = (z * z).sum()                                    # saves z
    row = torch.zeros(5)
    s.grad(z.detach(), torch.zeros((5, 1), dtype=torch.int64), row, row, torch.zeros((5, 1)), row, out=z.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


# ---- streams -------------------------------------------------------------------

class Stream:
    """A stream of a device that keeps what it was told to wait for."""

    def __init__(self, address):
        self.cuda_stream, self.waited = address, []

    def wait_stream(self, other):
        self.waited.append(other)


class Workspace:
    def __init__(self):
        self.used_on = []

    def record_stream(self, stream):
        self.used_on.append(stream)


class Device:
    """The current stream, and whether it is being captured into a graph."""

    def __init__(self, monkeypatch):
        self.stream, self.capturing = Stream(0), False
        monkeypatch.undo()                               # (the calls go through _on_stream here)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.stream)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)
        monkeypatch.setattr(train, "_current_stream", lambda index: self.stream.cuda_stream)

    def handle(self):
        h = train._OnStream()
        h._bind_device("cuda:0")
        h.workspace = Workspace()
        return h

    def call(self, h, stream, capturing=False):
        self.stream, self.capturing = stream, capturing
        assert h._on_stream(lambda *args: args, 1, 2) == (1, 2, stream.cuda_stream)


def test_the_workspace_is_kept_for_every_stream_that_it_was_used_on(monkeypatch):
    """It was allocated on the handle's first stream: given back with the handle, it may be that stream's next tensor while another stream's
    kernels still use it, unless the allocator knows of these."""
    d = Device(monkeypatch)
    a, b, c = d.stream, Stream(7), Stream(9)
    h = d.handle()
    d.call(h, a)
    assert h.workspace.used_on == []
    d.call(h, b)
    d.call(h, b)
    d.call(h, c)
    d.call(h, a)
    assert h.workspace.used_on[:2] == [b, c]
    assert b.waited == [a] and c.waited == [b] and a.waited == [c]


def test_a_captured_call_does_not_make_the_handle_forget_the_stream_before(monkeypatch):
    """Eager work on b, then a capture, then eager work on c: that has to wait for b's, which the capture's stream knows nothing of."""
    d = Device(monkeypatch)
    a, b, c, capture = d.stream, Stream(7), Stream(9), Stream(11)
    h = d.handle()
    d.call(h, b)
    d.call(h, capture, capturing=True)
    assert capture.waited == [] and capture not in h.workspace.used_on
    d.call(h, c)
    assert c.waited == [b]
    d.call(h, capture, capturing=True)
    d.call(h, c)
    assert c.waited == [b]


# ---- what is given as out ------------------------------------------------------

def test_outputs_of_which_some_are_left_out_or_exchanged():
    s = scorer_of(11, 1, 2)
    z, t = torch.zeros((5, 11)), torch.zeros((5, 1), dtype=torch.int64)
    lse = torch.zeros(5)
    out = s.outputs(5)._replace(lse=lse, entropy=None)
    assert s.score(z, t, out=out) is out
    assert CALLED[-1][5:9] == (out.logp, lse, None, out.top_logp)
    for wrong in (dict(lse=torch.zeros(6)), dict(logp=torch.zeros((5, 1), dtype=torch.float64)), dict(top_ids=torch.zeros((5, 2)))):
        with pytest.raises(AssertionError, match="out"):
            s.score(z, t, out=s.outputs(5)._replace(**wrong))
    with pytest.raises(AssertionError, match="out"):
        s.score(z, t, out=s.outputs(4))
    with pytest.raises(AssertionError, match="out"):
        s.score(z, t, out=scorer_of(11, 2, 2).outputs(5))
