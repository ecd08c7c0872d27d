"""What runner.Session enqueues through torch goes to the session's stream, not to torch's current one."""
import contextlib
import threading
import types

import numpy as np
import pytest

from paper_2306_15685_amd import binding as B
from paper_2306_15685_amd import runner, synth


def test_drawn_labels_are_copied_on_the_session_s_stream(monkeypatch):
    import torch
    from torch.utils._python_dispatch import TorchDispatchMode

    w = synth.scaled(synth.WORKLOADS["tiny"], channels=3, frames=7, chunk=4)
    session = types.SimpleNamespace(cuda_stream=77)
    current, done = ["current"], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    class Copies(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            if "copy_" in str(func):
                done.append(("copy", current[-1]))
            return func(*args, **(kwargs or {}))

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(B, "cbd_layer_apply", lambda *a, hip_stream, **kw: done.append(("layer", hip_stream)))
    monkeypatch.setattr(B, "cbd_sample_labels", lambda *a, **kw: done.append(("draw", None)))   # (on the sampler's own stream)
    s = object.__new__(runner.Session)
    s.torch, s.w, s.stream = torch, w, session
    s.inp = types.SimpleNamespace(hidden=[torch.zeros((3, 7, 8), dtype=torch.bfloat16)])
    s.layer, s.sampler, s.settings = "layer", "sampler", {}
    s.scores = torch.zeros(3 * 4 * w.num_pdfs)
    s.row_channels = {n: torch.arange(3, dtype=torch.int32).repeat_interleave(n) for n in (4, 3)}
    s.random = [[torch.zeros(12), torch.zeros(9)]]
    s.row_labels, s.row_logprobs = torch.arange(12, dtype=torch.int32), torch.arange(12) / 2
    s.drawn = [(torch.full((3, 7), -9, dtype=torch.int32), torch.full((3, 7), -9.0))]
    with Copies():
        s._chunk_scores(0, 0, 4)
        s._chunk_scores(0, 4, 3)
    assert done == [("layer", 77), ("draw", None), ("copy", session), ("copy", session)] * 2
    labels, logprobs = s.drawn[0]
    assert torch.equal(labels[:, :4], s.row_labels.view(3, 4)) and torch.equal(labels[:, 4:], s.row_labels[:9].view(3, 3))
    assert torch.equal(logprobs[:, :4], s.row_logprobs.view(3, 4)) and torch.equal(logprobs[:, 4:], s.row_logprobs[:9].view(3, 3))


@pytest.mark.gpu
def test_sessions_step_from_another_stream_or_thread():
    """A session made under a stream of its own and stepped under torch's default one, from this thread and from another,
    with the session's stream behind other work: labels and log-probabilities are those of a session on the current stream."""
    import torch
    w = synth.scaled(synth.WORKLOADS["tiny"], channels=6, frames=23, chunk=4, segments=2)
    inp = runner.make_inputs(w, hidden_features=40)
    draw = runner.Draw(temperature=0.9, top_p=0.9)
    plain = runner.Session(inp, draw=draw)
    try:
        finals = plain.step(keep_results=True)
        torch.cuda.synchronize()
        want = [(a.clone(), b.clone()) for a, b in plain.drawn]
    finally:
        plain.close()
    side = torch.cuda.Stream()
    work = torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        sess = runner.Session(inp, draw=draw)
    got = []

    def step():
        with torch.cuda.stream(side):
            for _ in range(20):
                work @ work
        got.append(sess.step(keep_results=True))

    try:
        for threaded in (False, True, False):
            for t in (t for pair in sess.drawn for t in pair):
                t.fill_(-9)
            torch.cuda.synchronize()
            if threaded:
                thread = threading.Thread(target=step)
                thread.start()
                thread.join()
            else:
                step()
            side.synchronize()
            for (a, b), (a2, b2) in zip(sess.drawn, want):
                assert torch.equal(a, a2) and torch.equal(b, b2), threaded
        assert len(got) == 3
        for r in got:
            for a, b in zip(r, finals):
                assert np.array_equal(a[0], b[0]) and all(np.array_equal(x, y) for x, y in zip(a[1], b[1]))
    finally:
        sess.close()
