"""The score rows' operators as they are used together: hidden vectors -> output layer -> decoding and drawn labels, a chunk
at a time (runner.Session), and a loop of layers that draws a label per step, captured and replayed."""
import numpy as np
import pytest

from paper_2306_15685_amd import runner, synth
from paper_2306_15685_amd import binding as B

import gpu_harness as GH
import score_reference as R
from oracle import OracleChannel, OracleGraph

pytestmark = pytest.mark.gpu


def logprob_error(value, num_labels):
    """Rounding to fp32, weights off by half a unit of 2^-50 each, and the labels' relative error of 2^-36."""
    return 2.0 ** -24 * abs(value) + num_labels * 2.0 ** -51 + 2.0 ** -36


@pytest.mark.parametrize("biased", [True, False])
def test_hidden_vectors_to_paths_and_labels(biased):
    """Frames in chunks of 20, 20 and 10 of two utterances with new lists each."""
    import torch
    w = synth.scaled(synth.WORKLOADS["tiny"], channels=5, frames=50, chunk=20, segments=2, partial_every_chunk=True)
    inp = runner.make_inputs(w, hidden_features=72)
    draw = runner.Draw(temperature=0.8, top_k=60, top_p=0.9, min_p=0.01)
    sess = runner.Session(inp, biased=biased, draw=draw)
    # (the settings reach the kernel as fp32: 0.8 is 0.80000001192... there, which moves a log-probability by 1.5e-8 of it)
    temperature, top_p, min_p = (float(np.float32(v)) for v in (draw.temperature, draw.top_p, draw.min_p))
    chunks = {}
    make = sess._chunk_scores

    def keep(s, t0, n):
        make(s, t0, n)
        chunks[s, t0] = sess.scores[:w.channels * n * w.num_pdfs].view(w.channels, n, w.num_pdfs).clone()

    sess._chunk_scores = keep
    try:
        finals = sess.step(keep_results=True)
        torch.cuda.synchronize()
        partials = {(s, t): r for s, t, r in sess.partials}
        assert sorted(chunks) == [(s, t) for s in (0, 1) for t in (0, 20, 40)]
        weight, bias = (t.cpu() for t in inp.output_layer)
        og = OracleGraph.from_graph(inp.g)
        first = [(a.clone(), b.clone()) for a, b in sess.drawn]
        for s in range(w.segments):
            scores = torch.cat([chunks[s, t] for t in (0, 20, 40)], dim=1).cpu()
            want, err = R.layer64(inp.hidden[s].cpu(), weight, bias, "none", 1.0, None, 1.0, "f32")
            assert ((scores.double() - want).abs() <= err).all()
            labels, logprobs = (t.cpu().numpy() for t in sess.drawn[s])
            lists, offs = inp.contexts[s]
            listed, boost = runner.listed_labels(inp.g, inp.contexts[s])
            assert any(len(x) for x in listed)
            for c in range(w.channels):
                # decoding of these very scores
                ch = OracleChannel(og, w.beam, w.max_active)
                ch.set_context(lists[c] if biased else np.zeros(0, np.int32), offs[c] if biased else 0.0)
                ch.reset()
                for t in (0, 20, 40):
                    ch.advance(scores[c, t:t + 20].numpy())
                    if t < 40:
                        st, wl, al, cost, na, nw = partials[s, t + 20]
                        GH.assert_best_equal((int(st[c]), wl[c], al[c], float(cost[c])), ch.best_path(False), f"{s} {c} {t}")
                st, wl, al, cost, na, nw = finals[s]
                GH.assert_best_equal((int(st[c]), wl[c], al[c], float(cost[c])), ch.best_path(True), f"{s} {c} final")
                # and labels drawn from them
                for t in range(w.frames):
                    n = min(20, w.frames - t // 20 * 20)
                    u = float(sess.random[s][t // 20][c * n + t % 20])
                    label, lp, _ = R.sample_row(scores[c, t].numpy(), u, temperature, draw.top_k, top_p, min_p, listed[c],
                                                boost[c] if biased else 0.0)
                    assert labels[c, t] == label, (s, c, t)
                    assert abs(logprobs[c, t] - lp) <= logprob_error(lp, w.num_pdfs), (s, c, t)
        sess.step()
        torch.cuda.synchronize()
        for (a, b), (a2, b2) in zip(first, sess.drawn):
            assert torch.equal(a, a2) and torch.equal(b, b2)
    finally:
        sess.close()


def test_decoding_is_that_of_the_same_scores_as_log_likelihoods():
    """The output layer's scores handed over as log-likelihoods decode to the same results, bit for bit."""
    import torch
    w = synth.scaled(synth.WORKLOADS["tiny"], channels=4, frames=33, chunk=8, partial_every_chunk=True)
    inp = runner.make_inputs(w, hidden_features=40)
    sess = runner.Session(inp)
    weight, bias = inp.output_layer
    scores = torch.empty((4, 33, w.num_pdfs), device="cuda")
    h = inp.hidden[0]
    try:
        got = sess.step(keep_results=True)[0]
        B.cbd_layer_apply(sess.layer, 4, 33, h.data_ptr(), h.stride(0), h.stride(1), scores.data_ptr(), scores.stride(0),
                          scores.stride(1), hip_stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    finally:
        sess.close()
    plain = runner.Session(runner.Inputs(w, inp.g, [scores], inp.contexts))
    try:
        want = plain.step(keep_results=True)[0]
    finally:
        plain.close()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("dtype,rows", [("f16", 3), ("bf16", 40), ("f32", 5)])
def test_loop_of_layers_and_draws(dtype, rows):
    """state = tanh(W state) + state / 2, scores = V state, a label per channel: a step captured once and replayed, with the
    program's own work between the replays, gives the numbers of the steps done one by one."""
    import torch
    T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    D, N, steps = 136, 333, 6
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device="cuda")   # noqa: E731
    wt, vt, bias = (rnd(D, D) / D ** 0.5).to(T), (rnd(N, D) * 3 / D ** 0.5).to(T), rnd(N)
    start, uniform = rnd(rows, D).to(T), torch.rand((steps, rows), generator=gen, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    inner = B.cbd_layer_create(wt.data_ptr(), D, D, B.DTYPES[dtype], activation=B.ACTIVATIONS["tanh"], hip_stream=st)
    outer = B.cbd_layer_create(vt.data_ptr(), D, N, B.DTYPES[dtype], bias_ptr=bias.data_ptr(), hip_stream=st)
    samplers = {}
    state, nxt, scores = start.clone(), torch.empty_like(start), torch.empty((rows, N), device="cuda")
    u, label, lp = torch.empty(rows, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    top_p = torch.full((rows,), 0.9, device="cuda")

    def one(stream, sampler):
        B.cbd_layer_apply(inner, rows, 1, state.data_ptr(), D, 0, nxt.data_ptr(), D, 0, output_dtype=B.DTYPES[dtype],
                          residual_ptr=state.data_ptr(), residual_channel_stride=D, residual_scale=0.5, hip_stream=stream)
        state.copy_(nxt)
        B.cbd_layer_apply(outer, rows, 1, state.data_ptr(), D, 0, scores.data_ptr(), N, 0, hip_stream=stream)
        B.cbd_sample_labels(sampler, rows, scores.data_ptr(), N, B.DTYPES["f32"], u.data_ptr(), label.data_ptr(),
                            top_p_ptr=top_p.data_ptr(), logprobs_ptr=lp.data_ptr())

    def result():
        torch.cuda.synchronize()
        return [t.clone() for t in (state, scores, label, lp)]

    side = torch.cuda.Stream()
    try:
        lists = [[c, 300 - c] for c in range(rows)]
        for name, s in (("own", st), ("side", side.cuda_stream)):
            samplers[name] = B.cbd_sampler_create(rows, N, hip_stream=s)
            B.cbd_sampler_set_contexts(samplers[name], range(rows), lists, [1.5] * rows)
        want = []
        for i in range(steps):
            u.copy_(uniform[i])
            before = state.clone()
            one(st, samplers["own"])
            want.append(result())
            full, err = R.layer64(before, wt, None, "tanh", 1.0, before, 0.5, dtype)
            assert ((state.double() - full).abs() <= err).all()
            full, err = R.layer64(state, vt, bias, "none", 1.0, None, 1.0, "f32")
            assert ((scores.double() - full).abs() <= err).all()
            for c in range(rows):
                ref, ref_lp, _ = R.sample_row(scores[c].cpu().numpy(), float(u[c]), top_p=float(np.float32(0.9)), listed=lists[c], offset=1.5)
                assert int(label[c]) == ref and abs(float(lp[c]) - ref_lp) <= logprob_error(ref_lp, N), (i, c)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            one(side.cuda_stream, samplers["side"])
        state.copy_(start)
        for i in range(steps):
            u.copy_(uniform[i])
            for t in (scores, label, lp):
                t.fill_(7)
            graph.replay()
            for got, ref in zip(result(), want[i]):
                assert torch.equal(got, ref), i
            assert float((rnd(64, 64) @ rnd(64, 64)).abs().sum()) > 0   # (the program's own work)
    finally:
        torch.cuda.synchronize()
        for s in samplers.values():
            B.cbd_sampler_free(s)
        B.cbd_layer_free(inner)
        B.cbd_layer_free(outer)
