"""Workload inputs as hidden vectors and an output layer: shapes, the scores' distribution, the labels of a context."""
import numpy as np
import pytest

from paper_2306_15685_amd import runner, synth


def small(**kw):
    return synth.scaled(synth.WORKLOADS["tiny"], **{**dict(channels=3, frames=7, chunk=4, segments=2), **kw})


def test_scores_of_hidden_vectors_are_log_likelihoods_but_for_a_small_constant():
    import torch
    w = small()
    inp = runner.make_inputs(w, device="cpu", hidden_features=64)
    assert inp.loglikes == [] and len(inp.hidden) == 2
    weight, bias = inp.output_layer
    assert weight.shape == (w.num_pdfs, 64) and bias.shape == (w.num_pdfs,)
    assert weight.dtype == torch.bfloat16 and bias.dtype == torch.float32
    for h in inp.hidden:
        assert h.shape == (3, 7, 64) and h.dtype == torch.bfloat16
        mass = torch.logsumexp(h.double() @ weight.double().t() + bias.double(), dim=-1)
        assert mass.abs().max() < 6.0   # (of N(0, 9) for 200 labels: the mean of the masses is 1, single frames vary)
    assert not torch.equal(inp.hidden[0], inp.hidden[1])
    again = runner.make_inputs(w, g=inp.g, device="cpu", hidden_features=64)
    assert torch.equal(again.hidden[1], inp.hidden[1]) and torch.equal(again.output_layer[0], weight)


def test_labels_of_a_context_are_those_its_arcs_read():
    w = small()
    inp = runner.make_inputs(w, device="cpu", hidden_features=8)
    g = inp.g
    eps, read = np.flatnonzero(g.ilabel == 0)[:2], np.flatnonzero(g.ilabel > 0)[:3]
    labels, boost = runner.listed_labels(g, ([np.concatenate([eps, read, read]), eps, np.zeros(0, np.int64)], np.float32([-2, -3, 0])))
    assert np.array_equal(labels[0], sorted({int(g.ilabel[a]) - 1 for a in read}))
    assert labels[1].size == 0 and labels[2].size == 0
    assert np.array_equal(boost, np.float32([2, 3, 0])) and boost.dtype == np.float32


def test_labels_are_drawn_from_hidden_vectors_only():
    inp = runner.make_inputs(small(segments=1), device="cpu")
    assert inp.hidden is None and len(inp.loglikes) == 1
    with pytest.raises(ValueError, match="drawn from the scores of hidden vectors"):
        runner.Session(inp, draw=runner.Draw())
