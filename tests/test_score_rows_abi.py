"""Host-side checks of the score-row calls that need no device: refused before anything is enqueued."""
import numpy as np
import pytest

from paper_2306_15685_amd import binding as B

import score_reference as R


def refused(call, *args, **kw):
    with pytest.raises(B.CbdError) as e:
        call(*args, **kw)
    assert e.value.status == B.CBD_E_INVALID, (args, kw)


def test_layers_refuse_bad_descriptions():
    some = 4096   # (an address that is never followed)
    for args in ((some, 0, 8, 0), (some, -1, 8, 0), (some, 65_537, 8, 0), (some, 8, 0, 0), (some, 8, 1_048_577, 0), (some, 8, 8, 3),
                 (some, 8, 8, -1), (0, 8, 8, 0), (some + 2, 8, 8, 0), (some + 1, 8, 8, 1), (some + 1, 8, 8, 2)):
        refused(B.cbd_layer_create, *args)
    for kw in (dict(activation=6), dict(activation=-1), dict(weight_stride=7), dict(weight_stride=-8), dict(weight_stride=1 << 41),
               dict(bias_ptr=some + 2)):
        refused(B.cbd_layer_create, some, 8, 8, 0, **kw)
    refused(B.cbd_layer_create, some, 65_536, 1_048_576, 0)   # (256 GB)
    refused(B.cbd_layer_apply, None, 1, 1, some, 8, 8, some, 8, 8)
    B.cbd_layer_free(None)


def test_samplers_refuse_bad_sizes():
    for args in ((0, 10), (-1, 10), (1, 0), (1, -5), (1, 1_048_577)):
        refused(B.cbd_sampler_create, *args)
    refused(B.cbd_sampler_set_contexts, None, [0], [[1]], [1.0])
    refused(B.cbd_sample_labels, None, 1, 4096, 10, 0, 4096, 4096)
    B.cbd_sampler_free(None)


def test_the_sampling_rule_by_hand():
    """Scores 0, ln 2, -inf, ln 5, 0, 0 -> weights 1 2 - 5 1 1 of 10, relative to the best 0.2 0.4 - 1 0.2 0.2."""
    x = np.array([0.0, np.log(2.0), -np.inf, np.log(5.0), 0.0, 0.0], np.float32)
    at = lambda u, **kw: R.sample_row(x, u, **kw)[::2]  # noqa: E731
    assert [at(u) for u in (0.05, 0.15, 0.35, 0.85, 0.95)] == [(0, 5), (1, 5), (3, 5), (4, 5), (5, 5)]
    assert at(0.1, top_k=1) == (3, 1) and at(0.1, top_k=2) == (1, 2) and at(0.99, top_k=3) == (3, 3)
    assert at(0.0, top_p=0.45) == (3, 1) and at(0.0, top_p=0.65) == (1, 2) and at(0.0, top_p=0.75) == (0, 3) and at(0.99, top_p=0.85) == (4, 4)
    assert at(0.0, min_p=0.3) == (1, 2) and at(0.0, min_p=0.15) == (0, 5) and at(0.5, min_p=1.0) == (3, 1)
    assert at(0.9, temperature=0.0) == (3, 1)
    # temperature 1/2: weights 1 4 - 25 1 1 of 32
    assert at(4.5 / 32, temperature=0.5) == (1, 5) and at(5.5 / 32, temperature=0.5) == (3, 5)
    # label 4 listed twice, raised to the best's level and beyond
    assert at(0.99, temperature=0.0, listed=[4, 4], offset=2.0) == (4, 1)
    assert R.sample_row(x, 0.05)[1] == pytest.approx(np.log(0.1), abs=1e-6)
    assert R.sample_row(np.full(3, -np.inf), 0.5) == (-1, -np.inf, 0)
