"""cbd_sample_labels where the kept labels end at an unusual place: a min_p whose test is the same for many scores around its
border, a cut among zeros, rows of as many labels as there may be.  Against the rule in 64 bits, as in test_gpu_sampling.py."""
import numpy as np
import pytest

import score_reference as R
import test_gpu_sampling as S

pytestmark = pytest.mark.gpu

DEV = "cuda"


# best score, temperature, scores this near to it have a weight of 1 in 64 bits, those this far away have not: exp(d) rounds
# to 1 for d > -2^-54 = -5.6e-17 and to less for d < -2^-53
PLATEAUS = [(5.0, 1e15, 0.03, 0.6), (3.0, 1e12, 3e-5, 6e-4), (1e-12, 1.0, 3e-17, 6e-16), (-2.0, 1e14, 3e-3, 6e-2)]


@pytest.mark.parametrize("labels", [700, 5_000, 20_000, 70_000])
@pytest.mark.parametrize("best,temperature,near,far", PLATEAUS)
def test_min_p_of_one_at_high_temperatures(best, temperature, near, far, labels):
    """min_p = 1 keeps the labels whose weight is 1: some, or more than a list holds, alone and behind other cuts."""
    import torch
    rng = np.random.default_rng(labels)
    rows = []
    for n in (1, 200, 300, labels // 2):
        x = best - np.float64(far) - np.abs(rng.uniform(0, 1, labels)) * abs(best)
        x[rng.permutation(labels)[:n]] = best - rng.uniform(0, near, n)
        x[rng.integers(0, labels)] = best
        rows.append(x.astype(np.float32))
    x = torch.from_numpy(np.stack(rows)).to(DEV)
    d = (x.cpu().numpy().astype(np.float64) - np.float64(np.float32(best))) / np.float64(np.float32(temperature))
    assert ((d > -2.0 ** -54) | (d < -2.0 ** -53)).all()   # (the test's own condition)
    s = S.Sampler(4, labels)
    t, one = [temperature] * 4, [1.0] * 4
    for kw in (dict(), dict(top_p=[0.999] * 4), dict(top_k=[labels - 1] * 4), dict(top_k=[labels // 2 + 30] * 4, top_p=[0.9999] * 4)):
        S.check_rows(s, x, rng.random(4), "f32", temperature=t, min_p=one, **kw)
    s.close()


@pytest.mark.parametrize("labels", [401, 3_000, 7_000, 20_000, 60_000])
def test_cuts_among_zeros(labels):
    """A best score just below a power of two, so that the borders between intervals of keys lie between the zeros and the
    largest negative scores; half of the labels zero, the others negative and next to zero."""
    import torch
    rng = np.random.default_rng(labels)
    rows, zeros = [], labels // 2
    for best in (1.9999999, 0.99999994, 3.9999998, 2.0 ** -100 * (2 - 2.0 ** -23), 1.9999999):
        x = -rng.uniform(5e-40, 2e-39, labels)
        x[rng.permutation(labels)[:zeros]] = 0.0
        x[rng.integers(0, labels)] = best
        rows.append(x)
    rows[3][rng.integers(0, labels, 20)] = -0.0
    rows[4][rows[4] < 0] *= 1e36   # (further away)
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DEV)
    s = S.Sampler(5, labels)
    for p in (0.3, 0.5, 0.75, 0.95):
        S.check_rows(s, x, rng.random(5), "f32", top_p=[p] * 5)
    for k in (2, 100, 150, 300, zeros // 2, zeros + 30):
        S.check_rows(s, x, rng.random(5), "f32", top_k=[k] * 5)
        S.check_rows(s, x, rng.random(5), "f32", top_k=[k] * 5, top_p=[0.75] * 5, min_p=[0.01] * 5)
    # 16-bit scores reach such a best score by their offset
    y = torch.zeros((2, labels), device=DEV)
    y[:, labels // 2:] = -1e-39
    y[0, labels - 3] = 1.0
    y[1, 5] = 3.0
    y = y.to(torch.bfloat16)
    lists, offsets = [[labels - 3], [5]], np.array([0.9999999, 0.9999998], np.float32)
    s.lists([0, 1], lists, offsets)
    for p in (0.3, 0.75):
        S.check_rows(s, y, rng.random(2), "bf16", lists, offsets, top_p=[p] * 2)
    s.close()


def test_as_many_list_entries_as_there_may_be():
    """2^31 - 1 entries, all but the last three label 0 of channel 1."""
    import torch
    from paper_2306_15685_amd import binding as B
    total, N = 2 ** 31 - 1, 40
    labels = np.zeros(total, np.int32)   # (pages that are only read take no memory)
    labels[-3:] = 5, 39, 7
    s = S.Sampler(3, N)
    print("setting the lists", flush=True)
    B.cbd_sampler_set_contexts(s.h, [1, 2], None, [2.0, 3.0], packed=(labels, np.array([0, total - 1, total], np.int32)))
    x = torch.from_numpy(np.random.default_rng(1).normal(0, 1, (3, N)).astype(np.float32)).to(DEV)
    for u in (0.05, 0.4, 0.9):
        S.check_rows(s, x, [u] * 3, "f32", [[], [0, 5, 39], [7]], [0.0, 2.0, 3.0], top_k=[4] * 3)
    s.close()


@pytest.mark.parametrize("labels,dtype", [(1_048_575, "bf16"), (1_048_576, "f32")])
def test_as_many_labels_as_there_may_be(labels, dtype):
    """Scores as they come, all equal (the largest sum of weights there is, cuts among the ties), and few distinct ones; random
    numbers at both ends."""
    import torch
    rng = np.random.default_rng(labels)
    rows = rng.normal(0, 2, (4, labels)).astype(np.float32)
    rows[1] = 3.0
    rows[2] = rng.integers(0, 3, labels)
    rows[3, 1:] = -np.inf
    rows[3, labels - 1] = rows[3, 0]
    x = torch.from_numpy(rows).to(DEV).to(S.T(dtype))
    s = S.Sampler(4, labels)
    for u in (0.0, 0.37, 0.9999999, 1.0):
        S.check_rows(s, x, [u] * 4, dtype)
        S.check_rows(s, x, [u] * 4, dtype, top_p=[0.3, 0.71, 0.6, 0.4])
    S.check_rows(s, x, rng.random(4), dtype, top_k=[100, 70_001, 800_000, 1])
    S.check_rows(s, x, rng.random(4), dtype, top_k=[900_000, 1_000_003, 500, 2], top_p=[0.9, 0.31, 0.95, 0.7], temperature=[0.7, 1.3, 2.0, 1.0])
    S.check_rows(s, x, rng.random(4), dtype, min_p=[0.05, 0.5, 0.3, 1.0])
    s.close()
