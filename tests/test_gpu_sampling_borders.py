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
