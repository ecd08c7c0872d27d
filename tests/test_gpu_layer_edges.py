"""cbd_layer_apply at the edges of its numbers: infinite weights, scales that leave the range, activations relative to their
own size, more tiles than a launch takes."""
import numpy as np
import pytest

import test_gpu_layers as L

pytestmark = pytest.mark.gpu

DEV = "cuda"
INF = float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (1, 40, 24), (5, 40, 24), (3, 70, 33), (70, 136, 100), (9, 300, 500), (300, 264, 520), (1067, 264, 1032)])
def test_an_infinite_weight_gives_infinities(dtype, rows, K, N):
    """... with the sign of what it is multiplied by, wherever along K it is: nothing is multiplied by it twice or by a zero
    that is not in the row.  Every kernel, with K that ends inside its steps."""
    import torch
    g = L.gen(rows + K)
    x, w = L.whole((1, rows, K), dtype, g), L.whole((N, K), dtype, g)
    x[x == 0] = 1
    for at in sorted({0, K // 2, K - 1}):
        v = w.clone()
        v[N - 1, at], v[0, at] = INF, -INF   # (N = 1: one weight)
        layer = L.Layer(v, None, dtype)
        got = layer.apply(x, torch.zeros((1, rows, N), device=DEV))[0]
        want = (x[0].double() @ w.double().t()).float()
        want[:, N - 1] = x[0, :, at].float() * INF
        want[:, 0] = x[0, :, at].float() * -INF
        assert torch.equal(got, want), at
        layer.close()
