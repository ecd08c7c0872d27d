"""cbd_layer_apply at the edges of its numbers: infinite weights, scales that leave the range, activations relative to their
own size, more tiles than a launch takes."""
import numpy as np
import pytest

import score_reference as R
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(5, 40, 24), (128, 64, 128), (1024, 64, 2048), (2560, 32, 3328), (4096, 576, 4352)])
def test_sums_that_only_a_scale_takes_out_of_range(dtype, rows, K, N):
    """scale * (sum + bias): the sum's and the bias's own multiples are beyond fp32, the result is not."""
    import torch
    g = L.gen(K)
    top = 2.0 ** 127
    x, w = torch.zeros((1, rows, K), device=DEV, dtype=L.T(dtype)), torch.zeros((N, K), device=DEV, dtype=L.T(dtype))
    small = L.whole((rows,), "f32", g)
    x[0, :, 0] = small.to(L.T(dtype)) / 8 + 1
    w[:, 0] = top
    bias = torch.full((N,), -top, device=DEV)
    layer = L.Layer(w, bias, dtype)
    for scale in (2.0, -2.0, 1.5, 1.0, 0.25):
        got = layer.apply(x, torch.zeros((1, rows, N), device=DEV), scale)
        assert torch.equal(got[0], (small / 8 * scale)[:, None].mul(top).expand(rows, N)), scale
    layer.close()


def test_more_tiles_than_one_launch_takes():
    """2^28 rows of 129 outputs: two launches of tiles, a few rows in the second.  Row r's input is r mod 32."""
    import torch
    rows, N = 2 ** 28 + 100, 129
    if torch.cuda.mem_get_info()[0] < 100 * 2 ** 30:
        pytest.skip("needs 100 GB of free device memory")
    x = (torch.arange(rows, device=DEV, dtype=torch.int32) % 32).float()
    w = (torch.arange(N, device=DEV) % 5 - 2).float()[:, None].contiguous()
    out = torch.full((rows + 1, N), 7.0, device=DEV, dtype=torch.bfloat16)
    layer = L.Layer(w, None, "f32")
    layer.apply(x.view(1, rows, 1), out[:rows].view(1, rows, N))
    want = (torch.arange(32, device=DEV).float()[:, None] * w[:, 0]).to(torch.bfloat16).repeat(2 ** 15, 1)   # of 2^20 rows
    for at in range(0, rows, 2 ** 20):
        n = min(2 ** 20, rows - at)
        assert torch.equal(out[at:at + n], want[:n]), at
    assert (out[rows] == 7.0).all()
    layer.close()
    del x, out, want
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,N", [(200, 40), (2048, 256)])
@pytest.mark.parametrize("act,steps", [("tanh", lambda y: 8 + 0 * y), ("gelu", lambda y: 20 + 0 * y),
                                       ("sigmoid", lambda y: 1.25 * y + 6), ("silu", lambda y: 1.25 * y + 6)])
def test_activations_relative_to_their_own_size(act, steps, rows, N):
    """One product, rounded as fp32 does: the activation itself, in fp32, over -12 .. 12 and at small |y|.  Half
    steps, largest first: tanh, the exponential's part at |y| = 0.6 is 0.86 of (1.5 for its argument + 2 + 1 + 2 for the quotient)
    and 1 for the sum.  gelu, 8 for t (3, of which g takes up to 2.7 times), 4 for the polynomial, 2 for its fit, 3 for the
    exponential, 1 for each of three products.  sigmoid, silu: 1.25 |y| + 2 for the exponential, 1 for the sum, 2 for the
    reciprocal, 1 for the product."""
    import torch
    g = L.gen(5)
    x = torch.rand((1, rows, 1), generator=g, device=DEV) * 2 - 1
    w = 2.0 ** torch.randint(-30, 4, (N, 1), generator=g, device=DEV).float() * torch.where(torch.rand((N, 1), generator=g, device=DEV) < 0.5, 1.5, 1.0)
    w[: N // 2] = torch.rand((N // 2, 1), generator=g, device=DEV) * 12
    y = (x[0] * w[:, 0]).double()   # (fp32 products, as the layer makes them)
    layer = L.Layer(w, None, "f32", act)
    got = layer.apply(x, torch.zeros((1, rows, N), device=DEV))[0].double()
    want = R.act64(act, y)
    error = (got - want).abs() / want.abs() * 2.0 ** 24   # (in half steps)
    print(act, "largest error in half steps", float(error.max()), flush=True)
    assert (want != 0).all() and (error <= steps(y.abs())).all()
    layer.close()
