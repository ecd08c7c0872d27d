"""cbd_layer_apply against the definition in 64 bits.

Inputs of small whole numbers make every fp32 sum exact, so that a wrong index shows as a wrong number; real-valued inputs
are held to the bound derived in score_reference.layer64."""
import numpy as np
import pytest

from paper_2306_15685_amd import binding as B

import score_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
INF = float("inf")


def T(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


class Layer:
    def __init__(self, weight, bias, dtype, act="none"):
        import torch
        self.weight, self.bias, self.dtype, self.act = weight, bias, dtype, act
        self.N, self.K = weight.shape
        self.h = B.cbd_layer_create(weight.data_ptr(), self.K, self.N, B.DTYPES[dtype], weight_stride=weight.stride(0),
                                    bias_ptr=bias.data_ptr() if bias is not None else 0, activation=B.ACTIVATIONS[act],
                                    hip_stream=torch.cuda.current_stream().cuda_stream)

    def apply(self, x, out, scale=1.0, residual=None, residual_scale=1.0, stream=None):
        """x, out, residual: [channels, frames, width] tensors of any strides with packed rows."""
        import torch
        names = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}
        assert x.stride(2) == 1 and out.stride(2) == 1
        B.cbd_layer_apply(self.h, x.shape[0], x.shape[1], x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0),
                          out.stride(1), B.DTYPES[names[out.dtype]], scale=scale,
                          residual_ptr=residual.data_ptr() if residual is not None else 0,
                          residual_channel_stride=residual.stride(0) if residual is not None else 0,
                          residual_frame_stride=residual.stride(1) if residual is not None else 0, residual_scale=residual_scale,
                          hip_stream=(stream or torch.cuda.current_stream()).cuda_stream)
        return out

    def close(self):
        B.cbd_layer_free(self.h)


def gen(seed):
    import torch
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def whole(shape, dtype, g, hi=3):
    import torch
    return torch.randint(-hi, hi + 1, shape, generator=g, device=DEV).to(T(dtype))


# channels, frames, inputs, outputs: single rows, tile borders and one beyond, odd widths, narrow and wide outputs
SHAPES = [(1, 1, 1, 1), (1, 1, 64, 16), (1, 1, 1024, 6000), (1, 3, 7, 5), (3, 1, 65, 33), (1, 16, 32, 16), (1, 17, 31, 17),
          (2, 16, 96, 48), (4, 16, 128, 64), (5, 13, 200, 1021), (1, 64, 512, 512), (1, 65, 72, 80), (8, 16, 1000, 100), (3, 43, 264, 130),
          (2, 64, 2048, 128), (16, 8, 129, 257), (1, 129, 136, 255), (4, 64, 256, 256), (5, 51, 520, 384), (7, 37, 771, 300),
          (32, 33, 256, 511), (11, 97, 264, 1032), (16, 128, 64, 600)]


# enough rows and outputs for each size of tile, none of them a whole number of tiles: 64 x 128, 64 x 256, 128 x 256 ...
LARGE = [(1, 1003, 40, 2001), (5, 501, 72, 3301), (3, 1411, 33, 4133), (70, 61, 100, 4101)]
# ... and with every tile whole
LARGE_WHOLE = [(2, 512, 64, 2048), (4, 640, 32, 3328), (8, 512, 96, 4352)]
# ... many rows of few outputs, and inputs long enough for the largest tiles in 16 bits
DEEP = [(1, 500, 1032, 500), (32, 33, 517, 511), (3, 1411, 577, 2001), (70, 61, 520, 4101), (4, 640, 544, 3328), (8, 512, 576, 4352)]


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32"), ("bf16", "bf16"), ("f16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("shape", LARGE + LARGE_WHOLE + DEEP)
def test_whole_numbers_are_exact_in_large_products(shape, dtype, out):
    import torch
    C, F, K, N = shape
    print(dtype, out, shape, flush=True)
    g = gen(K)
    x, w, b = whole((C, F, K), dtype, g, 2), whole((N, K), dtype, g, 2), whole((N,), "f32", g, 9)
    res = whole((C, F, N), out, g, 9)
    base = (x.reshape(-1, K).double() @ w.double().t()).reshape(C, F, N) + b.double()
    for act, residual in (("none", None), ("relu", res), ("none", res), ("relu", None)):
        layer = Layer(w, b, dtype, act)
        got = layer.apply(x, torch.full((C, F, N), 7.0, device=DEV, dtype=T(out)), 0.5, residual, 2.0)
        want = 0.5 * (base.clamp(min=0) if act == "relu" else base)
        if residual is not None:
            want = want + 2.0 * residual.double()
        assert torch.equal(got, want.float().to(T(out))), (shape, act)
        layer.close()


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f16", "f32"), ("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "f16")])
def test_whole_numbers_are_exact(dtype, out):
    import torch
    for n, shape in enumerate(SHAPES):
        C, F, K, N = shape
        print(dtype, out, shape, flush=True)
        g = gen(100 + n)
        x, w = whole((C, F, K), dtype, g), whole((N, K), dtype, g)
        b = whole((N,), "f32", g, 9) if n % 3 else None
        res = whole((C, F, N), out, g, 9) if n % 2 else None
        layer = Layer(w, b, dtype, "relu" if n % 5 == 4 else "none")
        got = layer.apply(x, torch.full((C, F, N), 7.0, device=DEV, dtype=T(out)), 0.5, res, 2.0)
        want = x.double() @ w.double().t()
        if b is not None:
            want = want + b.double()
        want = 0.5 * (want.clamp(min=0) if n % 5 == 4 else want)
        if res is not None:
            want = want + 2.0 * res.double()
        assert torch.equal(got, want.float().to(T(out))), shape
        layer.close()


@pytest.mark.parametrize("act", ["none", "relu", "sigmoid", "tanh", "gelu", "silu"])
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
def test_real_numbers_within_the_derived_bound(dtype, out, act):
    import torch
    for C, F, K, N in [(1, 1, 700, 90), (3, 11, 256, 129), (8, 40, 384, 260)]:
        g = gen(K + N)
        x = (torch.randn((C, F, K), generator=g, device=DEV) * 2).to(T(dtype))
        w = (torch.randn((N, K), generator=g, device=DEV) / K ** 0.5).to(T(dtype))
        b = torch.randn(N, generator=g, device=DEV)
        res = torch.randn((C, F, N), generator=g, device=DEV).to(T(out))
        layer = Layer(w, b, dtype, act)
        got = layer.apply(x, torch.empty((C, F, N), device=DEV, dtype=T(out)), 1.5, res, 0.66).double()
        want, bound = R.layer64(x, w, b, act, 1.5, res, float(np.float32(0.66)), out)
        worst = ((got - want).abs() / bound).max().item()
        assert worst <= 1.0, (C, F, K, N, worst)
        layer.close()


@pytest.mark.parametrize("dtype,out,act", [("bf16", "bf16", "silu"), ("f16", "f32", "gelu"), ("f32", "f32", "sigmoid"), ("f32", "f16", "tanh")])
def test_real_numbers_in_larger_products(dtype, out, act):
    import torch
    for C, F, K, N in [(7, 33, 771, 1021), (32, 33, 256, 511), (11, 97, 264, 1032), (5, 401, 90, 2101), (3, 1411, 577, 2001), (8, 512, 576, 4352)]:
        g = gen(K + N)
        x = (torch.randn((C, F, K), generator=g, device=DEV) * 2).to(T(dtype))
        w = (torch.randn((N, K), generator=g, device=DEV) / K ** 0.5).to(T(dtype))
        b, res = torch.randn(N, generator=g, device=DEV), torch.randn((C, F, N), generator=g, device=DEV).to(T(out))
        layer = Layer(w, b, dtype, act)
        got = layer.apply(x, res.clone(), 0.75, None, 0.0).double()
        want, err = R.layer64(x, w, b, act, 0.75, None, 0.0, out)
        assert ((got - want).abs() <= err).all(), (C, F, K, N)
        inout = res.clone()   # the residual in place
        layer.apply(x, inout, 0.75, inout, 0.5)
        want, err = R.layer64(x, w, b, act, 0.75, res, 0.5, out)
        assert ((inout.double() - want).abs() <= err).all(), (C, F, K, N)
        layer.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_million_rows_of_three_outputs(dtype):
    import torch
    g = gen(4)
    rows = 65_535 * 32 + 21   # (more blocks of 16 and of 32 rows than a grid's second dimension has)
    x, w = whole((1, rows, 8), dtype, g), whole((3, 8), dtype, g)
    layer = Layer(w, None, dtype)
    for n in (rows, 65_535 * 16, 65_535 * 16 + 1):
        got = layer.apply(x[:, :n], torch.full((1, n, 3), 7.0, device=DEV))
        assert torch.equal(got, (x[:, :n].double() @ w.double().t()).float())
    layer.close()


@pytest.mark.parametrize("act", ["sigmoid", "tanh", "gelu", "silu"])
def test_activations_at_the_ends_of_their_range(act):
    """One input, weight 1: the activation itself, at large values of both signs, at zero and at infinity."""
    import torch
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5.0, -5.0, 20.0, -20.0, 88.0, -88.0, 89.0, -89.0, 104.0, -104.0, 1e4, -1e4, 3e38, -3e38, INF, -INF], device=DEV)
    layer = Layer(torch.ones((1, 1), device=DEV), None, "f32", act)
    got = layer.apply(v[None, :, None], torch.empty((1, v.numel(), 1), device=DEV))[0, :, 0].double()
    want = R.act64(act, v.double())
    if act in ("gelu", "silu"):
        want[-1] = float("nan")   # (-inf times zero)
    ok = (got - want).abs() <= 8 * 2.0 ** -24 * v.double().abs().clamp(min=1.0, max=104.0)
    ok |= (got == want) | (got.isnan() & want.isnan()) | ((got - want).abs() <= 8 * 2.0 ** -24 * want.abs())
    assert ok.all(), (got, want)
    layer.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C,F,K,N", [(1, 1, 96, 40), (3, 5, 100, 70), (4, 9, 64, 64), (6, 50, 72, 270), (7, 33, 200, 1021),
                                     (32, 33, 100, 511), (11, 97, 72, 1032), (9, 300, 40, 1700)])
def test_layouts(dtype, C, F, K, N):
    """Chunks of longer buffers, frames outermost, rows that overlap, pointers aligned to one element only; what lies
    between the rows is neither read into results nor written."""
    import torch
    g = gen(C * F + K)
    w = whole((N, K + 5), dtype, g)
    w[:, K:] = float("nan")
    layer = Layer(w[:, :K], None, dtype)

    def check(x, make_out, name):
        out, everything = make_out(7.0)   # (the rows are a view of `everything`)
        layer.apply(x, out)
        assert torch.equal(out, (x.double() @ w[:, :K].double().t()).float()), name
        out.fill_(7.0)
        assert torch.equal(everything, torch.full_like(everything, 7.0)), name + ": something else was written"

    def packed(v):
        o = torch.full((C, F, N), v, device=DEV)
        return o, o

    def gaps(v):   # odd gaps after every row, a longer buffer
        o = torch.full((C, F + 2, N + 3), v, device=DEV)
        return o[:, 1:1 + F, 2:2 + N], o

    def frames_first(v):
        o = torch.full((F, C, N), v, device=DEV)
        return o.transpose(0, 1), o

    nan = float("nan")
    x0 = whole((C, F, K), dtype, g)
    for out_name, make in (("packed", packed), ("gaps", gaps), ("frames first", frames_first)):
        check(x0, make, out_name)
        long = torch.full((C, F + 7, K + 3), nan, device=DEV, dtype=T(dtype))
        long[:, 4:4 + F, 1:1 + K] = x0
        check(long[:, 4:4 + F, 1:1 + K], make, "part of a longer buffer, " + out_name)
        long = torch.full((C, F, K + 8), nan, device=DEV, dtype=T(dtype))
        long[:, :, :K] = x0
        check(long[:, :, :K], make, "padded rows, " + out_name)
        ff = x0.transpose(0, 1).contiguous().transpose(0, 1)
        check(ff, make, "frames first, " + out_name)
        flat = torch.full((C * F * K + 1,), nan, device=DEV, dtype=T(dtype))
        flat[1:] = x0.flatten()
        check(flat[1:].view(C, F, K), make, "one element off, " + out_name)
        step = 3 if K % 2 else 8
        line = whole((C, K + step * F), dtype, g)
        check(torch.as_strided(line, (C, F, K), (line.stride(0), step, 1)), make, "overlapping rows, " + out_name)
        check(x0[:1].expand(C, F, K), make, "one channel's rows for all, " + out_name)
    # the residual may be the output
    out = whole((C, F, N), "f32", g)
    want = (x0.double() @ w[:, :K].double().t()).float() - out
    layer.apply(x0, out, 1.0, out, -1.0)
    assert torch.equal(out, want)
    layer.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(5, 40, 24), (70, 136, 100), (300, 264, 520), (1067, 264, 1032), (1056, 136, 511)])
def test_what_is_not_finite_stays_in_its_row_and_column(dtype, rows, K, N):
    import torch
    g = gen(rows)
    x, w = whole((1, rows, K), dtype, g), whole((N, K), dtype, g)
    x[0, 3, K - 1] = float("nan")
    x[0, rows - 1, 0] = INF
    w[N - 1, 2] = float("nan")
    layer = Layer(w, None, dtype, "relu")
    got = layer.apply(x, torch.zeros((1, rows, N), device=DEV))[0]
    clean = torch.ones((rows, N), dtype=torch.bool, device=DEV)
    clean[3], clean[rows - 1], clean[:, N - 1] = False, False, False
    want = (x[0].double() @ w.double().t()).clamp(min=0).float()
    assert torch.equal(got[clean], want[clean])
    assert got[3].isnan().all() and got[:, N - 1].isnan().all()
    layer.close()


def test_rounding_to_the_output_type_saturates_to_infinity_and_keeps_small_values():
    import torch
    w = torch.ones((1, 1), device=DEV)
    layer = Layer(w, None, "f32")
    v = torch.tensor([65504.0, 65519.9, 65520.0, -70000.0, 2.0 ** -24, 2.0 ** -26, 1 + 2.0 ** -11, 1 + 3 * 2.0 ** -11], device=DEV)
    for out in ("f16", "bf16"):
        got = layer.apply(v[None, :, None], torch.empty((1, v.numel(), 1), device=DEV, dtype=T(out)))
        assert torch.equal(got[0, :, 0], v.to(T(out)))
    layer.close()


def test_far_rows():
    """Rows whose offset in elements passes 32 bits."""
    import torch
    K, N = 64, 32
    g = gen(5)
    w = whole((N, K), "bf16", g)
    layer = Layer(w, None, "bf16")
    big = torch.empty((2 ** 31 + 2 ** 20,), device=DEV, dtype=torch.bfloat16)
    x = whole((2, 3, K), "bf16", g)
    far = torch.as_strided(big, (2, 3, K), (2 ** 31 + 64, 128, 1))
    far.copy_(x)
    bigout = torch.empty((2 ** 31 + 2 ** 20,), device=DEV, dtype=torch.bfloat16)
    out = torch.as_strided(bigout, (2, 3, N), (2 ** 31 + 32, 64, 1))
    layer.apply(far, out)
    assert torch.equal(out, (x.double() @ w.double().t()).float().to(torch.bfloat16))
    layer.close()


def test_streams_graphs_and_repeats():
    """Two streams at once, a captured call replayed with new inputs between the program's own work, equal bits always."""
    import torch
    g = gen(9)
    K, N, C, F = 520, 300, 4, 24
    w = torch.randn((N, K), generator=g, device=DEV).to(torch.bfloat16)
    layer = Layer(w, None, "bf16", "gelu")
    x = torch.randn((C, F, K), generator=g, device=DEV).to(torch.bfloat16)
    out = layer.apply(x, torch.empty((C, F, N), device=DEV))
    first = out.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = torch.empty_like(out)
    for _ in range(3):
        layer.apply(x, other, stream=side)
        layer.apply(x, out)
    torch.cuda.synchronize()
    assert torch.equal(out, first) and torch.equal(other, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.apply(x, out)
    for k in range(4):
        x.copy_(torch.randn((C, F, K), generator=g, device=DEV))
        other = layer.apply(x, torch.empty_like(out))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other), k
    layer.close()


def test_refusals():
    import torch
    w = torch.zeros((8, 16), device=DEV)
    layer = Layer(w, None, "f32")
    x, o = torch.zeros((4, 4, 16), device=DEV), torch.full((4, 4, 8), 3.0, device=DEV)
    good = dict(n_channels=4, n_frames=4, input_ptr=x.data_ptr(), input_channel_stride=64, input_frame_stride=16,
                output_ptr=o.data_ptr(), output_channel_stride=32, output_frame_stride=8)
    bad = [dict(n_channels=-1), dict(n_frames=-1), dict(input_ptr=0), dict(output_ptr=0), dict(output_dtype=3),
           dict(output_dtype=-1), dict(scale=INF), dict(scale=float("nan")), dict(input_channel_stride=-1),
           dict(input_frame_stride=-16), dict(output_frame_stride=7), dict(output_channel_stride=31),
           dict(output_channel_stride=-32), dict(input_ptr=x.data_ptr() + 2), dict(output_ptr=o.data_ptr() + 1),
           dict(residual_ptr=o.data_ptr() + 2), dict(residual_ptr=o.data_ptr(), residual_channel_stride=32, residual_frame_stride=0),
           dict(residual_ptr=x.data_ptr(), residual_scale=INF), dict(residual_ptr=x.data_ptr(), residual_frame_stride=-1),
           dict(output_ptr=x.data_ptr()), dict(n_channels=65536, n_frames=65536, output_channel_stride=1 << 30),
           dict(n_channels=1 << 15, n_frames=1 << 14, output_channel_stride=1 << 18),
           dict(input_channel_stride=1 << 61), dict(output_channel_stride=8, output_frame_stride=9)]
    for kw in bad:
        with pytest.raises(B.CbdError) as e:
            B.cbd_layer_apply(layer.h, **{**good, **kw})
        assert e.value.status == B.CBD_E_INVALID, kw
    for kw in (dict(n_channels=0), dict(n_frames=0), dict(n_channels=0, input_ptr=0, output_ptr=0)):
        B.cbd_layer_apply(layer.h, **{**good, **kw})
    torch.cuda.synchronize()
    assert (o == 3.0).all()
    B.cbd_layer_apply(layer.h, **good)
    torch.cuda.synchronize()
    assert (o == 0.0).all()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(B.CbdError):
            B.cbd_layer_create(w.data_ptr(), 16, 8, 0, hip_stream=side.cuda_stream)
        o.zero_()
    layer.close()
