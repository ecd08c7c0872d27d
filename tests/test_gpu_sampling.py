"""cbd_sample_labels against the rule in 64 bits (score_reference.sample_row).  Labels and counts have to be equal;
log-probabilities are rounded to fp32 once (half a step, 2^-24) and their total is summed in units
of 2^-min(50, 62 - log2 labels) from weights with a relative error of 2^-36."""
import math

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


def logprob_error(value, num_labels):
    """Rounding to fp32, and weights off by half a unit each."""
    bits = min(50, 62 - math.ceil(math.log2(num_labels)) if num_labels > 1 else 62)
    return 2.0 ** -24 * abs(value) + num_labels * 2.0 ** -(bits + 1) + 2.0 ** -36


class Sampler:
    def __init__(self, channels, labels):
        import torch
        self.C, self.N = channels, labels
        self.h = B.cbd_sampler_create(channels, labels, hip_stream=torch.cuda.current_stream().cuda_stream)

    def lists(self, channels, lists, offsets):
        B.cbd_sampler_set_contexts(self.h, channels, lists, offsets)

    def draw(self, x, random, dtype, channels=None, temperature=None, top_k=None, top_p=None, min_p=None, n=None, stride=None):
        """x: tensor of rows; settings: sequences or None -> numpy (labels, logprobs, kept)."""
        import torch
        n = x.shape[0] if n is None else n
        dev = lambda v, t: None if v is None else torch.as_tensor(np.asarray(v), dtype=t, device=DEV)  # noqa: E731
        f, i = torch.float32, torch.int32
        a = dict(random=dev(random, f), channels=dev(channels, i), temperature=dev(temperature, f), top_k=dev(top_k, i),
                 top_p=dev(top_p, f), min_p=dev(min_p, f))
        self.out = labels, logprobs, kept = [torch.full((n + 2,), 77, device=DEV, dtype=t) for t in (i, f, i)]
        B.cbd_sample_labels(self.h, n, x.data_ptr(), x.stride(0) if stride is None else stride, B.DTYPES[dtype],
                            labels_ptr=labels.data_ptr(), logprobs_ptr=logprobs.data_ptr(), kept_ptr=kept.data_ptr(),
                            **{k + "_ptr": v.data_ptr() if v is not None else 0 for k, v in a.items()})
        torch.cuda.synchronize()
        for t in self.out:
            assert (t[n:] == 77).all()   # nothing behind the last row
        return [t[:n].cpu().numpy() for t in self.out]

    def close(self):
        B.cbd_sampler_free(self.h)


def check(got, want, num_labels, where):
    label, logprob, kept = got
    wl, wp, wk = want
    assert int(label) == wl and int(kept) == wk, (where, got, want)
    if wl < 0:
        assert logprob == -INF, where
    else:
        assert abs(float(logprob) - wp) <= logprob_error(wp, num_labels), (where, got, want)


def check_rows(s, x, random, dtype, lists=None, offsets=None, channels=None, **settings):
    got = s.draw(x, random, dtype, channels=channels, **settings)
    rows = x.float().cpu().numpy()
    f32 = lambda name, r: float(np.float32(settings[name][r])) if settings.get(name) is not None else None  # noqa: E731
    for r in range(rows.shape[0]):
        kw = {k: f32(k, r) for k in ("temperature", "top_p", "min_p") if settings.get(k) is not None}
        if settings.get("top_k") is not None:
            kw["top_k"] = int(settings["top_k"][r])
        c = r if channels is None else channels[r]
        if lists is not None:
            kw.update(listed=lists[c], offset=offsets[c])
        check([v[r] for v in got], R.sample_row(rows[r], float(np.float32(random[r])), **kw), s.N, (dtype, s.N, r, kw))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,labels", [(3, 1), (5, 2), (7, 40), (4, 63), (4, 64), (4, 65), (9, 200), (6, 1000), (5, 1023), (5, 1025), (8, 2049), (6, 4097),
                                         (5, 6000), (4, 8191), (3, 16385), (3, 20_000), (3, 33_000), (2, 65_537), (2, 131_075), (2, 200_000)])
def test_settings(dtype, rows, labels):
    """Every combination of the truncations, at several scales of the scores, with lists."""
    import torch
    rng = np.random.default_rng(labels)
    g = torch.Generator(device=DEV)
    g.manual_seed(labels)
    s = Sampler(rows, labels)
    lists = [rng.integers(0, labels, rng.integers(0, 30)) for _ in range(rows)]
    offsets = rng.uniform(-4, 4, rows).astype(np.float32)
    for n, sigma in enumerate((0.3, 1.0, 4.0)):
        x = torch.log_softmax(torch.randn((rows, labels), generator=g, device=DEV) * sigma, dim=1)
        if n == 1:
            x.masked_fill_(torch.rand((rows, labels), generator=g, device=DEV) < 0.4, -INF)
        x = x.to(T(dtype))
        if n == 2:
            s.lists(range(rows), lists, offsets)
        kw = dict(lists=lists, offsets=offsets) if n == 2 else {}
        u = lambda: rng.random(rows).astype(np.float32)  # noqa: E731
        t = rng.uniform(0.3, 2.0, rows)
        k = rng.integers(1, max(2, min(labels, 300)), rows)
        for case in (dict(), dict(temperature=t), dict(top_k=k), dict(top_p=rng.uniform(0.1, 0.99, rows)),
                     dict(min_p=rng.uniform(0.001, 0.5, rows)), dict(temperature=t, top_k=k, top_p=rng.uniform(0.5, 0.99, rows)),
                     dict(temperature=t, top_k=k, top_p=rng.uniform(0.5, 0.99, rows), min_p=rng.uniform(0.0001, 0.1, rows)),
                     dict(top_k=rng.integers(1, labels + 1, rows), min_p=rng.uniform(0.0001, 0.1, rows)),
                     dict(temperature=np.where(np.arange(rows) % 2, 0.0, t), top_p=rng.uniform(0.1, 0.99, rows))):
            check_rows(s, x, u(), dtype, **case, **kw)
    s.close()


def test_settings_at_their_borders():
    """Off values, values beyond the range, NaN, and random numbers at both ends."""
    import torch
    nan = float("nan")
    x = torch.tensor([[0.5, 2.0, -1.0, 2.0, 1.0, -INF]], device=DEV)
    s = Sampler(1, 6)
    one = lambda u=0.4, **kw: tuple(v[0] for v in s.draw(x, [u], "f32", **{k: [v] for k, v in kw.items()}))  # noqa: E731
    row = x[0].cpu().numpy()
    for kw, same in ((dict(top_k=0), {}), (dict(top_k=-3), {}), (dict(top_k=6), {}), (dict(top_k=2 ** 31 - 1), {}), (dict(top_p=1.0), {}),
                     (dict(top_p=7.0), {}), (dict(top_p=nan), {}), (dict(min_p=0.0), {}), (dict(min_p=-1.0), {}), (dict(min_p=nan), {}),
                     (dict(top_p=0.0), dict(top_k=1)), (dict(top_p=-1.0), dict(top_k=1)), (dict(min_p=1.0), dict(top_k=2)),
                     (dict(min_p=5.0), dict(top_k=2)), (dict(top_p=1e-30), dict(top_k=1)), (dict(temperature=INF, top_k=3), dict(temperature=1e30, top_k=3)),
                     (dict(temperature=1e-30), dict(temperature=1e-30)), (dict(temperature=1e30), {"temperature": 1e30})):
        for u in (0.0, 0.1, 0.3, 0.6, 0.99):
            check(one(u, **kw), R.sample_row(row, float(np.float32(u)), **same), 6, (kw, u))
    for t in (0.0, -0.0, -1.0, nan, -INF):
        assert one(0.9, temperature=t) == (1, 0.0, 1)
    for u, label in ((0.0, 0), (-1.0, 0), (nan, 0), (1.0, 4), (2.0, 4), (INF, 4), (1.0 - 2.0 ** -24, 4)):
        assert one(u)[0] == label, u
    assert one(0.0, top_k=2)[0] == 1 and one(1.0, top_k=2)[0] == 3
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("labels", [5, 300, 6_000, 70_000])
def test_rows_with_little_or_nothing_in_them(dtype, labels):
    import torch
    lowest = torch.finfo(T(dtype)).min
    x = torch.full((9, labels), -INF, device=DEV)
    x[1] = float("nan")
    x[2] = lowest                      # all equal: uniform
    x[3, labels - 1] = -1e4            # one label
    x[4] = lowest; x[4, 3] = 1.0       # masked by the lowest value: never chosen  # noqa: E702
    x[5, 2] = INF; x[5, 4] = INF; x[5, 1] = 5.0  # noqa: E702
    x[6] = -0.0; x[6, 3] = 0.0         # equal zeros  # noqa: E702
    x[7, 0] = float("nan"); x[7, 1] = 0.25; x[7, 4] = float("nan")  # noqa: E702
    x[8] = 3.0                         # all equal
    x = x.to(T(dtype))
    s = Sampler(9, labels)
    for u in (0.0, 0.3, 0.5, 0.999):
        for kw in ({}, dict(top_k=[3] * 9), dict(top_p=[0.5] * 9), dict(min_p=[0.3] * 9), dict(temperature=[0.0] * 9),
                   dict(temperature=[0.7] * 9, top_k=[4] * 9, top_p=[0.9] * 9)):
            check_rows(s, x, [u] * 9, dtype, **kw)
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("labels", [100, 3_000, 30_000, 150_000])
def test_ties(dtype, labels):
    """Few distinct values: the cut falls inside a run of equal scores, kept from the lowest label on."""
    import torch
    rng = np.random.default_rng(labels)
    rows = 6
    x = torch.from_numpy(rng.integers(0, 4, (rows, labels)).astype(np.float32)).to(DEV)
    x[4] = 1.0
    x[5, :] = 0.0
    x[5, labels // 2:] = 2.0
    x = x.to(T(dtype))
    s = Sampler(rows, labels)
    for _ in range(3):
        check_rows(s, x, rng.random(rows), dtype, top_k=rng.integers(1, labels, rows))
        check_rows(s, x, rng.random(rows), dtype, top_p=rng.uniform(0.05, 0.95, rows))
        check_rows(s, x, rng.random(rows), dtype, top_k=rng.integers(1, labels, rows), top_p=rng.uniform(0.05, 0.95, rows),
                   temperature=rng.uniform(0.5, 2, rows))
    check_rows(s, x, [0.5] * rows, dtype, top_p=[0.5] * rows)
    s.close()


@pytest.mark.parametrize("labels", [4_000, 120_000])
def test_scores_that_crowd_or_spread(labels):
    """Values one step apart, values over the whole range of fp32, and far outliers: the cut is found at any scale."""
    import torch
    rng = np.random.default_rng(5)
    base = np.float32(-7.5)
    crowd = (base.view(np.int32) + rng.integers(0, 50, labels)).astype(np.int32).view(np.float32)
    spread = (rng.integers(0, 2 ** 31 - 2 ** 24, labels).astype(np.int64) | (rng.integers(0, 2, labels) << 31)).astype(np.uint32).view(np.float32)
    spread = np.where(np.isfinite(spread), spread, 0.0).astype(np.float32)
    outlier = rng.normal(0, 1, labels).astype(np.float32)
    outlier[17] = 1e6
    deep = rng.normal(0, 1, labels).astype(np.float32)
    deep[rng.random(labels) < 0.9] = -1e5
    small = rng.normal(0, 1e-30, labels).astype(np.float32)
    x = torch.from_numpy(np.stack([crowd, spread, outlier, deep, small])).to(DEV)
    s = Sampler(5, labels)
    for k in (1, 7, 64, 1000, labels // 2, labels - 1):
        check_rows(s, x, rng.random(5), "f32", top_k=[k] * 5)
        check_rows(s, x, rng.random(5), "f32", top_k=[k] * 5, top_p=[0.8] * 5)
    for p in (1e-6, 0.3, 0.9, 0.999):
        check_rows(s, x, rng.random(5), "f32", top_p=[p] * 5)
        check_rows(s, x, rng.random(5), "f32", top_p=[p] * 5, temperature=[1e-3, 1e5, 1e5, 30.0, 1e-29])
    for m in (1e-6, 0.5, 0.99999):
        check_rows(s, x, rng.random(5), "f32", min_p=[m] * 5)
    s.close()


def test_rows_lists_and_strides():
    """Rows by channel, one channel several times, one row several times, odd strides and starts, channels out of range."""
    import torch
    rng = np.random.default_rng(11)
    C, N = 5, 777
    s = Sampler(C, N)
    lists = [rng.integers(0, N, n) for n in (0, 1, 50, 777, 3)]
    lists[2] = np.concatenate([lists[2], lists[2][::-1], [N - 1, 0, 0]])
    offsets = np.array([5.0, 3.0, -2.5, 1.0, 4.0], np.float32)
    s.lists(range(C), lists, offsets)
    for dtype in ("f32", "bf16", "f16"):
        for stride, start in ((777, 0), (777, 1), (780, 3), (800, 8)):
            buf = torch.full((12 * stride + start + 1,), float("nan"), device=DEV, dtype=T(dtype))
            x = torch.as_strided(buf, (8, N), (stride, 1), start)
            x.copy_(torch.from_numpy(rng.normal(0, 2, (8, N)).astype(np.float32)).to(DEV))
            check_rows(s, x, rng.random(8), dtype, lists, offsets, channels=[4, 2, 2, 0, 3, 1, 2, 4], top_p=[0.9] * 8)
        one = x[:1].expand(6, N)
        check_rows(s, one, rng.random(6), dtype, lists, offsets, channels=[2, 2, 2, 2, 2, 1], top_k=[40] * 6)
    got = s.draw(x.float().contiguous(), [0.5] * 4, "f32", channels=[1, -1, 5, 2 ** 31 - 1], n=4)
    assert got[0][0] >= 0 and (got[0][1:] == -1).all() and (got[1][1:] == -INF).all() and (got[2][1:] == 0).all()
    # lists replaced and cleared, the others as they were
    s.lists([3, 1], [[5, 6], []], [2.0, 9.0])
    lists[3], lists[1], offsets[3] = np.array([5, 6]), np.array([], int), 2.0
    x = torch.from_numpy(rng.normal(0, 2, (C, N)).astype(np.float32)).to(DEV)
    check_rows(s, x, rng.random(C), "f32", lists, offsets, min_p=[0.05] * C)
    s.close()


def test_long_lists_of_many_channels():
    """More list entries than one upload holds."""
    import torch
    rng = np.random.default_rng(3)
    C, N = 60, 5_000
    lists = [rng.integers(0, N, 2_000) for _ in range(C)]
    offsets = rng.uniform(0, 3, C).astype(np.float32)
    s = Sampler(C, N)
    s.lists(range(C), lists, offsets)
    x = torch.from_numpy(rng.normal(0, 1.5, (C, N)).astype(np.float32)).to(DEV)
    check_rows(s, x, rng.random(C), "f32", lists, offsets, top_p=[0.8] * C)
    s.close()


def test_far_rows():
    """Rows whose offset in elements passes 32 bits."""
    import torch
    N, rng = 300, np.random.default_rng(2)
    buf = torch.empty((2 ** 32 + 2 ** 12,), device=DEV, dtype=torch.bfloat16)
    x = torch.as_strided(buf, (3, N), (2 ** 31 + 10, 1))
    x.copy_(torch.from_numpy(rng.normal(0, 2, (3, N)).astype(np.float32)).to(DEV))
    s = Sampler(3, N)
    check_rows(s, x, rng.random(3), "bf16", top_k=[9] * 3)
    s.close()


def test_captured_call_replays_with_new_values():
    import torch
    rng = np.random.default_rng(8)
    C, N = 6, 9_000
    s = Sampler(C, N)
    stream = torch.cuda.Stream()
    B.cbd_sampler_free(s.h)
    s.h = B.cbd_sampler_create(C, N, hip_stream=stream.cuda_stream)
    x = torch.zeros((C, N), device=DEV)
    u, p = torch.zeros(C, device=DEV), torch.ones(C, device=DEV)
    label, lp, kept = torch.zeros(C, dtype=torch.int32, device=DEV), torch.zeros(C, device=DEV), torch.zeros(C, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.cbd_sample_labels(s.h, C, x.data_ptr(), N, 0, u.data_ptr(), label.data_ptr(), top_p_ptr=p.data_ptr(),
                            logprobs_ptr=lp.data_ptr(), kept_ptr=kept.data_ptr())
        with pytest.raises(B.CbdError):
            s.lists([0], [[1]], [1.0])
        with pytest.raises(B.CbdError):
            B.cbd_sampler_create(C, N, hip_stream=stream.cuda_stream)
        with pytest.raises(B.CbdError):
            B.cbd_sampler_free(s.h)
    for k in range(4):
        rows, uu, pp = rng.normal(0, 2, (C, N)).astype(np.float32), rng.random(C).astype(np.float32), rng.uniform(0.3, 0.95, C).astype(np.float32)
        x.copy_(torch.from_numpy(rows)); u.copy_(torch.from_numpy(uu)); p.copy_(torch.from_numpy(pp))  # noqa: E702
        lists = [rng.integers(0, N, 40) for _ in range(C)]
        s.lists(range(C), lists, [2.0] * C)
        torch.cuda.synchronize()
        label.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in (label, lp, kept)]
        for r in range(C):
            check([v[r] for v in got], R.sample_row(rows[r], float(uu[r]), top_p=float(pp[r]), listed=lists[r], offset=2.0), N, (k, r))
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("labels", [1_030, 4_099, 20_000, 40_003])
def test_few_labels_wherever_they_are(labels, dtype):
    """top_k and min_p on rows whose best labels lie behind one another, are equal, are few, or are infinite."""
    import torch
    rng = np.random.default_rng(labels)
    N = labels
    rows = [np.sort(rng.normal(0, 3, N)), np.sort(rng.normal(0, 3, N))[::-1], np.zeros(N), rng.normal(0, 3, N)]
    for n in (1, 49, 50, 51, 127, 128, 129, 300):   # labels that are not masked, in one stretch and spread
        near, spread = np.full(N, -INF), np.full(N, -INF)
        near[500:500 + n] = rng.normal(0, 2, n)
        spread[rng.choice(N, n, replace=False)] = rng.normal(0, 2, n)
        rows += [near, spread]
    for n in (40, 50, 300):   # equal best ones
        x = rng.normal(0, 1, N)
        x[rng.choice(N, n, replace=False)] = 9.0
        rows.append(x)
        rows.append(np.where(x == 9.0, INF, x))
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).to(DEV).to(T(dtype))
    s = Sampler(len(rows), N)
    for k in (1, 50, 128, 129):
        u = rng.random(len(rows))
        check_rows(s, x, u, dtype, top_k=[k] * len(rows))
        check_rows(s, x, u, dtype, top_k=[k] * len(rows), top_p=[0.75] * len(rows), temperature=[2.0] * len(rows))
    for m in (0.5, 1e-3, 1e-6):
        check_rows(s, x, rng.random(len(rows)), dtype, min_p=[m] * len(rows))
    s.close()


@pytest.mark.parametrize("with_channels", [True, False])
def test_more_rows_than_one_launch_takes(with_channels):
    """2^21 + 70 rows of five scores; row i's best label is i mod 5."""
    import torch
    n, N = 2 ** 21 + 70, 5
    s = Sampler(n if not with_channels else 3, N)
    at = torch.arange(n, device=DEV, dtype=torch.int32)
    x = torch.full((n, N), -100.0, device=DEV, dtype=torch.float16)
    x.scatter_(1, (at % N).long()[:, None], 100.0)
    u, labels, kept = torch.rand(n, device=DEV), torch.full((n + 1,), 77, device=DEV, dtype=torch.int32), torch.zeros(n, device=DEV, dtype=torch.int32)
    top_p = torch.full((n,), 0.5, device=DEV)
    which = 2 * (at >= 2 ** 21).int()
    # raised by 300: of channel 2 (the rows behind the first 2^21), or of one row there and one before it
    s.lists([2], [[3]], [300.0]) if with_channels else s.lists([2 ** 21 - 1, 2 ** 21 + 66], [[3], [4]], [300.0, 300.0])
    B.cbd_sample_labels(s.h, n, x.data_ptr(), N, B.DTYPES["f16"], u.data_ptr(), labels.data_ptr(), top_p_ptr=top_p.data_ptr(),
                        channels_ptr=which.data_ptr() if with_channels else 0, kept_ptr=kept.data_ptr())
    torch.cuda.synchronize()
    want = at % N
    if with_channels:
        want[2 ** 21:] = 3
    else:
        want[2 ** 21 - 1], want[2 ** 21 + 66] = 3, 4
    assert torch.equal(labels[:n], want) and int(labels[n]) == 77 and (kept == 1).all()
    s.close()


def test_two_samplers_beside_each_other():
    """Two threads, a stream and a sampler each, the same rows: both draw what one draws alone."""
    import threading
    import torch
    n, N = 300, 7_000
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x, u = torch.randn((n, N), generator=g, device=DEV) * 3, torch.rand(n, generator=g, device=DEV)
    p = torch.full((n,), 0.9, device=DEV)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros((20, n), dtype=torch.int32, device=DEV) for _ in range(3)]
    samplers = [B.cbd_sampler_create(n, N, hip_stream=st.cuda_stream) for st in [torch.cuda.current_stream()] + streams]
    torch.cuda.synchronize()

    def draw(i):
        torch.cuda.set_device(0)
        for j in range(20):
            B.cbd_sampler_set_contexts(samplers[i], range(n), [[(c + j) % N, 5] for c in range(n)], [2.0] * n)
            B.cbd_sample_labels(samplers[i], n, x.data_ptr(), N, 0, u.data_ptr(), outs[i][j].data_ptr(), top_p_ptr=p.data_ptr())

    draw(0)
    threads = [threading.Thread(target=draw, args=(i,)) for i in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    for s in samplers:
        B.cbd_sampler_free(s)


def test_frequencies_follow_the_weights():
    """Random numbers in equal steps choose every kept label in proportion to its weight: n steps of 1/n hit a label of
    probability q at least floor(q n) and at most ceil(q n) times."""
    import torch
    n = 4_096
    x = torch.tensor([[1.0, -INF, 0.0, 2.0, -1.0, 0.5, 0.0]], device=DEV)
    s = Sampler(1, 7)
    u = (np.arange(n) / n).astype(np.float32)
    label, _, _ = s.draw(x, u, "f32", channels=[0] * n, n=n, stride=0, temperature=[0.8] * n)
    q = np.exp(x[0].cpu().numpy().astype(np.float64) / float(np.float32(0.8)))
    q /= q.sum()
    hits = np.bincount(label, minlength=7)
    assert (hits >= np.floor(q * n)).all() and (hits <= np.ceil(q * n)).all() and hits[1] == 0
    s.close()


def test_refusals():
    import torch
    s = Sampler(4, 10)
    x, out = torch.zeros((4, 10), device=DEV), torch.full((4,), 5, dtype=torch.int32, device=DEV)
    u = torch.zeros(4, device=DEV)
    good = dict(n=4, scores_ptr=x.data_ptr(), row_stride=10, dtype=0, random_ptr=u.data_ptr(), labels_ptr=out.data_ptr())
    for kw in (dict(n=-1), dict(n=5), dict(scores_ptr=0), dict(random_ptr=0), dict(labels_ptr=0), dict(dtype=3), dict(dtype=-1),
               dict(row_stride=-1), dict(row_stride=1 << 61), dict(scores_ptr=x.data_ptr() + 2), dict(labels_ptr=out.data_ptr() + 2),
               dict(top_k_ptr=u.data_ptr() + 1), dict(channels_ptr=u.data_ptr() + 2)):
        with pytest.raises(B.CbdError) as e:
            B.cbd_sample_labels(s.h, **{**good, **kw})
        assert e.value.status == B.CBD_E_INVALID, kw
    B.cbd_sample_labels(s.h, **{**good, "n": 0})
    for args in (([4], [[1]], [1.0]), ([-1], [[1]], [1.0]), ([0, 0], [[1], [2]], [1.0, 1.0]), ([0], [[10]], [1.0]), ([0], [[-1]], [1.0]),
                 ([0], [[1]], [INF]), ([0], [[1]], [float("nan")]), ([], [], [])):
        with pytest.raises(B.CbdError) as e:
            s.lists(*args)
        assert e.value.status == B.CBD_E_INVALID, args
    for packed in (([1, 2], [1, 2]), ([1, 2], [0, -1])):
        with pytest.raises(B.CbdError):
            B.cbd_sampler_set_contexts(s.h, [0], None, [1.0], packed=tuple(np.array(v, np.int32) for v in packed))
    with pytest.raises(ValueError):
        s.lists([0, 1], [[1], [2]], [1.0])
    torch.cuda.synchronize()
    assert (out == 5).all()
    B.cbd_sample_labels(s.h, **good)   # none of the refused lists took effect: labels 0, equal scores
    torch.cuda.synchronize()
    assert (out == 0).all()
    s.close()
