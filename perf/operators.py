"""The operators on either side of the decoder's score rows, as timed passes: sizes, inputs, one pass, and the work it
cannot do without.

Kinds of case:
  layer   one affine layer of the network that makes the score rows, over a chunk of frames of every channel:
          out = scale * act(x W^T + bias) + residual_scale * residual  (`cbd_layer_apply`)
  sample  one label per row of scores, for models whose labels are drawn one after the other instead of being searched
          through a graph: boosted labels per channel, temperature, top-k, top-p, min-p  (`cbd_sample_labels`)

Rows of a layer are addressed by channel and frame, as in the decoder's log-likelihoods.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "sigmoid", "tanh", "gelu", "silu")


def _layer(name, channels, frames, held, inputs, outputs, dtype, out, act="none", scale=1.0, residual=0.0, bias=True):
    """held: frames of the buffer the chunk is a part of (channel stride); residual: its scale, 0 = none."""
    c = dict(kind="layer", channels=channels, frames=frames, held=held, inputs=inputs, outputs=outputs, dtype=dtype, out=out,
             act=act, scale=scale, residual=residual, bias=bias)
    return dict(c, name=name) if name else c


def _sample(name, rows, labels, dtype, sigma, listed=0, temperature="one", top_k=0, top_p=1.0, min_p=0.0, masked=0.0):
    """listed: boosted labels a channel; temperature: "one" = 1 for all rows, "rows" = another for each, some of them 0;
    top_k, top_p, min_p: 0, 1, 0 = off, otherwise drawn per row around the value; masked: share of scores at -inf."""
    c = dict(kind="sample", rows=rows, labels=labels, dtype=dtype, sigma=sigma, listed=listed, temperature=temperature,
             top_k=top_k, top_p=top_p, min_p=min_p, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one live stream, one frame: the output layer's weights are read for a single row
        _layer("layer_frame", 1, 1, 1, 1024, 6000, "bf16", "f32"),
        # a step of 32 streams through a feed-forward layer with half-step residual
        _layer("layer_step", 32, 1, 1, 2048, 512, "f16", "f16", "none", 0.5, 1.0),
        # ten frames of a live stream in full precision, the bypass of a factored time-delay layer
        _layer("layer_live", 1, 10, 60, 512, 512, "f32", "f32", "relu", 1.0, 0.66),
        # sizes that fit no tile: an odd input width, an odd label count, a handful of channels
        _layer("layer_odd", 7, 33, 151, 771, 1021, "f16", "f32", "sigmoid"),
        # the output layer over a chunk of 32 recordings, in full precision
        _layer("layer_precise", 32, 50, 333, 512, 3000, "f32", "f32"),
        # an online server: 256 streams x 50 frames into a feed-forward block and out of it
        _layer("layer_wide", 256, 50, 50, 1024, 4096, "bf16", "bf16", "silu"),
        _layer("layer_scores", 256, 50, 500, 1024, 6000, "bf16", "f32"),
        # one live stream of an end-to-end model over a few units
        _sample("sample_live", 1, 600, "f32", 3.0, 20, "one", 40, 0.95),
        # a server's step over word pieces, rows with settings of their own
        _sample("sample_step", 64, 20_000, "bf16", 3.0, 100, "rows", 50, 0.95),
        # many clients over the labels of the large graph, cut at a share of the best label's probability
        _sample("sample_clients", 2_048, 6_000, "f32", 4.0, 300, "rows", 0, 1.0, 0.02, 0.1),
        # flat rows cut by mass alone: no small set of labels holds it
        _sample("sample_flat", 512, 5_003, "f16", 1.0, 50, "rows", 0, 0.9, 0.0, 0.3),
        # whole words as labels
        _sample("sample_words", 256, 200_000, "f32", 2.5, 300, "rows", 0, 0.92, 0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        inputs, outputs = _log_int(rng, 64, 4_096), _log_int(rng, 100, 6_000)
        if rng.random() < 0.6:   # widths of a network are mostly multiples of 64; label counts are what they are
            inputs = (inputs + 63) // 64 * 64
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        # at most the operations of the largest listed case (a sixteenth of them in f32)
        most = 256 * 50 * 1024 * 6000 // (16 if dtype == "f32" else 1) // (inputs * outputs)
        channels = _log_int(rng, 1, max(1, min(512, most)))
        frames = _log_int(rng, 1, max(1, min(64, most // channels, 12_800 // channels)))
        out = rng.choice(["f32", dtype])
        residual = rng.choice([0.0, 0.0, 0.66, 1.0])
        return _layer("", channels, frames, frames + rng.choice([0, rng.randint(1, 50)]), inputs, outputs, dtype, out,
                      rng.choice(ACTIVATIONS), rng.choice([1.0, 0.5]), residual, rng.random() < 0.8)
    labels = _log_int(rng, 40, 200_000)
    rows = _log_int(rng, 1, min(2_048, 51_200_000 // labels))
    return _sample("", rows, labels, rng.choice(["f32", "f16", "bf16"]), round(rng.uniform(1.0, 4.0), 2),
                   rng.choice([0, _log_int(rng, 1, min(labels, 500))]), rng.choice(["one", "rows"]),
                   rng.choice([0, _log_int(rng, 1, max(2, min(labels, 1_000)))]), rng.choice([1.0, round(rng.uniform(0.5, 0.98), 3)]),
                   rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 4)]), rng.choice([0.0, 0.0, 0.3]))


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _layer_inputs(case, seed):
    """Normalised hidden vectors, weights that keep their scale, a bias as label priors leave it."""
    g, t = _generator(seed), TYPES[case["dtype"]]
    C, T, K, N = case["channels"], case["held"], case["inputs"], case["outputs"]
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    x = randn(C, T, K).to(t)
    weight = (randn(N, K) / math.sqrt(K)).to(t)
    bias = randn(N) if case["bias"] else None
    residual = randn(C, case["frames"], N).to(TYPES[case["out"]]) if case["residual"] else None
    return x[:, T - case["frames"]:], weight, bias, residual


def _sample_inputs(case, seed):
    """Log-probabilities of a network's rows, settings as clients choose them, one random number a row."""
    g = _generator(seed)
    R, N = case["rows"], case["labels"]
    x = torch.randn((R, N), generator=g, device=DEV).mul_(case["sigma"])
    x = torch.log_softmax(x, dim=-1)
    if case["masked"]:
        x.masked_fill_(torch.rand((R, N), generator=g, device=DEV) < case["masked"], float("-inf"))
    x = x.to(TYPES[case["dtype"]])
    rand = lambda: torch.rand(R, generator=g, device=DEV)  # noqa: E731
    d = dict(scores=x, random=rand(), temperature=None, top_k=None, top_p=None, min_p=None, lists=None, offsets=None)
    if case["temperature"] == "rows":
        d["temperature"] = torch.where(rand() < 0.1, 0.0, 0.5 + rand())
    if case["top_k"]:
        d["top_k"] = (1 + rand() * (2 * case["top_k"] - 1)).to(torch.int32)
    if case["top_p"] < 1.0:
        d["top_p"] = case["top_p"] + (rand() - 0.5) * 0.04
    if case["min_p"]:
        d["min_p"] = case["min_p"] * (0.5 + rand())
    if case["listed"]:
        d["lists"] = torch.randint(0, N, (R, case["listed"]), generator=g, device=DEV, dtype=torch.int32)
        d["offsets"] = 1.0 + 4.0 * rand()
    return d


class _State:
    """The inputs of one pass, and what a program keeps beside them: buffers for the results and, where the framework's
    calls are made, the layer or the sampler with its channels' lists."""

    def __init__(self, case, seed):
        self.case = case
        self.handle = None
        if case["kind"] == "layer":
            self.x, self.weight, self.bias, self.residual = _layer_inputs(case, seed)
            self.out = torch.empty((case["channels"], case["frames"], case["outputs"]), dtype=TYPES[case["out"]], device=DEV)
        else:
            d = _sample_inputs(case, seed)
            self.__dict__.update(d)
            R = case["rows"]
            self.labels = torch.empty(R, dtype=torch.int32, device=DEV)
            self.logprobs = torch.empty(R, dtype=torch.float32, device=DEV)
            self.kept = torch.empty(R, dtype=torch.int32, device=DEV)
            self.listed = None
            if self.lists is not None and not own:
                self.listed = torch.zeros((R, case["labels"]), dtype=torch.bool, device=DEV)
                self.listed.scatter_(1, self.lists.long(), True)
        if own:
            from paper_2306_15685_amd import binding as B
            self.B = B
            self.stream = torch.cuda.current_stream().cuda_stream
            if case["kind"] == "layer":
                self.handle = B.cbd_layer_create(
                    self.weight.data_ptr(), case["inputs"], case["outputs"], B.DTYPES[case["dtype"]],
                    bias_ptr=self.bias.data_ptr() if self.bias is not None else 0, activation=B.ACTIVATIONS[case["act"]],
                    hip_stream=self.stream)
            else:
                self.handle = B.cbd_sampler_create(case["rows"], case["labels"], hip_stream=self.stream)
                if self.lists is not None:
                    B.cbd_sampler_set_contexts(self.handle, range(case["rows"]), self.lists.cpu().numpy(),
                                               self.offsets.cpu().numpy())

    def __del__(self):
        if self.handle is not None:
            (self.B.cbd_layer_free if self.case["kind"] == "layer" else self.B.cbd_sampler_free)(self.handle)


def prepare(case, seed):
    return _State(case, seed)


# ---- one pass --------------------------------------------------------------------------------------------------------


def _activation(name, y):
    if name == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if name == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-y))
    if name == "tanh":
        return torch.tanh(y)
    if name == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if name == "silu":
        return y / (1.0 + torch.exp(-y))
    return y


def _plain_layer(s):
    c = s.case
    y = torch.matmul(s.x.float(), s.weight.float().t())
    if s.bias is not None:
        y = y + s.bias
    y = c["scale"] * _activation(c["act"], y)
    if s.residual is not None:
        y = y + c["residual"] * s.residual.float()
    return y.to(TYPES[c["out"]])


def _plain_sample(s):
    """Order, truncation and choice as sorted rows and running sums; masses in 64 bits, since a label is chosen where a
    sum passes a border."""
    inf = float("inf")
    x = s.scores.float()
    R, N = x.shape
    if s.listed is not None:
        x = torch.where(s.listed, x + s.offsets[:, None], x)
    x = torch.where(torch.isnan(x), -inf, x)
    ordered, order = torch.sort(x, dim=1, descending=True, stable=True)
    best = ordered[:, :1].double()
    rank = torch.arange(N, device=x.device)
    d = torch.where(best == inf, torch.where(ordered == inf, 0.0, -inf), ordered.double() - best)
    d = torch.where(ordered == -inf, -inf, d)
    allowed = d > -inf
    if s.temperature is not None:
        T = s.temperature.double()[:, None]
        greedy = ~(T > 0)
        d = torch.where(greedy, d, d / T)
        allowed = allowed & (~greedy | (rank == 0))
    if s.top_k is not None:
        k = s.top_k[:, None]
        allowed = allowed & ((rank < k) | (k <= 0))
    d = torch.where(allowed, d, -inf)
    w = torch.exp(d)
    if s.top_p is not None:
        p = s.top_p.double()[:, None]
        before = torch.cumsum(w, 1) - w
        allowed = allowed & ((before < p * w.sum(1, keepdim=True)) | ~(p < 1) | (rank == 0))
    if s.min_p is not None:
        m = s.min_p.double()[:, None].clamp(max=1.0)
        allowed = allowed & ((w >= m) | ~(m > 0))
    w = torch.where(allowed, w, 0.0)
    d = torch.zeros_like(d).scatter_(1, order, d)
    w = torch.zeros_like(w).scatter_(1, order, w)
    run_w = torch.cumsum(w, 1)
    total = run_w[:, -1:]
    label = (run_w > s.random.double()[:, None] * total).to(torch.int8).argmax(1)
    some = total[:, 0] > 0
    logprob = torch.where(some, d.gather(1, label[:, None])[:, 0] - torch.log(total[:, 0]), -inf)
    return {"label": torch.where(some, label, -1).to(torch.int32), "logprob": logprob.float(), "kept": allowed.sum(1).to(torch.int32)}


def _own_layer(s):
    c, x, out = s.case, s.x, s.out
    residual = s.residual
    s.B.cbd_layer_apply(
        s.handle, c["channels"], c["frames"], x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
        s.B.DTYPES[c["out"]], scale=c["scale"], residual_ptr=residual.data_ptr() if residual is not None else 0,
        residual_channel_stride=residual.stride(0) if residual is not None else 0,
        residual_frame_stride=residual.stride(1) if residual is not None else 0, residual_scale=c["residual"],
        hip_stream=s.stream)
    return out


def _own_sample(s):
    c = s.case
    at = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    s.B.cbd_sample_labels(
        s.handle, c["rows"], s.scores.data_ptr(), s.scores.stride(0), s.B.DTYPES[c["dtype"]], s.random.data_ptr(),
        s.labels.data_ptr(), temperature_ptr=at(s.temperature), top_k_ptr=at(s.top_k), top_p_ptr=at(s.top_p),
        min_p_ptr=at(s.min_p), logprobs_ptr=s.logprobs.data_ptr(), kept_ptr=s.kept.data_ptr())
    return {"label": s.labels, "logprob": s.logprobs, "kept": s.kept}


def run(state):
    if state.case["kind"] == "layer":
        return (_own_layer if own else _plain_layer)(state)
    return (_own_sample if own else _plain_sample)(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------


def _exact_layer(case, seed):
    x, weight, bias, residual = _layer_inputs(case, seed)
    C, T, N = case["channels"], case["frames"], case["outputs"]
    y = torch.empty((C * T, N), dtype=torch.float64, device=DEV)
    rows, w = x.reshape(C * T, -1), weight.double().t().contiguous()
    for r in range(0, C * T, 4096):
        y[r:r + 4096] = rows[r:r + 4096].double() @ w
    if bias is not None:
        y += bias.double()
    act = case["act"]
    if act == "relu":
        y = y.clamp(min=0.0)
    elif act == "sigmoid":
        y = torch.special.expit(y)
    elif act == "tanh":
        y = torch.tanh(y)
    elif act == "gelu":
        y = y * 0.5 * torch.special.erfc(y * -math.sqrt(0.5))
    elif act == "silu":
        y = y * torch.special.expit(y)
    y = case["scale"] * y.reshape(C, T, N)
    if residual is not None:
        y += case["residual"] * residual.double()
    return y


def _exact_sample(case, seed):
    """Row by row: the kept labels found one condition after the other, then the choice among them."""
    d = _sample_inputs(case, seed)
    R = case["rows"]
    label, logprob, kept = [], [], []
    for r in range(R):
        x = d["scores"][r].float()
        if d["lists"] is not None:
            own_labels = torch.unique(d["lists"][r].long())
            x[own_labels] = x[own_labels] + d["offsets"][r]   # (the definition's one addition in 32 bits)
        x = x.double()
        keep = torch.nonzero(x > float("-inf")).flatten()   # labels in ascending order; NaN is not above -inf
        T = float(d["temperature"][r]) if d["temperature"] is not None else 1.0
        k = int(d["top_k"][r]) if d["top_k"] is not None else 0
        p = float(d["top_p"][r]) if d["top_p"] is not None else 1.0
        m = float(d["min_p"][r]) if d["min_p"] is not None else 0.0
        if keep.numel() == 0:
            label.append(-1), logprob.append(float("-inf")), kept.append(0)
            continue
        if not T > 0:
            label.append(int(keep[torch.argmax(x[keep])])), logprob.append(0.0), kept.append(1)
            continue
        by = torch.argsort(x[keep], descending=True, stable=True)
        keep = keep[by]
        if 0 < k < keep.numel():
            keep = keep[:k]
        logw = (x[keep] - x[keep[0]]) / T
        w = torch.exp(logw)
        n = keep.numel()
        if p < 1.0:
            upto = torch.cumsum(w, 0)
            n = min(n, max(1, 1 + int((upto < p * upto[-1]).sum())))
        if m > 0.0:
            n = min(n, int((w >= min(m, 1.0)).sum()))
        keep, logw, w = keep[:n], logw[:n], w[:n]
        back = torch.argsort(keep)
        upto = torch.cumsum(w[back], 0)
        at = back[int((upto <= float(d["random"][r]) * upto[-1]).sum().clamp(max=n - 1))]
        label.append(int(keep[at])), kept.append(n)
        logprob.append(float(logw[at] - torch.log(upto[-1])))
    return {"label": torch.tensor(label, dtype=torch.int32, device=DEV), "logprob": torch.tensor(logprob, dtype=torch.float64, device=DEV),
            "kept": torch.tensor(kept, dtype=torch.int32, device=DEV)}


def exact(case, seed):
    return (_exact_layer if case["kind"] == "layer" else _exact_sample)(case, seed)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    """A layer: inputs, weights, bias and residual read once, outputs written once; two operations per product.  A row of
    scores: read once, with its list's bits and settings; a comparison, an exponential's few operations and a sum per
    label."""
    size = {"f32": 4, "f16": 2, "bf16": 2}
    if case["kind"] == "layer":
        R, K, N = case["channels"] * case["frames"], case["inputs"], case["outputs"]
        out = R * N * size[case["out"]]
        return {"bytes": size[case["dtype"]] * K * (R + N) + (4 * N if case["bias"] else 0) + out * (2 if case["residual"] else 1),
                "flops": 2 * R * K * N}
    R, N = case["rows"], case["labels"]
    return {"bytes": R * N * size[case["dtype"]] + 4 * R * min(case["listed"], N) + 32 * R, "flops": 4 * R * N}
