"""The operators of a worker's backward pass, timed from one token to the largest batch.

The p workers' tokens lie one under the other in matrices of `rows` rows; worker w has `sizes[w]`
consecutive ones.  Four operators take such a batch to the rows of the gradient matrix G [p, n]
that the aggregation reads:

    norm        layer norm, with or without an 8-bit checkpoint of the normalised rows
    norm_grad   its backward pass: dx, and every worker's dgamma and dbeta in that worker's row of G
    pack/unpack any activation as an 8-bit checkpoint, and back
    linear      every worker's weight and bias gradient of a linear layer from the checkpoint of
                its input, in that worker's row of G

A checkpoint holds blocks of 32 features of a row: s = 2^max(floor(log2 max|v|) - 6, -126) as the
byte 127 + log2 s, and the codes round(v / s) within +-127; rows of codes are padded to whole
blocks with zeros, rows of exponent bytes to multiples of four.  code * s has seven significant
bits, so it is given back in bf16 without another rounding.

    listed()            the cases that are timed
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has in hand before the call
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the outputs in 64 bits
"""
import math
import random

import torch

own = False

EPS = 1e-5
BLOCK = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
MOST_ELEMENTS = 65536 * 4096          # of one activation matrix, and of G
MOST_FLOPS = 2 * 65536 * 4096 * 4096  # of one linear layer's gradient


def listed():
    return [
        # one token in front of a head: latency alone
        dict(name="norm_token", op="norm", rows=1, features=768, dtype="bf16", params="f32", checkpoint=False),
        # 15 workers with a thousand tokens each, the forward pass of a training step
        dict(name="norm_batch", op="norm", rows=15 * 1024, features=768, dtype="bf16", params="f32", checkpoint=True),
        # a wide model's batch, evaluated without a checkpoint
        dict(name="norm_large", op="norm", rows=65536, features=4096, dtype="bf16", params="bf16", checkpoint=False),
        # a small model in 32 bits, odd width, ragged workers, backward from x
        dict(name="norm_grad_small", op="norm_grad", rows=1001, features=257, workers=7, ragged=True, dtype="f32",
             params="f32", grads="f32", source="x", residual=False),
        # the backward half of norm_batch, the residual branch's gradient added
        dict(name="norm_grad_batch", op="norm_grad", rows=15 * 1024, features=768, workers=15, ragged=False, dtype="bf16",
             params="f32", grads="f32", source="checkpoint", residual=True),
        # the wide model's batch spread over 32 workers, gradients in bf16
        dict(name="norm_grad_large", op="norm_grad", rows=65536, features=4096, workers=32, ragged=True, dtype="bf16",
             params="bf16", grads="bf16", source="checkpoint", residual=False),
        # an activation of odd width in 32 bits, kept in 8 and read back
        dict(name="pack_odd", op="pack", rows=9999, features=1111, dtype="f32"),
        # the wide model's activation read back for a backward pass
        dict(name="unpack_large", op="unpack", rows=65536, features=4096, dtype="bf16"),
        # a small layer, a few tokens for each of 7 workers: latency
        dict(name="linear_small", op="linear", rows=224, features=48, outputs=64, workers=7, ragged=False, dtype="f32",
             params="f32", grads="f32", affine=True),
        # the projection behind the norm of norm_batch
        dict(name="linear_batch", op="linear", rows=15 * 1024, features=768, outputs=2304, workers=15, ragged=False,
             dtype="bf16", params="f32", grads="f32", affine=True),
        # 60 ragged workers (some without a token), odd sizes, gradients of the outputs in 32 bits
        dict(name="linear_ragged", op="linear", rows=30011, features=1001, outputs=509, workers=60, ragged=True,
             dtype="f32", params="f32", grads="f32", affine=False),
        # the wide model's square projection, 16 workers with 4096 tokens each
        dict(name="linear_large", op="linear", rows=65536, features=4096, outputs=4096, workers=16, ragged=False,
             dtype="bf16", params="bf16", grads="bf16", affine=True),
    ]


def _between(rng, low, high):
    """A whole number between the two, spread over their logarithm; odd ones as often as not."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = min(high, max(low, v))
    if v >= 64 and rng.random() < 0.5:
        v -= v % 16          # a model's widths and batches are mostly multiples
    return v - 1 if v == 3072 else v


def draw(rng: random.Random):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "norm_grad", "pack", "unpack", "linear", "linear", "linear", "linear"])
    case = dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16"]))
    half = MOST_ELEMENTS if case["dtype"] == "bf16" else MOST_ELEMENTS // 2
    if op == "linear":
        case["features"] = _between(rng, 16, 4096)
        case["outputs"] = _between(rng, 16, 4096)
        case["workers"] = rng.choice([1, 2, 3, 7, 15, 32, 60, 64])
        case["workers"] = max(1, min(case["workers"], MOST_ELEMENTS // (case["features"] * case["outputs"])))
        flops = MOST_FLOPS if case["dtype"] == "bf16" else MOST_FLOPS // 8
        most = min(65536, flops // (2 * case["features"] * case["outputs"]), half // max(case["features"], case["outputs"]))
        case["rows"] = _between(rng, min(64, most), most)
        case["affine"] = rng.random() < 0.5
    else:
        case["features"] = _between(rng, 16, 16384)
        case["rows"] = _between(rng, 1, min(262144, half // case["features"]))
    if op == "norm":
        case["checkpoint"] = rng.random() < 0.5
    if op == "norm_grad":
        case["workers"] = rng.choice([1, 2, 3, 7, 15, 32, 60, 64])
        case["source"] = rng.choice(["x", "checkpoint", "checkpoint"])
        case["residual"] = rng.random() < 0.5
    if op in ("norm", "norm_grad", "linear"):
        case["params"] = rng.choice(["f32", "bf16"])
    if op in ("norm_grad", "linear"):
        case["ragged"] = rng.random() < 0.5
        case["grads"] = rng.choice(["f32", "bf16"])
    return case


def _sizes(case):
    """Rows of every worker: even, or ragged with some workers that have none."""
    p, rows = case["workers"], case["rows"]
    if not case["ragged"]:
        return [rows // p + (1 if w < rows % p else 0) for w in range(p)]
    rng = random.Random(1000 * rows + p)
    share = [0.0 if p > 3 and rng.random() < 0.1 else rng.uniform(0.3, 1.7) for _ in range(p)]
    share[rng.randrange(p)] = 1.0
    total = sum(share)
    sizes = [int(rows * s / total) for s in share]
    sizes[max(range(p), key=lambda w: sizes[w])] += rows - sum(sizes)
    return sizes


def _activation(gen, rows, features, dtype):
    """Rows of a residual stream: every feature its own mean and scale, a few of them far out."""
    scale = torch.exp(0.5 * torch.randn(features, generator=gen, device="cuda"))
    scale = torch.where(torch.rand(features, generator=gen, device="cuda") < 0.01, scale * 20, scale)
    mean = 0.3 * torch.randn(features, generator=gen, device="cuda")
    return (torch.randn(rows, features, generator=gen, device="cuda").mul_(scale).add_(mean)).to(dtype)


def _gradient(gen, rows, features, dtype):
    """Gradients of outputs: small, tokens of very different size, a few rows that are masked out."""
    token = 1e-3 * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
    token = torch.where(torch.rand(rows, 1, generator=gen, device="cuda") < 0.05, torch.zeros_like(token), token)
    return (torch.randn(rows, features, generator=gen, device="cuda").mul_(token)).to(dtype)


def _params(gen, features, dtype):
    gamma = 1 + 0.2 * torch.randn(features, generator=gen, device="cuda")
    beta = 0.1 * torch.randn(features, generator=gen, device="cuda")
    return gamma.to(dtype), beta.to(dtype)


def _pack(v):
    """Codes and exponent bytes of a matrix in 32 bits."""
    rows, features = v.shape
    pitch = -(-features // BLOCK) * BLOCK
    v = torch.nn.functional.pad(v, (0, pitch - features)).view(rows, -1, BLOCK)
    most = v.abs().amax(2)
    power = ((most.view(torch.int32) >> 23) - 6).clamp(min=1)       # 127 + log2 s
    inverse = ((254 - power) << 23).view(torch.float32)             # 1 / s
    codes = torch.round(v * inverse.unsqueeze(2)).clamp(-127, 127)
    codes = codes.to(torch.int8).view(rows, pitch)
    power = torch.nn.functional.pad(power.to(torch.uint8), (0, -power.shape[1] % 4))
    return codes, power.contiguous()


def _unpack(codes, power, features):
    """The values that a checkpoint stands for, in 32 bits."""
    rows = codes.shape[0]
    scale = (power[:, : codes.shape[1] // BLOCK].to(torch.int32) << 23).view(torch.float32)
    return (codes.view(rows, -1, BLOCK).float() * scale.unsqueeze(2)).view(rows, -1)[:, :features]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, rows, features = case["op"], case["rows"], case["features"]
    dtype = TYPES[case["dtype"]]
    s = dict(case=case, dtype=dtype)
    if op in ("norm", "norm_grad", "linear"):
        s["gamma"], s["beta"] = _params(gen, features, TYPES[case["params"]])
    if op in ("norm", "pack"):
        s["x"] = _activation(gen, rows, features, dtype)
    elif op == "unpack":
        s["codes"], s["power"] = _pack(_activation(gen, rows, features, torch.float32))
    else:
        x = _activation(gen, rows, features, dtype)
        s["mean"], s["rstd"], xhat = _normalised(x)
        s["codes"], s["power"] = _pack(xhat)
        s["x"] = x
        s["sizes"] = _sizes(case)
        s["count"] = torch.tensor(s["sizes"], device="cuda")
        s["dy"] = _gradient(gen, rows, case.get("outputs", features), dtype)
        s["residual"] = _gradient(gen, rows, features, dtype) if case.get("residual") else None
        # G's row: the slices that the pass writes, in the order in which a model's parameters lie
        p, outputs = case["workers"], case.get("outputs")
        n = 2 * features if op == "norm_grad" else outputs * features + outputs
        G = torch.zeros(p, -(-n // 8) * 8, dtype=TYPES[case["grads"]], device="cuda")
        if op == "norm_grad":
            s["dgamma"], s["dbeta"] = G[:, :features], G[:, features:2 * features]
        else:
            s["dbias"], s["dweight"] = G[:, :outputs], G[:, outputs:n].unflatten(1, (outputs, features))
    return s


def _normalised(x):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    return mean.squeeze(1), rstd.squeeze(1), c * rstd


def _worker_sums(count, v):
    """[p, features]: the sum of every worker's rows, as a product with the 0/1 matrix of who has which."""
    end = count.cumsum(0).unsqueeze(1)
    row = torch.arange(v.shape[0], device=v.device)
    return ((row < end) & (row >= end - count.unsqueeze(1))).float() @ v


def _by_worker(count, most, v):
    """[p, most, features]: every worker's rows, padded with zeros."""
    count = count.unsqueeze(1)
    first = count.cumsum(0) - count
    row = torch.arange(most, device=v.device)
    return v[(first + row).clamp(max=v.shape[0] - 1)] * (row < count).unsqueeze(2)


def _plain(s):
    case, op, features, dtype = s["case"], s["case"]["op"], s["case"]["features"], s["dtype"]
    if op == "norm":
        mean, rstd, xhat = _normalised(s["x"])
        out = dict(y=(xhat * s["gamma"].float() + s["beta"].float()).to(dtype), mean=mean, rstd=rstd)
        if case["checkpoint"]:
            out["values"] = _unpack(*_pack(xhat), features).to(torch.bfloat16)
        return out
    if op == "pack":
        return _unpack(*_pack(s["x"].float()), features).to(torch.bfloat16)
    if op == "unpack":
        return _unpack(s["codes"], s["power"], features).to(dtype)
    dy = s["dy"].float()
    if op == "norm_grad":
        if case["source"] == "x":
            xhat = (s["x"].float() - s["mean"].unsqueeze(1)) * s["rstd"].unsqueeze(1)
        else:
            xhat = _unpack(s["codes"], s["power"], features)
        h = dy * s["gamma"].float()
        a, b = h.mean(1, keepdim=True), (h * xhat).mean(1, keepdim=True)
        dx = s["rstd"].unsqueeze(1) * (h - a - xhat * b)
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        s["dgamma"].copy_(_worker_sums(s["count"], dy * xhat))
        s["dbeta"].copy_(_worker_sums(s["count"], dy))
        return dict(dx=dx.to(dtype), dgamma=s["dgamma"], dbeta=s["dbeta"])
    v = _unpack(s["codes"], s["power"], features)
    if case["affine"]:
        v = v * s["gamma"].float() + s["beta"].float()
    dy, v = _by_worker(s["count"], max(s["sizes"]), dy), _by_worker(s["count"], max(s["sizes"]), v)
    s["dweight"].copy_(torch.bmm(dy.transpose(1, 2), v))
    s["dbias"].copy_(dy.sum(1))
    return dict(dweight=s["dweight"], dbias=s["dbias"])


def _own(s):
    import paper_2302_05865_amd as fa
    case, op, features = s["case"], s["case"]["op"], s["case"]["features"]
    if op == "norm":
        kept = fa.Checkpoint.empty(case["rows"], features) if case["checkpoint"] else None
        y, mean, rstd = fa.fa_layer_norm(s["x"], s["gamma"], s["beta"], EPS, checkpoint=kept)
        out = dict(y=y, mean=mean, rstd=rstd)
        if kept is not None:
            out["values"] = fa.fa_checkpoint_unpack(kept, torch.bfloat16)
        return out
    if op == "pack":
        return fa.fa_checkpoint_unpack(fa.fa_checkpoint_pack(s["x"]), torch.bfloat16)
    kept = fa.Checkpoint(s["codes"], s["power"], features)
    if op == "unpack":
        return fa.fa_checkpoint_unpack(kept, s["dtype"])
    if op == "norm_grad":
        source = dict(x=s["x"], mean=s["mean"]) if case["source"] == "x" else dict(checkpoint=kept)
        dx = fa.fa_layer_norm_backward(s["dy"], s["rstd"], s["sizes"], s["dgamma"], s["dbeta"], gamma=s["gamma"],
                                       residual=s["residual"], **source)
        return dict(dx=dx, dgamma=s["dgamma"], dbeta=s["dbeta"])
    affine = dict(gamma=s["gamma"], beta=s["beta"]) if case["affine"] else {}
    fa.fa_linear_grad(s["dy"], kept, s["sizes"], s["dweight"], s["dbias"], **affine)
    return dict(dweight=s["dweight"], dbias=s["dbias"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    op, n = case["op"], case["rows"] * case["features"]
    es, kept = BYTES[case["dtype"]], n * (1 + 1 / BLOCK)
    if op == "norm":
        more = 2 * n if case["checkpoint"] else 0
        return dict(bytes=2 * n * es + more + 8 * case["rows"] + 2 * case["features"] * BYTES[case["params"]], flops=8 * n)
    if op == "pack":
        return dict(bytes=n * es + 2 * n, flops=3 * n)
    if op == "unpack":
        return dict(bytes=kept + n * es, flops=n)
    gs = BYTES[case["grads"]]
    if op == "norm_grad":
        x = n * es if case["source"] == "x" else kept
        return dict(bytes=(3 if case["residual"] else 2) * n * es + x + 2 * case["workers"] * case["features"] * gs, flops=12 * n)
    o, f = case["outputs"], case["features"]
    return dict(bytes=case["rows"] * o * es + kept + case["workers"] * (o * f + o) * gs, flops=2 * case["rows"] * o * f)


def _exact_values(s):
    """A checkpoint's values from its definition, in 64 bits."""
    codes, blocks = s["codes"].double(), s["codes"].shape[1] // BLOCK
    power = s["power"][:, :blocks].double().repeat_interleave(BLOCK, 1) - 127
    return (codes * torch.exp2(power))[:, : s["case"]["features"]]


def _exact_rounded(v):
    """What a checkpoint of v stands for, from its definition, in 64 bits, a block at a time."""
    got = torch.empty_like(v)
    for j in range(0, v.shape[1], BLOCK):
        part = v[:, j:j + BLOCK]
        power = torch.frexp(part.abs().amax(1, keepdim=True))[1].double() - 7       # floor(log2) - 6
        step = torch.exp2(power.clamp(min=-126))
        got[:, j:j + BLOCK] = (part / step).round().clamp(-127, 127) * step
    return got


def exact(case, seed):
    s = prepare(case, seed)
    op, features = case["op"], case["features"]
    if op == "norm":
        x = s["x"].double()
        variance, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = (variance + EPS) ** -0.5
        xhat = (x - mean) * rstd
        out = dict(y=torch.addcmul(s["beta"].double(), xhat, s["gamma"].double()), mean=mean[:, 0], rstd=rstd[:, 0])
        if case["checkpoint"]:
            out["values"] = _exact_rounded(xhat)
        return out
    if op == "pack":
        return _exact_rounded(s["x"].double())
    if op == "unpack":
        return _exact_values(s)
    p, dy, ends = case["workers"], s["dy"].double(), [0]
    for rows in s["sizes"]:
        ends.append(ends[-1] + rows)
    parts = list(zip(ends, ends[1:]))
    if op == "norm_grad":
        rstd = s["rstd"].double()[:, None]
        xhat = (s["x"].double() - s["mean"].double()[:, None]) * rstd if case["source"] == "x" else _exact_values(s)
        gamma = s["gamma"].double()
        along = (dy * xhat) @ gamma / features
        dx = rstd * (dy * gamma - (dy @ gamma / features)[:, None] - xhat * along[:, None])
        if case["residual"]:
            dx = dx + s["residual"].double()
        return dict(dx=dx, dgamma=torch.stack([(dy[a:b] * xhat[a:b]).sum(0) for a, b in parts]),
                    dbeta=torch.stack([dy[a:b].sum(0) for a, b in parts]))
    v = _exact_values(s)
    dweight = torch.empty(p, case["outputs"], features, dtype=torch.float64, device="cuda")
    dbias = torch.empty(p, case["outputs"], dtype=torch.float64, device="cuda")
    for w, (a, b) in enumerate(parts):
        dbias[w] = dy[a:b].sum(0)
        dweight[w] = dy[a:b].t() @ v[a:b]
        if case["affine"]:
            dweight[w] = dweight[w] * s["gamma"].double() + dbias[w][:, None] * s["beta"].double()
    return dict(dweight=dweight, dbias=dbias)
