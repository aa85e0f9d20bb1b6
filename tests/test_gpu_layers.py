"""Layer norm, its backward pass, 8-bit checkpoints and linear gradients on the GPU against the
64-bit formulas.

Bounds (u = 2^-24, one fp32 rounding; outputs in bf16 add 2^-8 of their size):
 * a sum of n terms, each lane adding its at most 64 in turn and the partial sums joined in a tree
   of at most ten levels, is off by at most 80 u of the sum of magnitudes; the workers' sums over
   rows add at most 300 values in turn (rows of a chunk, then its worker's chunks).
 * xhat = (x - mean) rstd: the mean's error d = 80 u mean|x| enters as it is; in the variance only
   its square, because the centred values add up to nothing.
 * a linear layer's sums: products are exact, at most rows/8 + 32 additions in turn of the matrix
   core (2 u each, its sums need not be rounded to nearest).
"""
import numpy as np
import pytest
import torch

from oracle import layers_oracle as lo
from paper_2302_05865_amd import (Checkpoint, FaError, fa_checkpoint_pack, fa_checkpoint_unpack, fa_layer_norm,
                                  fa_layer_norm_backward, fa_linear_grad)

from gpu_util import announce

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UB = 2.0 ** -8            # bf16: half of 2^-7, the spacing above 1, of a value's size
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MARK = -77.0              # what lies around an output

WIDTHS = [1, 2, 7, 31, 32, 33, 64, 127, 128, 129, 255, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8193, 16384]


def _rng(*seed):
    return np.random.default_rng([int(abs(hash(str(s))) % 1000) if isinstance(s, str) else int(s) for s in seed])


def _seed_of(dtype):
    return 1 if dtype == "f32" else 2


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _store(v, dtype):
    """Half a step of the output's type at v, on top of its fp32 value."""
    return np.abs(v) * (UB if dtype == "bf16" else 0) + 1e-38


def _placed(values, dtype, offset=0, gap=0):
    """A device matrix with these values, `offset` elements into its memory and `gap` between rows; all else is MARK."""
    rows, width = values.shape
    flat = torch.full((offset + rows * (width + gap) + 8,), MARK, dtype=TYPES[dtype], device="cuda")
    view = flat[offset:offset + rows * (width + gap)].view(rows, width + gap)[:, :width]
    view.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return view, flat


def _around_is_untouched(view, flat):
    keep = flat.clone()
    keep.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(MARK)
    return bool((keep == MARK).all())


def _activations(rng, rows, width, offset=0.5):
    return rng.normal(size=(rows, width)) * np.exp(rng.normal(size=width)) + offset


# ---- the checkpoint -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_pack_and_unpack_are_the_definition(width, dtype):
    announce("pack", width, dtype)
    rng = _rng(width, _seed_of(dtype))
    rows = 1 if width % 3 == 0 else 37
    v = _activations(rng, rows, width)
    v[rng.random(v.shape) < 0.05] = 0
    v *= np.exp2(rng.integers(-160, 120, size=(rows, 1)))              # every range, subnormal ones too
    x, _ = _placed(np.clip(v, -3e38, 3e38), dtype, offset=width % 5, gap=width % 4)
    v = _host(x)
    kept = fa_checkpoint_pack(x)
    codes, exponents = lo.pack(v)
    assert np.array_equal(kept.codes.cpu().numpy(), codes)
    assert np.array_equal(kept.exponents.cpu().numpy()[:, :exponents.shape[1]], exponents)
    want = lo.unpack(codes, exponents, width)
    for to in ("f32", "bf16"):
        out, flat = _placed(np.zeros((rows, width)), to, offset=width % 3, gap=1)
        assert fa_checkpoint_unpack(kept, out=out) is out
        assert np.array_equal(_host(out), want) and _around_is_untouched(out, flat)
    assert fa_checkpoint_unpack(kept).dtype == torch.float32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_that_are_not_finite(dtype):
    v = np.ones((5, 70))
    v[0, 3], v[1, 40], v[2, 69], v[3, 31] = np.inf, -np.inf, np.nan, np.nan
    if dtype == "f32":
        v[4, 5] = np.float64(np.finfo(np.float32).max)
    x, _ = _placed(v, dtype)
    back = _host(fa_checkpoint_unpack(fa_checkpoint_pack(x)))
    bad = np.zeros((5, 70), bool)
    bad[0, :32] = bad[1, 32:64] = bad[2, 64:] = bad[3, :32] = True
    assert np.array_equal(np.isnan(back), bad)
    assert (back[:4][~bad[:4]] == 1).all() and np.isfinite(back[4]).all()


def test_checkpoint_of_no_rows():
    kept = fa_checkpoint_pack(torch.empty((0, 40), device="cuda"))
    assert kept.rows == 0 and fa_checkpoint_unpack(kept, torch.bfloat16).shape == (0, 40)


# ---- layer norm --------------------------------------------------------------------------------------------------------------

def _norm_bounds(x, gamma, beta, mean, rstd, xhat):
    """Bounds of mean, rstd, xhat and y in fp32."""
    d = 80 * U * np.abs(x).mean(axis=1)
    rel = 100 * U + 0.5 * (rstd * d) ** 2
    bx = rstd[:, None] * (d[:, None] + 2 * U * np.abs(x - mean[:, None])) + np.abs(xhat) * (rel[:, None] + 2 * U)
    by = np.abs(gamma) * bx + 4 * U * (np.abs(xhat * gamma) + np.abs(beta))
    return d, rstd * rel, bx, by


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_layer_norm(width, dtype):
    announce("norm", width, dtype)
    rng = _rng(width, _seed_of(dtype), 7)
    rows = 41 if width < 300 else 5
    x, _ = _placed(_activations(rng, rows, width), dtype, offset=width % 3, gap=width % 5)
    params = "f32" if width % 2 else "bf16"
    gamma, beta = (torch.from_numpy(rng.normal(size=width)).to("cuda", TYPES[params]) for _ in range(2))
    eps = 1e-5
    want, mean, rstd, xhat = lo.layer_norm(_host(x), _host(gamma), _host(beta), eps)
    d, br, bx, by = _norm_bounds(_host(x), _host(gamma), _host(beta), mean, rstd, xhat)
    out, flat = _placed(np.zeros((rows, width)), dtype, offset=width % 4, gap=width % 3)
    kept = Checkpoint.empty(rows, width)
    y, m, r = fa_layer_norm(x, gamma, beta, eps, checkpoint=kept, out=out)
    assert y is out and _around_is_untouched(out, flat)
    assert (np.abs(_host(m) - mean) <= d + U * np.abs(mean) + 1e-38).all()
    assert (np.abs(_host(r) - rstd) <= br + U * rstd).all()
    assert (np.abs(_host(y) - want) <= by + _store(want, dtype) + UB * by).all()
    # the checkpoint: a code's value is within half a step of xhat, within one where it was held at 127
    codes, exponents = kept.codes.cpu().numpy(), kept.exponents.cpu().numpy()
    values = lo.unpack(codes, exponents, width)
    step = np.repeat(2.0 ** (exponents[:, :-(-width // 32)].astype(float) - 127), 32, axis=1)[:, :width]
    held = np.abs(codes[:, :width]) == 127
    assert (np.abs(values - xhat) <= np.where(held, 1.0, 0.5) * step + bx).all()
    for of, e in ((xhat - bx, -1), (xhat + bx, 1)):       # the exponent is that of a value within the bound
        shift = np.sign(xhat) * np.abs(xhat - of) * e
        _, edge = lo.pack(xhat + shift)
        got = exponents[:, :edge.shape[1]].astype(int)
        assert (got >= edge.astype(int)).all() if e < 0 else (got <= edge.astype(int)).all()
    assert not codes[:, width:].any()
    # without statistics, without parameters, with only one of them
    assert torch.equal(fa_layer_norm(x, gamma, beta, eps, stats=False)[0], out)
    plain, m, r = fa_layer_norm(x, eps=eps, stats=False)
    assert m is None and r is None
    assert (np.abs(_host(plain) - xhat) <= bx + _store(xhat, dtype) + UB * bx).all()
    only = _host(fa_layer_norm(x, beta=beta, eps=eps)[0])
    wantb, _, _, _ = lo.layer_norm(_host(x), None, _host(beta), eps)
    _, _, _, by = _norm_bounds(_host(x), np.ones(width), _host(beta), mean, rstd, xhat)
    assert (np.abs(only - wantb) <= by + _store(wantb, dtype) + UB * by).all()


@pytest.mark.parametrize("width", [48, 700, 3000, 12001])
def test_layer_norm_rows_do_not_mix(width):
    """Rows with a NaN, an infinity, a constant, zeros: theirs alone; a large mean costs no more than its bound."""
    rng = _rng(width, 3)
    x = rng.normal(size=(9, width))
    x[1, width // 2], x[3, 0], x[5], x[6] = np.nan, np.inf, 4.0, 0.0
    x[7] += 500.0
    dev, _ = _placed(x, "f32")
    kept = Checkpoint.empty(9, width)
    y, mean, rstd = fa_layer_norm(dev, checkpoint=kept)
    y, back = _host(y), _host(fa_checkpoint_unpack(kept))
    assert np.isnan(y[[1, 3]]).all() and np.isnan(back[[1, 3]]).all()
    assert (y[[5, 6]] == 0).all() and (back[[5, 6]] == 0).all()
    good = [0, 2, 4, 7, 8]
    want, m, r, xhat = lo.layer_norm(_host(dev)[good])
    _, _, bx, _ = _norm_bounds(_host(dev)[good], 1.0, 0.0, m, r, xhat)
    assert (np.abs(y[good] - want) <= bx).all()


def test_layer_norm_of_no_rows_and_of_many():
    y, m, r = fa_layer_norm(torch.empty((0, 100), device="cuda"))
    assert y.shape == (0, 100) and m.shape == (0,) and r.shape == (0,)
    x = torch.randn(50_001, 24, device="cuda")
    y, m, r = fa_layer_norm(x)
    x = x.double()
    want = (x - x.mean(1, keepdim=True)) * (x.var(1, correction=0, keepdim=True) + 1e-5) ** -0.5
    assert float((y.double() - want).abs().max()) < 1e-5        # |xhat| < 5: 200 u of it, twice over


# ---- its backward pass ---------------------------------------------------------------------------------------------------------

SPLITS = [[1], [0, 3, 0], [5, 1, 30, 0, 64], [0, 0], [33] * 7, [2] * 64]


def _backward_bounds(dy, xhat, rstd, gamma, residual, sizes):
    h = dy * gamma
    a, b = np.abs(h).mean(axis=1, keepdims=True), np.abs(h * xhat).mean(axis=1, keepdims=True)
    inner = 82 * U * a + np.abs(xhat) * 86 * U * b + 6 * U * (np.abs(h) + np.abs(xhat) * b + a)
    bdx = rstd[:, None] * inner
    if residual is not None:
        bdx = bdx + 2 * U * np.abs(residual)
    return bdx, 304 * U * lo.worker_sums(np.abs(dy * xhat), sizes), 304 * U * lo.worker_sums(np.abs(dy), sizes)


def _check_backward(sizes, width, dtype, params, grads, source, with_residual, seed):
    rng = _rng(seed, width, len(sizes))
    rows, p = sum(sizes), len(sizes)
    x = _activations(rng, rows, width)
    dyv = rng.normal(size=(rows, width)) * np.exp(2 * rng.normal(size=(rows, 1))) * (rng.random((rows, 1)) > 0.1)
    dy, _ = _placed(dyv, dtype, offset=width % 3, gap=width % 2)
    xd, _ = _placed(x, dtype, offset=width % 2, gap=3)
    gamma = torch.from_numpy(rng.normal(size=width)).to("cuda", TYPES[params])
    res = _placed(rng.normal(size=(rows, width)), dtype, gap=1)[0] if with_residual else None
    _, mean, rstd, xhat = lo.layer_norm(_host(xd))
    mean, rstd = (torch.from_numpy(t).float().cuda() for t in (mean, rstd))
    if source == "x":
        given = dict(x=xd, mean=mean)
        xhat = (_host(xd) - _host(mean)[:, None]) * _host(rstd)[:, None]
    else:
        kept = fa_checkpoint_pack(torch.from_numpy(xhat).float().cuda())
        given = dict(checkpoint=kept)
        xhat = lo.unpack(kept.codes.cpu().numpy(), kept.exponents.cpu().numpy(), width)
    # G's rows: some other parameter, gamma, beta, some other parameter
    G = torch.full((p, 2 * width + 12), MARK, dtype=TYPES[grads], device="cuda")
    dgamma, dbeta = G[:, 3:3 + width], G[:, 3 + width:3 + 2 * width]
    out, flat = _placed(np.zeros((rows, width)), dtype, offset=1, gap=2)
    dx = fa_layer_norm_backward(dy, rstd, sizes, dgamma, dbeta, gamma=gamma, residual=res, out=out, **given)
    assert dx is out and _around_is_untouched(out, flat)
    assert bool((G[:, :3] == MARK).all()) and bool((G[:, 3 + 2 * width:] == MARK).all())
    r = _host(res) if with_residual else None
    want, wg, wb = lo.layer_norm_backward(_host(dy), xhat, _host(rstd), sizes, _host(gamma), r)
    bdx, bg, bb = _backward_bounds(_host(dy), xhat, _host(rstd), _host(gamma), r, sizes)
    if rows:
        assert (np.abs(_host(dx) - want) <= bdx + _store(want, dtype) + UB * bdx).all()
    assert (np.abs(_host(dgamma) - wg) <= bg + _store(wg, grads) + UB * bg).all()
    assert (np.abs(_host(dbeta) - wb) <= bb + _store(wb, grads) + UB * bb).all()
    for w, n in enumerate(sizes):
        if n == 0:
            assert not dgamma[w].any() and not dbeta[w].any()
    # the same again, and each output alone
    again = torch.empty_like(G)
    a, b = again[:, 3:3 + width], again[:, 3 + width:3 + 2 * width]
    assert torch.equal(fa_layer_norm_backward(dy, rstd, sizes, a, b, gamma=gamma, residual=res, **given), dx)
    assert torch.equal(a, dgamma) and torch.equal(b, dbeta)
    a.zero_()
    assert torch.equal(fa_layer_norm_backward(dy, rstd, sizes, a, None, gamma=gamma, residual=res, **given), dx)
    assert torch.equal(a, dgamma)
    b.zero_()
    fa_layer_norm_backward(dy, rstd, sizes, None, b, gamma=gamma, residual=res, **given)
    assert torch.equal(b, dbeta)
    assert torch.equal(fa_layer_norm_backward(dy, rstd, sizes, gamma=gamma, residual=res, **given), dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("source", ["x", "checkpoint"])
@pytest.mark.parametrize("width", WIDTHS)
def test_backward_over_widths(width, source, dtype):
    announce("norm backward", width, source, dtype)
    sizes = [3, 0, 9, 1] if width > 300 else [13, 0, 70, 5]
    _check_backward(sizes, width, dtype, "f32" if width % 2 else "bf16", "bf16" if width % 3 else "f32", source, width % 4 < 2,
                    _seed_of(dtype))


@pytest.mark.parametrize("sizes", SPLITS)
@pytest.mark.parametrize("width", [20, 100, 300, 1500])
def test_backward_over_workers(sizes, width):
    announce("norm backward", sizes, width)
    _check_backward(sizes, width, "f32", "f32", "f32", "checkpoint", True, 11)
    _check_backward(sizes, width, "bf16", "bf16", "bf16", "x", False, 12)


@pytest.mark.parametrize("rows,width", [(9000, 24), (5003, 200), (2111, 1024), (1500, 2500)])
def test_backward_over_many_rows(rows, width):
    """More rows than workgroups: every team has several, every worker several chunks."""
    announce("norm backward", rows, width)
    _check_backward([rows // 2, 0, rows - rows // 2 - 1, 1], width, "bf16", "f32", "f32", "checkpoint", True, 13)


def test_backward_without_gamma_and_against_differences():
    rng = _rng(5)
    x, dyv = rng.normal(size=(4, 6)), rng.normal(size=(4, 6))
    eps = 1e-2
    xd = torch.from_numpy(x).float().cuda()
    dy = torch.from_numpy(dyv).float().cuda()
    x, dyv = _host(xd), _host(dy)
    _, mean, rstd = fa_layer_norm(xd, eps=eps)
    dgamma, dbeta = torch.empty((2, 2, 6), device="cuda")
    dx = _host(fa_layer_norm_backward(dy, rstd, [1, 3], dgamma, dbeta, x=xd, mean=mean))
    h = 1e-5                                        # 64-bit differences: h^2 and 1e-16 / h, both below 1e-9
    for k in np.ndindex(4, 6):
        keep, f = x[k], []
        for s in (h, -h):
            x[k] = keep + s
            f.append(float((lo.layer_norm(x, None, None, eps)[0] * dyv).sum()))
        x[k] = keep
        assert abs(dx[k] - (f[0] - f[1]) / (2 * h)) < 2e-5       # |terms| < 30: 100 u of them, and a margin of ten
    _, _, _, xhat = lo.layer_norm(x, None, None, eps)
    assert np.allclose(_host(dgamma), lo.worker_sums(dyv * xhat, [1, 3]), atol=1e-5)
    assert np.allclose(_host(dbeta), lo.worker_sums(dyv, [1, 3]), atol=1e-5)


def test_a_row_that_is_not_finite_stays_with_its_worker():
    rng = _rng(9)
    dy = torch.from_numpy(rng.normal(size=(12, 80))).float().cuda()
    x = torch.from_numpy(rng.normal(size=(12, 80))).float().cuda()
    x[5, 7] = float("nan")
    kept = Checkpoint.empty(12, 80)
    _, _, rstd = fa_layer_norm(x, checkpoint=kept)
    dgamma, dbeta = torch.empty((2, 3, 80), device="cuda")
    dx = fa_layer_norm_backward(dy, rstd, [4, 4, 4], dgamma, dbeta, checkpoint=kept)
    assert bool(torch.isnan(dx[5]).all()) and bool(torch.isfinite(dx[[0, 1, 2, 3, 4, 6, 7, 8, 9, 10, 11]]).all())
    assert bool(torch.isnan(dgamma[1]).all()) and bool(torch.isfinite(dgamma[[0, 2]]).all())
    assert bool(torch.isfinite(dbeta).all())


# ---- linear gradients ----------------------------------------------------------------------------------------------------------

def _check_linear(sizes, features, outputs, dtype, params, grads, affine, seed, gap=0):
    rng = _rng(seed, features, outputs, len(sizes))
    rows, p = sum(sizes), len(sizes)
    dyv = rng.normal(size=(rows, outputs)) * np.exp(2 * rng.normal(size=(rows, 1))) * (rng.random((rows, 1)) > 0.1)
    dy, _ = _placed(dyv, dtype, offset=outputs % 3, gap=gap)
    kept = fa_checkpoint_pack(torch.from_numpy(_activations(rng, rows, features)).float().cuda())
    v = lo.unpack(kept.codes.cpu().numpy(), kept.exponents.cpu().numpy(), features)
    gamma = beta = None
    if affine:
        gamma, beta = (torch.from_numpy(rng.normal(size=features)).to("cuda", TYPES[params]) for _ in range(2))
    n = outputs * features
    G = torch.full((p, n + outputs + 9), MARK, dtype=TYPES[grads], device="cuda")
    dbias, dweight = G[:, 1:1 + outputs], G[:, 1 + outputs:1 + outputs + n].unflatten(1, (outputs, features))
    fa_linear_grad(dy, kept, sizes, dweight, dbias, gamma=gamma, beta=beta)
    assert bool((G[:, :1] == MARK).all()) and bool((G[:, 1 + outputs + n:] == MARK).all())
    g, b = (_host(gamma), _host(beta)) if affine else (np.ones(features), np.zeros(features))
    P, wb = lo.linear_grad(_host(dy), v, sizes)
    bw = P * g + wb[:, :, None] * b
    turns = (2 * (np.array(sizes) / 8 + 32) * U)[:, None]
    mb = lo.worker_sums(np.abs(_host(dy)), sizes)
    bb = turns * mb
    mp, _ = lo.linear_grad(np.abs(_host(dy)), np.abs(v), sizes)
    bp = np.abs(g) * turns[:, :, None] * mp + np.abs(b) * bb[:, :, None] + 4 * U * (np.abs(P * g) + np.abs(wb[:, :, None] * b))
    assert (np.abs(_host(dweight) - bw) <= bp + _store(bw, grads) + UB * bp).all()
    assert (np.abs(_host(dbias) - wb) <= bb + _store(wb, grads) + UB * bb).all()
    for w, k in enumerate(sizes):
        if k == 0:
            assert not dweight[w].any() and not dbias[w].any()
    again = torch.empty((p, outputs, features), dtype=TYPES[grads], device="cuda")
    fa_linear_grad(dy, kept, sizes, again, gamma=gamma, beta=beta)
    assert torch.equal(again, dweight)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("features,outputs", [(1, 1), (1, 130), (33, 7), (64, 48), (31, 257), (128, 128), (129, 127), (256, 64), (300, 200),
                                              (511, 129), (512, 256), (520, 264), (100, 1000)])
def test_linear_over_shapes(features, outputs, dtype):
    announce("linear", features, outputs, dtype)
    _check_linear([40, 0, 1, 75], features, outputs, dtype, "f32" if features % 2 else "bf16", "bf16" if outputs % 3 else "f32",
                  features % 4 < 2, _seed_of(dtype), gap=outputs % 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", SPLITS + [[15], [16], [17], [31], [32], [33], [63], [64], [65], [127], [129], [255, 257]])
def test_linear_over_workers(sizes, dtype):
    announce("linear", sizes, dtype)
    _check_linear(sizes, 70, 50, dtype, "f32", "f32", True, 21)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,features,outputs", [([3000], 65, 40), ([1999, 0, 1100, 3], 200, 130), ([700] * 3, 300, 260), ([5003], 260, 300)])
def test_linear_of_few_tiles_and_many_rows(sizes, features, outputs, dtype):
    """The rows of a worker are cut into parts that are joined in order."""
    announce("linear", sizes, features, outputs, dtype)
    _check_linear(sizes, features, outputs, dtype, "bf16", "f32", True, 31)
    _check_linear(sizes, features, outputs, dtype, "f32", "bf16", False, 32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_of_whole_tiles(dtype):
    _check_linear([256, 128], 1024, 768, dtype, "f32", "f32", True, 41)


def test_linear_range_of_fp32():
    """Every piece of an fp32 value counts: the largest, tiny ones, values that differ in the last bit; infinities and NaN
    reach the outputs of their feature block and no one else's."""
    dyv = np.array([[3.4028234e38, 1.0, 1e-30], [-3.4028234e38, 1 + 2.0 ** -23, 3e-30], [0, -2.0, 0]], np.float32)
    v = np.zeros((3, 40))
    v[:, 0], v[:, 35] = 1.0, [0.5, 0.5, 0.25]
    kept = fa_checkpoint_pack(torch.from_numpy(v).float().cuda())
    dw, db = torch.empty((1, 3, 40), device="cuda"), torch.empty((1, 3), device="cuda")
    fa_linear_grad(torch.from_numpy(dyv).cuda(), kept, [3], dw, db)
    want = dyv.astype(np.float64).T @ v
    assert np.allclose(_host(dw)[0], want, rtol=4 * U, atol=0) and _host(dw)[0, 1, 0] == 2.0 ** -23
    for bad in (np.inf, np.nan):
        dy = torch.ones((6, 5), device="cuda")
        dy[4, 2] = bad
        kept = fa_checkpoint_pack(torch.ones((6, 70), device="cuda"))
        dw, db = torch.empty((2, 5, 70), device="cuda"), torch.empty((2, 5), device="cuda")
        fa_linear_grad(dy, kept, [3, 3], dw, db)
        hit = ~torch.isfinite(dw)
        assert bool(hit[1, 2].all()) and int(hit.sum()) == 70 and int((~torch.isfinite(db)).sum()) == 1
        if bad == np.inf:
            assert bool((dw[1, 2] == bad).all()) and float(db[1, 2]) == bad


# ---- streams, graphs, refusals ---------------------------------------------------------------------------------------------------

def _step(x, gamma, beta, dy, sizes, G, kept):
    D, O = x.shape[1], dy.shape[1]
    y, mean, rstd = fa_layer_norm(x, gamma, beta, checkpoint=kept)
    dx = fa_layer_norm_backward(x, rstd, sizes, G[:, :D], G[:, D:2 * D], gamma=gamma, checkpoint=kept)
    fa_linear_grad(dy, kept, sizes, G[:, 2 * D + O:].unflatten(1, (O, D)), G[:, 2 * D:2 * D + O], gamma=gamma, beta=beta)
    return y, dx


def test_on_another_stream_and_in_a_graph():
    announce("stream and graph")
    D, O, sizes = 96, 40, [700, 0, 811]
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(sum(sizes), k, generator=gen, device="cuda") for k in (D, O))
    gamma, beta = torch.randn(2, D, generator=gen, device="cuda")
    G = torch.zeros(3, 2 * D + O + O * D, device="cuda")
    kept = Checkpoint.empty(sum(sizes), D)
    y, dx = _step(x, gamma, beta, dy, sizes, G, kept)
    want = [t.clone() for t in (y, dx, G)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        H = torch.zeros_like(G)
        other = Checkpoint.empty(sum(sizes), D)
        y, dx = _step(x, gamma, beta, dy, sizes, H, other)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, H)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = _step(x, gamma, beta, dy, sizes, H, other)
    for turn in range(4):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        H.zero_()
        graph.replay()
        torch.cuda.synchronize()
        y2, dx2 = _step(x, gamma, beta, dy, sizes, G, kept)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(H, G), turn


def test_refusals():
    x = torch.randn(6, 40, device="cuda")
    kept = fa_checkpoint_pack(x)
    g = torch.ones(40, device="cuda")
    rstd = torch.ones(6, device="cuda")
    G = torch.zeros(2, 80, device="cuda")
    ok = dict(checkpoint=kept)
    for call in (
        lambda: fa_checkpoint_pack(x.cpu()), lambda: fa_checkpoint_pack(x.half()), lambda: fa_checkpoint_pack(x[0]),
        lambda: fa_checkpoint_pack(x.t()), lambda: fa_checkpoint_pack(x, out=Checkpoint.empty(6, 41)),
        lambda: fa_checkpoint_pack(x, out=Checkpoint.empty(5, 40)),
        lambda: fa_checkpoint_unpack(kept, torch.float16), lambda: fa_checkpoint_unpack(kept, out=torch.empty(6, 41, device="cuda")),
        lambda: fa_checkpoint_unpack(kept, torch.bfloat16, out=torch.empty(6, 40, device="cuda")),
        lambda: Checkpoint(kept.codes[:, :32], kept.exponents, 40), lambda: Checkpoint(kept.codes, kept.exponents, 80),
        lambda: Checkpoint(kept.codes, kept.exponents[:5], 40), lambda: Checkpoint(kept.codes, kept.exponents, 0),
        lambda: Checkpoint(kept.codes.float(), kept.exponents, 40),
        lambda: fa_layer_norm(x, g[:39]), lambda: fa_layer_norm(x, g, g.bfloat16()), lambda: fa_layer_norm(x, g.half()),
        lambda: fa_layer_norm(x, g.cpu()), lambda: fa_layer_norm(x, out=x), lambda: fa_layer_norm(x, out=torch.empty(6, 40, device="cuda").bfloat16()),
        lambda: fa_layer_norm(x, checkpoint=Checkpoint.empty(7, 40)), lambda: fa_layer_norm(x.expand(6, 40)[:, ::2]),
        lambda: fa_layer_norm(x[:1].expand(6, 40)),
        lambda: fa_layer_norm_backward(x, rstd, [6], G[:1, :40]), lambda: fa_layer_norm_backward(x, rstd, [6], x=x),
        lambda: fa_layer_norm_backward(x, rstd, [6], x=x, mean=rstd, checkpoint=kept),
        lambda: fa_layer_norm_backward(x, None, [6], **ok), lambda: fa_layer_norm_backward(x, rstd[:5], [6], **ok),
        lambda: fa_layer_norm_backward(x, rstd.bfloat16(), [6], **ok),
        lambda: fa_layer_norm_backward(x, rstd, [5], **ok), lambda: fa_layer_norm_backward(x, rstd, [7, -1], **ok),
        lambda: fa_layer_norm_backward(x, rstd, [], **ok), lambda: fa_layer_norm_backward(x, rstd, [6] + [0] * 64, **ok),
        lambda: fa_layer_norm_backward(x, rstd, [3, 3], G[:1, :40], G[:, :40], **ok),
        lambda: fa_layer_norm_backward(x, rstd, [3, 3], G[:, :40], G[:, 40:].bfloat16(), **ok),
        lambda: fa_layer_norm_backward(x, rstd, [3, 3], G[:, :39], G[:, 40:], **ok),
        lambda: fa_layer_norm_backward(x, rstd, [6], out=x, **ok), lambda: fa_layer_norm_backward(x, rstd, [6], residual=x.bfloat16(), **ok),
        lambda: fa_layer_norm_backward(x.bfloat16(), rstd, [6], x=x, mean=rstd),
        lambda: fa_linear_grad(x, kept, [3, 3], torch.zeros(2, 40, 39, device="cuda")),
        lambda: fa_linear_grad(x, kept, [3, 3], torch.zeros(2, 40, 40, device="cuda").transpose(1, 2)[:, :, :]),
        lambda: fa_linear_grad(x, kept, [3, 3], torch.zeros(2, 40, 80, device="cuda")[:, :, :40]),
        lambda: fa_linear_grad(x, kept, [3, 3], torch.zeros(1, 40, 40, device="cuda").expand(2, 40, 40)),
        lambda: fa_linear_grad(x, kept, [6], torch.zeros(1, 40, 40, device="cuda"), gamma=g),
        lambda: fa_linear_grad(x[:5], kept, [5], torch.zeros(1, 40, 40, device="cuda")),
        lambda: fa_linear_grad(x, kept, [6], torch.zeros(1, 40, 40, device="cuda"), torch.zeros(1, 40, device="cuda").bfloat16()),
        lambda: fa_linear_grad(x.half(), kept, [6], torch.zeros(1, 40, 40, device="cuda")),
    ):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(FaError):
        fa_layer_norm(torch.zeros(2, 16385, device="cuda"))
    with pytest.raises(FaError):
        fa_layer_norm(x, eps=-1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_far_apart(dtype):
    """Rows of dy and dx 2^24 elements apart: offsets in bytes inside a tile and a matrix pass 32 bits."""
    announce("rows far apart", dtype)
    rows, width, apart = 66 if dtype == "f32" else 130, 24, (1 << 24) + 1
    rng = _rng(3, _seed_of(dtype))
    flat = torch.zeros(rows * apart, dtype=TYPES[dtype], device="cuda")
    dy = flat.view(rows, apart)[:, :width]
    dy.copy_(torch.from_numpy(rng.normal(size=(rows, width))))
    x = torch.from_numpy(rng.normal(size=(rows, 40))).float().cuda()
    kept = fa_checkpoint_pack(x)
    dw, db = torch.empty((2, width, 40), device="cuda"), torch.empty((2, width), device="cuda")
    fa_linear_grad(dy, kept, [rows - 3, 3], dw, db)
    other, ob = torch.empty_like(dw), torch.empty_like(db)
    fa_linear_grad(dy.contiguous(), kept, [rows - 3, 3], other, ob)
    v = lo.unpack(kept.codes.cpu().numpy(), kept.exponents.cpu().numpy(), 40)
    want, wb = lo.linear_grad(_host(dy), v, [rows - 3, 3])
    for got, b in ((dw, db), (other, ob)):
        assert np.allclose(_host(got), want, rtol=0, atol=1e-4) and np.allclose(_host(b), wb, rtol=0, atol=1e-4)   # |terms| < 20 x 130
    y, mean, rstd = fa_layer_norm(dy)
    z, m, r = fa_layer_norm(dy.contiguous())
    assert torch.equal(y, z) and torch.equal(mean, m) and torch.equal(rstd, r)
    dx = fa_layer_norm_backward(dy, rstd, [rows], x=dy.contiguous(), mean=mean)
    again = flat.view(rows, apart)[:, width:2 * width]
    assert fa_layer_norm_backward(dy, rstd, [rows], x=dy, mean=mean, out=again) is again and torch.equal(dx, again)
