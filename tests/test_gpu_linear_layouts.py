"""Linear gradients where the layout of dy matters: a single row with any leading dimension, pitches and
widths of either parity, rows of a step nearly 2^24 bytes apart, tiles of either size.

Bounds (u = 2^-24; a gradient stored in bf16 adds 2^-8 of its size): products are exact; a matrix instruction adds 16 rows of
one piece of dy (one piece of bf16, three of fp32) to a sum, in at most two additions in turn of 2 u each; 32 more join
lanes and parts; gamma P + beta b costs 4 u of its terms.
"""
import numpy as np
import pytest
import torch

from linear_shapes import WIDE_IN_PARTS, WIDE_ONE_PART
from oracle import layers_oracle as lo
from paper_2302_05865_amd import fa_checkpoint_pack, fa_linear_grad

from gpu_util import announce

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UB = 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _gradient(rng, rows, outputs):
    return rng.normal(size=(rows, outputs)) * np.exp(rng.normal(size=(rows, 1))) * (rng.random((rows, 1)) > 0.1)


def _pitched(values, dtype, offset, gap):
    """`offset` elements into its memory, `gap` between rows, NaN in everything that is not an element."""
    rows, width = values.shape
    flat = torch.full((offset + rows * (width + gap) + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
    view = flat.as_strided((rows, width), (width + gap, 1), offset)
    view.copy_(torch.from_numpy(values))
    return view


def _check(dy, dtype, sizes, features, affine, grads, rng):
    rows, outputs = dy.shape
    p = len(sizes)
    kept = fa_checkpoint_pack(torch.from_numpy(rng.normal(size=(rows, features)) + 0.3).float().cuda())
    v = lo.unpack(kept.codes.cpu().numpy(), kept.exponents.cpu().numpy(), features)
    gamma = beta = None
    if affine:
        gamma, beta = (torch.from_numpy(rng.normal(size=features)).float().cuda() for _ in range(2))
    dweight = torch.full((p, outputs, features), -77.0, dtype=TYPES[grads], device="cuda")
    dbias = torch.full((p, outputs), -77.0, dtype=TYPES[grads], device="cuda")
    fa_linear_grad(dy, kept, sizes, dweight, dbias, gamma=gamma, beta=beta)
    g, b = (_host(gamma), _host(beta)) if affine else (np.ones(features), np.zeros(features))
    d, ends = _host(dy), np.concatenate([[0], np.cumsum(sizes)])
    for w in range(p):
        at, vw = d[ends[w]:ends[w + 1]], v[ends[w]:ends[w + 1]]
        turns = 2 * U * ((3 if dtype == "f32" else 1) * sizes[w] / 8 + 32)
        P, wb, most, mb = at.T @ vw, at.sum(0), np.abs(at).T @ np.abs(vw), np.abs(at).sum(0)
        want = P * g + wb[:, None] * b
        bound = np.abs(g) * turns * most + np.abs(b) * turns * mb[:, None] + 4 * U * (np.abs(P * g) + np.abs(wb[:, None] * b)) + 1e-38
        got, bias = _host(dweight[w]), _host(dbias[w])
        store = UB if grads == "bf16" else 0
        assert (np.abs(got - want) <= bound + store * (np.abs(want) + bound)).all(), w
        assert (np.abs(bias - wb) <= turns * mb + store * (np.abs(wb) + turns * mb) + 1e-38).all(), w


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [0, 1, 0]])
@pytest.mark.parametrize("outputs", [2, 8, 63, 64, 200])
def test_one_row_has_no_pitch(outputs, sizes, dtype):
    """With one row its leading dimension has no meaning, whatever it is."""
    announce("linear, one row", outputs, sizes, dtype)
    rng = np.random.default_rng([outputs, len(sizes)])
    values = torch.from_numpy(rng.normal(size=outputs)).to("cuda", TYPES[dtype])
    for ld in (0, 1, outputs // 2, outputs - 1, outputs, 1 << 30):
        for affine in (False, True):
            _check(values.as_strided((1, outputs), (ld, 1)), dtype, sizes, 70, affine, "f32", np.random.default_rng(ld))
    _check(values.view(outputs, 1).t(), dtype, sizes, 33, True, "f32", rng)
    _check(values.expand(5, outputs)[:1], dtype, sizes, 33, True, "bf16", rng)


def test_an_infinity_in_one_row_stays_with_its_output():
    for dtype in TYPES.values():
        dy = torch.ones(64, device="cuda", dtype=dtype)
        dy[40] = float("inf")
        kept = fa_checkpoint_pack(torch.ones((1, 40), device="cuda"))
        dweight, dbias = torch.empty((1, 64, 40), device="cuda"), torch.empty((1, 64), device="cuda")
        fa_linear_grad(dy.as_strided((1, 64), (1, 1)), kept, [1], dweight, dbias)
        want = torch.ones(64, device="cuda")
        want[40] = float("inf")
        assert torch.equal(dbias[0], want) and torch.equal(dweight[0], want[:, None].expand(64, 40))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_worker_without_rows_gets_zeros_whatever_the_parameters(bad):
    """Its sums have no terms: an infinite gamma or beta does not come into them, in one part or joined from several."""
    for sizes, outputs in (([0, 3, 0], 40), ([0, 9000], 8)):
        for dtype in TYPES.values():
            gen = torch.Generator(device="cuda").manual_seed(1)
            dy = torch.randn(sum(sizes), outputs, generator=gen, device="cuda").to(dtype)
            kept = fa_checkpoint_pack(torch.randn(sum(sizes), 70, generator=gen, device="cuda"))
            gamma, beta = torch.ones(2, 70, device="cuda")
            gamma[3], beta[5] = bad, bad
            dweight, dbias = torch.full((len(sizes), outputs, 70), -77.0, device="cuda"), torch.full((len(sizes), outputs), -77.0, device="cuda")
            fa_linear_grad(dy, kept, sizes, dweight, dbias, gamma=gamma, beta=beta)
            for w, n in enumerate(sizes):
                if n == 0:
                    assert not dweight[w].any() and not dbias[w].any()
                else:
                    finite = torch.isfinite(dweight[w])
                    assert not finite[:, [3, 5]].any() and int(finite.sum()) == outputs * 68


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gap", [0, 1, 2, 3])
@pytest.mark.parametrize("outputs", [2, 7, 50, 127, 129, 130])
def test_pitches_of_either_parity(outputs, gap, dtype):
    """Rows that begin at every place of a word and end there; one step and several, last steps of even and odd lengths."""
    announce("linear, pitches", outputs, gap, dtype)
    for sizes in ([1, 2], [63, 64], [65, 66, 0, 1], [127, 130, 191, 192], [129, 200]):
        rng = np.random.default_rng([outputs, gap, sizes[0]])
        for offset in (0, 1):
            dy = _pitched(_gradient(rng, sum(sizes), outputs), dtype, offset, gap)
            _check(dy, dtype, sizes, 70, offset == 1, "f32" if gap < 2 else "bf16", rng)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_farthest_rows_of_a_step(dtype):
    """A pitch just below 2^22 elements: a step of fp32 is nearly 2^30 bytes long."""
    announce("linear, far rows in a step", dtype)
    rows, outputs, apart = 131, 24, (1 << 22) - 1
    rng = np.random.default_rng(5)
    flat = torch.full((rows * apart,), float("nan"), dtype=TYPES[dtype], device="cuda")
    dy = flat.view(rows, apart)[:, :outputs]
    dy.copy_(torch.from_numpy(_gradient(rng, rows, outputs)))
    _check(dy, dtype, [rows - 2, 2], 40, True, "f32", rng)


@pytest.mark.parametrize("dtype,shape", [(t, s) for t in TYPES for s in WIDE_ONE_PART[t] + WIDE_IN_PARTS[t]],
                         ids=lambda s: s if isinstance(s, str) else f"{len(s[0])}x{sum(s[0])}x{s[1]}x{s[2]}")
def test_wide_tiles(shape, dtype):
    sizes, features, outputs = shape
    for gap, affine, grads in ((0, True, "f32"), (1, False, "bf16")):
        announce("linear, wide tiles", len(sizes), sum(sizes), features, outputs, dtype, gap)
        rng = np.random.default_rng([features, outputs, gap])
        dy = _pitched(_gradient(rng, sum(sizes), outputs), dtype, gap, gap)
        _check(dy, dtype, sizes, features, affine, grads, rng)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiny_gradients(dtype):
    """bf16 is exact down to its subnormals.  Of fp32 dy the lowest piece ends at 2^-133, the last place of bf16: exact from
    2^-110 on, below that each dy cut off by less than 2^-133.  (Products are taken of one row: no sum rounds them, but the
    three pieces' to 2 u each and the result's to half of 2^-149.)"""
    rng = np.random.default_rng(8)
    bits = 23 if dtype == "f32" else 7
    for power in (-100, -109, -110, -111, -117, -118, -119, -125, -126, -127, -133, -140, -149):
        values = np.concatenate([[1.0, 2 - 2.0 ** -bits], 1 + rng.integers(0, 1 << bits, size=60) * 2.0 ** -bits]) * 2.0 ** power
        dy = torch.from_numpy(values).to("cuda", TYPES[dtype])[None]
        d = _host(dy)[0]
        kept = fa_checkpoint_pack(torch.from_numpy(rng.normal(size=(1, 33))).float().cuda())
        v = lo.unpack(kept.codes.cpu().numpy(), kept.exponents.cpu().numpy(), 33)[0]
        dweight, dbias = torch.empty((1, 62, 33), device="cuda"), torch.empty((1, 62), device="cuda")
        fa_linear_grad(dy, kept, [1], dweight, dbias)
        cut = np.where((np.abs(d) >= 2.0 ** -110) | (dtype == "bf16"), 0.0, 2.0 ** -133)
        want = d[:, None] * v
        assert (np.abs(_host(dweight)[0] - want) <= cut[:, None] * np.abs(v) + 6 * U * np.abs(want) + 2.0 ** -148).all(), power
        assert (np.abs(_host(dbias)[0] - d) <= cut + 6 * U * np.abs(d) + 2.0 ** -148).all(), power


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[2500] + [0] * 63, [0] * 40 + [2001, 1, 0, 70], [3] * 30 + [3001]])
def test_workers_of_very_different_lengths(sizes, dtype):
    announce("linear, uneven workers", max(sizes), len(sizes), dtype)
    rng = np.random.default_rng(len(sizes))
    dy = _pitched(_gradient(rng, sum(sizes), 131), dtype, 1, 2)
    _check(dy, dtype, sizes, 150, True, "f32", rng)
