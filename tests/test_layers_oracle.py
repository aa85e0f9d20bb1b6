"""The 64-bit formulas of the workers' backward pass: gradients against differences, the
checkpoint's format against its definition, and what the library refuses without a GPU."""
import ctypes

import numpy as np
import pytest

import paper_2302_05865_amd as fa
from oracle import layers_oracle as lo
from paper_2302_05865_amd import _ctypes_defs as defs


def _differences(f, x, h=1e-6):
    """df/dx of a scalar function by central differences, in 64 bits: truncation ~h^2, rounding ~1e-16/h."""
    g = np.zeros_like(x)
    for k in np.ndindex(*x.shape):
        keep = x[k]
        x[k] = keep + h
        up = f()
        x[k] = keep - h
        g[k] = (up - f()) / (2 * h)
        x[k] = keep
    return g


@pytest.mark.parametrize("features", [1, 2, 5, 12])
def test_norm_gradients_against_differences(features):
    rng = np.random.default_rng(features)
    sizes = [2, 0, 3]
    x = rng.normal(size=(5, features)) * 2 + 1
    gamma, beta, dy = rng.normal(size=features), rng.normal(size=features), rng.normal(size=(5, features))
    eps = 1e-2
    _, _, rstd, xhat = lo.layer_norm(x, gamma, beta, eps)
    dx, dgamma, dbeta = lo.layer_norm_backward(dy, xhat, rstd, sizes, gamma)

    def loss(rows=slice(None)):
        return float((lo.layer_norm(x[rows], gamma, beta, eps)[0] * dy[rows]).sum())

    assert np.allclose(dx, _differences(loss, x), atol=1e-7)
    for w, rows in enumerate([slice(0, 2), slice(2, 2), slice(2, 5)]):
        if rows.start == rows.stop:
            assert not dgamma[w].any() and not dbeta[w].any()
            continue
        assert np.allclose(dgamma[w], _differences(lambda: loss(rows), gamma), atol=1e-7)
        assert np.allclose(dbeta[w], _differences(lambda: loss(rows), beta), atol=1e-7)


def test_linear_gradients_against_differences():
    rng = np.random.default_rng(5)
    sizes, outputs, features = [1, 3, 0, 2], 3, 4
    v, dy = rng.normal(size=(6, features)), rng.normal(size=(6, outputs))
    gamma, beta = rng.normal(size=features), rng.normal(size=features)
    W, b = rng.normal(size=(outputs, features)), rng.normal(size=outputs)
    dweight, dbias = lo.linear_grad(dy, v, sizes, gamma, beta)
    ends = np.concatenate([[0], np.cumsum(sizes)])
    for w in range(len(sizes)):
        rows = slice(ends[w], ends[w + 1])

        def loss():
            return float((((v[rows] * gamma + beta) @ W.T + b) * dy[rows]).sum())

        assert np.allclose(dweight[w], _differences(loss, W), atol=1e-7)
        assert np.allclose(dbias[w], _differences(loss, b), atol=1e-7)


def test_checkpoint_of_chosen_blocks():
    v = np.zeros((6, 33))
    v[0, :4] = [1.0, -1.984375, 1.9921875, 0.0078125]   # floor(log2) 0: s = 2^-6; 127.0, 127.5 -> held; 0.5 -> 0
    v[1, 0], v[1, 32] = 2.0 ** -140, 2.0 ** -126        # below s = 2^-126; exactly s
    v[2, 5] = np.float64(np.finfo(np.float32).max)
    v[3, 7], v[3, 32] = np.inf, 3.0
    v[4, 31] = np.nan
    codes, exponents = lo.pack(v)
    assert codes.shape == (6, 64) and exponents.shape == (6, 2)
    assert list(codes[0, :4]) == [64, -127, 127, 0] and exponents[0, 0] == 121
    assert codes[1, 0] == 0 and codes[1, 32] == 1 and list(exponents[1]) == [1, 1]
    assert codes[2, 5] == 127 and exponents[2, 0] == 248
    assert exponents[3, 0] == 255 and not codes[3, :32].any() and codes[3, 32] == 96 and exponents[3, 1] == 122
    back = lo.unpack(codes, exponents, 33)
    assert np.isnan(back[3, :32]).all() and back[3, 32] == 3.0 and np.isnan(back[4, :32]).all() and back[4, 32] == 0.0
    assert np.isfinite(back[[0, 1, 2, 5]]).all() and (back[5] == 0).all()


def test_checkpoint_pitches():
    lib = fa.load_library()
    for features, pitch, epitch in [(1, 32, 4), (32, 32, 4), (33, 64, 4), (128, 128, 4), (129, 160, 8), (4096, 4096, 128)]:
        assert lib.fa_checkpoint_code_pitch(features) == pitch
        assert lib.fa_checkpoint_exponent_pitch(features) == epitch
    assert lib.fa_checkpoint_code_pitch(0) == 0 and lib.fa_checkpoint_exponent_pitch(-3) == 0


def test_refusals_come_before_any_device_call():
    """Bad arguments are refused on the host; the addresses below are never followed."""
    lib = fa.load_library()
    ARG, OK = defs.FA_ERR_ARG, defs.FA_OK
    A = 1 << 20                                               # some aligned address
    wide = defs.FA_NORM_FEATURES_MAX + 1

    def pack(x=A, ld=64, rows=2, features=64, dtype=0, codes=A, exps=A):
        return lib.fa_checkpoint_pack(x, ld, rows, features, dtype, codes, exps, None)

    for bad in (dict(x=None), dict(x=A + 2), dict(x=A + 1, dtype=1), dict(ld=63), dict(rows=-1), dict(features=0), dict(dtype=2),
                dict(features=defs.FA_FEATURES_MAX + 1, ld=1 << 20), dict(codes=None), dict(codes=A + 8), dict(exps=A + 2),
                dict(rows=(1 << 40) + 1)):
        assert pack(**bad) == ARG, bad
    assert pack(rows=0, x=None, codes=None, exps=None) == OK  # nothing to do
    assert lib.fa_checkpoint_unpack(A, A, 2, 64, 0, None, 64, None) == ARG
    assert lib.fa_checkpoint_unpack(None, A, 2, 64, 0, A, 64, None) == ARG

    def norm(x=A, ld=64, rows=2, features=64, dtype=0, gamma=A, beta=A, pdt=0, eps=1e-5, y=2 * A, ldy=64, mean=A, rstd=A, codes=None,
             exps=None):
        return lib.fa_layer_norm(x, ld, rows, features, dtype, gamma, beta, pdt, eps, y, ldy, mean, rstd, codes, exps, None)

    for bad in (dict(x=None), dict(y=None), dict(y=A), dict(ld=63), dict(ldy=63), dict(features=wide, ld=wide, ldy=wide),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(gamma=A + 2), dict(beta=A + 1, pdt=1),
                dict(pdt=3), dict(mean=A + 2), dict(rstd=A + 1), dict(codes=A), dict(exps=A), dict(codes=A + 4, exps=A),
                dict(dtype=-1), dict(rows=-5)):
        assert norm(**bad) == ARG, bad
    assert norm(rows=0, x=None, y=None) == OK

    def sizes(*k):
        return (ctypes.c_int64 * len(k))(*k)

    def back(dy=A, ld=64, sz=sizes(1, 2), p=2, features=64, dtype=0, x=2 * A, ldx=64, mean=A, rstd=A, codes=None, exps=None,
             gamma=A, pdt=0, res=None, ldr=64, dx=3 * A, lddx=64, dg=A, lddg=64, db=A, lddb=64, gdt=0, ws=A, n=1 << 30):
        return lib.fa_layer_norm_backward(dy, ld, sz, p, features, dtype, x, ldx, mean, rstd, codes, exps, gamma, pdt, res, ldr, dx,
                                          lddx, dg, lddg, db, lddb, gdt, ws, n, None)

    need = lib.fa_layer_norm_backward_workspace(sizes(1, 2), 2, 64)
    assert need > 0
    for bad in (dict(dy=None), dict(sz=None), dict(p=0), dict(p=65), dict(sz=sizes(-1, 2)), dict(features=0), dict(x=None),
                dict(codes=A, exps=A), dict(x=None, codes=A), dict(mean=None), dict(rstd=None), dict(res=A + 2), dict(dx=None),
                dict(dx=A), dict(dx=2 * A), dict(res=3 * A), dict(lddx=63), dict(lddg=63), dict(lddb=1), dict(gdt=2), dict(ws=None),
                dict(ws=A + 4), dict(n=need - 1), dict(sz=sizes(1 << 40, 1))):
        assert back(**bad) == ARG, bad
    assert lib.fa_layer_norm_backward_workspace(sizes(1, -2), 2, 64) == -1
    assert lib.fa_layer_norm_backward_workspace(sizes(1, 2), 2, wide) == -1
    assert lib.fa_layer_norm_backward_workspace(None, 2, 64) == -1

    def linear(dy=A, ld=48, sz=sizes(3, 0), p=2, features=64, outputs=48, dtype=0, codes=A, exps=A, gamma=None, beta=None, pdt=0,
               dw=A, lddw=64 * 48, db=A, lddb=48, gdt=0, ws=A, n=1 << 40):
        return lib.fa_linear_grad(dy, ld, sz, p, features, outputs, dtype, codes, exps, gamma, beta, pdt, dw, lddw, db, lddb, gdt, ws,
                                  n, None)

    for bad in (dict(dy=None), dict(ld=47), dict(sz=sizes(-1, 3)), dict(p=65), dict(features=0), dict(outputs=0),
                dict(outputs=defs.FA_FEATURES_MAX + 1), dict(codes=None), dict(exps=None), dict(gamma=A), dict(beta=A), dict(dw=None),
                dict(lddw=64 * 48 - 1), dict(lddb=47), dict(dw=A + 2), dict(db=A + 1, gdt=1), dict(dtype=5), dict(gdt=9), dict(pdt=-1)):
        assert linear(**bad) == ARG, bad
    # one worker with many rows and a small layer: the rows are cut, the pieces need a place
    long = sizes(1 << 16)
    need = lib.fa_linear_grad_workspace(long, 1, 64, 48, 0)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=A + 8), dict(n=need - 1)):
        assert linear(sz=long, p=1, **bad) == ARG, bad
    assert lib.fa_linear_grad_workspace(long, 1, 0, 48, 0) == -1 and lib.fa_linear_grad_workspace(long, 1, 64, 48, 7) == -1
