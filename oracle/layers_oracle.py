"""The workers' backward pass in 64 bits on the CPU, from its formulas (test infrastructure only).

Layer norm, its backward pass, the 8-bit checkpoint and a linear layer's gradients, every worker's
apart.  NumPy; shares no code with the library.
"""
import numpy as np

BLOCK = 32


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd, xhat)"""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    centred = x - mean[:, None]
    rstd = 1.0 / np.sqrt((centred ** 2).mean(axis=1) + eps)
    xhat = centred * rstd[:, None]
    y = xhat if gamma is None else xhat * gamma
    return (y if beta is None else y + beta), mean, rstd, xhat


def layer_norm_backward(dy, xhat, rstd, sizes, gamma=None, residual=None):
    """(dx, dgamma [p, D], dbeta [p, D])"""
    dy, xhat = np.asarray(dy, np.float64), np.asarray(xhat, np.float64)
    h = dy if gamma is None else dy * gamma
    a = h.mean(axis=1, keepdims=True)
    b = (h * xhat).mean(axis=1, keepdims=True)
    dx = np.asarray(rstd, np.float64)[:, None] * (h - a - xhat * b)
    if residual is not None:
        dx = dx + residual
    return dx, worker_sums(dy * xhat, sizes), worker_sums(dy, sizes)


def worker_sums(v, sizes):
    ends = np.concatenate([[0], np.cumsum(sizes)])
    return np.stack([v[a:b].sum(axis=0) for a, b in zip(ends[:-1], ends[1:])])


def pack(v):
    """(codes [rows, padded], exponents [rows, blocks]) of a checkpoint of v."""
    v = np.asarray(v, np.float64)
    rows, features = v.shape
    blocks = -(-features // BLOCK)
    padded = np.zeros((rows, blocks * BLOCK))
    padded[:, :features] = v
    by_block = padded.reshape(rows, blocks, BLOCK)
    finite = np.isfinite(by_block).all(axis=2)
    most = np.abs(np.where(finite[:, :, None], by_block, 0.0)).max(axis=2)
    floor_log2 = np.where(most > 0, np.frexp(most)[1] - 1, -1000)
    power = np.maximum(floor_log2 - 6, -126)
    codes = np.rint(np.where(finite[:, :, None], by_block, 0.0) * 2.0 ** -power[:, :, None].astype(np.float64))
    codes = np.clip(codes, -127, 127)
    return codes.reshape(rows, blocks * BLOCK).astype(np.int8), np.where(finite, power + 127, 255).astype(np.uint8)


def unpack(codes, exponents, features):
    rows = codes.shape[0]
    blocks = -(-features // BLOCK)
    e = exponents[:, :blocks].astype(np.int64)
    scale = np.where(e == 255, np.nan, 2.0 ** (np.where(e == 255, 127, e) - 127.0))
    return (codes.reshape(rows, blocks, BLOCK) * scale[:, :, None]).reshape(rows, blocks * BLOCK)[:, :features]


def linear_grad(dy, v, sizes, gamma=None, beta=None):
    """(dweight [p, outputs, features], dbias [p, outputs])"""
    dy, v = np.asarray(dy, np.float64), np.asarray(v, np.float64)
    into = v if gamma is None else v * gamma + beta
    ends = np.concatenate([[0], np.cumsum(sizes)])
    dweight = np.stack([dy[a:b].T @ into[a:b] for a, b in zip(ends[:-1], ends[1:])])
    return dweight, worker_sums(dy, sizes)
