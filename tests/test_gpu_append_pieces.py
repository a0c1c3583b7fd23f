"""cobra_append_tokens on vectors and bases that bf16 pieces represent as badly as they can: every element just below
the middle between two bf16 values, with what two pieces leave of it of the sign that adds up.  The codes are still those
of the exact projection."""
import numpy as np
import pytest
import torch

from oracle import rope, serve
from paper_2609_24298_gb300 import cobra

from .serve_util import D, Cache
from .test_gpu_append_run import run

pytestmark = pytest.mark.gpu
THETA = 10000.0


def as_bf16(x):
    return torch.tensor(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def bad_vector(pos):
    """x [128] of bf16 values whose turned first half lies just above powers of two (1 .. 1 + 2^-8, |second half| less
    than a quarter of it), and the fp32 column w that adds up what the pieces drop."""
    a = pos * THETA ** (-2.0 * np.arange(64) / D)
    m = (128 + np.arange(128)) / 128.0
    few = np.concatenate([s * m * 2.0 ** e for e in range(-6, 1) for s in (1, -1)])
    A, B = np.meshgrid(m, few, indexing="ij")
    x = np.zeros(D)
    for j, (c, s) in enumerate(zip(np.cos(a), np.sin(a))):
        best = -1.0
        for P, Q in ((A, B), (B, A)):
            ya, yb = P * c - Q * s, P * s + Q * c
            e = np.floor(np.log2(np.abs(ya) + 1e-300))
            y = (np.abs(ya) / 2.0 ** e).astype(np.float32)
            p1 = as_bf16(y)
            p2 = as_bf16(y - p1)
            left = np.clip((y - p1 - p2).astype(np.float64) * 2.0 ** 17, -1, 1)
            worth = np.where((np.abs(yb) < 0.25 * np.abs(ya)) & (y < 1 + 2.0 ** -8), 128.0 * (y - 1) + 0.25 * left - 0.5 * (yb / (ya + 1e-300)) ** 2, -1)
            k = np.unravel_index(np.argmax(worth), worth.shape)
            if worth[k] > best:
                best, x[j], x[j + 64] = worth[k], P[k] / 2.0 ** e[k], Q[k] / 2.0 ** e[k]
    assert np.array_equal(as_bf16(x).astype(np.float64), x)
    y = rope.rotate(x[None], np.array([pos]), THETA)[0]
    w = np.zeros(D, np.float32)
    w[:64] = np.sign(y[:64]) * np.float32(1 + 2.0 ** -8 - 0.51 * 2.0 ** -16)
    return x, y, w


@pytest.mark.parametrize("n", [1, 40, 100])
@pytest.mark.parametrize("turn", [True, False])
@pytest.mark.parametrize("past", [2e-4, 8e-4])
def test_least_favourable_pieces(n, turn, past):
    """The exact projection lies `past` of a cell above a border, what the pieces make of it below."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()
    pos = 8001
    x, y, w = bad_vector(pos)
    if not turn:  # plain vectors are bf16 themselves: one piece
        y = x
        w[:] = np.sign(x) * np.float32(1 + 2.0 ** -8 - 0.51 * 2.0 ** -16)
    W = np.zeros((D, 2), np.float32)
    W[:, 0], W[64:, 1] = w, 1.0
    exact = w.astype(np.float64) @ y
    k = dict(r=2, b=8, W=W, mu=np.zeros(D, np.float32), delta=np.float32(exact / (126.0 + past)))
    cache = Cache([k, dict(k, W=W[::-1].copy())], 1, 1, [0, 0, 0], cap=8192).upload()
    g = np.random.default_rng(n)
    xs = as_bf16(g.standard_normal((2, 1, 3, n, 1, D))).astype(np.float64)
    at = [0, n // 2, n - 1]
    for s in range(3):
        xs[0, 0, s, at[s], 0] = x
    got, want = run(cache, [pos - j for j in at], [n] * 3, x=xs, theta=THETA if turn else None)
    for s in range(3):
        assert serve.new_codes(x[None], k, np.array([pos]) if turn else None, THETA)[0, 0] == 254
    assert np.array_equal(got, want)
