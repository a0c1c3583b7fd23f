"""NaN and infinities where a query looks: the definition gives NaN, and so does cobra_tree_attn; only a token that
sees nothing gives zeros.  What does not see them keeps its result."""
import numpy as np
import pytest
import torch

from oracle import attention
from paper_2609_24298_gb300 import cobra

from .serve_util import D, DEV, Cache, bf16, heads
from .test_gpu_tree import Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()


def outputs(call):
    call.run()
    assert cobra.cobra_check() == cobra.COBRA_OK
    L, S, N = call.o_v.shape[:3]
    return call.o_v[..., :call.c.kv * call.G * D].float().cpu().numpy().reshape(L, S, N, -1, D)


def put(call):
    """The call's (changed) q, kd and vd to its device buffers, as they are."""
    for a, d in ((call.q, call.q_d), (call.kd, call.k_d), (call.vd, call.v_d)):
        d[:a.size] = bf16(a.reshape(-1))[1]


def near(call):
    """Twice 2^-8 (probabilities) of the spread of the values, and twice 2^-8 (outputs) of the largest."""
    v = call.c.params[1]
    values = [attention.reconstruct(call.c.codes[1, s], v["W"], v["delta"], v["b"], v["mu"]) for s in range(call.S)]
    top = max(np.abs(x).max() for x in values + [call.vd])
    return 2.0 * 2.0 ** -8 * (2.0 * top + top)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("N,G", [(1, 4), (2, 8), (8, 4), (16, 8)])
@pytest.mark.parametrize("rk,q_scale,cap,slope", [(64, 1.0, 0.0, 0.0), (64, 40.0, 0.0, 0.0), (0, 1.0, 0.0, 0.0), (64, 1.0, 0.0, 0.01),
                                                   (40, 1.0, 30.0, 0.0), (40, 40.0, 100.0, -0.01)])
def test_queries(bad, N, G, rk, q_scale, cap, slope):
    """One element of one head's query of one token; a token that sees nothing has one too."""
    lens = [400, 130]
    cache = Cache(heads([(rk, 3), (32, 2), (48, 4), (128, 1)], 51), 1, 2, lens).upload()
    pos = np.array([[T + i for i in range(N)] for T in lens])
    pos[1, N - 1] = -3
    mask = [np.tril(np.ones((N, N), bool)) for _ in lens]
    mask[1][N - 1] = False
    slopes = np.full(2 * G, slope, np.float32) if slope else None
    call = Call(cache, G, N, mask=mask, pos=pos, q_scale=q_scale, cap=cap, slopes=slopes)
    want = outputs(call)
    assert np.isfinite(want).all()
    at = [(0, 0, 1, 5), (0, N - 1, 2 * G - 1, 127), (1, N - 1, 0, 64)]
    for s, i, h, d in at:
        call.q[0, s, i, h, d] = bad
        want[0, s, i, h] = np.nan if (s, i) != (1, N - 1) else 0.0
    put(call)
    got = outputs(call)
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("drafts_alone", [False, True])
@pytest.mark.parametrize("N,G", [(2, 4), (8, 4), (16, 8), (64, 2)])
def test_drafted_keys(N, G, drafts_alone):
    """A drafted key with a NaN, or whose score is +inf: NaN to the tokens that see it.  A score of -inf has no weight,
    unless it is all that a token sees."""
    lens = [0, 0] if drafts_alone else [400, 130]
    cache = Cache(heads([(64, 3), (48, 4)], 52), 1, 1, lens, cap=512).upload()
    mask = [np.eye(N, dtype=bool) for _ in lens]
    for m in mask:
        m[N - 1, 0] = True  # the last token sees the first one too
    call = Call(cache, G, N, mask=mask)
    call.q[..., 7] = 1.0  # (the sign of an infinite score is the key's)
    put(call)
    want = outputs(call)
    assert np.isfinite(want).all()
    good = call.kd.copy()
    for bad in (np.nan, np.inf, -np.inf):
        call.kd = good.copy()
        call.kd[:, :, 0, :, 7] = bad
        put(call)
        got = outputs(call)
        hit = np.zeros(want.shape, bool)
        if bad != -np.inf:
            hit[:, :, [0, N - 1]] = True
        elif drafts_alone:
            hit[:, :, 0] = True
        assert np.array_equal(np.isnan(got), hit), bad
        other = ~hit
        if bad == -np.inf:
            other[:, :, [0, N - 1]] = False
            # what the tokens 0 and N - 1 still see: the same without the first key
            alone = Call(cache, G, N, mask=[np.where(np.arange(N) == 0, False, m) for m in mask])
            alone.q, alone.kd = call.q, good
            put(alone)
            ref = outputs(alone)
            assert np.array_equal(got[:, :, N - 1], ref[:, :, N - 1])
            if not drafts_alone:
                assert np.array_equal(got[:, :, 0], ref[:, :, 0])
        assert np.array_equal(got[other], want[other])


def test_drafted_values():
    """An infinite drafted value is an infinity, or a NaN, to the tokens that see it, however small its weight."""
    cache = Cache(heads([(64, 3), (48, 4)], 53), 1, 1, [300]).upload()
    for scale in (1.0, 200.0):
        call = Call(cache, 4, 5, mask=[np.eye(5, dtype=bool) | (np.arange(5) == 1)], q_scale=scale)
        want = outputs(call)
        call.vd[0, 0, 1, 0, 9], call.vd[0, 0, 3, 0, 100] = np.inf, np.nan
        put(call)
        got = outputs(call)
        hit = np.zeros(want.shape, bool)
        hit[..., 9] = True
        hit[0, 0, 3, :, 100] = True
        assert np.array_equal(np.isfinite(got), ~hit)
        assert np.array_equal(got[~hit], want[~hit])


@pytest.mark.parametrize("slope", [np.inf, -np.inf, np.nan])
def test_infinite_slopes(slope):
    """slope * distance of a token to itself is NaN: so is a head's output; the other heads' are as they were, but for
    what another way to the softmax's reference changes (each way: probabilities rounded by 2^-8, outputs by 2^-8)."""
    cache = Cache(heads([(64, 3), (48, 4)], 54), 1, 1, [300]).upload()
    slopes = np.array([0.0, 0.01, 0.5, 0.0], np.float32)
    for kw in (dict(N=6), dict(N=1, drafts=False, pos=np.array([[299]]))):
        want = outputs(Call(cache, 4, slopes=slopes, **kw))
        call = Call(cache, 4, slopes=np.where(np.arange(4) == 1, slope, slopes).astype(np.float32), **kw)
        got = outputs(call)
        assert np.isnan(got[:, :, :, 1]).all()
        rest = [0, 2, 3]
        assert np.all(np.abs(got[:, :, :, rest] - want[:, :, :, rest]) <= near(call))


@pytest.mark.parametrize("slope", [1e25, 1e32, -1e25])
def test_steepest_slopes(slope):
    """Biases of up to -1e35 leave the last token seen (negative slopes: the first one), not nothing."""
    T = 300
    cache = Cache(heads([(64, 3), (48, 4)], 56), 1, 1, [T]).upload()
    slopes = np.array([slope, 0.01, 0.5, 0.0], np.float32)
    call = Call(cache, 4, 1, drafts=False, slopes=slopes, pos=np.array([[T + 2]]), window=200)
    got = outputs(call)
    v = cache.params[1]
    at = T - 1 if slope > 0 else T + 3 - 200
    want = attention.reconstruct(cache.codes[1, 0], v["W"], v["delta"], v["b"], v["mu"])[at]
    assert np.all(np.abs(got[0, 0, 0, 0] - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -16)
