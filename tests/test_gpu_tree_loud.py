"""Queries far beyond f16 next to ordinary ones of the same kv head and sequence."""
import numpy as np
import pytest
import torch

from paper_2609_24298_gb300 import cobra

from .serve_util import D, Cache, bf16, heads
from .test_gpu_tree import Call
from .test_gpu_tree_nonfinite import near, outputs, put

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()


@pytest.mark.parametrize("N,G", [(1, 4), (8, 4), (16, 8)])
def test_loud_query_leaves_the_others_alone(N, G):
    """Queries far beyond f16 (scaled by powers of two) next to ordinary ones of the same kv head."""
    cache = Cache(heads([(64, 3), (48, 4)], 55), 1, 1, [700]).upload()
    call = Call(cache, G, N, q_scale=4.0).run().check()
    for scale in (2.0 ** 20, 2.0 ** 60, 2.0 ** 110):
        call.q[0, 0, N // 2, 1] = bf16(scale * np.random.default_rng(1).standard_normal(D))[0]
        put(call)
        got = outputs(call)
        loud = call.q[0, 0, N // 2, 1].copy()
        assert np.isfinite(got).all()
        # one token takes all of the loud one: one of those with the highest scores
        k, v = cache.params
        keys = k["mu"] + float(k["delta"]) * (cache.codes[0, 0] - 3.5) @ k["W"].T.astype(np.float64)
        values = v["mu"] + float(v["delta"]) * (cache.codes[1, 0] - 7.5) @ v["W"].T.astype(np.float64)
        keys, values = (np.concatenate([a, b[0, 0, :N // 2 + 1, 0]]) for a, b in ((keys, call.kd), (values, call.vd)))
        best = np.argsort(keys @ loud)[::-1][:6]
        assert np.abs(values[best] - got[0, 0, N // 2, 1]).max(axis=1).min() <= 2.0 ** -7 * np.abs(values).max()
        # the others' as without it
        quiet = Call(cache, G, N, q_scale=4.0)
        quiet.q[0, 0, N // 2, 1] = 0.0
        put(quiet)
        want = outputs(quiet)
        other = np.ones(want.shape, bool)
        other[0, 0, N // 2, 1] = False
        assert np.all(np.abs(got - want)[other] <= near(call))
