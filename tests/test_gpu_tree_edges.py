"""Where what a query sees begins and ends, against 64 bits within a bound that one token more or less breaks
(oracle.serve.tree_attend_close): the tokens on either side of each edge outweigh all others, and the one that is not seen
outweighs the one that is."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2609_24298_gb300 import cobra

from .serve_util import D, Cache, bf16, heads
from .test_gpu_tree import Call
from .tree_util import close_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()


def unit_heads(rk, bk, rv, bv, seed, kv=1, k_delta=1.0):
    """K heads then V heads whose bases are unit vectors: a query's projections are its own elements."""
    g = np.random.default_rng(seed)
    eye = np.eye(D, dtype=np.float32)
    out = []
    for r, b, delta in [(rk, bk, k_delta)] * kv + [(rv, bv, 0.03)] * kv:
        out.append(dict(r=r, b=b, W=eye[:, :r].copy(), delta=np.float32(delta), mu=(0.2 * g.standard_normal(D)).astype(np.float32)))
    return out


@pytest.mark.parametrize("amp,cap", [(0.28, 0.0), (1.1, 0.0), (0.28, 20.0), (1.1, 60.0), (4.0, 500.0)])
@pytest.mark.parametrize("N,G", [(1, 4), (6, 4), (16, 8)])
@pytest.mark.parametrize("window", [0, 1, 100, 128, 129, 1000])
def test_edges(window, N, G, amp, cap):
    """Score in log2 units of a code's step: amp; every token's channel i is its score for query token i.  The last token
    before a window and the first behind a position have the largest code, the ones inside of them a large one."""
    lens = [1500, 700, 129, 128, 127, 5]
    cache = Cache(unit_heads(16, 8, 32, 8, 7), 1, 1, lens, cap=1536, paged=N == 6)
    S, g = len(lens), np.random.default_rng(window + N)
    pos = np.array([[max(T - 1 - (61 * i) % T, 0) if i % 2 else T - 1 + i + s % 3 for i in range(N)] for s, T in enumerate(lens)])
    for s, T in enumerate(lens):
        k = np.full((1536, 16), 128)
        for i in range(N):
            p, end = int(pos[s, i]), min(T, int(pos[s, i]) + 1)
            if window and p - window >= 0:
                k[p - window, i] = 255
            for t, c in ((max(p - window + 1, 0) if window else 0, 200), (end - 1, 200), (end, 255)):
                if 0 <= t < 1536 and k[t, i] != 255:
                    k[t, i] = c
        v = g.integers(0, 256, (1536, 32))
        cache.put(cache.host, 0, s, 0, k)  # (behind the sequence's last token too)
        cache.put(cache.host, 1, s, 0, v)
        cache.codes[0, s], cache.codes[1, s] = k, v
    cache.upload()
    call = Call(cache, G, N, drafts=False, pos=pos, window=window, cap=cap)
    # q . e_i / sqrt d log2e = amp
    q = np.zeros((1, S, N, G, D))
    for i in range(N):
        q[:, :, i, :, i] = amp * np.sqrt(D) / serve.LOG2E * (1.0 + 0.05 * np.arange(G))
    call.q, q_d = bf16(q)
    call.q_d[:q_d.numel()] = q_d.reshape(-1)
    call.run()
    wrong = [(1, 0, 0), (-1, 0, 0), (0, -1, 0)] + ([(0, 0, 1), (0, 0, -1)] if window > 1 else [])
    close_check(call, pos, None, wrong)


def rows_cache(levels, kv, seqs, bv, rv, seed):
    """One score level per code row (a single K channel of 8 bits, `levels` codes), values that are a row's own."""
    g = np.random.default_rng(seed)
    rows = len(levels)
    cache = Cache(unit_heads(2, 8, rv, bv, seed, kv), 1, kv, [128 * rows - 50 * (s % 2) for s in range(seqs)], cap=128 * rows)
    for h in range(kv):  # (the sequences of a head hold the same, up to their lengths)
        k = np.full((128 * rows, 2), 128)
        k[:, 0] = np.repeat(levels, 128)
        v = np.repeat(g.integers(0, 2 ** bv, (rows, rv)), 128, axis=0)
        for i, codes in ((h, k), (kv + h, v)):
            cache.put(cache.host, i, 0, 0, codes)
            first, size = cache.address(i, 0, 0), rows * 16 * cache.params[i]["r"] * cache.params[i]["b"]
            for s, T in enumerate(cache.lens):
                at = cache.address(i, s, 0)
                cache.host[at:at + size] = cache.host[first:first + size]
                cache.codes[i, s] = codes[:T]
    return cache.upload()


PROFILES = {
    # each row 61 log2 units above the one before; each 61 below; slow rises whose jumps come every second or third row;
    # a row that stays below the slack and outweighs what the next rise leaves of it
    "rising": [0, 61, 122, 183, 244, 305, 366, 427, 488, 549],
    "falling": [549, 488, 427, 366, 305, 244, 183, 122, 61, 0],
    "slow": [0, 25, 50, 75, 100, 125, 150, 175, 200, 201],
    "shares": [0, 59, 61, 60, 61, 120, 122, 121, 121, 122],
    "peak in the middle": [0, 300, 301, 300, 10, 290, 301, 5, 0, 1],
}


@pytest.mark.parametrize("profile", PROFILES)
@pytest.mark.parametrize("N,G,rv,cap,slope", [(1, 4, 30, 0.0, 0.0), (2, 8, 128, 0.0, 0.0), (5, 5, 62, 0.0, 0.0), (9, 5, 128, 0.0, 0.0),
                                              (1, 4, 128, 700.0, 0.0), (5, 5, 128, 700.0, -0.25), (9, 5, 64, 700.0, 0.0),
                                              (2, 8, 64, 0.0, 0.125), (9, 5, 30, 0.0, -0.25)])
def test_reference_moves_within_a_part(profile, N, G, rv, cap, slope):
    """Some eight rows per CTA, each with a level and values of its own, so that a sum
    that is not rescaled, a stale reference or a part taken with the wrong weight shows as another row's values."""
    kv, seqs, amp = 4, 16, 2.25  # (amp: log2 units per code step)
    codes = np.round(np.tile(PROFILES[profile], 2) / amp).astype(np.int64)
    cache = rows_cache(codes, kv, seqs, 8, rv, len(profile) + N)
    slopes = None if not slope else np.resize([slope, 0.0, slope / 2], kv * G).astype(np.float32)
    call = Call(cache, G, N, drafts=N > 1, cap=cap, slopes=slopes)
    q = np.zeros((1, seqs, N, kv * G, D))
    q[..., 0] = amp * np.sqrt(D) / serve.LOG2E
    call.q, q_d = bf16(q)
    call.q_d[:q_d.numel()] = q_d.reshape(-1)
    call.kd[..., 0] = -120.0  # (the drafted keys are below every row's level in question)
    call.k_d[:call.kd.size] = bf16(call.kd.reshape(-1))[1]
    call.run()
    for h, s in ((0, 0), (1, 5), (3, 15)):
        ref, bound = close_check(call, None, [(h, s)])
        # what could be wrong lies outside of the bound: nothing, the mean of all rows, and that of the highest
        # and the one before it (the earlier one's sum not rescaled)
        p = cache.params[kv + h]
        values = p["mu"] + float(p["delta"]) * (cache.codes[kv + h, s] - 127.5) @ p["W"].T
        best = 128 * max(int(np.argmax(codes)), 1)
        for wrong in (0.0, values.mean(axis=0), 0.5 * (values[best] + values[best - 1])):
            assert (np.abs(ref - wrong) > bound).any(axis=-1).all()


@pytest.mark.parametrize("N,G", [(1, 4), (2, 8), (5, 5), (9, 5)])
@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("rv", [40, 128])
def test_loud_queries_with_biases(N, G, window, rv):
    """Biases of both signs on scores without a bound, over rows that are seen whole and in part."""
    cache = Cache(heads([(64, 2), (40, 3), (rv, 3), (64, 1)], 71), 1, 2, [900, 131, 1], paged=True).upload()
    slopes = np.resize([0.5, -0.5, 0.0, 3.0, -0.01, 0.004, 20.0, -7.0], 2 * G).astype(np.float32)
    pos = np.maximum(np.array([[T + i - (5 if i % 3 == 2 else 0) for i in range(N)] for T in cache.lens]), 0)
    call = Call(cache, G, N, drafts=N > 1, slopes=slopes, window=window, pos=pos, q_scale=12.0).run()
    close_check(call, pos)
