"""Calls that the interface allows and one layer's tests do not make: parameter blocks in another order than K then V, a
part of a block's heads, outputs and drafts with strides of their own, more sequences and heads than a block of threads
counts at once, the most columns a head can have, calls with nothing to do."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2609_24298_gb300 import cobra

from .serve_util import D, DEV, Cache, bf16, heads
from .test_gpu_tree import Call
from .tree_util import close_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()


def reordered(cache, order):
    """The cache's parameter block with its heads in another order (None: a head of another model part)."""
    p = [cache.params[i if i is not None else 0] for i in order]
    pick = [i if i is not None else 0 for i in order]
    r, b = cache.r[pick], cache.b[pick]
    nbytes = cobra.cobra_params_bytes(r)
    block = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    cobra.cobra_params_build(block, nbytes, r, b, np.array([x["delta"] for x in p]), np.asarray(cache.offs)[pick],
                             [x["W"] for x in p], np.stack([x["mu"] for x in p]).reshape(-1))
    return block


RBS = [(64, 2), (30, 3), (128, 1), (16, 8), (48, 2), (96, 1), (20, 5), (64, 3)]


@pytest.mark.parametrize("drafts", [True, False])
def test_interleaved_block_and_strides(drafts):
    """Two layers of [V, other, K, other] heads behind three others; outputs, queries and drafts each with gaps."""
    L, H, G, S, N = 2, 2, 4, 3, 5
    cache = Cache(heads(RBS, 91), L, H, [300, 77, 0], cap=384, paged=True).upload()
    call = Call(cache, G, N, drafts=drafts, n_draft=[5, 2, 4])
    order = [None] * 3
    for l in range(L):
        order += [4 + 2 * l, 5 + 2 * l, None, 2 * l, 2 * l + 1, None, None]
    cache.block = reordered(cache, order)
    q = torch.full((S, N, L, H * G * D + 24), float("nan"), dtype=torch.bfloat16, device=DEV)
    k, v = (torch.full((N, H, S, L, D + 8), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    o = torch.full((N, L, S, H * G * D + 3), 123.0, dtype=torch.bfloat16, device=DEV)
    q[..., :H * G * D] = bf16(call.q.reshape(L, S, N, -1).transpose(1, 2, 0, 3))[1]
    for dst, src in ((k, call.kd), (v, call.vd)):
        dst[..., :D] = bf16(src.transpose(2, 3, 1, 0, 4))[1]
    d = call.desc
    d.v_head0, d.k_head0, d.layer_stride = 3, 6, 7
    d.q_stride_layer, d.q_stride_seq, d.q_stride_tok = q.stride(2), q.stride(0), q.stride(1)
    d.d_stride_layer, d.d_stride_seq, d.d_stride_tok, d.d_stride_head = k.stride(3), k.stride(2), k.stride(0), k.stride(1)
    d.o_stride_layer, d.o_stride_seq, d.o_stride_tok = o.stride(1), o.stride(2), o.stride(0)
    cobra.cobra_tree_attn(cache.block, d, q, k if drafts else None, v if drafts else None, call.n_d, None, None, None, cache.dev,
                          cache.lens_d, cache.table_d, o, call.ws, call.ws_bytes)
    call.o_v = o.permute(1, 2, 0, 3)
    call.check()


def test_many_sequences():
    """700 sequences (three blocks of 256), a third of them empty."""
    g = np.random.default_rng(92)
    S = 700
    lens = [int(x) if i % 3 else 0 for i, x in enumerate(g.integers(1, 200, S))]
    n = g.integers(0, 4, S)
    cache = Cache(heads([(20, 3), (32, 2)], 92), 1, 1, lens, cap=256, paged=True).upload()
    call = Call(cache, 2, 3, n_draft=n).run()
    call.S = S
    close_check(call, None, [(0, s) for s in range(0, S, 13) if n[s]])
    o = call.o_v.float().cpu().numpy()
    for s in range(S):
        assert np.all(o[0, s, n[s]:] == 123.0) and np.all(o[0, s, :n[s], :2 * D] != 123.0)


def test_many_heads():
    """280 kv heads of a call (two blocks of 256), of a few kinds."""
    kinds = heads([(2, 8), (16, 3), (0, 1), (30, 2)], 93)
    H = 280
    params = [kinds[i % 4] for i in range(H)] + [kinds[(i // 4) % 4] for i in range(H)]
    cache = Cache(params, 1, H, [130, 40]).upload()
    call = Call(cache, 1, 2).run()
    close_check(call, None, [(h, s) for h in range(0, H, 11) for s in range(2)])


def test_most_columns():
    """64 drafted tokens of 16 query heads: 1024 columns, sixteen tiles."""
    cache = Cache(heads([(64, 2), (40, 3)], 94), 1, 1, [333, 1], cap=384).upload()
    Call(cache, 16, 64, n_draft=[64, 51]).run().check()


def test_nothing_in_use():
    cache = Cache(heads([(64, 2), (40, 3)], 95), 1, 1, [333, 10]).upload()
    call = Call(cache, 4, 3, n_draft=[0, 0]).run().check()
    cache.lens_d.zero_()
    call = Call(cache, 4, 3, drafts=False).run()
    assert cobra.cobra_check() == cobra.COBRA_OK
    assert bool((call.o_v[..., :4 * D] == 0.0).all())


def test_append_to_an_interleaved_block():
    """Two layers of [V, other, K, other], the token rows of K and V in another order; some runs of none."""
    L, H, S, N = 2, 2, 3, 5
    cache = Cache(heads(RBS, 96), L, H, [0] * S, cap=384, paged=True).upload()
    order = [None]
    for l in range(L):
        order += [4 + 2 * l, 5 + 2 * l, None, 2 * l, 2 * l + 1, None, None]
    cache.block = reordered(cache, order)
    g = np.random.default_rng(96)
    x = bf16(1.3 * g.standard_normal((2, L, S, N, H, D)))[0]
    dev = []
    for side in range(2):
        t = torch.full((N, H, L, S, D + 2), float("nan"), dtype=torch.bfloat16, device=DEV)
        t[..., :D] = bf16(x[side].transpose(2, 3, 0, 1, 4))[1]
        dev.append(t)
    t = dev[0]
    desc = cobra.append_desc(v_head0=1, k_head0=4, layer_stride=7, n_layers=L, n_kv_heads=H, n_seqs=S, max_new=N, n_src=N,
                             pages_per_seq=cache.pps, x_stride_layer=t.stride(2), x_stride_seq=t.stride(3),
                             x_stride_tok=t.stride(0), x_stride_head=t.stride(1))
    pos, n = [126, 7, 300], [5, 0, 3]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    cobra.cobra_append_tokens(cache.block, desc, dev[0], dev[1], i32(pos), i32(n), None, None, 0, cache.dev, cache.table_d)
    assert cobra.cobra_check() == cobra.COBRA_OK
    want = cache.host.copy()
    for i in range(2 * L * H):
        side, l, h = i // (L * H), i // H % L, i % H
        for s in range(S):
            cache.put(want, i, s, pos[s], serve.new_codes(x[side, l, s, :n[s], h], cache.params[i]))
    assert np.array_equal(cache.dev.cpu().numpy(), want)
    # no run at all
    cobra.cobra_append_tokens(cache.block, desc, dev[0], dev[1], i32(pos), i32([0, 0, 0]), None, None, 0, cache.dev, cache.table_d)
    assert cobra.cobra_check() == cobra.COBRA_OK
    assert np.array_equal(cache.dev.cpu().numpy(), want)
