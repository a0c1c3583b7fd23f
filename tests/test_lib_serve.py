"""Refusals of the calls for serving with drafted tokens (cobra_norm_rope, cobra_append_tokens,
cobra_tree_attn, cobra_rope_table64): every check runs on the host before anything is launched, so the
addresses here are made up."""
import pytest

from paper_2609_24298_gb300 import cobra

A = 1 << 20  # an address aligned to anything
EINVAL, EALIGN, ESPACE = cobra.COBRA_EINVAL, cobra.COBRA_EALIGN, cobra.COBRA_ESPACE


def status(fn, *args):
    try:
        fn(*args)
    except cobra.CobraError as e:
        return e.status
    return cobra.COBRA_OK


def norm_args(**kw):
    d = dict(n_tok=3, n_q_heads=4, n_k_heads=2, norm=1, eps=1e-6, q_stride_tok=512, q_stride_head=128, k_stride_tok=256,
             k_stride_head=128, qo_stride_tok=512, qo_stride_head=128, ko_stride_tok=256, ko_stride_head=128)
    a = dict(q=A, k=A, qw=A, kw=A, pos=A, table=A, max_pos=100, qo=A, ko=A)
    for k, v in kw.items():
        (d if k in d else a)[k] = v
    return (cobra.norm_rope_desc(**d), *a.values())


@pytest.mark.parametrize("kw,want", [
    (dict(n_tok=-1), EINVAL), (dict(n_q_heads=-1), EINVAL), (dict(n_k_heads=-1), EINVAL),
    (dict(n_q_heads=0, n_k_heads=0), EINVAL), (dict(norm=0, table=None), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(qo=None), EINVAL),
    (dict(ko=None), EINVAL), (dict(pos=None), EINVAL), (dict(max_pos=0), EINVAL), (dict(max_pos=(1 << 22) + 1), EINVAL),
    (dict(norm=0), EINVAL), (dict(q=A + 8), EALIGN), (dict(ko=A + 2), EALIGN), (dict(q_stride_tok=516), EALIGN),
    (dict(ko_stride_head=129), EALIGN), (dict(qw=A + 4), EALIGN), (dict(table=A + 4), EALIGN), (dict(pos=A + 1), EALIGN),
    (dict(n_tok=0, q=None, k=None, pos=None), cobra.COBRA_OK),
])
def test_norm_rope(kw, want):
    assert status(cobra.cobra_norm_rope, *norm_args(**kw)) == want


def append_args(**kw):
    d = dict(k_head0=0, v_head0=8, layer_stride=8, n_layers=2, n_kv_heads=8, n_seqs=3, max_new=5, n_src=5, rows_per_seq=4,
             pages_per_seq=0)
    a = dict(params=A, desc=None, k=A, v=A, pos=A, n_new=A, index=A, table=A, max_pos=512, cache=A, page_table=None)
    for k, v in kw.items():
        (d if k in d else a)[k] = v
    a["desc"] = cobra.append_desc(**d)
    return tuple(a.values())


@pytest.mark.parametrize("kw,want", [
    (dict(params=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(pos=None), EINVAL),
    (dict(cache=None), EINVAL), (dict(k_head0=-1), EINVAL), (dict(v_head0=-1), EINVAL), (dict(n_layers=0), EINVAL),
    (dict(n_kv_heads=0), EINVAL), (dict(layer_stride=7), EINVAL), (dict(n_seqs=0), EINVAL), (dict(max_new=-1), EINVAL),
    (dict(n_src=0), EINVAL), (dict(n_src=4, index=None), EINVAL), (dict(rows_per_seq=0), EINVAL),
    (dict(page_table=A), EINVAL), (dict(pages_per_seq=-1), EINVAL), (dict(max_pos=0), EINVAL),
    (dict(k_head0=0x7ffffff0), EINVAL), (dict(n_seqs=0x7fffffff, max_new=0x7fffffff, n_src=0x7fffffff), EINVAL),
    (dict(params=A + 128), EALIGN), (dict(cache=A + 16), EALIGN), (dict(k=A + 1), EALIGN), (dict(pos=A + 2), EALIGN),
    (dict(table=A + 8), EALIGN), (dict(index=A + 2), EALIGN), (dict(max_new=0), cobra.COBRA_OK),
])
def test_append_tokens(kw, want):
    assert status(cobra.cobra_append_tokens, *append_args(**kw)) == want


def tree_args(**kw):
    d = dict(k_head0=0, v_head0=8, layer_stride=8, n_layers=2, n_kv_heads=8, group=4, n_seqs=3, rows_per_seq=4,
             pages_per_seq=0, max_draft=8, window=0, softcap=0.0)
    a = dict(params=A, desc=None, q=A, k=A, v=A, n_draft=A, mask=A, q_pos=A, slopes=A, cache=A, lens=A, page_table=None,
             out=A, ws=A, ws_bytes=1 << 40)
    for k, v in kw.items():
        (d if k in d else a)[k] = v
    a["desc"] = cobra.tree_desc(**d)
    return tuple(a.values())


@pytest.mark.parametrize("kw,want", [
    (dict(params=None), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(cache=None), EINVAL), (dict(lens=None), EINVAL), (dict(out=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(group=0), EINVAL), (dict(group=17), EINVAL), (dict(max_draft=0), EINVAL), (dict(max_draft=65), EINVAL),
    (dict(window=-1), EINVAL), (dict(softcap=-1.0), EINVAL), (dict(softcap=float("nan")), EINVAL),
    (dict(softcap=float("inf")), EINVAL), (dict(n_seqs=0), EINVAL), (dict(layer_stride=7), EINVAL),
    (dict(rows_per_seq=0), EINVAL), (dict(page_table=A), EINVAL), (dict(rows_per_seq=1 << 24), EINVAL),
    (dict(n_seqs=1 << 22), EINVAL), (dict(k_head0=-1), EINVAL), (dict(v_head0=0x7ffffffa), EINVAL),
    (dict(ws=A + 16), EALIGN), (dict(out=A + 1), EALIGN), (dict(mask=A + 4), EALIGN), (dict(q_pos=A + 2), EALIGN),
    (dict(params=A + 64), EALIGN), (dict(ws_bytes=1000), ESPACE),
])
def test_tree_attn(kw, want):
    assert status(cobra.cobra_tree_attn, *tree_args(**kw)) == want


def test_tree_workspace_size():
    size = lambda **kw: cobra.cobra_tree_workspace_size(tree_args(**kw)[1])
    assert size(max_draft=1) < size() < size(max_draft=64)
    assert size(n_seqs=6) > size()
    assert size() % 256 == 0
    assert status(cobra.cobra_tree_workspace_size, tree_args(group=0)[1]) == EINVAL


def test_rope_table64():
    assert cobra.cobra_rope_table64_bytes(1) == 17 * 128 * 8
    assert cobra.cobra_rope_table64_bytes(17) == 18 * 128 * 8
    assert status(cobra.cobra_rope_table64_bytes, 0) == EINVAL
    assert status(cobra.cobra_rope_table64_bytes, (1 << 22) + 1) == EINVAL
    assert status(cobra.cobra_rope_table64, 0.0, 16, A, 1 << 20) == EINVAL
    assert status(cobra.cobra_rope_table64, 1e4, 16, A + 8, 1 << 20) == EALIGN
    assert status(cobra.cobra_rope_table64, 1e4, 16, A, 1000) == ESPACE
    assert status(cobra.cobra_rope_table64, 1e4, 16, None, 1 << 20) == EINVAL


def test_header_names_the_calls_that_read_parameters_early():
    """Kernels that read the block ahead of their wait for the kernel in front are calls behind which a block must not be
    written: their names are in the header's paragraph on it."""
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = lambda *p: open(os.path.join(root, *p)).read()
    text = re.search(r"must not be written by the kernel directly ahead(.*?)plain stream order", src("include", "cobra.h"), re.S).group(1)
    early, ordered = text.split("finishes.")
    for file, kernel, call in (("append_run.cuh", " append_run_kernel(RunArgs", "cobra_append_tokens"),
                               ("tree.cuh", " tree_project(const TreeArgs", "cobra_tree_attn")):
        body = src("paper_2609_24298_gb300", "csrc", file)
        body = body[body.index(kernel):]
        first = min(body.index(x) for x in ("param_pool(", "head_table(", "tree_head(") if x in body)
        assert call in (early if first < body.index("grid_dep_wait();") else ordered)
