"""Caps of any size: within the close bound (oracle.serve.tree_attend_close), which holds nothing that grows with the
cap; a cap far above the scores changes nothing."""
import numpy as np
import pytest
import torch

from paper_2609_24298_gb300 import cobra

from .serve_util import Cache, heads
from .test_gpu_tree import Call
from .tree_util import close_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()


@pytest.mark.parametrize("N,G", [(1, 4), (4, 4), (4, 8), (9, 7)])
@pytest.mark.parametrize("q_scale", [0.5, 3.0, 12.0])
@pytest.mark.parametrize("cap", [1e-45, 1e-38, 1e-3, 5.0, 50.0, 55.0, 56.0, 200.0, 3e3, 1e5, 1e6, 1e7, 1e15, 9.9e29])
def test_caps(cap, q_scale, N, G):
    cache = Cache(heads([(64, 2), (40, 3), (20, 4), (128, 1)], 61, mu_scale=0.5), 1, 2, [513, 77], paged=True).upload()
    call = Call(cache, G, N, drafts=N > 1, cap=cap, q_scale=q_scale).run()
    close_check(call, None, [(0, 0), (1, 1)])


@pytest.mark.parametrize("N,G", [(1, 4), (4, 8), (9, 7)])
def test_large_caps_with_biases_and_windows(N, G):
    slopes = np.resize([0.5, 0.0, -0.03, 0.004], 2 * G).astype(np.float32)
    cache = Cache(heads([(64, 2), (40, 3), (20, 4), (128, 1)], 62), 1, 2, [900, 200], paged=True).upload()
    for cap in (60.0, 1e6, 1e20):
        call = Call(cache, G, N, drafts=N > 1, cap=cap, q_scale=8.0, slopes=slopes, window=300).run()
        close_check(call, None, [(0, 0), (1, 1)])
