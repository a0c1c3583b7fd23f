"""cobra_norm_rope over all of bf16's range: vectors whose squares leave fp32's, within the bound of
test_gpu_norm_rope.py."""
import numpy as np
import pytest
import torch

from paper_2609_24298_gb300 import cobra

from .serve_util import D, DEV, bf16
from .test_gpu_norm_rope import THETA, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-12, 1e-6, 1e30])
@pytest.mark.parametrize("weight", [True, False])
def test_range(eps, weight):
    """Vectors of every size, one per (token, head), neighbours far apart; one element alone; the largest and smallest."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cobra.lib()
    g = np.random.default_rng(int(eps > 0) + weight)
    T, h = 60, 9
    x = g.standard_normal((T, h, D)) * 10.0 ** g.uniform(-38, 37.5, (T, h, 1))
    x[::5] *= np.arange(D) == 70  # a single element
    x[1::5] *= 10.0 ** g.uniform(-8, 0, (T // 5, h, D))  # elements of all sizes
    x[2, :, :] = 3.3895313892515355e38
    x[3, :, :] = 1e-38
    x[4, 0, :], x[4, 1, :] = 2.0 ** -133, 0.0 if eps else 2.0 ** -130
    x = bf16(np.clip(x, -3.38e38, 3.38e38))[0]
    if eps == 0.0:
        x[np.abs(x).max(axis=2) == 0.0] = 1.0  # (0 / 0 otherwise)
    w = [1.0 + 0.2 * g.standard_normal(D).astype(np.float32) for _ in range(2)] if weight else [None, None]
    pos = g.integers(0, 1000, T).astype(np.int32)
    nbytes = cobra.cobra_rope_table_bytes(1000)
    table = torch.empty(nbytes // 4, dtype=torch.float32, device=DEV)
    cobra.cobra_rope_table(THETA, 1000, table, nbytes)
    xd = bf16(x)[1]
    out = torch.empty((2, T, h, D), dtype=torch.bfloat16, device=DEV)
    desc = cobra.norm_rope_desc(n_tok=T, n_q_heads=h, n_k_heads=h, norm=1, eps=eps, q_stride_tok=h * D, q_stride_head=D,
                                k_stride_tok=h * D, k_stride_head=D, qo_stride_tok=h * D, qo_stride_head=D, ko_stride_tok=h * D,
                                ko_stride_head=D)
    wd = [None if v is None else torch.tensor(v, device=DEV, dtype=torch.float32) for v in w]
    for rotate in (False, True):
        cobra.cobra_norm_rope(desc, xd, xd, wd[0], wd[1], torch.tensor(pos, device=DEV) if rotate else None,
                              table if rotate else None, 1000 if rotate else 0, out[0], out[1])
        assert cobra.cobra_check() == cobra.COBRA_OK
        for side in range(2):
            check(out[side].double().cpu().numpy(), x, w[side], float(np.float32(eps)), pos if rotate else None, THETA)
