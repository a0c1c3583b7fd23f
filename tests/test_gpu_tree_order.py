"""Stream order covers the parameter block of cobra_tree_attn: the kernel directly ahead writes a head's basis (here the
angle table's, whose 16 + 112 rows of 128 floats are a basis of rank 128), and the call uses the finished one."""
import pytest
import torch

from paper_2609_24298_gb300 import cobra

from .serve_util import Cache, heads
from .test_gpu_tree import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head", [0, 1])
@pytest.mark.parametrize("N", [1, 12])
def test_parameters_written_by_the_kernel_ahead(N, head):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache = Cache(heads([(128, 2), (128, 2)], 81), 1, 1, [900, 40]).upload()
    # the pool is behind the header and two head entries, at a multiple of 256 bytes: W, mu, W^T mu of each head
    w_ptr = cache.block.data_ptr() + 256 + head * 4 * (128 * 128 + 128 + 128)
    a, b = Call(cache, 4, N), Call(cache, 4, N)
    got = []
    for theta in (3.0, 500000.0, 3.0):
        torch.cuda.synchronize()
        cobra.cobra_rope_table(theta, 16 * 112, w_ptr, 128 * 128 * 4)
        a.run()  # directly behind
        torch.cuda.synchronize()
        b.run()
        assert cobra.cobra_check() == cobra.COBRA_OK
        assert torch.equal(a.o_v, b.o_v)
        got.append(a.o_v.clone())
    assert torch.equal(got[0], got[2]) and not torch.equal(got[0], got[1])
