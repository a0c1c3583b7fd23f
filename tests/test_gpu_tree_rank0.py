"""cobra_tree_attn with K heads that have no channels, from parameter images whose offset of the (absent) basis
is none that could be read: behind the pool's last float, or off the 16-byte grid.  Nothing is read there."""
import struct

import numpy as np
import pytest
import torch

from paper_2609_24298_gb300 import cobra

from .serve_util import DEV, Cache, heads
from .test_gpu_tree import Call
from .test_lib_params import resign

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("place", ["end", "odd"])
@pytest.mark.parametrize("G,N", [(1, 1), (4, 6), (8, 9)])
def test_basis_of_no_channels_is_not_read(place, G, N):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache = Cache(heads([(0, 1), (0, 1), (40, 3), (64, 2)], 41), 1, 2, [300, 17]).upload()
    p = cache.params
    raw = bytearray(cobra.cobra_params_image(cache.r, cache.b, np.array([x["delta"] for x in p]), cache.offs,
                                             [x["W"] for x in p], np.stack([x["mu"] for x in p]).reshape(-1)).tobytes())
    floats = struct.unpack_from("<Q", raw, 32)[0]
    for h in range(2):
        struct.pack_into("<Q", raw, 64 + 64 * h + 24, floats if place == "end" else 2 * h + 1)
    img = resign(raw)
    assert cobra.cobra_params_verify(img) == cobra.COBRA_OK
    cobra.cobra_params_upload(cache.block, cache.block.numel(), img)
    Call(cache, G, N).run().check()
