"""Checks of a call of cobra_tree_attn (test_gpu_tree.Call) that tell one token more or less apart."""
from __future__ import annotations

import numpy as np

from oracle import serve
from paper_2609_24298_gb300 import cobra

from .serve_util import D


def close_check(call, pos, pairs=None, may_be_wrong=()):
    """Within the close bound at the (kv head, sequence) pairs of the first layer (None: all); and each of `may_be_wrong`, a change
    of (length, positions, window), breaks it somewhere."""
    assert cobra.cobra_check() == cobra.COBRA_OK
    c, G = call.c, call.G
    v0 = c.layers * c.kv
    o = call.o_v.double().cpu().numpy()
    broken = [False] * len(may_be_wrong)
    for h, s in pairs or [(h, s) for h in range(c.kv) for s in range(call.S)]:
        n = int(call.n[s])

        def want(n, T, p, window):
            kd, vd = (x[0, s, :n, h] if call.drafts else None for x in (call.kd, call.vd))
            return serve.tree_attend_close(call.q[0, s, :n, h * G:(h + 1) * G], c.codes[h, s][:T], c.codes[v0 + h, s][:T],
                                           c.params[h], c.params[v0 + h], kd, vd,
                                           None if call.mask is None else call.mask[s][:n, :n], p, window, call.cap,
                                           None if call.slopes is None else call.slopes[h * G:(h + 1) * G])

        T = c.lens[s]
        at = T + np.arange(n) if pos is None else np.asarray(pos[s][:n])
        ref, bound = want(n, T, at, call.window)
        got = o[0, s, :n, h * G * D:(h + 1) * G * D].reshape(n, G, D)
        assert np.all(np.abs(got - ref) <= bound), (h, s, np.abs(got - ref).max(), bound.max())
        m = min(n, 3)
        for k, (dT, dp, dw) in enumerate(may_be_wrong):
            if not broken[k]:
                other, _ = want(m, T + dT, at[:m] + dp, call.window + dw)
                broken[k] = bool((np.abs(other - ref[:m]) > 2 * bound[:m]).any())
    assert all(broken), broken
    return ref, bound
