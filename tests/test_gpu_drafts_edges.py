"""Drafted tokens over the cache where attention and its certificate are most easily wrong: against oracle/drafts.py, with the tolerances of
test_gpu_drafts.py."""
import numpy as np
import pytest

import oracle
import workloads
from helpers import GpuLayerCache
from oracle import drafts
from test_gpu_drafts import assert_nodes, random_tree, tree_call

pytestmark = pytest.mark.gpu


def sequences(x, bt):
    """Four sequences over and over."""
    return np.tile(x, ((bt + 3) // 4,) + (1,) * (x.ndim - 1))[:bt]


# 33 .. 64, 65 .. 128 and up to 256 rows; a workgroup has a sequence, more than 64 blocks of it and not a multiple of 32
@pytest.mark.parametrize("n,n_tokens", [(13, 1157), (13, 1293), (27, 1093), (27, 1347), (64, 1093), (64, 1285)])
def test_widths_of_two_blocks_do_not_meet(n, n_tokens):
    """The first blocks are wide in one half of the channels, all others in the other half: a Delta over channels of two blocks is up to
    twice that of any block."""
    print("tree widths", n, n_tokens, flush=True)
    rng = np.random.default_rng(60 + n_tokens)
    bt = 256 if n * 4 <= 64 else 160
    k = rng.standard_normal((4, 1, n_tokens, 128)) * 0.05
    k[:, :, :64, :64] *= 20.0
    k[:, :, 64:, 64:] *= 20.0
    k, kd = k.astype(np.float16), workloads.normal_f16(rng, (4, 1, n, 128))
    v, vd = workloads.normal_f16(rng, (4, 1, n_tokens, 128)), workloads.normal_f16(rng, (4, 1, n, 128))
    q = workloads.normal_f16(rng, (4, n, 4, 128))
    seen = random_tree(rng, 4, n)
    nodes = np.unique([0, 1, n // 2, n - 1])
    oc = oracle.OracleLayerCache(4, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q[:, nodes], kd, vd, seen[:, nodes], oracle.Tolerances())
    with GpuLayerCache(bt, 4, 1, n_tokens, tier2=False) as gc:
        gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)))
    for at in range(4):
        for y in (O, flags, *cert.values()):
            assert all(np.array_equal(z, y[at]) for z in y[at::4])
        assert_nodes(ref[at:at + 1], O[at:at + 1, nodes], {f: y[at:at + 1, nodes] for f, y in cert.items()}, flags[at:at + 1, nodes], at)
