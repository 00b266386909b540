"""The what-ifs of activations fused into the products beside them: on the captured CNN
trace through the oracle, and the iteration itself against the plain one."""
import os

import numpy as np
import pytest

from paper_2006_03318_amd import fused_iteration as F
from paper_2006_03318_amd import recipes as R
from paper_2006_03318_amd import trace as TR
from paper_2006_03318_amd import workloads as W

GOLD = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "rocprof_cnn")


def test_elementwise_kernels_of_the_layers_go(oracle_mod):
    """A trace whose layers carry the iteration's own names."""
    tg = TR.build_graph(TR.read_rocprof_csv(GOLD), iterations=[2, 3])
    tg.layer_names = [n.split()[0] + " mlp %d" % i if "BatchNorm" in n or "ReLU" in n else n for i, n in enumerate(tg.layer_names)]
    mlps = [i for i, n in enumerate(tg.layer_names) if "mlp" in n]
    g = tg.graph
    elem = (g.kind == W.K_ELEM) & R.in_layers(g, mlps)
    assert elem.any()
    base, _, _ = F.what_if(tg)
    g2, vs, names = F.what_if_products(tg)
    assert len(names) == vs.n_variants == 2
    gone = ((vs.remove_bits[:, 0]) & 1).astype(bool)
    assert np.array_equal(np.nonzero(gone & R.is_kernel(g))[0], np.nonzero(elem)[0])
    assert np.all(gone[g.launch_of[elem]])
    _, plain, _ = F.what_if(tg)
    _, _, before, _ = oracle_mod.run(base, plain)
    _, _, after, _ = oracle_mod.run(g2, vs)
    assert after[0] < before[0] and after[1] <= before[4]


@pytest.mark.gpu
def test_iteration_on_the_librarys_products():
    """The same training as with the framework's own products: five steps' losses, each off by the few roundings
    of 16 bits in which the two differ."""
    from tests.gpu_common import require_gpu
    require_gpu()
    _, plain = F.train(hidden=256, layers=3, rows=500, steps=2, fused=True)
    _, own = F.train(hidden=256, layers=3, rows=500, steps=2, fused=True, products=True)
    assert len(own) == 5 and np.allclose(own, plain, rtol=2.0 ** -8, atol=0)
