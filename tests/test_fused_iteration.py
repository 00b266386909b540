"""The what-ifs of the fused iteration on the captured CNN trace, through the
oracle."""
import os

import numpy as np

from paper_2006_03318_amd import fused_iteration as F
from paper_2006_03318_amd import recipes as R
from paper_2006_03318_amd import trace as TR

GOLD = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "rocprof_cnn")


def _trace():
    return TR.build_graph(TR.read_rocprof_csv(GOLD), iterations=[2, 3])


def test_variants(oracle_mod):
    tg = _trace()
    g, vs, names = F.what_if(tg)
    assert len(names) == vs.n_variants == 5
    _, _, ms, _ = oracle_mod.run(g, vs)
    assert abs(int(ms[0]) - tg.measured_span) <= 0.01 * tg.measured_span      # as traced
    assert ms[1] <= ms[0] and ms[2] <= ms[0] and ms[3] <= ms[1] and ms[4] <= ms[3]


def test_update_becomes_one_kernel():
    tg = _trace()
    g, vs, _ = F.what_if(tg)
    update = tg.layer_names.index("weight update")
    k = R.is_kernel(g) & (g.layer == update)
    bits = (vs.remove_bits[:, 0] >> 1) & 1          # variant 1: fused update
    for it in (2, 3):
        ids = np.nonzero(k & (g.iteration == it))[0]
        assert ids.size > 1 and int((bits[ids] == 0).sum()) == 1
        p, q = R.task_ratios(vs, g, 1)
        keep = ids[bits[ids] == 0][0]
        assert g.dur[keep] * p[keep] // q[keep] == g.dur[ids].sum()
        p, q = R.task_ratios(vs, g, 4)              # a quarter, kernel by kernel
        quarter = g.dur[keep] * p[keep] // q[keep]
        assert g.dur[ids].sum() // 4 - ids.size <= quarter <= g.dur[ids].sum() // 4


def test_fused_layers_keep_their_longest_kernel():
    tg = _trace()
    g = tg.graph
    layers = [i for i, n in enumerate(tg.layer_names) if "BatchNorm" in n]
    assert layers
    g2, vs = R.compile_sweep(g, [[], [F.FuseLayers(layers)]])
    gone = ((vs.remove_bits[:, 0] >> 1) & 1).astype(bool)
    k = R.is_kernel(g)
    for la in layers:
        for it in (2, 3):
            ids = np.nonzero(k & (g.layer == la) & (g.iteration == it))[0]
            if ids.size:
                left = ids[~gone[ids]]
                assert left.size == 1 and g.dur[left[0]] == g.dur[ids].max()
                assert np.all(gone[g.launch_of[ids[gone[ids]]]])
    assert not np.any(gone[k & ~np.isin(g.layer, layers)])


def test_norms_become_one_kernel_a_pass(oracle_mod):
    """A trace whose layers carry the iteration's own names: each pass through
    a norm keeps one kernel, and the iteration is shorter for it."""
    tg = _trace()
    tg.layer_names = [n.split()[0] + " norm %d" % i if "BatchNorm" in n else n for i, n in enumerate(tg.layer_names)]
    norms = [i for i, n in enumerate(tg.layer_names) if "norm" in n]
    g, vs, names = F.what_if(tg)
    k = R.is_kernel(g)
    for v, name in enumerate(names):
        gone = ((vs.remove_bits[:, 0] >> v) & 1).astype(bool)
        for la in norms:
            for it in (2, 3):
                ids = np.nonzero(k & (g.layer == la) & (g.iteration == it))[0]
                assert ids.size == (2 if tg.layer_names[la].startswith("fwd") else 1)
                fused = name in ("fused norms", "both", "both, update in one pass")
                assert int(gone[ids].sum()) == (ids.size - 1 if fused else 0)
    _, _, ms, _ = oracle_mod.run(g, vs)
    assert ms[2] < ms[0] and ms[3] < ms[1] and ms[3] < ms[2]
