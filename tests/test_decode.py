"""The decode step's tile graph: the work it stands for, and the block shapes of the kernels."""
import numpy as np
import pytest

from paper_2607_11262_gb300 import decode
from paper_2607_11262_gb300 import workloads as W


@pytest.mark.parametrize("case", decode.CASES)
def test_graph_holds_the_steps_work(case):
    g = decode.graph(**case)
    assert g.n_ctas <= decode.SMS
    sizes = np.diff(g.tpl_node_off.astype(np.int64))
    per = [g.work[o:o + n][(g.type[o:o + n] == W.LOAD)].astype(np.int64).sum() for o, n in zip(g.tpl_node_off, sizes)]
    loads = sum(per[t] for t in g.cta_template)
    rows = -(-case["seqs"] * 4 // decode.ROWS)
    want = 2 * 8 * 256 * (case["prefix"] * rows + case["seqs"] * case["own"])
    assert want <= loads <= 1.1 * want + decode.SMS * (decode.ROWS * 256 + 2 * 32768)


def test_params_are_a_valid_row():
    p = decode.gb300_params()
    assert p[W.P_NUM_SMS] == decode.SMS and p[W.P_HBM_BPC] == 3531
