"""CTAs of the tree attention that refuse to work leave nothing behind that the joining kernel could take for theirs."""
import numpy as np
import pytest
import torch

from attn_util import Attn
from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import synth

pytestmark = pytest.mark.gpu

RECORDS = 32 * 160                     # bytes of the workspace in front of the sums: what the join is to do for each CTA


def test_hook_is_exported_but_not_declared():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert hasattr(speca.lib(), "speca_test_misplace_shared_memory")
    assert "speca_test_misplace" not in open(os.path.join(root, "include", "speca.h")).read()


@pytest.mark.parametrize("H,HK,d,n", [(6, 3, 64, 4), (9, 3, 128, 20), (24, 3, 128, 40), (24, 3, 256, 40)])
def test_refused_shared_memory_joins_nothing(H, HK, d, n):
    """The workspace holds, for every CTA, a record of two parts that lies inside this problem (layer 2, head 2, node 2, two rows
    from row 2): joined, it would overwrite outputs with the quotient of two zeros."""
    a = Attn(1, 3, H, HK, d, 16, [9000, 40], [synth.random_tree_parent(n, 8, 4, np.random.default_rng(n)), synth.chain_parent(n)])
    a.ws.zero_()
    a.ws[:RECORDS].view(torch.int32).fill_(2)
    hook = speca.lib().speca_test_misplace_shared_memory
    hook(1)
    try:
        a.attend()
        torch.cuda.synchronize()
    finally:
        hook(0)
    assert a.status_value() == speca.STATUS_TIMEOUT
    assert bool((a.o == 7).all())
    a.status.zero_()
    a.attend()
    assert a.status_value() == 0
    a.check()
