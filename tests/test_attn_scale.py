"""Scales of the attention that fp32 does not hold: softmax(scale s) is formed as 2^(scale log2(e) s), so that product has to be
finite.  On the host, before anything is launched (no GPU needed)."""
import ctypes
import math

import pytest

from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import build as speca_build

FAKE = ctypes.c_void_p(0x1000)         # aligned, never dereferenced: there are no nodes
MOST = 2.0 ** 128 * (1 - 2.0 ** -24) / math.log2(math.e)


@pytest.mark.parametrize("scale,code", [(3.39e38, -4), (2.5e38, -4), (MOST * (1 + 2.0 ** -20), -4), (MOST * (1 - 2.0 ** -20), 0), (1e38, 0), (1.0, 0), (1e-30, 0)])
def test_scales(scale, code):
    speca_build.build()
    d = speca.AttnDims(1, 1, 2, 1, 64, scale, 1, 16, 1, 1).c()
    assert speca.lib().speca_attend_tree(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, 0, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                         FAKE, None) == code
