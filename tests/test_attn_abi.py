"""Refusals of the attention layers' calls on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import build as speca_build

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)     # never dereferenced: validation fails first
NULL, UNSUPPORTED, ALIGN, RANGE, WORKSPACE = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def lib():
    speca_build.build()
    return speca.lib()


def dims(**change):
    a = dict(n_layers=2, batch=3, heads=8, kv_heads=2, d_head=128, scale=0.1, max_nodes=8, page_size=16, n_pages=10, max_pages=4)
    a.update(change)
    return speca.AttnDims(**a)


def call(lib, what, d, **change):
    p = d.c()
    ref = ctypes.byref(p)
    f = dict(q=FAKE, k=FAKE, v=FAKE, offs=FAKE, T=0, parent=FAKE, kc=FAKE, vc=FAKE, table=FAKE, len=FAKE, o=FAKE, ws=FAKE,
             bytes=1 << 40, status=FAKE, wq=FAKE, wk=FAKE, eps=1e-6, freq=FAKE, rot=64, ql=1 << 20, qt=1 << 12, kl=1 << 20,
             kt=1 << 12, out=FAKE, depth=8, path=FAKE, plen=FAKE, src=FAKE, dst=FAKE, n=0)
    f.update(change)
    if what == "attend":
        return lib.speca_attend_tree(ref, f["q"], f["k"], f["v"], f["offs"], f["T"], f["parent"], f["kc"], f["vc"], f["table"],
                                     f["len"], f["o"], f["ws"], f["bytes"], f["status"], None)
    if what == "norm":
        return lib.speca_norm_rope(ref, f["q"], f["ql"], f["qt"], f["k"], f["kl"], f["kt"], f["wq"], f["wk"], f["eps"], f["freq"],
                                   f["rot"], 0, 1.0, f["offs"], f["T"], f["parent"], f["len"], f["o"], f["out"], f["status"], None)
    if what == "commit":
        return lib.speca_commit_kv(ref, f["kc"], f["vc"], f["table"], f["len"], f["k"], f["v"], f["offs"], f["T"], f["parent"],
                                   f["depth"], f["path"], f["plen"], f["out"], f["status"], None)
    return lib.speca_copy_pages(ref, f["kc"], f["vc"], f["src"], f["dst"], f["n"], f["status"], None)


CALLS = ["attend", "norm", "commit", "copy"]


@pytest.mark.parametrize("what", CALLS)
@pytest.mark.parametrize("change,code", [
    (dict(n_layers=0), RANGE), (dict(batch=0), RANGE), (dict(heads=0), RANGE), (dict(kv_heads=0), RANGE), (dict(kv_heads=3), UNSUPPORTED),
    (dict(d_head=96), UNSUPPORTED), (dict(d_head=512), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
    (dict(page_size=512), UNSUPPORTED), (dict(n_pages=0), RANGE), (dict(max_pages=0), RANGE), (dict(max_nodes=0), RANGE),
    (dict(max_nodes=8193), RANGE), (dict(n_pages=1 << 30), RANGE), (dict(max_pages=1 << 28), RANGE), (dict(batch=1 << 25), RANGE)])
def test_shapes_that_are_refused(lib, what, change, code):
    assert call(lib, what, dims(**change)) == code
    if what == "attend":
        d = dims(**change).c()
        assert lib.speca_attn_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("what,names", [("attend", "offs kc vc table len status"), ("norm", "offs len status freq"),
                                        ("commit", "kc vc table len offs out status path plen"), ("copy", "kc vc status")])
def test_missing_pointers(lib, what, names):
    for name in names.split():
        assert call(lib, what, dims(), **{name: None}) == NULL, name


@pytest.mark.parametrize("what,names", [("attend", "q k v o"), ("norm", "q k o out"), ("commit", "k v")])
def test_missing_packed_arrays(lib, what, names):
    for name in names.split():
        assert call(lib, what, dims(), T=4, **{name: None}) == NULL, name


@pytest.mark.parametrize("what,names", [("attend", "q k v kc vc o"), ("norm", "q k o out wq wk"), ("commit", "kc vc k v"),
                                        ("copy", "kc vc")])
def test_misaligned_pointers(lib, what, names):
    for name in names.split():
        assert call(lib, what, dims(), **{name: ODD}) == ALIGN, name


@pytest.mark.parametrize("what", ["attend", "norm", "commit"])
def test_node_counts(lib, what):
    assert call(lib, what, dims(), T=-1) == RANGE
    assert call(lib, what, dims(), T=25) == RANGE                       # batch * max_nodes is 24
    assert call(lib, what, dims(max_nodes=1025), T=4) == RANGE          # with a parent array
    assert call(lib, what, dims(n_layers=60000, max_nodes=1000, batch=100), T=100000) == RANGE


def test_rest(lib):
    assert call(lib, "norm", dims(), T=0) == 0                          # complete, nothing to do
    assert call(lib, "attend", dims(), T=0) == 0
    assert call(lib, "copy", dims()) == 0
    for rot, code in ((-16, UNSUPPORTED), (8, UNSUPPORTED), (24, UNSUPPORTED), (144, UNSUPPORTED)):
        assert call(lib, "norm", dims(), rot=rot) == code
    assert call(lib, "norm", dims(), rot=0, freq=None) == 0
    assert call(lib, "norm", dims(), wq=None, wk=None) == 0
    assert call(lib, "norm", dims(), eps=-1.0) == RANGE
    assert call(lib, "norm", dims(), T=4, qt=8 * 128 - 8) == RANGE      # tokens that overlap
    assert call(lib, "norm", dims(), T=4, kt=2 * 128 + 4) == ALIGN
    assert call(lib, "norm", dims(), T=4, ql=-8) == RANGE
    assert call(lib, "norm", dims(), T=4, kl=12) == ALIGN
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(lib, "attend", dims(scale=scale)) == RANGE
    d = dims().c()
    need = lib.speca_attn_workspace_bytes(ctypes.byref(d))
    assert need > 0
    assert call(lib, "attend", dims(), bytes=need - 1) == WORKSPACE
    assert call(lib, "attend", dims(), ws=None) == WORKSPACE
    assert call(lib, "attend", dims(), ws=ODD) == WORKSPACE
    for depth in (0, 17):
        assert call(lib, "commit", dims(), depth=depth) == RANGE
    assert call(lib, "copy", dims(), n=-1) == RANGE
    assert call(lib, "copy", dims(), n=11) == RANGE                     # more destinations than there are pages
    assert call(lib, "copy", dims(), n=3, src=None) == NULL
    assert lib.speca_attn_workspace_bytes(None) == 0
