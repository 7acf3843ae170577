"""Tree attention over a paged cache against the definition in 64 bits: head layouts, lengths, pages, trees, what is masked."""
import numpy as np
import pytest
import torch

from attn_util import Attn, dev
from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import synth

pytestmark = pytest.mark.gpu


def trees(sizes, seed=0, depth=8, kids=4):
    rng = np.random.default_rng(seed)
    return [synth.random_tree_parent(n, depth, kids, rng) if n > 1 else synth.chain_parent(n) for n in sizes]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("H,HK", [(1, 1), (4, 4), (6, 2), (8, 1), (28, 4)])
def test_head_layouts(d, H, HK):
    a = Attn(1, 1, H, HK, d, 16, [300, 17, 0, 129], trees([5, 33, 12, 1]))
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_lengths_around_pages_and_tiles(d, page):
    lens = [0, 1, 2, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 513, 700]
    a = Attn(2, 1, 4, 2, d, page, lens, trees([1 + i % 9 for i in range(len(lens))]))
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("d,H,HK", [(64, 4, 4), (128, 8, 2), (256, 16, 2)])
def test_tree_sizes(d, H, HK):
    sizes = [1, 2, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 200]
    a = Attn(3, 1, H, HK, d, 32, [37 * i % 300 for i in range(len(sizes))], trees(sizes))
    a.attend()
    assert a.status_value() == 0
    a.check()


def test_large_trees_and_a_deep_one():
    rng = np.random.default_rng(4)
    parents = [synth.random_tree_parent(1024, 16, 4, rng), synth.chain_parent(700), np.full(300, -1), synth.chain_parent(1)]
    a = Attn(4, 1, 2, 1, 128, 16, [50, 3, 700, 0], parents)
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("d,H,HK", [(64, 14, 2), (128, 8, 2), (256, 4, 1)])
def test_prompts(d, H, HK):
    a = Attn(5, 1, H, HK, d, 16, [0, 100, 513, 1, 0], [np.zeros(n) for n in (1, 300, 64, 1300, 129)], chain=True)
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("H,HK,d", [(32, 8, 128), (16, 2, 256), (8, 8, 64)])
def test_long_contexts_are_split_and_joined(H, HK, d):
    a = Attn(6, 1, H, HK, d, 64, [20000, 1, 7777], trees([7, 3, 40]))
    a.attend()
    assert a.status_value() == 0
    a.check()


def test_many_short_sequences_and_layers():
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 90, 150)
    a = Attn(7, 3, 4, 2, 64, 16, lens, trees(rng.integers(0, 12, 150)))
    a.attend()
    assert a.status_value() == 0
    a.check()


def test_scores_that_grow_along_the_context():
    """Later keys score ever higher, so that what was summed before has to be scaled down again and again; and a
    context whose first key outweighs the rest."""
    a = Attn(8, 1, 4, 1, 128, 16, [900, 900], trees([4, 4]))
    for b, up in ((0, True), (1, False)):
        for i in range(900):
            f = (i if up else 899 - i) / 900 * 4
            page, row = int(a.table[b, i // 16]), i % 16
            a.k_cache[0, page, 0, row] = (a.q[0, int(a.offs[b]), 0] * f).to(torch.bfloat16)
    a.attend()
    assert a.status_value() == 0
    # scores up to 4 |q|^2 / sqrt(d) ~ 180: an error of 2^-24 d times that is 3e-3, above what check() allows for
    o, size = a.expected()
    assert float(((a.o.double() - o).abs() / (2.0 ** -6 * size)).max()) <= 1.0


def test_values_that_are_not_finite_reach_only_who_attends_them():
    parents = [np.array([-1, 0, 0, 1]), np.array([-1, 0])]
    a = Attn(9, 1, 4, 2, 128, 16, [40, 40], parents)
    a.v[0, 2] = float("inf")                      # node 2 of sequence 0: a leaf
    a.k[0, 4 + 1] = float("nan")                  # node 1 of sequence 1: a leaf
    a.attend()
    assert a.status_value() == 0
    assert not torch.isfinite(a.o[0, [2, 5]]).any()
    a.v[0, 2], a.k[0, 5] = 0, 0                   # (what nobody else attends does not enter the others' definition)
    want, size = a.expected()
    keep = [0, 1, 3, 4]
    assert float(((a.o[:, keep].double() - want[:, keep]).abs() / (2.0 ** -6 * size[:, keep])).max()) <= 1.0


def test_bad_sequences_are_skipped_and_reported():
    def faulty(change, bit):
        a = Attn(10, 2, 4, 2, 64, 16, [100, 200, 300], trees([6, 9, 4]))
        change(a)
        a.attend()
        assert a.status_value() == bit
        a.check(sequences=[0, 2])                 # sequence 1 keeps the 7 it was filled with
        assert bool((a.o[:, int(a.offs[1]):int(a.offs[2])] == 7).all())

    def parent(a):
        a.parent[6 + 3] = 3

    def table(value):
        def change(a):
            a.page_table[1, 200 // 16] = value
        return change

    def length(value):
        def change(a):
            a.kv_len[1] = value
        return change

    faulty(parent, speca.STATUS_BAD_PARENT)
    for value in (-1, 10 ** 6, 1 << 30):
        faulty(table(value), speca.STATUS_BAD_PAGE)
    for value in (-1, 16 * 100, (1 << 31) - 1, -(1 << 31)):
        faulty(length(value), speca.STATUS_BAD_PAGE)


def test_bad_offsets_are_skipped_and_reported():
    a = Attn(11, 1, 4, 2, 64, 16, [100, 200, 300], trees([6, 9, 4]))
    a.node_offsets[2] = 3                          # decreasing: sequence 1 is bad, and 2 begins inside 0
    a.attend()
    assert a.status_value() & speca.STATUS_BAD_OFFSETS
    a = Attn(11, 1, 4, 2, 64, 16, [100, 200], trees([6, 9]))
    a.dims.max_nodes = 8
    a.attend()
    assert a.status_value() == speca.STATUS_TOO_MANY
    a.check(sequences=[0])


def test_captured_and_replayed_with_other_lengths():
    a = Attn(12, 1, 8, 2, 128, 16, [5000, 333, 64], trees([9, 17, 1]))
    a.attend()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.attend()
    for lens in ([5000, 333, 64], [1, 200, 0], [4999, 1, 63]):
        a.lens = lens
        a.kv_len.copy_(dev(np.array(lens)))
        a.ws.fill_(255)                            # what an earlier call left in the workspace does not matter
        a.o.fill_(7)
        g.replay()
        assert a.status_value() == 0
        a.check()


def test_on_another_stream_and_deterministic():
    a = Attn(13, 1, 32, 8, 128, 16, [9000, 4000], trees([20, 64]))
    first = a.attend().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            a.o.fill_(0)
            a.attend()
            assert torch.equal(a.o, first)
    torch.cuda.synchronize()
    a.check()
