"""Tree attention where units are cut into pieces: in several layers and heads, in batches of more than 32 sequences, and with
inputs that show a single key that is lost or taken twice."""
import numpy as np
import pytest
import torch

from attn_util import BF16, Attn
from paper_2607_16673_b200 import synth

pytestmark = pytest.mark.gpu

# query heads, key heads, columns, nodes: units of few rows, of up to 128, of more, and of 256 columns with few rows and with many
FORMS = [(4, 4, 64, 5), (8, 2, 128, 4), (14, 2, 64, 9), (8, 2, 128, 20), (32, 2, 64, 24), (32, 2, 128, 20), (2, 2, 256, 7), (16, 2, 256, 40)]


def trees(sizes, seed):
    rng = np.random.default_rng(seed)
    return [synth.random_tree_parent(n, 8, 4, rng) if n > 1 else synth.chain_parent(n) for n in sizes]


@pytest.mark.parametrize("H,HK,d,n", FORMS)
def test_cut_units_of_several_layers(H, HK, d, n):
    a = Attn(1, 3, H, HK, d, 32, [7001, 0, 2500], trees([n, 1, max(1, n // 2)], n))
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("H,HK,d,n", FORMS)
def test_cut_units_of_more_than_32_sequences(H, HK, d, n):
    rng = np.random.default_rng(n)
    sizes = rng.integers(1, n + 1, 75)
    sizes[[0, 40, 74]] = n
    lens = rng.integers(0, 1500, 75)
    lens[[3, 33, 64, 74]] = [5000, 3500, 0, 4100]
    a = Attn(2, 2, H, HK, d, 16, lens, trees(sizes, n))
    a.attend()
    assert a.status_value() == 0
    a.check()


@pytest.mark.parametrize("H,HK,d,n", FORMS)
@pytest.mark.parametrize("page", [16, 128])
def test_every_key_counts_once(H, HK, d, n, page):
    """All keys are zero, so that the rows a node attends weigh the same, and in every call each column of V is zero but for one
    row, another for each column, layer and head: an output is that row's value over the number of rows, zero where the node does
    not attend it, and twice or nothing where it is taken twice or lost.  Calls go on until every row had its turn.

    Weights are one, every sum is exact, the quotient is off by fp32's rounding and the output by bf16's."""
    L, lens, sizes = 2, [2900, 1300, 70], [n, max(1, n // 2), 1]
    a = Attn(3, L, H, HK, d, page, lens, trees(sizes, n))
    for cache in (a.k_cache, a.v_cache):
        cache.mul_(0.0)                                      # (what is not a number, in rows that nobody has, stays so)
    a.k.zero_()
    a.v.zero_()
    table = torch.from_numpy(a.table.astype(np.int64)).cuda()
    cols = torch.arange(d, device="cuda")
    seen = [a.seen(b).cuda() for b in range(3)]
    value, group = 2048.0, H // HK
    for call in range(-(-max(x + y for x, y in zip(lens, sizes)) // d)):
        want = torch.zeros(L, a.T, H, d, dtype=torch.float64, device="cuda")
        marks = []
        for b in range(3):
            lo, hi = int(a.offs[b]), int(a.offs[b + 1])
            share = value / (lens[b] + seen[b].sum(1, keepdim=True).double())            # of one row, by node
            for l in range(L):
                for h in range(HK):
                    key = (call * d + cols + 37 * (l * HK + h)) % (lens[b] + sizes[b])
                    at, node = key.clamp(max=max(0, lens[b] - 1)), (key - lens[b]).clamp(min=0)
                    cached = key < lens[b]
                    marks.append((a.v_cache[l, :, h], (table[b, at // page][cached], (at % page)[cached], cols[cached])))
                    marks.append((a.v[l, lo:hi, h], (node[~cached], cols[~cached])))
                    want[l, lo:hi, h * group:(h + 1) * group] = torch.where(cached | seen[b][:, node], share, 0.0)[:, None]
        for rows, index in marks:
            rows[index] = value
        a.o.fill_(7)
        a.attend()
        assert bool(((a.o.double() - want).abs() <= (BF16 + 2.0 ** -20) * want).all()), call
        for rows, index in marks:
            rows[index] = 0
    assert a.status_value() == 0
