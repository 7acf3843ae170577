"""Contexts of nearly 2^31 rows, the most that a page table may describe: tree attention behind them, commits to their end."""
import pytest
import torch

from attn_util import BF16, dev
from paper_2607_16673_b200 import binding as speca

pytestmark = pytest.mark.gpu


# units of few rows in tiles of 128 and of 64 keys, of up to 128 rows, of more, and of 256 columns
@pytest.mark.parametrize("H,d,n", [(1, 64, 3), (1, 256, 2), (8, 64, 4), (64, 64, 4), (8, 256, 4)])
def test_lengths_next_to_the_limit(H, d, n):
    """One sequence as long as the table is wide but for five rows, behind a short one.  All keys are zero, so every row weighs the
    same, and page p of four has ones in the columns c with c % 4 == p: an output is the share of its page among the rows.

    Counts stay below 2^24 in every sum of a piece (2^31 / 148 rows), which makes those exact; joining the pieces rounds each of
    some 160 additions of the sums and of the weights' sum by 2^-24, 2^-15 in all, and the output is rounded once to bf16."""
    page, max_pages = 32, (1 << 26) - 1
    length = max_pages * page - 5
    if torch.cuda.mem_get_info()[0] < 4 << 30:
        pytest.skip("needs 4 GB of device memory")
    gen = torch.Generator("cuda").manual_seed(d + H)
    k_cache = torch.zeros(1, 4, 1, page, d, dtype=torch.bfloat16, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    for p in range(4):
        v_cache[0, p, 0, :, p::4] = 1
    table = torch.full((2, max_pages), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 2
    # the second half of the pages is drawn from three of the four, so that its loss or repetition shows
    table[1].random_(0, 4, generator=gen)
    table[1, max_pages // 2:] %= 3
    lens = [17, length]
    q = torch.empty(1, 2 * n, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    k, v = torch.zeros(1, 2 * n, 1, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2 * n, 1, d, dtype=torch.bfloat16, device="cuda")
    o, status = torch.full_like(q, 7.0), dev([0])
    dims = speca.AttnDims(1, 2, H, 1, d, d ** -0.5, n, page, 4, max_pages)
    speca.attend_tree(dims, q, k, v, dev([0, n, 2 * n]), 2 * n, None, k_cache, v_cache, table, dev(lens), o,
                      speca.alloc_attn_workspace(dims), status)
    torch.cuda.synchronize()
    assert int(status) == 0
    rows = torch.stack([(table[1, :-1] == p).sum() for p in range(4)]).double() * page
    rows[int(table[1, -1])] += page - 5
    for i in range(n):
        short = torch.zeros(d, dtype=torch.float64, device="cuda")
        short[2::4] = 17 / (18 + i)
        far = rows.repeat(d // 4) / (length + i + 1)
        for at, want in ((i, short), (n + i, far)):
            assert bool(((o[0, at].double() - want).abs() <= (BF16 + 2.0 ** -14) * want).all()), (at, i)


@pytest.mark.parametrize("extra,in_place", [(0, False), (0, True), (1, False), (1, True)])
def test_commit_up_to_the_limit(extra, in_place):
    """Four rows appended where four are left, and where three are: then nothing is, and it is said."""
    page, max_pages, d = 32, (1 << 26) - 1, 64
    length = max_pages * page - 4 + extra
    if torch.cuda.mem_get_info()[0] < 2 << 30:
        pytest.skip("needs 2 GB of device memory")
    cache = [torch.zeros(1, 2, 1, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rec = [torch.empty(1, 4, 1, d, dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2)]
    table = torch.zeros(1, max_pages, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    kv_len, status = dev([length]), dev([0])
    out = kv_len if in_place else torch.zeros_like(kv_len)
    dims = speca.AttnDims(1, 1, 1, 1, d, 1.0, 4, page, 2, max_pages)
    speca.commit_kv(dims, *cache, table, kv_len, *rec, dev([0, 4]), 4, None, None, None, out, status)
    torch.cuda.synchronize()
    for x, y in zip(cache, rec):
        assert int(x[0, 0].count_nonzero()) == 0
        assert torch.equal(x[0, 1, 0, -4:], torch.zeros_like(y[0, :, 0]) if extra else y[0, :, 0])
        assert int(x[0, 1, 0, :-4].count_nonzero()) == 0
    assert out.tolist() == [length if extra else length + 4]
    assert int(status) == (speca.STATUS_BAD_PAGE if extra else 0)
