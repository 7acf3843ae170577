"""Norm and rotation, commit to the cache and copies of pages, against their definitions in 64 bits (or bit for bit)."""
import numpy as np
import pytest
import torch

from attn_util import BF16, Attn, dev
from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import synth

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ norm and rotation
def norm_case(seed, L, H, HK, d, lens, parents, rot, inter, weights=True, fused=False, scale=1.0, base=1e4):
    """Inputs, the call's outputs, and the 64-bit outputs with the sizes their errors are measured by."""
    gen = torch.Generator("cuda").manual_seed(seed)
    chain = parents is None or isinstance(parents, list) and all(isinstance(p, int) for p in parents)
    sizes = parents if chain else [len(p) for p in parents]
    offs = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    T, B = int(offs[-1]), len(sizes)
    x = torch.empty(L, T, (H + 2 * HK) * d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=gen)
    q = x[..., :H * d].unflatten(-1, (H, d))
    k = x[..., H * d:(H + HK) * d].unflatten(-1, (HK, d))
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    wq, wk = ((1 + 0.3 * torch.randn(L, d, device="cuda", generator=gen)) if weights else None for _ in range(2))
    half = rot // 2
    freq = (base ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(1, half))).float()
    out = [torch.full_like(t, 7.0, memory_format=torch.contiguous_format) for t in (q, k)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dims = speca.AttnDims(L, B, H, HK, d, max_nodes=max([1] + list(sizes)))
    parent = None if chain else dev(np.concatenate(parents))
    kv = dev(np.array(lens))
    args = (dims, q, k, wq, wk, 1e-6, freq, rot, inter, scale, dev(offs), T, parent, kv, out[0], out[1], status)
    speca.norm_rope(*args)
    torch.cuda.synchronize()
    assert int(status) == 0
    pos = []
    for b in range(B):
        depth = []
        for i in range(sizes[b]):
            up = i - 1 if chain else int(parents[b][i])
            depth.append(1 if up < 0 else depth[up] + 1)
        pos += [lens[b] + e - 1 for e in depth]
    angle = torch.outer(torch.tensor(pos, dtype=torch.float64, device="cuda"), freq.double())[None, :, None, :]
    for y, src, w in ((out[0], q, wq), (out[1], k, wk)):
        z = src.double()
        if w is not None:
            z = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()[:, None, None, :]
        first = torch.arange(half, device="cuda") * (2 if inter else 1)
        second = first + (1 if inter else half)
        a, b = z[..., first], z[..., second]
        want, size = z.clone(), z.abs()
        want[..., first] = scale * (a * angle.cos() - b * angle.sin())
        want[..., second] = scale * (a * angle.sin() + b * angle.cos())
        for e in (first, second):
            size[..., e] = scale * (a.abs() + b.abs())
        # one rounding to bf16, and fp32 before it: the norm's sum of d squares, square root and two products stay under
        # (d + 8) 2^-24 of the value, the angle (formed in 64 bits, rounded to fp32 as a part of a turn) and its sine and
        # cosine under 2^-21 of the pair
        off = (y.double() - want).abs()
        allowed = BF16 * want.abs() + ((d + 8) * 2.0 ** -24 + 2.0 ** -21) * size
        assert off.numel() == 0 or float((off / (allowed + 1e-30)).max()) <= 1.0
    return args


TREES = [synth.random_tree_parent(30, 8, 4, np.random.default_rng(0)), synth.chain_parent(1), np.full(5, -1),
         synth.chain_parent(16)]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (64, 16), (128, 128), (128, 48), (128, 0), (256, 256), (256, 64), (256, 176)])
def test_rotated_parts_and_layouts(d, rot, inter):
    norm_case(1, 2, 6, 2, d, [0, 5, 1000, 70000], TREES, rot, inter)


@pytest.mark.parametrize("H,HK", [(1, 1), (3, 1), (5, 5), (28, 4), (32, 8), (64, 1)])
def test_norm_head_layouts_and_strides(H, HK):
    norm_case(2, 3, H, HK, 128, [17, 0, 3, 9], TREES, 128, False, fused=True)
    norm_case(2, 1, H, HK, 64, [17], [1], 64, True, fused=True)


def test_far_positions():
    """Positions up to the largest length: the angle's whole turns are taken off in 64 bits."""
    far = [(1 << 31) - 40, 1 << 24, (1 << 20) + 1]
    norm_case(3, 1, 4, 2, 128, far, [33, 7, 1], 128, False, base=5e5)
    norm_case(3, 1, 4, 2, 128, far, [33, 7, 1], 64, True)


def test_without_norm_and_scaled():
    norm_case(4, 2, 4, 1, 64, [5, 100], [9, 30], 64, False, weights=False, scale=1.25)
    norm_case(4, 2, 4, 1, 256, [5, 100], [9, 30], 128, True, scale=0.5)


def test_many_tokens_and_layers():
    norm_case(5, 5, 8, 2, 128, list(range(60)), [1 + i % 90 for i in range(60)], 128, False, fused=True)


def test_norm_reports_bad_sequences_and_leaves_their_rows():
    parents = [np.array([-1, 0, 0]), np.array([-1, 0, 1, 1]), np.array([-1, -1])]
    args = list(norm_case(6, 2, 4, 2, 64, [3, 4, 5], parents, 64, False))
    dims, out, status = args[0], (args[14], args[15]), args[16]
    want = [x.clone() for x in out]

    def again(bit, bad):
        for x in out:
            x.fill_(7)
        status.zero_()
        speca.norm_rope(*args)
        torch.cuda.synchronize()
        assert int(status) == bit
        for x, w in zip(out, want):
            for t in range(9):
                assert bool((x[:, t] == 7).all()) if t in bad else torch.equal(x[:, t], w[:, t])

    args[12][3 + 2] = 2                           # a parent that is not before its node
    again(speca.STATUS_BAD_PARENT, range(3, 7))
    args[12][3 + 2] = 1
    args[13][1] = -2
    again(speca.STATUS_BAD_PAGE, range(3, 7))
    args[13][1] = 4
    dims.max_nodes = 3
    again(speca.STATUS_TOO_MANY, range(3, 7))


# ------------------------------------------------------------------------------------------------ commit
def commit_expected(a, order):
    k, v = a.k_cache.clone(), a.v_cache.clone()
    for b, nodes in enumerate(order):
        for i, t in enumerate(nodes):
            at = a.lens[b] + i
            page, row = int(a.table[b, at // a.page]), at % a.page
            k[:, page, :, row] = a.k[:, int(a.offs[b]) + t]
            v[:, page, :, row] = a.v[:, int(a.offs[b]) + t]
    return k, v


def bits(x):
    return x.view(torch.int16)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L,HK,d,page", [(1, 1, 64, 16), (3, 2, 128, 16), (2, 4, 256, 32), (2, 8, 128, 256)])
def test_commit_appends_the_accepted_path(L, HK, d, page, in_place):
    rng = np.random.default_rng(20)
    parents = [synth.random_tree_parent(n, 8, 4, rng) for n in (30, 12, 5, 64)] + [synth.chain_parent(8)]
    lens = [0, page - 1, 3 * page, page - 3, 40]
    a = Attn(20, L, HK, HK, d, page, lens, parents, room=16)
    order = [synth.root_path(p, int(np.argmax(synth.depth_of(p)))) for p in parents]
    order[1], order[2] = [], order[2][:1]
    path, plen = np.full((5, 8), -1, np.int32), np.zeros(5, np.int32)
    for b, p in enumerate(order):
        path[b, :len(p)], plen[b] = p, len(p)
    want = commit_expected(a, order)
    out = a.kv_len if in_place else torch.full_like(a.kv_len, -9)
    speca.commit_kv(a.dims, a.k_cache, a.v_cache, a.page_table, a.kv_len, a.k, a.v, a.node_offsets, a.T, a.parent, dev(path),
                    dev(plen), out, a.status)
    assert a.status_value() == 0
    assert out.tolist() == [n + len(p) for n, p in zip(lens, order)]
    assert torch.equal(bits(a.k_cache), bits(want[0])) and torch.equal(bits(a.v_cache), bits(want[1]))


@pytest.mark.parametrize("HK,d,page", [(2, 64, 16), (3, 128, 64), (1, 256, 128)])
def test_commit_appends_prompts(HK, d, page):
    sizes, lens = [300, 0, 1, 77, 1025], [0, 9, page, page - 1, 5]
    a = Attn(21, 2, HK, HK, d, page, lens, [np.zeros(n) for n in sizes], chain=True, room=1025)
    want = commit_expected(a, [range(n) for n in sizes])
    speca.commit_kv(a.dims, a.k_cache, a.v_cache, a.page_table, a.kv_len, a.k, a.v, a.node_offsets, a.T, None, None, None,
                    a.kv_len, a.status)
    assert a.status_value() == 0 and a.kv_len.tolist() == [n + m for n, m in zip(lens, sizes)]
    assert torch.equal(bits(a.k_cache), bits(want[0])) and torch.equal(bits(a.v_cache), bits(want[1]))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("fault", ["index", "chain", "deep", "page", "full", "length"])
def test_commit_skips_and_reports_a_bad_sequence(fault, in_place):
    parents = [np.array([-1, 0, 0, 2]), np.array([-1, 0, 1, 0]), np.array([-1, 0, 1])]
    lens = [5, 30, 2]
    a = Attn(22, 2, 2, 2, 64, 16, lens, parents, room=8)
    path = np.array([[0, 2, 3], [0, 1, 2], [0, 1, 2]], np.int32)
    plen = np.array([3, 3, 2], np.int32)
    bit = speca.STATUS_BAD_PATH
    if fault == "index":
        path[1, 2] = 4
    elif fault == "chain":
        path[1, 2] = 3                            # a sibling of node 1, not its child
    elif fault == "deep":
        plen[1], bit = 4, speca.STATUS_TOO_DEEP
    elif fault == "page":                         # the last of its new rows is on a page that is none
        a.page_table[1, 32 // 16] = a.n_pages
        bit = speca.STATUS_BAD_PAGE
    elif fault == "full":
        a.kv_len[1] = a.max_pages * 16 - 2
        bit = speca.STATUS_BAD_PAGE
    else:
        a.kv_len[1] = -1
        bit = speca.STATUS_BAD_PAGE
    before = a.kv_len.tolist()
    want = commit_expected(a, [[0, 2, 3], [], [0, 1]])
    out = a.kv_len if in_place else torch.full_like(a.kv_len, -9)
    speca.commit_kv(a.dims, a.k_cache, a.v_cache, a.page_table, a.kv_len, a.k, a.v, a.node_offsets, a.T, a.parent, dev(path),
                    dev(plen), out, a.status)
    assert a.status_value() == bit
    assert out.tolist() == [before[0] + 3, before[1], before[2] + 2]
    assert torch.equal(bits(a.k_cache), bits(want[0])) and torch.equal(bits(a.v_cache), bits(want[1]))


def test_commit_of_nothing():
    a = Attn(23, 1, 2, 2, 64, 16, [5, 3], [np.zeros(0), np.zeros(0)], chain=True)
    out = torch.full_like(a.kv_len, -9)
    want = bits(a.k_cache).clone()
    speca.commit_kv(a.dims, a.k_cache, a.v_cache, a.page_table, a.kv_len, a.k, a.v, a.node_offsets, 0, None, None, None, out,
                    a.status)
    assert a.status_value() == 0 and out.tolist() == [5, 3] and torch.equal(bits(a.k_cache), want)


# ------------------------------------------------------------------------------------------------ copies
def copy_case(seed, L, HK, d, page, n_pages, src, dst):
    gen = torch.Generator("cuda").manual_seed(seed)
    k, v = (torch.empty(L, n_pages, HK, page, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    dims = speca.AttnDims(L, 1, HK, HK, d, page_size=page, n_pages=n_pages)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = k.clone(), v.clone()
    speca.copy_pages(dims, k, v, dev(np.array(src)), dev(np.array(dst)), status)
    torch.cuda.synchronize()
    return (k, v), want, int(status)


@pytest.mark.parametrize("L,HK,d,page", [(1, 1, 64, 16), (3, 2, 128, 32), (2, 3, 256, 64), (2, 8, 128, 256)])
def test_pages_are_copied_in_every_layer(L, HK, d, page):
    rng = np.random.default_rng(30)
    ids = rng.permutation(60)
    src, dst = np.concatenate([ids[:10], ids[:10], ids[3:4]]), ids[20:41]
    got, want, status = copy_case(30, L, HK, d, page, 60, src, dst)
    for x, w in zip(got, want):
        w[:, torch.from_numpy(dst).cuda()] = w[:, torch.from_numpy(src).cuda()]
        assert torch.equal(x, w)
    assert status == 0


def test_copies_that_depend_on_an_order_are_not_made():
    #       good    twice the same target   source that is written   onto itself   out of range
    src = [0,       1, 2,                   5, 6,                    9,            40, 1, -1]
    dst = [10,      11, 11,                 6, 12,                   9,            13, 40, 14]
    got, want, status = copy_case(31, 2, 2, 64, 16, 40, src, dst)
    assert status == speca.STATUS_BAD_PAGE
    for x, w in zip(got, want):
        w[:, 10] = w[:, 0]
        w[:, 12] = w[:, 6]                        # 6 is not written: the pair that would have is refused
        assert torch.equal(x, w)


def test_more_copies_than_a_block_has_threads():
    src, dst = np.arange(700) % 300, np.arange(700) + 300
    got, want, status = copy_case(32, 1, 1, 64, 16, 1000, src, dst)
    assert status == 0
    for x, w in zip(got, want):
        w[:, 300:] = w[:, torch.from_numpy(src).cuda()]
        assert torch.equal(x, w)
