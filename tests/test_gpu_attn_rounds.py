"""The attention layers' calls as a serving loop makes them: a prompt, speculative rounds, a fork, captured rounds; and what the
documentation allows beyond that."""
import numpy as np
import pytest
import torch

from attn_util import BF16, Attn, dev
from paper_2607_16673_b200 import binding as speca
from paper_2607_16673_b200 import synth

pytestmark = pytest.mark.gpu


class Layer:
    """An attention layer of a stack over a paged cache, driven by the library's calls, and beside it every sequence's accepted
    tokens with their unrotated queries, keys and values, from which any output can be formed again in 64 bits."""

    def __init__(self, seed, B, H=8, HK=2, d=128, page=16, max_pages=40):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.B, self.H, self.HK, self.d, self.page = B, H, HK, d, page
        self.n_pages, self.max_pages = B * max_pages + 7, max_pages
        ids = self.rng.permutation(self.n_pages)
        self.free = list(ids[B * max_pages:])
        self.table = dev(ids[:B * max_pages].reshape(B, max_pages))
        shape = (1, self.n_pages, HK, page, d)
        self.k_cache, self.v_cache = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.wq, self.wk = (1 + 0.2 * torch.randn(1, d, device="cuda", generator=self.gen) for _ in range(2))
        self.freq = (1e4 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2))).float()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.kept = [(torch.zeros(HK, 0, d, device="cuda", dtype=torch.bfloat16),) * 2 for _ in range(B)]

    def records(self, sizes):
        T = int(sum(sizes))
        x = torch.empty(1, T, (self.H + 2 * self.HK) * self.d, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=self.gen)
        q = x[..., :self.H * self.d].unflatten(-1, (self.H, self.d))
        k = x[..., self.H * self.d:(self.H + self.HK) * self.d].unflatten(-1, (self.HK, self.d))
        v = x[..., (self.H + self.HK) * self.d:].unflatten(-1, (self.HK, self.d)).contiguous()
        return dev(np.concatenate([[0], np.cumsum(sizes)])), T, q, k, v

    def forward(self, sizes, parents):
        offs, T, q, k, v = self.records(sizes)
        dims = speca.AttnDims(1, self.B, self.H, self.HK, self.d, self.d ** -0.5, max(sizes), self.page, self.n_pages, self.max_pages)
        parent = None if parents is None else dev(np.concatenate(parents))
        qr, kr, o = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(v), None
        o = torch.empty_like(qr)
        speca.norm_rope(dims, q, k, self.wq, self.wk, 1e-6, self.freq, self.d, False, 1.0, offs, T, parent, self.kv_len, qr, kr, self.status)
        ws = speca.alloc_attn_workspace(dims)
        speca.attend_tree(dims, qr, kr, v, offs, T, parent, self.k_cache, self.v_cache, self.table, self.kv_len, o, ws, self.status)
        return dims, offs, T, parent, q, qr, kr, v, o

    def check(self, sizes, parents, offs, q, qr, kr, v, o):
        """q, k against their definition at the node's position, o against attention over what was accepted before and the path."""
        offs, at = offs.tolist(), [k.shape[1] for k, _ in self.kept]
        for b in range(self.B):
            p = np.arange(sizes[b]) - 1 if parents is None else parents[b]
            depth, seen = np.zeros(sizes[b], int), np.zeros((sizes[b], sizes[b]), bool)
            for i, up in enumerate(p):
                if up >= 0:
                    depth[i], seen[i] = depth[up] + 1, seen[up]
                seen[i, i] = True
            pos = torch.from_numpy(at[b] + depth).cuda().double()
            y = q[0, offs[b]:offs[b + 1]].double()
            y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * self.wq[0].double()
            ang = torch.outer(pos, self.freq.double())[:, None]
            a, c = y.chunk(2, -1)
            y = torch.cat([a * ang.cos() - c * ang.sin(), a * ang.sin() + c * ang.cos()], -1)
            mine = qr[0, offs[b]:offs[b + 1]].double()
            # one rounding, and fp32 before it: 2^-20 of the pair covers what test_gpu_kvcache.py derives
            pair = y.reshape(*y.shape[:-1], 2, -1).norm(dim=-2).repeat(1, 1, 2)
            assert bool(((mine - y).abs() <= BF16 * y.abs() + 2.0 ** -15 * pair).all())
            blocked = torch.cat([torch.zeros(sizes[b], at[b], dtype=torch.bool), ~torch.from_numpy(seen)], 1).cuda()
            for h in range(self.HK):
                keys = torch.cat([self.kept[b][0][h], kr[0, offs[b]:offs[b + 1], h]]).double()
                vals = torch.cat([self.kept[b][1][h], v[0, offs[b]:offs[b + 1], h]]).double()
                for g in range(h * (self.H // self.HK), (h + 1) * (self.H // self.HK)):
                    w = torch.softmax((mine[:, g] @ keys.T * self.d ** -0.5).masked_fill(blocked, -float("inf")), -1)
                    want, size = w @ vals, w @ vals.abs()
                    off = (o[0, offs[b]:offs[b + 1], g].double() - want).abs()
                    assert bool((off <= BF16 * want.abs() + (BF16 + 2.0 ** -10) * size).all())      # as attn_util.check()

    def keep(self, b, nodes, offs, kr, v):
        rows = [int(offs[b]) + i for i in nodes]
        self.kept[b] = tuple(torch.cat([old, new[0, rows].transpose(0, 1)], 1) for old, new in zip(self.kept[b], (kr, v)))


def test_prompt_rounds_and_a_fork():
    s = Layer(1, 3)
    # prompts, of which one arrives in two chunks
    for sizes in ([37, 200, 16], [1, 64, 5]):
        dims, offs, T, parent, q, qr, kr, v, o = s.forward(sizes, None)
        s.check(sizes, None, offs, q, qr, kr, v, o)
        speca.commit_kv(dims, s.k_cache, s.v_cache, s.table, s.kv_len, kr, v, offs, T, None, None, None, s.kv_len, s.status)
        for b in range(3):
            s.keep(b, range(sizes[b]), offs, kr, v)
    assert s.kv_len.tolist() == [38, 264, 21]
    # sequence 2 goes on as a copy of sequence 0: full pages are shared, the open one is copied
    table = s.table.tolist()
    own = table[2]
    full = 38 // s.page
    table[2] = table[0][:full] + own[full:]
    s.table.copy_(dev(np.array(table)))
    dims = speca.AttnDims(1, 3, s.H, s.HK, s.d, page_size=s.page, n_pages=s.n_pages)
    speca.copy_pages(dims, s.k_cache, s.v_cache, dev(np.array(table[0][full:full + 1])), dev(np.array(table[2][full:full + 1])), s.status)
    s.kv_len[2] = s.kv_len[0]
    s.kept[2] = s.kept[0]
    # rounds: trees of other sizes each, greedy acceptance, commit in place
    for step in range(6):
        sizes = [int(x) for x in s.rng.integers(1, 40, 3)]
        parents = [synth.random_tree_parent(n, 8, 4, s.rng) if n > 1 else synth.chain_parent(n) for n in sizes]
        dims, offs, T, parent, q, qr, kr, v, o = s.forward(sizes, parents)
        s.check(sizes, parents, offs, q, qr, kr, v, o)
        tok = dev(s.rng.integers(0, 3, T))
        target, root = dev(s.rng.integers(0, 3, T)), dev(s.rng.integers(0, 3, 3))
        path, plen, nxt = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((3, 8), 3, 3))
        speca.greedy_accept(3, 8, offs, parent, tok, target, root, path, plen, nxt, s.status)
        speca.commit_kv(dims, s.k_cache, s.v_cache, s.table, s.kv_len, kr, v, offs, T, parent, path, plen, s.kv_len, s.status)
        for b in range(3):
            s.keep(b, path[b, :int(plen[b])].tolist(), offs, kr, v)
        assert s.kv_len.tolist() == [k.shape[1] for k, _ in s.kept]
    assert int(s.status) == 0


def test_a_round_captured_and_replayed():
    """norm, attention, acceptance and commit in one graph; every replay finds the lengths the last one left."""
    s = Layer(2, 4, H=4, HK=1, d=64)
    s.kv_len.copy_(dev(np.array([0, 16, 31, 300])))
    s.k_cache.normal_(generator=s.gen)
    s.v_cache.normal_(generator=s.gen)
    parents = [synth.random_tree_parent(n, 8, 4, s.rng) for n in (12, 9, 30, 2)]
    sizes = [len(p) for p in parents]
    offs, T, q, k, v = s.records(sizes)
    dims = speca.AttnDims(1, 4, 4, 1, 64, 0.125, max(sizes), 16, s.n_pages, s.max_pages)
    parent = dev(np.concatenate(parents))
    qr, kr, o = torch.empty(1, T, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(v), torch.empty(1, T, 4, 64, dtype=torch.bfloat16, device="cuda")
    tok, target, root = dev(np.zeros(T)), dev(np.zeros(T)), dev(np.zeros(4))           # everything matches: the deepest path
    path, plen, nxt = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((4, 8), 4, 4))
    ws = speca.alloc_attn_workspace(dims)

    def round_():
        speca.norm_rope(dims, q, k, s.wq, s.wk, 1e-6, s.freq, 64, True, 1.0, offs, T, parent, s.kv_len, qr, kr, s.status)
        speca.attend_tree(dims, qr, kr, v, offs, T, parent, s.k_cache, s.v_cache, s.table, s.kv_len, o, ws, s.status)
        speca.greedy_accept(4, 8, offs, parent, tok, target, root, path, plen, nxt, s.status)
        speca.commit_kv(dims, s.k_cache, s.v_cache, s.table, s.kv_len, kr, v, offs, T, parent, path, plen, s.kv_len, s.status)

    start = [x.clone() for x in (s.kv_len, s.k_cache, s.v_cache)]
    round_()
    torch.cuda.synchronize()
    for x, y in zip((s.kv_len, s.k_cache, s.v_cache), start):
        x.copy_(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        round_()
    got = []
    for _ in range(3):
        g.replay()
        got.append((o.clone(), s.kv_len.clone()))
    captured = [x.clone() for x in (s.k_cache, s.v_cache)]
    for x, y in zip((s.kv_len, s.k_cache, s.v_cache), start):
        x.copy_(y)
    for want, lens in got:
        round_()
        assert torch.equal(o, want) and torch.equal(s.kv_len, lens)
    assert torch.equal(captured[0].view(torch.int16), s.k_cache.view(torch.int16))
    assert torch.equal(captured[1].view(torch.int16), s.v_cache.view(torch.int16))
    assert int(s.status) == 0


def test_two_calls_at_once_with_a_workspace_each():
    a, b = Attn(3, 1, 32, 8, 128, 16, [6000, 900], [synth.chain_parent(4)] * 2), Attn(4, 1, 16, 2, 256, 32, [3000, 77, 12], [synth.chain_parent(9)] * 3)
    first = [x.attend().clone() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for x, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                x.attend()
    torch.cuda.synchronize()
    for x, want in zip((a, b), first):
        assert torch.equal(x.o, want) and x.status_value() == 0
        x.check()


@pytest.mark.parametrize("lens", [[20000, 40], [150, 40]])
def test_a_bad_page_anywhere_in_a_split_context(lens):
    """The CTA that meets the page and those that do not agree on leaving the sequence alone."""
    a = Attn(5, 1, 8, 2, 128, 16, lens, [synth.chain_parent(20), synth.chain_parent(3)])
    for at in (0, lens[0] // 32, (lens[0] - 1) // 16):
        a.status.zero_()
        a.o.fill_(7)
        keep = int(a.page_table[0, at])
        a.page_table[0, at] = -1
        a.attend()
        a.page_table[0, at] = keep
        assert a.status_value() == speca.STATUS_BAD_PAGE
        a.check(sequences=[1])


@pytest.mark.parametrize("H,HK,d,n", [(64, 1, 128, 3), (128, 1, 64, 1), (48, 3, 256, 2), (256, 1, 64, 5)])
def test_many_query_heads_to_a_key_head(H, HK, d, n):
    a = Attn(6, 1, H, HK, d, 16, [100, 0, 513], [synth.chain_parent(n), synth.chain_parent(1), synth.chain_parent(n)])
    a.attend()
    assert a.status_value() == 0
    a.check()


def test_values_that_are_not_finite_in_each_kernel():
    """A leaf's value that is not finite, for units of few rows, of up to 128 and of more; split and whole contexts."""
    for H, HK, d, n in ((4, 4, 64, 9), (8, 1, 128, 12), (16, 1, 128, 40), (16, 2, 256, 17)):
        for lens in ([20, 300], [9000, 5]):
            a = Attn(7, 1, H, HK, d, 16, lens, [synth.random_tree_parent(n, 8, 4, np.random.default_rng(n)), synth.chain_parent(n)])
            p = a.parents[0]
            leaf = max(i for i in range(n) if i not in p)
            a.v[0, leaf, :, ::3] = float("inf")
            a.v[0, leaf, :, 1::3] = float("nan")
            a.attend()
            assert a.status_value() == 0
            got = a.o[0, leaf].clone()
            assert bool(torch.isinf(got[:, ::3]).all()) and bool(torch.isnan(got[:, 1::3]).all()) and bool(torch.isfinite(got[:, 2::3]).all())
            a.v[0, leaf] = 0
            want, size = a.expected()
            a.o[0, leaf], size[0, leaf] = want[0, leaf].to(torch.bfloat16), float("inf")
            assert float(((a.o.double() - want).abs() / ((BF16 + 2.0 ** -10) * size + BF16 * want.abs())).max()) <= 1.0


def test_caches_beyond_32_bits():
    """Pages whose elements lie past 2^32, for every call that takes the cache."""
    HK, d, page = 8, 128, 64
    n_pages = (1 << 32) // (HK * d * page) + 40
    if torch.cuda.mem_get_info()[0] < 6 * n_pages * HK * d * page:
        pytest.skip("needs 26 GB of device memory")
    k, v = (torch.empty(1, n_pages, HK, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a = Attn(8, 1, 16, HK, d, page, [200, 500], [synth.chain_parent(2), synth.chain_parent(20)], room=64)
    move = np.arange(n_pages - a.n_pages, n_pages)                  # the problem's pages, at the end of the large pool
    k[:, move[0]:], v[:, move[0]:] = a.k_cache, a.v_cache
    a.table = np.where((a.table >= 0) & (a.table < a.n_pages), a.table + move[0], -1).astype(np.int32)
    a.k_cache, a.v_cache, a.n_pages = k, v, n_pages
    a.dims.n_pages = n_pages
    a.page_table = dev(a.table)
    a.attend()
    assert a.status_value() == 0
    a.check()
    out = torch.empty_like(a.kv_len)
    speca.commit_kv(a.dims, k, v, a.page_table, a.kv_len, a.k, a.v, a.node_offsets, a.T, None, None, None, out, a.status)
    assert a.status_value() == 0 and out.tolist() == [202, 520]
    for b in range(2):
        for i in range(len(a.parents[b])):
            at = a.lens[b] + i
            page_at = int(a.table[b, at // page])
            assert torch.equal(k[0, page_at, :, at % page], a.k[0, int(a.offs[b]) + i])
            assert torch.equal(v[0, page_at, :, at % page], a.v[0, int(a.offs[b]) + i])
    src, dst = int(a.table[0, 0]), 3
    speca.copy_pages(a.dims, k, v, dev(np.array([src, dst])), dev(np.array([dst + 1, n_pages - 1])), a.status)
    assert a.status_value() == 0
    assert torch.equal(k[0, src].view(torch.int16), k[0, dst + 1].view(torch.int16))
    assert torch.equal(v[0, dst].view(torch.int16), v[0, n_pages - 1].view(torch.int16))


def test_refusals_of_the_binding_name_the_argument():
    a = Attn(9, 1, 4, 2, 64, 16, [20], [synth.chain_parent(3)])
    wide = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16, device="cuda")[..., ::2]
    with pytest.raises(speca.SpecaError, match="q"):
        speca.attend_tree(a.dims, wide, a.k, a.v, a.node_offsets, a.T, a.parent, a.k_cache, a.v_cache, a.page_table, a.kv_len, a.o,
                          a.ws, a.status)
    with pytest.raises(speca.SpecaError, match="kv_len"):
        speca.attend_tree(a.dims, a.q, a.k, a.v, a.node_offsets, a.T, a.parent, a.k_cache, a.v_cache, a.page_table,
                          a.kv_len.long(), a.o, a.ws, a.status)
    with pytest.raises(speca.SpecaError, match="workspace"):
        speca.attend_tree(a.dims, a.q, a.k, a.v, a.node_offsets, a.T, a.parent, a.k_cache, a.v_cache, a.page_table, a.kv_len,
                          a.o, a.ws[:256], a.status)
    freq = torch.ones(32, device="cuda")
    with pytest.raises(speca.SpecaError, match="dense"):
        speca.norm_rope(a.dims, wide, a.k, None, None, 1e-6, freq, 64, False, 1.0, a.node_offsets, a.T, a.parent, a.kv_len, a.o,
                        torch.empty_like(a.k), a.status)
    with pytest.raises(speca.SpecaError, match="inv_freq"):
        speca.norm_rope(a.dims, a.q, a.k, None, None, 1e-6, freq, 32, False, 1.0, a.node_offsets, a.T, a.parent, a.kv_len, a.o,
                        torch.empty_like(a.k), a.status)


@pytest.mark.parametrize("H,HK,d,n", [(4, 4, 64, 4), (8, 2, 128, 20), (8, 1, 128, 40), (16, 2, 256, 9)])
def test_a_wait_that_runs_out_is_reported(H, HK, d, n):
    """A CTA whose first keys never come gives up after its bounded wait, says so and leaves; the next call is as ever."""
    a = Attn(10, 1, H, HK, d, 16, [300, 40], [synth.random_tree_parent(n, 8, 4, np.random.default_rng(n)), synth.chain_parent(n)])
    hook = speca.lib().speca_test_withhold_first_load
    hook(1)
    try:
        a.attend()
        torch.cuda.synchronize()
    finally:
        hook(0)
    assert a.status_value() & speca.STATUS_TIMEOUT
    a.status.zero_()
    a.o.fill_(7)
    a.attend()
    assert a.status_value() == 0
    a.check()
