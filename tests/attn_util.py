"""Problems of the attention layers on the GPU, and what the calls have to give, in 64 bits and sequence by sequence."""
import numpy as np
import torch

from paper_2607_16673_b200 import binding as speca

BF16 = torch.finfo(torch.bfloat16).eps / 2          # a rounding to bf16 is off by at most this, relative to the value


def dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


class Attn:
    """A batch with committed lengths `lens` and drafts `parents` (arrays; with chain=True only their sizes count).  Pages are
    handed out in random order; table entries and rows that no sequence has are filled with what must never be used."""

    def __init__(self, seed, L, H, HK, d, page, lens, parents, chain=False, room=0, std_q=2.0):
        self.rng = np.random.default_rng(seed)
        gen = torch.Generator("cuda").manual_seed(seed)
        self.L, self.B, self.H, self.HK, self.d, self.page = L, len(lens), H, HK, d, page
        self.lens, self.chain = [int(x) for x in lens], chain
        self.parents = [np.arange(len(p)) - 1 if chain else np.asarray(p) for p in parents]
        self.offs = np.concatenate([[0], np.cumsum([len(p) for p in parents])]).astype(np.int32)
        self.T = T = int(self.offs[-1])
        need = [-(-(n + room) // page) for n in self.lens]
        self.max_pages, used = max(1, max(need)) + 1, sum(need)
        self.n_pages = used + 4
        ids = self.rng.permutation(self.n_pages)
        self.table = self.rng.choice(np.array([-1, -5, 1 << 30, self.n_pages], np.int32), (self.B, self.max_pages))
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.free = ids[at:]

        def normal(*shape, std=1.0):
            return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)

        self.k_cache, self.v_cache = normal(L, self.n_pages, HK, page, d), normal(L, self.n_pages, HK, page, d)
        live = torch.zeros(self.n_pages, page, dtype=torch.bool, device="cuda")
        for b, n in enumerate(self.lens):
            for i in range(-(-n // page)):
                live[int(self.table[b, i]), :min(page, n - i * page)] = True
        for cache in (self.k_cache, self.v_cache):
            cache.masked_fill_(~live[None, :, None, :, None], float("nan"))
        self.q, self.k, self.v = normal(L, T, H, d, std=std_q), normal(L, T, HK, d), normal(L, T, HK, d)
        self.o = torch.full((L, T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
        most = max([1] + [len(p) for p in parents])
        self.dims = speca.AttnDims(L, self.B, H, HK, d, d ** -0.5, most, page, self.n_pages, self.max_pages)
        self.node_offsets, self.page_table, self.kv_len = dev(self.offs), dev(self.table), dev(np.array(self.lens))
        flat = np.concatenate(self.parents) if self.parents else np.zeros(0)
        self.parent = None if chain else dev(flat)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = speca.alloc_attn_workspace(self.dims)

    def attend(self):
        speca.attend_tree(self.dims, self.q, self.k, self.v, self.node_offsets, self.T, self.parent, self.k_cache,
                          self.v_cache, self.page_table, self.kv_len, self.o, self.ws, self.status)
        return self.o

    def status_value(self):
        torch.cuda.synchronize()
        return int(self.status.item())

    def rows(self, cache, l, h, b):
        """Committed rows of one head of one sequence."""
        pages = torch.from_numpy(self.table[b, :-(-self.lens[b] // self.page)].astype(np.int64)).to(cache.device)
        return cache[l, pages, h].reshape(-1, self.d)[:self.lens[b]]

    def seen(self, b):
        """Whether node j is node i or its ancestor."""
        p = self.parents[b]
        m = np.zeros((len(p), len(p)), bool)
        for i, up in enumerate(p):
            if up >= 0:
                m[i] = m[up]
            m[i, i] = True
        return torch.from_numpy(m)

    def expected(self, sequences=None):
        """o in 64 bits, and the sum of weights times |v|, which its error is measured by."""
        o = torch.full((self.L, self.T, self.H, self.d), 7.0, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(o)
        for b in range(self.B) if sequences is None else sequences:
            lo, hi = int(self.offs[b]), int(self.offs[b + 1])
            if lo == hi:
                continue
            blocked = torch.cat([torch.zeros(hi - lo, self.lens[b], dtype=torch.bool), ~self.seen(b)], 1).cuda()
            for l in range(self.L):
                for h in range(self.HK):
                    k = torch.cat([self.rows(self.k_cache, l, h, b), self.k[l, lo:hi, h]]).double()
                    v = torch.cat([self.rows(self.v_cache, l, h, b), self.v[l, lo:hi, h]]).double()
                    for g in range(h * (self.H // self.HK), (h + 1) * (self.H // self.HK)):
                        s = (self.q[l, lo:hi, g].double() @ k.T * self.dims.scale).masked_fill(blocked, -float("inf"))
                        w = torch.softmax(s, -1)
                        o[l, lo:hi, g] = w @ v
                        size[l, lo:hi, g] = w @ v.abs()
        return o, size

    def check(self, sequences=None):
        """Every output within what rounding allows; rows of other sequences as they were.

        A weight is rounded to bf16 (off by BF16 of itself), o once more; both at worst add up along the sum.  The rest is
        fp32: a score is a sum of d products, off by at most d 2^-24 of scale sum |q||k|, which for d = 256 and these inputs
        (|q| ~ 2, |k| ~ 1, 20 of scale sum) is 3e-4; the weight follows the score, its denominator as well: 2^-10 covers
        both, and the exponential's and the sums' own 2^-20."""
        o, size = self.expected(sequences)
        allowed = BF16 * o.abs() + (BF16 + 2.0 ** -10) * size + 1e-30
        off = (self.o.double() - o).abs()
        assert torch.isfinite(self.o).all()
        worst = float((off / allowed).max()) if off.numel() else 0.0
        assert worst <= 1.0, worst
