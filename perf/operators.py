"""The attention layers of a hybrid stack in a speculative round, as measurable cases.

Between its gated-delta-rule layers such a stack has layers with softmax attention over a paged cache of keys and values.
A round takes a draft through them by four calls: queries and keys are normed and rotated by their place in the tree
(``norm``), every node attends the committed context and its own ancestors (``attend``), the keys and values of the accepted
path are appended to the cache (``commit``), and a forked sequence gets its own copy of the pages it will write
(``copy``).

Layouts: q, o bf16 [L, T, Hq, d]; k, v bf16 [L, T, Hkv, d]; caches bf16 [L, pages, Hkv, page, d]; page table int32
[B, max_pages], -1 where a sequence has no page; kv_len int32 [B]; nodes packed over the batch by node_offsets, parent
local to the sequence (-1: child of the committed context), no parent array at all for chains and prompts.
"""
import math

import numpy as np
import torch

own = False                                 # whether run() makes the library's calls

DEV = "cuda"
EPS = 1e-6


def _case(op, L, B, Hq, Hkv, d, page, lo, hi, kind, nlo, nhi, rot=0, inter=False, base=1e4):
    # L layers in the call, B sequences with lo..hi committed tokens, kind/nlo..nhi the draft (one: a single token, chain,
    # tree, prompt: a chunk of a prompt); rot, inter, base: rotated part of a head, pair layout, frequency base
    return dict(op=op, L=L, B=B, Hq=Hq, Hkv=Hkv, d=d, page=page, lo=lo, hi=hi, kind=kind, nlo=nlo, nhi=nhi, rot=rot,
                inter=inter, base=base)


def listed():
    def c(name, *a, **k):
        return dict(name=name, **_case(*a, **k))

    return [
        # one user, a short conversation, a chain of four drafted tokens: the smallest call, latency counts
        c("attend_chain4_1user", "attend", 1, 1, 32, 8, 128, 16, 1000, 1000, "chain", 4, 4),
        # a serving batch, ragged contexts, ragged draft trees
        c("attend_tree_b32", "attend", 1, 32, 32, 8, 128, 16, 500, 8000, "tree", 8, 32),
        # a round without drafts at the largest batch: one token per sequence over long contexts
        c("attend_single_b64", "attend", 1, 64, 32, 8, 128, 64, 2000, 16001, "one", 1, 1),
        # wide heads, eight query heads to a key head, full trees over long contexts: many rows to a key
        c("attend_tree64_d256", "attend", 1, 16, 16, 2, 256, 32, 2001, 30000, "tree", 40, 64),
        # a chunk of a prompt behind what is cached already, two users
        c("attend_prompt_b2", "attend", 1, 2, 32, 8, 128, 16, 1500, 4096, "prompt", 1024, 1024),
        # one user, one layer, one token: all of it is launch and latency
        c("norm_one", "norm", 1, 1, 32, 8, 128, 16, 777, 777, "one", 1, 1, rot=128),
        # a full batch of trees in twelve layers, wide heads, a quarter of the head rotated, interleaved pairs
        c("norm_tree_b128", "norm", 12, 128, 16, 2, 256, 16, 100, 30000, "tree", 24, 64, rot=64, inter=True, base=1e7),
        # prompt chunks of one layer at far positions
        c("norm_prompt_b8", "norm", 1, 8, 32, 8, 128, 16, 1000, 500000, "prompt", 1024, 1024, rot=128, base=5e5),
        # accepted paths of a full batch of trees, all attention layers of the stack
        c("commit_tree_b128", "commit", 12, 128, 32, 8, 128, 16, 100, 2000, "tree", 24, 64),
        # prompt chunks of four users go into the cache
        c("commit_prompt_b4", "commit", 12, 4, 16, 2, 256, 64, 1, 1500, "prompt", 700, 1024),
        # one fork of one user's conversation
        c("copy_one", "copy", 12, 1, 16, 2, 256, 64, 900, 900, "one", 1, 1),
        # open pages of a full batch, forked four ways
        c("copy_b256", "copy", 12, 256, 32, 8, 128, 32, 100, 900, "one", 4, 4),
    ]


_HEADS = [(8, 8, 64), (14, 2, 64), (32, 8, 128), (24, 8, 128), (28, 4, 128), (16, 2, 256), (8, 2, 256), (16, 16, 128)]


def draw(rng):
    """One more case of the ranges above; cost bounded by the largest listed case's."""
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["attend"] * 5 + ["norm"] * 3 + ["commit"] * 2 + ["copy"])
    Hq, Hkv, d = rng.choice(_HEADS)
    page = rng.choice([16, 32, 64, 128])
    B = log_int(1, 64 if op == "attend" else 128)
    kind = rng.choice(["one", "chain", "tree", "tree", "prompt"])
    nhi = {"one": 1, "chain": rng.randint(2, 16), "tree": rng.randint(9, 64), "prompt": log_int(65, 1024)}[kind]
    nlo = nhi if kind == "one" else rng.randint(max(1, nhi // 4), nhi)
    hi = log_int(8, 30000)
    L = 1 if op == "attend" else rng.choice([1, 4, 12])
    if op == "attend":
        # keys of the batch, and scores of the padded batch
        hi = min(hi, (1 << 29) // (B * Hkv * d))
        if kind == "prompt":
            B = min(B, 4)
            hi = min(hi, 8000)
        hi = max(8, min(hi, (1 << 30) // (B * Hq * nhi)))
    elif op == "norm":
        if kind == "prompt":
            B, L = min(B, 8), 1
        hi = hi * rng.choice([1, 16])
    elif op == "commit":
        if kind == "prompt":
            B = min(B, 4)
        hi = max(8, min(hi, 2000, (1 << 28) // (B * Hkv * d * L)))
    else:
        kind, nlo, nhi = "one", 1, rng.randint(1, 4)
        nlo = nhi
        hi = max(8, min(hi, 900, (1 << 28) // (B * Hkv * d * L)))
    rot, inter, base = 0, False, 1e4
    if op == "norm":
        rot = rng.choice([d, d, d // 2, d // 4])
        inter = rng.random() < 0.4
        base = rng.choice([1e4, 5e5, 1e7])
    lo = 0 if op != "copy" and rng.random() < 0.2 else rng.randint(1, hi)
    while True:
        case = _case(op, L, B, Hq, Hkv, d, page, lo, hi, kind, nlo, nhi, rot, inter, base)
        if B == 1 or max(map(_cost, listed())) >= _cost(case):
            return case
        B = -(-B // 2)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _sizes(case):
    """Context lengths and node counts of the sequences, spread evenly over their ranges, in a fixed random order."""
    rng = np.random.RandomState(7)
    lens = np.linspace(case["lo"], case["hi"], case["B"]).round().astype(np.int64) if case["B"] > 1 else np.array([case["hi"]])
    nodes = np.linspace(case["nlo"], case["nhi"], case["B"]).round().astype(np.int64) if case["B"] > 1 else np.array([case["nhi"]])
    return rng.permutation(lens), rng.permutation(nodes)


def _tree(n, rng, max_depth=8, max_kids=4):
    """A random draft tree of n nodes: parents precede children, at most max_kids children a node."""
    parent, depth, kids = np.full(n, -1, np.int64), np.ones(n, np.int64), np.zeros(n + 1, np.int64)
    for i in range(1, n):
        ok = [j for j in range(-1, i) if kids[j] < max_kids and (j < 0 or depth[j] < max_depth)]
        j = ok[rng.randint(len(ok))] if ok else -1
        parent[i], depth[i] = j, 1 if j < 0 else depth[j] + 1
        kids[j] += 1
    return parent


def _on(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV, dtype)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _set_up(s)
    return s


def _inputs(case, seed):
    L, B, Hq, Hkv, d, page = (case[k] for k in ("L", "B", "Hq", "Hkv", "d", "page"))
    rng = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(DEV).manual_seed(seed)
    lens, nodes = _sizes(case)
    offs = np.concatenate([[0], np.cumsum(nodes)])
    T = int(offs[-1])
    tree = case["kind"] == "tree"
    parents = [_tree(int(n), rng) for n in nodes] if tree else None
    s = dict(case=case, T=T, max_nodes=int(nodes.max()), offs=_on(offs), kv_len=_on(lens),
             status=torch.zeros(1, dtype=torch.int32, device=DEV), parent=_on(np.concatenate(parents)) if tree else None)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=gen)

    if case["op"] == "norm":
        # queries and keys as the fused projection of a layer leaves them: slices of one row per token
        x = normal(L, T, (Hq + 2 * Hkv) * d, std=2.0)
        s["q"] = x[..., :Hq * d].unflatten(-1, (Hq, d))
        s["k"] = x[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d))
        s["wq"], s["wk"] = (1 + 0.2 * torch.randn(L, d, device=DEV, generator=gen) for _ in range(2))
        half = case["rot"] // 2
        s["inv_freq"] = (case["base"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        s["q_out"] = torch.empty(L, T, Hq, d, dtype=torch.bfloat16, device=DEV)
        s["k_out"] = torch.empty(L, T, Hkv, d, dtype=torch.bfloat16, device=DEV)
        s["n_pages"], s["max_pages"] = 1, 1
        return s
    # pages of the sequences, in random order over the pool; room for what a commit appends
    need = -(-(lens + (nodes if case["op"] == "commit" else 0)) // page)
    s["max_pages"] = max(1, int(need.max()))
    forks = case["nhi"] if case["op"] == "copy" else 0
    used = int(need.sum())
    s["n_pages"] = n_pages = used + 3 + forks * B
    ids = rng.permutation(n_pages)
    table = np.full((B, s["max_pages"]), -1, np.int64)
    table[np.arange(s["max_pages"])[None, :] < need[:, None]] = ids[:used]
    s["table"] = _on(table)
    s["k_cache"], s["v_cache"] = normal(L, n_pages, Hkv, page, d), normal(L, n_pages, Hkv, page, d)
    if case["op"] == "attend":
        s["q"], s["k"], s["v"] = normal(L, T, Hq, d, std=2.0), normal(L, T, Hkv, d), normal(L, T, Hkv, d)
        s["o"] = torch.empty(L, T, Hq, d, dtype=torch.bfloat16, device=DEV)
    elif case["op"] == "commit":
        s["k"], s["v"] = normal(L, T, Hkv, d), normal(L, T, Hkv, d)
        s["new_len"] = torch.empty(B, dtype=torch.int32, device=DEV)
        s["path"], s["path_len"] = None, None
        if tree:
            # root paths of random nodes, cut at random: what an acceptance leaves
            path, plen = np.full((B, 8), -1, np.int64), np.zeros(B, np.int64)
            for b, p in enumerate(parents):
                i, walk = rng.randint(len(p)), []
                while i >= 0:
                    walk.append(i)
                    i = p[i]
                plen[b] = rng.randint(len(walk) + 1)
                path[b, :plen[b]] = walk[::-1][:plen[b]]
            s["path"], s["path_len"] = _on(path), _on(plen)
    else:
        s["src"] = _on(np.repeat(table[np.arange(B), need - 1], forks))
        s["dst"] = _on(ids[used:used + forks * B])
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _where(s):
    """Sequence and local index of every packed node, and the largest node count."""
    offs = s["offs"].long()
    t = torch.arange(s["T"], device=DEV)
    seq = torch.bucketize(t, offs[1:], right=True)
    return seq, t - offs[seq], int(_sizes(s["case"])[1].max())


def _ancestors(s, seq, local, n):
    """[B, n, n]: whether node j of the sequence is node i or one of its ancestors."""
    B = s["case"]["B"]
    if s["parent"] is None:
        return torch.ones(n, n, dtype=torch.bool, device=DEV).tril().expand(B, n, n)
    up = torch.eye(n, device=DEV).repeat(B, 1, 1)
    has = s["parent"] >= 0
    up[seq[has], local[has], s["parent"][has].long()] = 1
    return torch.linalg.matrix_power(up, 16) > 0            # trees here are at most eight levels deep


def _plain_norm(s):
    c = s["case"]
    seq, local, n = _where(s)
    depth = _ancestors(s, seq, local, n).sum(-1)[seq, local] if s["parent"] is not None else local + 1
    pos = s["kv_len"].long()[seq] + depth - 1
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[None, :, None, :], angle.sin().float()[None, :, None, :]
    half, rot = c["rot"] // 2, c["rot"]

    def turn(x, w):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w[:, None, None, :]
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["inter"] else (y[..., :half], y[..., half:rot])
        p, q = a * cos - b * sin, a * sin + b * cos
        turned = torch.stack([p, q], -1).flatten(-2) if c["inter"] else torch.cat([p, q], -1)
        return torch.cat([turned, y[..., rot:]], -1).bfloat16()

    return turn(s["q"], s["wq"]), turn(s["k"], s["wk"])


def _plain_attend(s):
    c = s["case"]
    L, B, Hq, Hkv, d, page = (c[k] for k in ("L", "B", "Hq", "Hkv", "d", "page"))
    seq, local, n = _where(s)
    width = s["max_pages"] * page
    # context and draft, padded to the longest of the batch
    ids = s["table"].clamp(min=0).long()
    there = torch.arange(width, device=DEV)[None, :] < s["kv_len"][:, None]
    drafted = torch.zeros(B, n, dtype=torch.bool, device=DEV)
    drafted[seq, local] = True
    sees = torch.cat([there[:, None, :].expand(B, n, width), _ancestors(s, seq, local, n) & drafted[:, None, :]], -1)

    def gathered(cache, rec):
        x = cache[:, ids].permute(0, 1, 3, 2, 4, 5).reshape(L, B, Hkv, width, d).float()
        y = torch.zeros(L, B, n, Hkv, d, device=DEV)
        y[:, seq, local] = rec.float()
        return torch.cat([x, y.transpose(2, 3)], 3)

    q = torch.zeros(L, B, n, Hq, d, device=DEV)
    q[:, seq, local] = s["q"].float()
    q = q.reshape(L, B, n, Hkv, Hq // Hkv, d).permute(0, 1, 3, 2, 4, 5).reshape(L, B, Hkv, n * (Hq // Hkv), d)
    scores = q @ gathered(s["k_cache"], s["k"]).transpose(-1, -2) * d ** -0.5
    sees = sees[None, :, None].repeat_interleave(Hq // Hkv, 3)
    scores = torch.where(sees, scores, -math.inf)
    # a padded row of the batch may see nothing: it is not returned, and must not spread NaN either
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    o = (p @ gathered(s["v_cache"], s["v"])) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.reshape(L, B, Hkv, n, Hq // Hkv, d).permute(0, 1, 3, 2, 4, 5).reshape(L, B, n, Hq, d)
    return o[:, seq, local].bfloat16()


def _plain_commit(s):
    c = s["case"]
    if s["path"] is None:
        seq, local, _ = _where(s)
        rank, node, count = local, torch.arange(s["T"], device=DEV), s["offs"].diff()
    else:
        count = s["path_len"]
        seq, rank = (torch.arange(s["path"].shape[1], device=DEV)[None, :] < count[:, None]).nonzero(as_tuple=True)
        node = s["offs"].long()[seq] + s["path"].long()[seq, rank]
    at = s["kv_len"].long()[seq] + rank
    page, row = s["table"].long()[seq, at // c["page"]], at % c["page"]
    s["k_cache"][:, page, :, row] = s["k"][:, node].transpose(0, 1)
    s["v_cache"][:, page, :, row] = s["v"][:, node].transpose(0, 1)
    return s["k_cache"], s["v_cache"], s["kv_len"] + count


def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    s["k_cache"][:, dst] = s["k_cache"][:, src]
    s["v_cache"][:, dst] = s["v_cache"][:, src]
    return s["k_cache"], s["v_cache"]


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _set_up(s):
    # shapes and workspace, which a program makes once and keeps from call to call
    from paper_2607_16673_b200 import binding as speca
    c = s["case"]
    s["dims"] = speca.AttnDims(c["L"], c["B"], c["Hq"], c["Hkv"], c["d"], scale=c["d"] ** -0.5,
                               max_nodes=s["max_nodes"], page_size=c["page"], n_pages=s["n_pages"],
                               max_pages=s["max_pages"])
    s["ws"] = speca.alloc_attn_workspace(s["dims"]) if c["op"] == "attend" else None


def _own(s):
    from paper_2607_16673_b200 import binding as speca
    if "dims" not in s:                     # inputs that were made for the plain forms
        _set_up(s)
    c, D = s["case"], s["dims"]
    if c["op"] == "attend":
        speca.attend_tree(D, s["q"], s["k"], s["v"], s["offs"], s["T"], s["parent"], s["k_cache"], s["v_cache"],
                          s["table"], s["kv_len"], s["o"], s["ws"], s["status"])
        return s["o"]
    if c["op"] == "norm":
        speca.norm_rope(D, s["q"], s["k"], s["wq"], s["wk"], EPS, s["inv_freq"], c["rot"], c["inter"], 1.0, s["offs"],
                        s["T"], s["parent"], s["kv_len"], s["q_out"], s["k_out"], s["status"])
        return s["q_out"], s["k_out"]
    if c["op"] == "commit":
        speca.commit_kv(D, s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["k"], s["v"], s["offs"], s["T"],
                        s["parent"], s["path"], s["path_len"], s["new_len"], s["status"])
        return s["k_cache"], s["v_cache"], s["new_len"]
    speca.copy_pages(D, s["k_cache"], s["v_cache"], s["src"], s["dst"], s["status"])
    return s["k_cache"], s["v_cache"]


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return (_plain_attend if op == "attend" else _plain_norm if op == "norm" else
            _plain_commit if op == "commit" else _plain_copy)(state)


def work(case):
    L, B, Hq, Hkv, d, page = (case[k] for k in ("L", "B", "Hq", "Hkv", "d", "page"))
    lens, nodes = _sizes(case)
    T = int(nodes.sum())
    if case["op"] == "norm":
        return {"bytes": 4 * L * T * (Hq + Hkv) * d, "flops": 10 * L * T * (Hq + Hkv) * d}
    if case["op"] == "commit":
        # a path is as long as half a random node's depth on average: about two rows of a tree's
        rows = T if case["kind"] != "tree" else 2 * B
        return {"bytes": 8 * L * rows * Hkv * d, "flops": 0}
    if case["op"] == "copy":
        return {"bytes": 8 * L * B * case["nhi"] * Hkv * page * d, "flops": 0}
    if case["kind"] == "tree":
        pairs = float(((lens + 4) * nodes).sum())               # about four ancestors a node
    else:
        pairs = float((lens * nodes + nodes * (nodes + 1) / 2).sum())
    return {"bytes": 4 * L * (int(lens.sum()) * Hkv * d + T * (Hq + Hkv) * d), "flops": 4 * L * d * Hq * pairs}


# ---------------------------------------------------------------------------------------------------------------
# the definition, in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    L, B, Hq, Hkv, d, page = (case[k] for k in ("L", "B", "Hq", "Hkv", "d", "page"))
    offs, lens = s["offs"].tolist(), s["kv_len"].tolist()
    par = s["parent"].tolist() if s["parent"] is not None else None
    if case["op"] == "copy":
        for j, (a, b) in enumerate(zip(s["src"].tolist(), s["dst"].tolist())):
            for cache in (s["k_cache"], s["v_cache"]):
                cache[:, b].copy_(cache[:, a])
        return s["k_cache"], s["v_cache"]
    if case["op"] == "commit":
        table = s["table"].tolist()
        new = []
        for b in range(B):
            n = offs[b + 1] - offs[b]
            if s["path"] is None:
                order = list(range(n))
            else:
                order = s["path"][b, :int(s["path_len"][b])].tolist()
            new.append(lens[b] + len(order))
            first = 0
            while first < len(order):                          # the rows that fall into one page
                at = lens[b] + first
                take = min(page - at % page, len(order) - first)
                rows = torch.tensor([offs[b] + i for i in order[first:first + take]], device=DEV)
                for cache, rec in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
                    cache[:, table[b][at // page], :, at % page:at % page + take] = rec[:, rows].transpose(1, 2)
                first += take
        return s["k_cache"], s["v_cache"], torch.tensor(new, dtype=torch.int32, device=DEV)
    if case["op"] == "norm":
        pos = []
        for b in range(B):
            depth = []
            for i in range(offs[b + 1] - offs[b]):
                up = i - 1 if par is None else par[offs[b] + i]
                depth.append(1 if up < 0 else depth[up] + 1)
            pos += [lens[b] + x - 1 for x in depth]
        pos = torch.tensor(pos, dtype=torch.float64, device=DEV)
        outs = []
        for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
            out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
            for l in range(L):
                y = x[l].double()
                y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w[l].double()
                pairs = case["rot"] // 2
                first = torch.arange(pairs, device=DEV) * (2 if case["inter"] else 1)
                second = first + (1 if case["inter"] else pairs)
                turned = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(len(pos), pairs),
                                     torch.outer(pos, s["inv_freq"].double()))[:, None, :]
                z = torch.complex(y[..., first], y[..., second]) * turned
                y[..., first], y[..., second] = z.real, z.imag
                out[l] = y
            outs.append(out)
        return tuple(outs)
    out = torch.empty(L, s["T"], Hq, d, dtype=torch.float64, device=DEV)
    for b in range(B):
        n = offs[b + 1] - offs[b]
        seen = torch.zeros(n, n, dtype=torch.bool)
        if par is None:
            seen = torch.arange(n)[None, :] <= torch.arange(n)[:, None]
        else:
            for i in range(n):
                up = par[offs[b] + i]
                if up >= 0:
                    seen[i] = seen[up]
                seen[i, i] = True
        blocked = torch.cat([torch.zeros(n, lens[b], dtype=torch.bool), ~seen], 1).to(DEV)
        pages = s["table"][b, :-(-lens[b] // page)].long()
        for l in range(L):
            for h in range(Hkv):
                k, v = (torch.cat([cache[l, pages, h].reshape(-1, d)[:lens[b]], rec[l, offs[b]:offs[b + 1], h]]).double()
                        for cache, rec in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])))
                for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    x = (s["q"][l, offs[b]:offs[b + 1], g].double() @ k.T / math.sqrt(d)).masked_fill(blocked, -math.inf)
                    out[l, offs[b]:offs[b + 1], g] = torch.softmax(x, -1) @ v
    return out
