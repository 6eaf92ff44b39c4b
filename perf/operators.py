"""Performance cases of the operators that a long, bounded KV cache needs beside the verification step.

`listed()` names them, `draw(rng)` gives another of the same ranges, `prepare(case, seed)` makes what a serving loop holds
on the GPU before the call, `run(state)` is one pass, `work(case)` the bytes and operations a pass cannot do without,
`exact(case, seed)` the outputs from the definitions in 64 bits.

Three kinds of case:
  attend   tree attention of one layer whose scores are capped by a tanh and biased by slopes over the keys' positions,
           with the log-sum-exp of every row
  weigh    the attention weight that the accepted path's rows gave to every cache row, added to the rows' totals
  evict    the cache cut down to a budget: the most recent rows and those of the largest totals stay; rows that stay but
           lie behind the budget move into the places of evicted ones

`own` chooses the library's calls; otherwise everything is computed by elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ES = {"f32": 4, "bf16": 2, "f16": 2}


def _attend(name, B, Hq, Hkv, D, dtype, P, N, levels, cap, bias, page=0, ragged=False):
    """bias: "none", "rows" (positions are row numbers) or "kept" (positions of a cache that rows were evicted from)"""
    case = {"kind": "attend", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "P": P, "N": N, "levels": levels, "cap": cap,
            "bias": bias, "page": page, "ragged": ragged}
    return dict(case, name=name) if name else case


def _weigh(name, B, Hq, Hkv, D, dtype, P, N, accepted, cap, bias, page=0, ragged=False):
    """accepted: drafted tokens on the path; the path's accepted + 1 rows are the last ones of the P in the cache"""
    case = {"kind": "weigh", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "P": P, "N": N, "accepted": accepted, "cap": cap,
            "bias": bias, "page": page, "ragged": ragged}
    return dict(case, name=name) if name else case


def _evict(name, layers, B, Hkv, D, dtype, P, budget, recent, page=0, ragged=False):
    case = {"kind": "evict", "layers": layers, "B": B, "Hkv": Hkv, "D": D, "dtype": dtype, "P": P, "budget": budget, "recent": recent,
            "page": page, "ragged": ragged}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: a toy model in fp32 with both score changes, nothing but latency
        _attend("attend tiny f32", 1, 4, 4, 64, "f32", 128, 15, 4, 20.0, "rows"),
        # one user of a 7B model whose scores are capped: the paper's operating point (batch 1)
        _attend("attend 7b b1 capped", 1, 32, 32, 128, "bf16", 1024, 60, 6, 50.0, "none"),
        # a serving batch of grouped queries over a cache that rows were evicted from: positions are looked up
        _attend("attend gqa8b b8 kept", 8, 32, 8, 128, "bf16", 8192, 64, 8, 0.0, "kept"),
        # the largest: long contexts, full trees, capped scores
        _attend("attend 70b-long b16 capped", 16, 64, 8, 128, "bf16", 32768, 128, 10, 30.0, "none"),
        # single tokens (no draft) of a ragged batch over a paged cache, head size 64, biased by distance
        _attend("attend one token d64 paged", 13, 32, 8, 64, "f16", 5003, 1, 1, 0.0, "rows", 64, True),
        # the step after the 7B model's verification: five rows were appended
        _weigh("weigh 7b b1", 1, 32, 32, 128, "bf16", 1029, 60, 4, 50.0, "none"),
        # the serving batch, positions looked up, paged and ragged
        _weigh("weigh gqa8b b8 kept paged", 8, 32, 8, 128, "f16", 8197, 64, 4, 0.0, "kept", 128, True),
        # long contexts: one pass over a gigabyte of keys
        _weigh("weigh 70b-long b16", 16, 64, 8, 128, "bf16", 32768, 128, 6, 30.0, "none"),
        # a prompt that is taken in by pieces of 128 tokens (a chain of nodes, all of them accepted)
        _weigh("weigh prompt piece", 2, 32, 8, 128, "bf16", 4096, 128, 127, 0.0, "none"),
        # a toy cache in fp32: latency
        _evict("evict tiny f32", 1, 1, 4, 64, "f32", 160, 128, 32),
        # every layer of a 7B model, one user: a quarter of the rows go
        _evict("evict 7b 32 layers f16", 32, 1, 32, 128, "f16", 1367, 1024, 256),
        # a layer of a large batch, paged and ragged: half of the rows go
        _evict("evict 70b-long b16 paged", 1, 16, 8, 128, "bf16", 32768, 16384, 4096, 256, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "weigh", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    D = rng.choice([64, 128, 128])
    B = _log(rng, 1, 16)
    G = rng.choice([1, 2, 4, 4, 8])
    Hkv = rng.choice([2, 4, 8, 8, 16]) if G > 1 else rng.choice([4, 8, 16, 32, 40])
    page = rng.choice([0, 0, 64, 128, 256])
    ragged = rng.random() < 0.5
    P = _log(rng, 64, 32768)
    while P > 64 and B * Hkv * P * D * ES[dtype] > 1.0e9:
        P = P * 2 // 3
    if kind == "evict":
        layers = rng.choice([1, 1, _log(rng, 2, 32)])
        while layers > 1 and layers * B * Hkv * P * D * ES[dtype] > 6.0e8:
            layers //= 2
        budget = max(1, int(P * rng.uniform(0.3, 1.0)))
        return _evict(None, layers, B, Hkv, D, dtype, P, budget, int(budget * rng.choice([0.0, 0.1, 0.25, 0.5])), page, ragged)
    cap = rng.choice([0.0, 20.0, 30.0, 50.0])
    bias = rng.choice(["none", "rows", "kept"])
    N = rng.choice([1, rng.randint(2, 128), rng.randint(2, 128)])
    if kind == "weigh":
        accepted = rng.choice([0, min(N - 1, rng.randint(0, 8)), min(N - 1, rng.randint(0, 8)), N - 1])
        while P > 256 and 2.0 * B * Hkv * G * (accepted + 1) * P * D > (4e9 if dtype == "f32" else 1e11):
            P = P * 2 // 3
        return _weigh(None, B, Hkv * G, Hkv, D, dtype, max(P, accepted + 1), N, accepted, cap, bias, page, ragged)
    most = 2.0e12 if dtype != "f32" and D == 128 else 2e10 if dtype != "f32" else 8e9
    while P > 64 and 4.0 * B * Hkv * max(G * N, 32) * P * D > most:
        P = P * 2 // 3
    return _attend(None, B, Hkv * G, Hkv, D, dtype, P, N, 1 if N == 1 else rng.randint(2, min(N, 10)), cap, bias, page, ragged)


# ---------------------------------------------------------------------------------------------- inputs
def _randn(g, shape, dtype, std=1.0):
    """N(0, std) in `dtype`, drawn in slices so that the fp32 draw of a large cache stays small."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat, step = out.view(-1), 1 << 27
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.numel(), device="cuda", generator=g).mul_(std))
    return out


def _parents(B, N, levels, seed):
    """Random trees: every level has a node at least, nodes are numbered level by level."""
    out = np.full((B, N), -1, dtype=np.int32)
    for b in range(B):
        r = np.random.default_rng([seed, b])
        depth = np.sort(np.concatenate([np.arange(1, levels), r.integers(1, max(levels, 2), max(0, N - levels))]))[:N - 1] if N > 1 else []
        depth = np.concatenate([[0], depth]).astype(int)
        for i in range(1, N):
            above = np.nonzero(depth[:i] == depth[i] - 1)[0]
            out[b, i] = r.choice(above)
    return out


def _ancestors(parent):
    """[B][N][N] truth values: column j is row i's node itself or one of its ancestors"""
    B, N = parent.shape
    m = np.zeros((B, N, N), dtype=bool)
    for i in range(N):
        m[:, i, i] = True
        if i:
            b = np.arange(B)
            m[b, i] |= m[b, parent[:, i]]
    return m


class _State:
    pass


def _slopes(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device="cuda")


def _cache(s, case, g, lead, rows, dt):
    """K and V caches, contiguous [lead][B][Hkv][rows][D] or pools [lead][pages][Hkv][page][D] behind a shuffled block table;
    returns the row capacity"""
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    s.block_table = None
    if page:
        blocks = -(-rows // page)
        rows, pages = blocks * page, B * blocks
        s.block_table = torch.randperm(pages, device="cuda", generator=g).view(B, blocks).to(torch.int32).contiguous()
        shape = lead + (pages, Hkv, page, D)
    else:
        shape = lead + (B, Hkv, rows, D)
    s.k_cache = _randn(g, shape, dt)
    if case["kind"] != "weigh":
        s.v_cache = _randn(g, shape, dt)
    return rows


def _positions(g, lead, S, lengths, end):
    """Positions [lead][S] of rows of a cache that rows were evicted from: the last quarter in order up to `end` - 1, the others
    distinct ones from before, in any order."""
    out = torch.zeros(lead + (S,), dtype=torch.int32, device="cuda")
    for b in range(lead[-2]):
        n = int(lengths[b])
        tail = n // 4
        first = int(end[b]) - tail
        pick = torch.rand(lead[:-2] + (lead[-1], first), device="cuda", generator=g).argsort(-1)[..., :n - tail]
        out[..., b, :, :n - tail] = pick.to(torch.int32)
        out[..., b, :, n - tail:n] = torch.arange(first, int(end[b]), device="cuda", dtype=torch.int32)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case, s.kind = case, case["kind"]
    dt = DTYPES[case["dtype"]]
    B, Hkv, D, P = case["B"], case["Hkv"], case["D"], case["P"]
    i32 = dict(dtype=torch.int32, device="cuda")
    host = np.full(B, P)
    if case["ragged"]:
        least = max(1, case.get("accepted", 0) + 1)
        host = np.random.default_rng([seed, 77]).integers(max(P // 2, least), P + 1, B)
    s.host_len = host
    s.cache_len = torch.from_numpy(host.astype(np.int32)).cuda()
    s.status = torch.empty(B, **i32)

    if s.kind == "evict":
        Ly, budget = case["layers"], case["budget"]
        S = s.S = _cache(s, case, g, (Ly,), P, dt)
        # totals of attention weights: a few rows have most of it
        s.weight = torch.randn(Ly, B, Hkv, S, device="cuda", generator=g).mul_(2.0).exp_()
        s.next_pos = s.cache_len + (s.cache_len // 2)
        s.key_pos = _positions(g, (Ly, B, Hkv), S, host, host + host // 2)
        s.weight_out, s.key_pos_out = torch.zeros_like(s.weight), torch.zeros_like(s.key_pos)
        s.new_len = torch.empty(B, **i32)
        s.kept = torch.empty(Ly, B, Hkv, budget, **i32)
        if own:
            from paper_2506_14158_amd import binding
            s.ws = binding.alloc_workspace(binding.s4c_kv_evict_workspace_size(Ly, B, Hkv, budget, S))
        return s

    Hq, N = case["Hq"], case["N"]
    s.slopes = _slopes(Hq) if case["bias"] != "none" else None
    s.key_pos = s.root_pos = None
    s.q = _randn(g, (B, N, Hq, D), dt, 2.0)
    if s.kind == "attend":
        S = s.S = _cache(s, case, g, (), P, dt)
        parent = _parents(B, N, case["levels"], seed)
        s.parent = torch.from_numpy(parent).cuda()
        s.k_tree, s.v_tree = _randn(g, (B, N, Hkv, D), dt), _randn(g, (B, N, Hkv, D), dt)
        if case["bias"] == "kept":
            s.root_pos = s.cache_len + (s.cache_len // 2)
            s.key_pos = _positions(g, (B, Hkv), S, host, host + host // 2)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(B, N, Hq, device="cuda")
        if own:
            from paper_2506_14158_amd import binding
            code = {"f32": binding.S4C_F32, "bf16": binding.S4C_BF16, "f16": binding.S4C_F16}[case["dtype"]]
            shape = binding.AttnShape(B, Hq, Hkv, D, N, S, code)
            s.ws = binding.alloc_workspace(binding.s4c_tree_attn_workspace_size(shape, P))
            s.score = binding.Score(case["cap"], s.slopes, s.key_pos, s.root_pos)
        return s

    # weigh: what the attention before it and the appended path left
    L = case["accepted"]
    S = s.S = _cache(s, case, g, (), P, dt)
    r = np.random.default_rng([seed, 78])
    path = np.stack([np.concatenate([[0], 1 + np.sort(r.permutation(N - 1)[:L])]) for _ in range(B)]).astype(np.int32)
    s.path = torch.from_numpy(path).cuda()
    s.accept_len = torch.full((B,), L, **i32)
    first = s.cache_len - (L + 1)
    if case["bias"] == "kept":
        s.root_pos = first + (first // 2)
        h0 = host - (L + 1)
        s.key_pos = _positions(g, (B, Hkv), S, h0, h0 + h0 // 2)
    s.weight = torch.randn(B, Hkv, S, device="cuda", generator=g).mul_(2.0).exp_()
    s.weight_out = torch.zeros_like(s.weight)
    s.lse = torch.zeros(B, N, Hq, device="cuda")
    for b in range(B):
        x = _path_scores(s, b, torch.float32)
        s.lse[b, s.path[b].long()] = torch.logsumexp(x, -1).permute(2, 0, 1).reshape(L + 1, Hq)
    if own:
        from paper_2506_14158_amd import binding
        s.score = binding.Score(case["cap"], s.slopes, s.key_pos, s.root_pos)
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _rows(s, cache, b, n):
    """the first n cache rows of sequence b: [Hkv][n][D]"""
    page = s.case["page"]
    if not page:
        return cache[b, :, :n]
    t = s.block_table[b, :-(-n // page)].long()
    return cache[t].transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def _changed(s, x, rel):
    """scores x [Hkv][G][R][n] of the type of the arithmetic, capped and biased; rel [Hkv][n]: the keys' positions from the root's"""
    if s.case["cap"] > 0:
        x = s.case["cap"] * torch.tanh(x / s.case["cap"])
    if s.slopes is not None:
        Hkv, G = x.shape[:2]
        x = x + s.slopes.to(x.dtype).view(Hkv, G, 1, 1) * rel.to(x.dtype).view(rel.shape[0], 1, 1, rel.shape[1])
    return x


def _relative(s, b, n):
    """positions of the n cached rows of sequence b before its drafted ones, from the root's: [Hkv or 1][n]"""
    if s.key_pos is not None:
        return s.key_pos[b, :, :n] - s.root_pos[b]
    return torch.arange(-n, 0, device="cuda").view(1, n)


def _path_scores(s, b, dt):
    """scores of the path's rows of sequence b: [Hkv][G][L+1][n], -inf behind the query's own key"""
    Hkv, D, L, n = s.case["Hkv"], s.case["D"], s.case["accepted"], int(s.host_len[b])
    q = s.q[b, s.path[b].long()].to(dt)                                   # [L+1][Hq][D]
    q = q.view(L + 1, Hkv, -1, D).permute(1, 2, 0, 3)                     # [Hkv][G][L+1][D]
    k = _rows(s, s.k_cache, b, n).to(dt)
    x = torch.matmul(q.reshape(Hkv, -1, D), k.transpose(1, 2).contiguous()).view(Hkv, -1, L + 1, n) / math.sqrt(D)
    rel = _relative(s, b, n - L - 1)
    rel = torch.cat([rel, torch.arange(L + 1, device="cuda").expand(rel.shape[0], L + 1)], 1)
    x = _changed(s, x, rel)
    seen = torch.arange(n, device="cuda") < (torch.arange(L + 1, device="cuda") + (n - L)).view(-1, 1)
    return x.masked_fill(~seen, -math.inf)


def _plain_attend(s):
    c = s.case
    Hkv, D, N = c["Hkv"], c["D"], c["N"]
    parent = s.parent.long()
    seen = torch.eye(N, dtype=torch.bool, device="cuda").repeat(c["B"], 1, 1)
    depth = torch.zeros_like(parent)
    for i in range(1, N):
        up = parent[:, i]
        seen[:, i] |= seen.gather(1, up.view(-1, 1, 1).expand(-1, 1, N))[:, 0]
        depth[:, i] = depth.gather(1, up.view(-1, 1))[:, 0] + 1
    for b in range(c["B"]):
        n = int(s.host_len[b])
        q = s.q[b].float().view(N, Hkv, -1, D).permute(1, 2, 0, 3)                     # [Hkv][G][N][D]
        G = q.shape[1]
        k = torch.cat([_rows(s, s.k_cache, b, n), s.k_tree[b].transpose(0, 1)], 1).float()
        x = torch.matmul(q.reshape(Hkv, G * N, D), k.transpose(1, 2).contiguous()).view(Hkv, G, N, n + N) / math.sqrt(D)
        del k
        rel = _relative(s, b, n)
        rel = torch.cat([rel, depth[b].expand(rel.shape[0], N).to(rel.dtype)], 1)
        x = _changed(s, x, rel)
        x[..., n:].masked_fill_(~seen[b], -math.inf)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - m)
        del x
        l = p.sum(-1, keepdim=True)
        v = torch.cat([_rows(s, s.v_cache, b, n), s.v_tree[b].transpose(0, 1)], 1).float()
        o = torch.matmul(p.view(Hkv, G * N, n + N), v).view(Hkv, G, N, D) / l
        s.out[b] = o.permute(2, 0, 1, 3).reshape(N, -1, D).to(s.out.dtype)
        s.lse[b] = (m + torch.log(l)).squeeze(-1).permute(2, 0, 1).reshape(N, -1)
    return {"out": s.out, "lse": s.lse}


def _plain_weigh(s):
    Hkv, L = s.case["Hkv"], s.case["accepted"]
    for b in range(s.case["B"]):
        n = int(s.host_len[b])
        x = _path_scores(s, b, torch.float32)                                          # [Hkv][G][L+1][n]
        lse = s.lse[b, s.path[b].long()].view(L + 1, Hkv, -1).permute(1, 2, 0).unsqueeze(-1)
        got = torch.exp(x - lse).sum((1, 2))
        got[:, :n - L - 1] += s.weight[b, :, :n - L - 1]
        s.weight_out[b, :, :n] = got
        if s.key_pos is not None:
            s.key_pos[b, :, n - L - 1:n] = s.root_pos[b] + torch.arange(L + 1, device="cuda", dtype=torch.int32)
    return _weigh_outputs(s)


def _weigh_outputs(s):
    return {"weight": s.weight_out} if s.key_pos is None else {"weight": s.weight_out, "key_pos": s.key_pos}


def _at(s, ly, b, h, j):
    """indices into a cache [..][D] viewed as rows of it, of row j of (layer, sequence, KV head)"""
    c, page = s.case, s.case["page"]
    if not page:
        return ((ly * c["B"] + b) * c["Hkv"] + h) * s.S + j
    t = s.block_table[b, j // page].long()
    return ((ly * s.block_table.numel() + t) * c["Hkv"] + h) * page + j % page


def _plain_evict(s):
    c = s.case
    n = s.cache_len.long().view(1, -1, 1, 1)
    m = n.clamp(max=c["budget"])
    S = s.S
    j = torch.arange(S, device="cuda").view(1, 1, 1, S)
    worth = torch.where(s.key_pos >= (s.next_pos - c["recent"]).view(1, -1, 1, 1), math.inf, s.weight)
    worth = torch.where(j < n, worth, -math.inf)
    order = torch.sort(worth, dim=-1, descending=True, stable=True).indices
    stays = torch.zeros_like(worth, dtype=torch.bool).scatter_(-1, order, (j < m).expand_as(order))
    hole, mover = ((j < m) & ~stays).nonzero(as_tuple=True), ((j >= m) & stays).nonzero(as_tuple=True)
    D = c["D"]
    for cache in (s.k_cache, s.v_cache):
        rows = cache.view(-1, D)
        rows[_at(s, *hole)] = rows[_at(s, *mover)]
    front = torch.arange(c["budget"], device="cuda", dtype=torch.int32).view(1, 1, 1, -1)
    s.kept.copy_(torch.where(front < m, front, -1))
    s.kept[hole] = mover[3].to(torch.int32)
    take = s.kept.clamp(min=0).long()
    live = s.kept >= 0
    s.weight_out[..., :c["budget"]] = torch.where(live, s.weight.gather(-1, take), s.weight_out[..., :c["budget"]])
    s.key_pos_out[..., :c["budget"]] = torch.where(live, s.key_pos.gather(-1, take), s.key_pos_out[..., :c["budget"]])
    s.new_len.copy_(m.view(-1))
    return _evict_outputs(s)


def _evict_outputs(s):
    return {"k_cache": s.k_cache, "v_cache": s.v_cache, "weight": s.weight_out, "key_pos": s.key_pos_out, "kept": s.kept,
            "cache_len": s.new_len}


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return {"attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[s.kind](s)
    from paper_2506_14158_amd import binding
    c = s.case
    if s.kind == "attend":
        if c["page"]:
            binding.s4c_tree_attn_scored_paged(s.q, s.k_tree, s.v_tree, s.k_cache, s.v_cache, s.block_table, s.cache_len, s.parent, c["P"],
                                               s.score, s.out, s.lse, 0.0, s.status, s.ws)
        else:
            binding.s4c_tree_attn_scored(s.q, s.k_tree, s.v_tree, s.k_cache, s.v_cache, s.cache_len, s.parent, c["P"], s.score, s.out,
                                         s.lse, 0.0, s.status, s.ws)
        return {"out": s.out, "lse": s.lse}
    if s.kind == "weigh":
        if c["page"]:
            binding.s4c_kv_weigh_paged(s.q, s.k_cache, s.block_table, s.lse, s.cache_len, s.path, s.accept_len, c["P"], s.score, s.weight,
                                       s.weight_out, 0.0, s.status)
        else:
            binding.s4c_kv_weigh(s.q, s.k_cache, s.lse, s.cache_len, s.path, s.accept_len, c["P"], s.score, s.weight, s.weight_out, 0.0,
                                 s.status)
        return _weigh_outputs(s)
    if c["page"]:
        binding.s4c_kv_evict_paged(s.k_cache, s.v_cache, s.block_table, s.weight, s.key_pos, s.cache_len, s.next_pos, c["budget"],
                                   c["recent"], s.weight_out, s.key_pos_out, s.new_len, s.ws, s.kept, s.status)
    else:
        binding.s4c_kv_evict(s.k_cache, s.v_cache, s.weight, s.key_pos, s.cache_len, s.next_pos, c["budget"], c["recent"], s.weight_out,
                             s.key_pos_out, s.new_len, s.ws, s.kept, s.status)
    return _evict_outputs(s)


# ---------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    es = ES[case["dtype"]]
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    n = case["P"] * (0.75 if case["ragged"] else 1.0)
    if case["kind"] == "evict":
        units = case["layers"] * B * Hkv
        m = min(n, case["budget"])
        recent, gone = min(case["recent"], m), n - m
        # the most recent rows lie at the end; of the others any is as likely to stay
        moved = min(recent, gone) + max(0.0, gone - recent) * ((m - recent) / max(1.0, n - recent)) if gone > 0 else 0.0
        return {"bytes": units * (8.0 * n + 12.0 * m + 4.0 * moved * D * es), "flops": 2.0 * units * n}
    Hq, N = case["Hq"], case["N"]
    looked_up = 4.0 * B * Hkv * n if case["bias"] == "kept" else 0.0
    if case["kind"] == "weigh":
        R = case["accepted"] + 1
        return {"bytes": B * Hkv * n * (D * es + 8.0) + looked_up + B * R * Hq * (D * es + 4.0), "flops": 2.0 * B * R * Hq * n * D}
    return {"bytes": 2.0 * B * Hkv * (n + N) * D * es + looked_up + B * N * Hq * (2.0 * D * es + 4.0),
            "flops": 4.0 * B * Hq * N * (n + case["levels"] / 2.0) * D}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_score(case, h, q, k, pos):
    """scores [R][n] of query head h in 64 bits; pos [n]: the keys' positions from the root's"""
    x = q.double() @ k.double().t().contiguous() * (1.0 / math.sqrt(case["D"]))
    if case["cap"] > 0:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    if case["bias"] != "none":
        x += 2.0 ** (-8.0 * (h + 1) / case["Hq"]) * pos.double()
    return x


def _exact_rows(case, s, cache, b, kvh, n):
    if not case["page"]:
        return cache[b, kvh, :n]
    j = torch.arange(n, device="cuda")
    return cache[s.block_table[b].long()[j // case["page"]], kvh, j % case["page"]]


def exact(case, seed):
    s = prepare(case, seed)
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["kind"] == "evict":
        return _exact_evict(case, s)
    Hq, N = case["Hq"], case["N"]
    G = Hq // Hkv
    if case["kind"] == "weigh":
        R = case["accepted"] + 1
        total = s.weight_out.double()
        pos = None if s.key_pos is None else s.key_pos.clone()
        for b in range(B):
            n = int(s.host_len[b])
            for kvh in range(Hkv):
                k = _exact_rows(case, s, s.k_cache, b, kvh, n)
                rel = torch.arange(n, device="cuda") - (n - R)
                if pos is not None:
                    pos[b, kvh, n - R:n] = s.root_pos[b] + torch.arange(R, device="cuda", dtype=torch.int32)
                    rel = pos[b, kvh, :n].long() - s.root_pos[b].long()
                got = torch.zeros(n, dtype=torch.float64, device="cuda")
                got[:n - R] = s.weight[b, kvh, :n - R].double()
                for h in range(kvh * G, (kvh + 1) * G):
                    x = _exact_score(case, h, s.q[b, s.path[b].long(), h], k, rel)
                    p = torch.exp(x - s.lse[b, s.path[b].long(), h].double().view(-1, 1))
                    got += torch.tril(p, n - R).sum(0)
                total[b, kvh, :n] = got
        return {"weight": total} if pos is None else {"weight": total, "key_pos": pos}
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, N, Hq, dtype=torch.float64, device="cuda")
    tree = _ancestors(_parents(B, N, case["levels"], seed))
    for b in range(B):
        n = int(s.host_len[b])
        deep = torch.from_numpy(tree[b].sum(1) - 1).cuda()
        for kvh in range(Hkv):
            k = torch.cat([_exact_rows(case, s, s.k_cache, b, kvh, n), s.k_tree[b, :, kvh]])
            v = torch.cat([_exact_rows(case, s, s.v_cache, b, kvh, n), s.v_tree[b, :, kvh]]).double()
            rel = torch.arange(-n, 0, device="cuda") if s.key_pos is None else s.key_pos[b, kvh, :n].long() - s.root_pos[b].long()
            rel = torch.cat([rel, deep])
            for h in range(kvh * G, (kvh + 1) * G):
                x = _exact_score(case, h, s.q[b, :, h], k, rel)
                x[:, n:][torch.from_numpy(~tree[b]).cuda()] = -math.inf
                lse[b, :, h] = torch.logsumexp(x, 1)
                out[b, :, h] = torch.exp(x - lse[b, :, h].view(-1, 1)) @ v
    return {"out": out, "lse": lse}


def _exact_evict(case, s):
    kept = np.full(tuple(s.kept.shape), -1, dtype=np.int32)
    w, pos, nxt = s.weight.cpu().numpy(), s.key_pos.cpu().numpy(), s.next_pos.cpu().numpy()
    for ly in range(case["layers"]):
        for b in range(case["B"]):
            n = int(s.host_len[b])
            m = min(n, case["budget"])
            for h in range(case["Hkv"]):
                new = pos[ly, b, h, :n] >= nxt[b] - case["recent"]
                best = np.lexsort((np.arange(n), -w[ly, b, h, :n].astype(np.float64), ~new))[:m]
                src = np.arange(m)
                src[np.setdiff1d(src, best)] = np.sort(best[best >= m])
                kept[ly, b, h, :m] = src
    weight, key_pos = s.weight_out.clone(), s.key_pos_out.clone()
    k, v = s.k_cache.clone(), s.v_cache.clone()
    for ly in range(case["layers"]):
        for b in range(case["B"]):
            m = min(int(s.host_len[b]), case["budget"])
            to = torch.arange(m, device="cuda")
            for h in range(case["Hkv"]):
                src = torch.from_numpy(kept[ly, b, h, :m]).long().cuda()
                weight[ly, b, h, :m] = s.weight[ly, b, h, src]
                key_pos[ly, b, h, :m] = s.key_pos[ly, b, h, src]
                for new, old in ((k, s.k_cache), (v, s.v_cache)):
                    if case["page"]:
                        t = s.block_table[b].long()
                        new[ly, t[to // case["page"]], h, to % case["page"]] = old[ly, t[src // case["page"]], h, src % case["page"]]
                    else:
                        new[ly, b, h, :m] = old[ly, b, h, src]
    return {"k_cache": k, "v_cache": v, "weight": weight, "key_pos": key_pos, "kept": torch.from_numpy(kept).cuda(),
            "cache_len": s.cache_len.clamp(max=case["budget"])}
