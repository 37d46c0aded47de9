"""The operators of speculative decoding over a paged private KV store, as measured cases.

A request's drafted tokens are a tree: its nodes are consecutive rows, a parent before its children, and `parents` holds
each node's parent within the request (-1: none; node 0 is the token sampled last).  Three operators that follow one
another in a step: attention of the nodes over the cache whose last tokens they are ("tree"), verification of the
drafted tokens against the target's probabilities from given random numbers ("verify"), and keeping the rows of the
accepted path in the cache ("commit").  Pages are bf16 [n_pages][page_size][Hkv][D], or 4-bit: E2M1 codes with one f16
scale per (token, KV head, 32 dimensions), 16 tokens of a head to a block of bytes.

`run` computes the plain form with elementary torch operations, or, with `own` set, makes the calls
of the package.  `exact` gives the same results in 64 bits, written apart from both.
"""
import math

import numpy as np
import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_SCALE = 10912.0  # largest f16 whose sixfold is still finite in f16


# ---- cases ---------------------------------------------------------------------------------------
def _tree(name, fmt, R, Hq, Hkv, D, nodes_min, nodes, len_min, len_max, page):
    """R requests with trees of nodes_min..nodes nodes that end contexts of len_min..len_max tokens."""
    return {"name": name, "kind": "tree", "fmt": fmt, "R": R, "Hq": Hq, "Hkv": Hkv, "D": D, "nodes_min": nodes_min,
            "nodes": nodes, "len_min": len_min, "len_max": len_max, "page": page}


def _verify(name, R, nodes_min, nodes, width, V, dtype, drafts):
    """R requests with trees of nodes_min..nodes nodes, `width` children a node, over a vocabulary of V;
    `drafts`: the drafts' own probabilities are at hand."""
    return {"name": name, "kind": "verify", "R": R, "nodes_min": nodes_min, "nodes": nodes, "width": width, "V": V,
            "dtype": dtype, "drafts": drafts}


def _commit(name, fmt, R, Hkv, D, nodes, path, ctx, page):
    """Up to `path` of `nodes` rows kept for each of R requests, behind contexts of up to ctx tokens."""
    return {"name": name, "kind": "commit", "fmt": fmt, "R": R, "Hkv": Hkv, "D": D, "nodes": nodes, "path": path,
            "ctx": ctx, "page": page}


def listed():
    return [
        # one request alone with a small tree: latency counts
        _tree("tree bf16 1x8 of 1000", "bf16", 1, 32, 8, 128, 8, 8, 1000, 1000, 32),
        # the 64-request workload's private contexts, 16 nodes a request
        _tree("tree bf16 64x16 of 4096", "bf16", 64, 32, 8, 128, 16, 16, 4096, 4096, 64),
        # large trees of the serving workload's heads, ragged contexts: bound by arithmetic
        _tree("tree bf16 24x60 of 1K-16K", "bf16", 24, 64, 8, 128, 60, 60, 1024, 16384, 128),
        # the smaller head dimension, trees of different sizes
        _tree("tree bf16 100x5-33 d64", "bf16", 100, 16, 4, 64, 5, 33, 700, 3100, 16),
        # the same in 4-bit pages: eight nodes a request
        _tree("tree fp4 64x8 of 4096", "fp4", 64, 32, 8, 128, 8, 8, 4096, 4096, 64),
        # large trees over 4-bit pages
        _tree("tree fp4 32x64 of 1K-8K", "fp4", 32, 64, 8, 128, 64, 64, 1024, 8192, 32),
        # one request, a chain of five drafted tokens
        _verify("verify 1x6 of 32000", 1, 6, 6, 1, 32000, "float32", True),
        # a batch with trees and the drafts' probabilities
        _verify("verify 64x16 of 128256", 64, 16, 16, 3, 128256, "float32", True),
        # a large batch of drafts picked without chance (a lookup in the prompt), odd vocabulary
        _verify("verify 200x5-25 of 50257", 200, 5, 25, 2, 50257, "float32", False),
        # up to six tokens kept for each of 64 requests
        _commit("commit bf16 64x16", "bf16", 64, 8, 128, 16, 6, 300, 64),
        # a large batch over 4-bit pages
        _commit("commit fp4 300x33", "fp4", 300, 8, 128, 33, 9, 200, 32),
        _commit("commit bf16 512x64", "bf16", 512, 8, 128, 64, 17, 100, 16),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["tree", "tree", "verify", "verify", "commit"])
    fmt = rng.choice(["bf16", "fp4"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if kind == "tree":
        nodes = log(2, 64)
        nodes_min = rng.choice([nodes, rng.randint(1, nodes)])
        R = log(1, 200)
        G = rng.choice([1, 2, 3, 4, 5, 7, 8])
        most = max(256, min(16000, 24 * 60 * 8 * 9000 // (R * nodes * G)))
        len_min = log(128, most)
        len_max = min(most, len_min + log(1, most))
        case = _tree("", fmt, R, Hkv * G, Hkv, D, nodes_min, nodes, len_min, max(len_min, len_max), page)
    elif kind == "verify":
        nodes = log(2, 64)
        V = log(1000, 160000)
        R = min(log(1, 300), max(1, (1 << 28) // (V * nodes)))
        case = _verify("", R, rng.choice([nodes, rng.randint(1, nodes)]), nodes, rng.randint(1, 4), V,
                       rng.choice(["float32", "float32", "bfloat16"]), rng.random() < 0.6)
    else:
        path = log(2, 20)
        nodes = min(64, 2 * path + log(1, 30))
        case = _commit("", fmt, log(1, 512), Hkv, D, nodes, path, log(1, 300), page)
    return {k: v for k, v in case.items() if k != "name"}


def _spread(n, lo, hi):
    """n whole numbers spread evenly from lo to hi, the same for every seed."""
    return np.round(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([max(lo, hi)], dtype=np.int64)


def _token_bytes(case):
    D, Hkv = case["D"], case["Hkv"]
    return 4 * D * Hkv if case["fmt"] == "bf16" else (D + D // 8) * Hkv


def work(case):
    R = case["R"]
    if case["kind"] == "tree":
        T = _spread(R, case["nodes_min"], case["nodes"])
        n = _spread(R, case["len_min"], case["len_max"])
        rows = int(T.sum()) * case["Hq"]
        return {"bytes": int(n.sum()) * _token_bytes(case) + rows * (4 * case["D"] + 4) + int(T.sum()) * 4,
                "flops": 4 * case["D"] * case["Hq"] * int((n * T).sum())}
    if case["kind"] == "verify":
        # every walk ends in one row of the vocabulary; where a test failed there, the drafts' row too
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": R * case["V"] * size * (2 if case["drafts"] else 1) + 12 * R * case["nodes"], "flops": 0}
    moved = int((_spread(R, 1, case["path"]) - 1).sum())  # the first row of a path stays where it is
    reads = R * case["nodes"] * (_token_bytes(case) + 4 * case["D"] * case["Hkv"]) if case["fmt"] == "fp4" else 0  # read back as bf16
    return {"bytes": 2 * moved * _token_bytes(case) + reads + 4 * R * (case["path"] + 3), "flops": 0}


# ---- inputs --------------------------------------------------------------------------------------
def _quantise(x):
    """fp32 [..., D] -> (codes uint8 [..., D] in 0..15, scales f16 [..., D / 32])."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    a = g.abs()
    s = torch.clamp(a.amax(-1) / 6.0, max=MAX_SCALE).to(torch.float16)
    t = s.float().unsqueeze(-1)
    code = ((a > 0.25 * t).to(torch.uint8) + (a >= 0.75 * t).to(torch.uint8) + (a > 1.25 * t).to(torch.uint8)
            + (a >= 1.75 * t).to(torch.uint8) + (a > 2.5 * t).to(torch.uint8) + (a >= 3.5 * t).to(torch.uint8)
            + (a > 5.0 * t).to(torch.uint8))
    code = code + 8 * (g < 0).to(torch.uint8)
    return code.reshape(x.shape), s


def _unswizzle(D, device):
    """Chunk g of token pair p of a block's value codes sits at position [p][g] of this table."""
    p = torch.arange(8, device=device).unsqueeze(1)
    g = torch.arange(8, device=device).unsqueeze(0)
    return g ^ (2 * (p % 4) if D == 128 else 4 * ((p // 2) % 2))


def _pack_blocks(kc, ks, vc, vs, D):
    """Codes [n][16][D] and scales [n][16][D / 32] of n blocks -> bytes [n][18 D]."""
    n, J = kc.shape[0], D // 32
    kb = kc.reshape(n, 16, J, 4, 4, 2).permute(0, 1, 3, 2, 4, 5)  # [n][token][c][j][byte][nibble]
    kb = (kb[..., 0] | (kb[..., 1] << 4)).reshape(n, 8 * D)
    vb = vc.reshape(n, 8, 2, 8, D // 16, 2).permute(0, 1, 3, 2, 4, 5)  # [n][pair][g][token][byte][nibble]
    vb = vb[..., 0] | (vb[..., 1] << 4)
    at = _unswizzle(D, kc.device).reshape(1, 8, 8, 1, 1).expand(n, 8, 8, 2, D // 16)
    vb = torch.zeros_like(vb).scatter_(2, at, vb).reshape(n, 8 * D)
    kz = ks.contiguous().reshape(n, 16 * J).view(torch.uint8)
    vz = vs.transpose(1, 2).contiguous().reshape(n, 16 * J).view(torch.uint8)
    return torch.cat([kb, vb, kz, vz], 1)


def _parents(rng, T, width):
    """A tree of T nodes, level by level, each node with up to `width` children; a random shape."""
    up = np.full(T, -1, dtype=np.int32)
    room = [width] * T
    first = 0
    for j in range(1, T):
        while room[first] == 0:
            first += 1
        at = first + int(rng.integers(0, max(1, min(j - first, 3))))
        at = at if room[at] > 0 else first
        up[j] = at
        room[at] -= 1
    return up


def _paged(case, gen, rng, length):
    """Pages of contexts of the given lengths in random order, with their table."""
    D, Hkv, page, R = case["D"], case["Hkv"], case["page"], case["R"]

    def fill(shape, outlier):
        """Normal values in bf16; with `outlier` every 16th dimension of the last axis is four times as large."""
        x = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
        step = max(1, (1 << 25) // int(np.prod(shape[1:])))
        for i in range(0, shape[0], step):
            y = torch.randn((min(step, shape[0] - i),) + tuple(shape[1:]), generator=gen, device="cuda")
            if outlier:
                y[..., ::16] *= 4.0
            x[i:i + step] = y.to(torch.bfloat16)
        return x

    pages = -(-length // page)
    n_pages = int(pages.sum()) + 3
    order = rng.permutation(n_pages)
    table = np.full((R, int(pages.max())), -1, dtype=np.int32)  # unused entries hold no page
    for r in range(R):
        at = int(pages[:r].sum())
        table[r, :pages[r]] = order[at:at + pages[r]]
    s = {"case": dict(case), "page_table": torch.from_numpy(table).cuda(),
         "kv_len": torch.from_numpy(length.astype(np.int32)).cuda(), "max_len": int(length.max())}
    if case["fmt"] == "bf16":
        s["k_pages"] = fill((n_pages, page, Hkv, D), True)
        s["v_pages"] = fill((n_pages, page, Hkv, D), False)
    else:
        pool = torch.empty((n_pages, Hkv, page // 16, 18 * D), device="cuda", dtype=torch.uint8)
        step = max(1, (1 << 25) // (page * Hkv * D))
        for i in range(0, n_pages, step):
            n = min(step, n_pages - i) * Hkv * (page // 16)
            kc, ks = _quantise(fill((n, 16, D), True).float())
            vc, vs = _quantise(fill((n, 16, D), False).float())
            pool[i:i + step] = _pack_blocks(kc, ks, vc, vs, D).reshape(-1, Hkv, page // 16, 18 * D)
        s["pages4"] = pool
    return s, fill


def _rows(s, T):
    """Where each request's nodes begin; None in a call where all have as many."""
    first = np.concatenate([[0], np.cumsum(T)]).astype(np.int32)
    s["row_start"] = torch.from_numpy(first).cuda()
    s["uniform"] = bool((T == T[0]).all())
    s["B"], s["T"] = int(first[-1]), int(T.max())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    R = case["R"]
    if case["kind"] == "commit":
        n_path = rng.permutation(_spread(R, 1, case["path"]))
        length = case["nodes"] + rng.permutation(_spread(R, 0, case["ctx"]))
        s, _ = _paged(case, gen, rng, length)
        # kept nodes lie behind all places that they move to (levels are stored one after another): the same
        # call again finds the same rows
        path = np.full((R, case["path"]), -1, dtype=np.int32)
        path[:, 0] = 0
        for r in range(R):
            path[r, 1:n_path[r]] = np.sort(rng.choice(np.arange(case["path"], case["nodes"]), n_path[r] - 1, replace=False))
        s["path"] = torch.from_numpy(path).cuda()
        s["n_path"] = torch.from_numpy(n_path.astype(np.int32)).cuda()
        return s
    T = rng.permutation(_spread(R, case["nodes_min"], case["nodes"]))
    if case["kind"] == "tree":
        order = np.argsort(np.argsort(T, kind="stable"), kind="stable")
        length = np.maximum(_spread(R, case["len_min"], case["len_max"])[order], T)  # as in work(): the longest with the most nodes
        s, fill = _paged(case, gen, rng, length)
        _rows(s, T)
        s["q"] = fill((s["B"], case["Hq"], case["D"]), False)
        s["parents"] = torch.from_numpy(np.concatenate([_parents(rng, int(t), 3) for t in T])).cuda()
        return s
    s = {"case": dict(case)}
    _rows(s, T)
    B, V = s["B"], case["V"]
    parents = np.concatenate([_parents(rng, int(t), case["width"]) for t in T])
    first = np.repeat(s["row_start"].cpu().numpy()[:-1], T)
    above = torch.from_numpy(np.where(parents >= 0, parents + first, np.arange(B))).cuda()  # the row of each node's parent
    dtype = getattr(torch, case["dtype"])
    s["target_probs"] = torch.empty(B, V, device="cuda", dtype=dtype)
    draft = torch.empty(B, V, device="cuda", dtype=dtype)
    step = max(1, (1 << 26) // V)
    for i in range(0, B, step):  # peaked distributions, the draft's near the target's
        x = 4.0 * torch.randn(min(step, B - i), V, generator=gen, device="cuda")
        s["target_probs"][i:i + step] = torch.softmax(x, 1).to(dtype)
        draft[i:i + step] = torch.softmax(x + torch.randn(x.shape, generator=gen, device="cuda"), 1).to(dtype)
    s["tokens"] = torch.empty(B, device="cuda", dtype=torch.int32)
    for i in range(0, B, step):  # each node's token is drawn from the draft at its parent
        s["tokens"][i:i + step] = torch.multinomial(draft[above[i:i + step]].float(), 1, generator=gen).squeeze(1).int()
    s["draft_probs"] = draft if case["drafts"] else None
    s["parents"] = torch.from_numpy(parents).cuda()
    s["u_accept"] = torch.rand(B, generator=gen, device="cuda")
    s["u_next"] = torch.rand(R, generator=gen, device="cuda")
    return s


# ---- the plain forms -----------------------------------------------------------------------------
def _grid(s):
    """Rows of the requests' nodes [R][T], and which of them exist."""
    first = s["row_start"].long()
    node = torch.arange(s["T"], device=first.device)
    at = first[:-1].unsqueeze(1) + node
    there = at < first[1:].unsqueeze(1)
    return torch.where(there, at, first[:-1].unsqueeze(1)), there


def _unpack_blocks(b, D):
    """Bytes [..., 18 D] of blocks -> keys and values fp32 [..., 16, D]."""
    J, lead = D // 32, b.shape[:-1]
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=b.device)
    kb = b[..., :8 * D].reshape(*lead, 16, 4, J, 4).transpose(-2, -3)  # [token][j][c][byte]
    k = lut[torch.stack([kb & 15, kb >> 4], -1).int()].reshape(*lead, 16, J, 32)
    ks = b[..., 16 * D:17 * D].contiguous().view(torch.float16).reshape(*lead, 16, J, 1)
    k = (k * ks).reshape(*lead, 16, D)
    vb = b[..., 8 * D:16 * D].reshape(*lead, 8, 8, D // 8)
    vb = torch.gather(vb, -2, _unswizzle(D, b.device).unsqueeze(-1).expand(*lead, 8, 8, D // 8))
    vb = vb.reshape(*lead, 8, 8, 2, D // 16).transpose(-2, -3)  # [pair][token][g][byte]
    v = lut[torch.stack([vb & 15, vb >> 4], -1).int()].reshape(*lead, 16, J, 32)
    vs = b[..., 17 * D:].contiguous().view(torch.float16).reshape(*lead, J, 16).transpose(-1, -2).unsqueeze(-1)
    return k, (v * vs).reshape(*lead, 16, D)


def _contexts(s):
    """Keys and values of the whole contexts in fp32 [R][Hkv][tokens][D]."""
    c = s["case"]
    R, Hkv, D = c["R"], c["Hkv"], c["D"]
    table = s["page_table"].long().clamp(min=0)
    if c["fmt"] == "bf16":
        return tuple(s[n][table].reshape(R, -1, Hkv, D).permute(0, 2, 1, 3).float() for n in ("k_pages", "v_pages"))
    k, v = _unpack_blocks(s["pages4"][table].permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, 18 * D), D)
    return k.reshape(R, Hkv, -1, D), v.reshape(R, Hkv, -1, D)


def _tree_plain(s):
    c = s["case"]
    R, Hq, Hkv, D, T = c["R"], c["Hq"], c["Hkv"], c["D"], s["T"]
    G = Hq // Hkv
    k, v = _contexts(s)
    at, there = _grid(s)
    up = torch.where(there, s["parents"].long()[at], torch.full_like(at, -1))
    # reach[r][i][a]: a is i or above it; the parents' parents, one level a step
    node = torch.arange(T, device=at.device)
    reach = node.expand(R, T).unsqueeze(-1) == node
    cur = up
    for _ in range(T - 1):
        reach = reach | (cur.unsqueeze(-1) == node)
        cur = torch.where(cur >= 0, torch.gather(up, 1, cur.clamp(min=0)), cur)
    committed = s["kv_len"].long() - there.sum(1)
    token = torch.arange(k.shape[2], device=k.device)
    drafted = token - committed.unsqueeze(1)  # [R][tokens]: which node a token is
    seen = torch.gather(reach, 2, drafted.clamp(0, T - 1).unsqueeze(1).expand(R, T, -1))
    seen = (drafted < 0).unsqueeze(1) | (seen & (drafted < there.sum(1, keepdim=True)).unsqueeze(1))
    hidden = ~seen.repeat_interleave(G, 1).unsqueeze(1)  # [R][1][T G][tokens]
    q = s["q"].float()[at].reshape(R, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, T * G, D)
    p = q @ k.transpose(-1, -2) * (1.0 / math.sqrt(D))
    p = p.masked_fill_(hidden, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = ((p @ v) / total).reshape(R, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(R, T, Hq, D)
    lse = (top + torch.log(total)).reshape(R, Hkv, T, G).permute(0, 2, 1, 3).reshape(R, T, Hq)
    return out[there].to(torch.bfloat16), lse[there]


def _verify_plain(s):
    """All requests at once, node after node; 64 bits: a border decides which token comes next."""
    c = s["case"]
    R, T, V = c["R"], s["T"], c["V"]
    at, there = _grid(s)
    up, token = s["parents"].long()[at], s["tokens"].long()[at]
    u = s["u_accept"].double()[at]
    each = torch.arange(R, device=at.device)
    cur = torch.zeros(R, dtype=torch.int64, device=at.device)
    p = s["target_probs"][at[:, 0]].double()
    z = torch.ones(R, dtype=torch.float64, device=at.device)
    path = torch.full((R, T), -1, dtype=torch.int32, device=at.device)
    path[:, 0] = 0
    n_path = torch.ones(R, dtype=torch.int32, device=at.device)
    for j in range(1, T):
        x = token[:, j]
        tried = there[:, j] & (up[:, j] == cur) & (x >= 0) & (x < V)
        x = x.clamp(0, V - 1)
        px = p[each, x]
        row = at[each, cur]
        qx = s["draft_probs"][row, x].double() if c["drafts"] else torch.ones_like(px)
        taken = tried & (px > 0) & (u[:, j] * qx * z < px)
        failed = tried & ~taken
        if c["drafts"]:
            left = (p / z.unsqueeze(1) - s["draft_probs"][row].double()).clamp_(min=0.0)
            sum_left = left.sum(1)
            moves = failed & (sum_left > 0)
            p = torch.where(moves.unsqueeze(1), left, p)
            z = torch.where(moves, sum_left, z)
        else:
            z = torch.where(failed, z - px, z)
            p[each, x] = torch.where(failed, torch.zeros_like(px), px)
        p = torch.where(taken.unsqueeze(1), s["target_probs"][at[:, j]].double(), p)
        z = torch.where(taken, torch.ones_like(z), z)
        cur = torch.where(taken, torch.full_like(cur, j), cur)
        path.scatter_(1, torch.where(taken, n_path.long(), torch.zeros_like(cur)).unsqueeze(1),
                      torch.where(taken, cur, torch.zeros_like(cur)).int().unsqueeze(1))
        n_path = n_path + taken.int()
    sums = p.cumsum(1)
    over = (sums > (s["u_next"].double() * sums[:, -1]).unsqueeze(1)) & (p > 0)
    last = V - 1 - (p > 0).flip(1).int().argmax(1)
    nxt = torch.where(over.any(1), over.int().argmax(1), last)
    return path, n_path, torch.where((p > 0).any(1), nxt, torch.full_like(nxt, -1)).int()


def _block_bytes(D, device):
    """Bytes of each of a block's 16 tokens inside it [16][9 D / 8], as places in the block."""
    t = torch.arange(16, device=device).unsqueeze(1)
    keys = t * (D // 2) + torch.arange(D // 2, device=device)
    chunk = torch.arange(8, device=device).repeat_interleave(D // 16)
    swap = 2 * ((t // 2) % 4) if D == 128 else 4 * ((t // 4) % 2)
    values = 8 * D + (t // 2) * D + (chunk ^ swap) * (D // 8) + (t % 2) * (D // 16) + torch.arange(D // 16, device=device).repeat(8)
    two = torch.arange(D // 16, device=device)
    key_scales = 16 * D + t * (D // 16) + two
    value_scales = 17 * D + 2 * ((two // 2) * 16 + t) + two % 2
    return torch.cat([keys, values, key_scales, value_scales], 1)


def _commit_plain(s):
    c = s["case"]
    R, D, Hkv, P, page = c["R"], c["D"], c["Hkv"], c["path"], c["page"]
    committed = s["kv_len"].long() - c["nodes"]
    j = torch.arange(P, device=committed.device)
    kept = j < s["n_path"].unsqueeze(1)
    req = torch.arange(R, device=committed.device).unsqueeze(1).expand(R, P)[kept]
    to = (committed.unsqueeze(1) + j)[kept]
    source = (committed.unsqueeze(1) + s["path"].long())[kept]
    table = s["page_table"].long()
    to_page, from_page = table[req, to // page], table[req, source // page]
    kv_len = (committed + s["n_path"]).int()
    if c["fmt"] == "bf16":
        for n in ("k_pages", "v_pages"):
            s[n][to_page, to % page] = s[n][from_page, source % page]
        return s["k_pages"], s["v_pages"], kv_len
    pool, where = s["pages4"], _block_bytes(D, committed.device)
    heads = torch.arange(Hkv, device=committed.device).reshape(1, Hkv, 1)

    def rows(at_page, token):
        return at_page.reshape(-1, 1, 1), heads, (token % page // 16).reshape(-1, 1, 1), where[token % 16].unsqueeze(1)

    pool[rows(to_page, to)] = pool[rows(from_page, source)]
    # the nodes' rows read back, as the values that they stand for
    k, v = _contexts(s)
    token = (committed.unsqueeze(1) + torch.arange(c["nodes"], device=committed.device)).reshape(R, 1, -1, 1).expand(R, Hkv, -1, D)
    k, v = (torch.gather(x, 2, token).transpose(1, 2).reshape(-1, Hkv, D).to(torch.bfloat16) for x in (k, v))
    return k, v, kv_len


# ---- the package's calls -------------------------------------------------------------------------
def _handle(s):
    """The store over the pages and, for attention, its scratch: made once and kept by a user's program."""
    if "store" not in s:
        from paper_2511_06010_b200 import paged, speculative

        c = s["case"]
        if c["fmt"] == "bf16":
            s["store"] = paged.PagedKvStore(k_pages=s["k_pages"], v_pages=s["v_pages"])
        else:
            s["store"] = paged.PagedKvStore(pages4=s["pages4"], page_size=c["page"])
        if c["kind"] == "tree":
            s["attention"] = speculative.TreeAttention(s["B"], c["Hq"], c["Hkv"], c["D"], s["max_len"], n_requests=c["R"],
                                                       max_nodes=s["T"], fmt=c["fmt"])
    return s["store"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"tree": _tree_plain, "verify": _verify_plain, "commit": _commit_plain}[c["kind"]](s)
    if c["kind"] == "verify":
        from paper_2511_06010_b200 import speculative

        return speculative.verify(s["target_probs"], s["tokens"], s["parents"], s["u_accept"], s["u_next"],
                                  draft_probs=s["draft_probs"], row_start=s["row_start"], max_nodes=s["T"])
    store = _handle(s)
    if c["kind"] == "tree":
        return s["attention"](s["q"], store, s["page_table"], s["kv_len"], s["parents"],
                              row_start=None if s["uniform"] else s["row_start"])
    kv_len = store.commit(s["page_table"], s["kv_len"], s["path"], s["n_path"], max_nodes=c["nodes"])
    if c["fmt"] == "bf16":
        return store.k_pages, store.v_pages, kv_len
    k, v = store.gather(s["page_table"], s["kv_len"], c["R"] * c["nodes"], q_len=c["nodes"])
    return k, v, kv_len


# ---- the definition in 64 bits -------------------------------------------------------------------
def _byte_map(D):
    """(byte, shift) of dimension d of token t in a block, for keys and for values, and where their scales are."""
    t, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    kbyte = t * (D // 2) + ((d % 32) // 8) * (D // 8) + (d // 32) * 4 + (d % 8) // 2
    width = D // 8                     # dimensions of one chunk
    pair, chunk = t // 2, d // width
    swap = 2 * (pair % 4) if D == 128 else 4 * ((pair // 2) % 2)
    vbyte = 8 * D + pair * D + (chunk ^ swap) * width + (t % 2) * (width // 2) + (d % width) // 2
    kscale = 8 * D + t * (D // 32) + d // 32           # in units of two bytes
    vscale = 8 * D + D // 2 + (d // 32) * 16 + t
    return [torch.from_numpy(x.reshape(-1)).cuda() for x in (kbyte, vbyte, kscale, vscale, 4 * (d % 2))]


def _exact_context(s, r, n):
    """Keys and values [Hkv][n][D] of request r in 64 bits."""
    c = s["case"]
    where = s["page_table"][r, :-(-n // c["page"])].long()
    if c["fmt"] == "bf16":
        return [s[x][where].flatten(0, 1)[:n].double().transpose(0, 1) for x in ("k_pages", "v_pages")]
    value = torch.tensor(E2M1 + tuple(-x for x in E2M1), dtype=torch.float64, device="cuda")
    kbyte, vbyte, kscale, vscale, shift = _byte_map(c["D"])
    b = s["pages4"][where].transpose(0, 1).flatten(1, 2)  # [Hkv][blocks][bytes]
    f = b.contiguous().view(torch.float16).double()
    k = (value[(b[..., kbyte].int() >> shift) & 15] * f[..., kscale]).reshape(c["Hkv"], -1, c["D"])[:, :n]
    v = (value[(b[..., vbyte].int() >> shift) & 15] * f[..., vscale]).reshape(c["Hkv"], -1, c["D"])[:, :n]
    return k, v


def _exact_tree(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    first, length, parents = s["row_start"].tolist(), s["kv_len"].tolist(), s["parents"].tolist()
    out = torch.empty(s["B"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["B"], Hq, dtype=torch.float64, device="cuda")
    for r in range(c["R"]):
        a, b, n = first[r], first[r + 1], length[r]
        T = b - a
        k, v = _exact_context(s, r, n)
        sees = np.ones((T, n), dtype=bool)
        sees[:, n - T:] = False
        for i in range(T):
            up = i
            while up >= 0:
                sees[i, n - T + up] = True
                up = parents[a + up]
        q = s["q"][a:b].double().reshape(T, Hkv, G, D)
        w = torch.einsum("ihgd,htd->higt", q, k) / math.sqrt(D)
        w.masked_fill_(torch.from_numpy(~sees).cuda().reshape(1, T, 1, n), -math.inf)
        lse[a:b] = torch.logsumexp(w, -1).permute(1, 0, 2).reshape(T, Hq)
        out[a:b] = torch.einsum("higt,htd->ihgd", torch.softmax(w, -1), v).reshape(T, Hq, D)
    return out, lse


def _exact_verify(s):
    """One request after the other, on the host; sums that do not round on the way."""
    c = s["case"]
    V, T = c["V"], s["T"]
    first, parents, tokens = s["row_start"].tolist(), s["parents"].tolist(), s["tokens"].tolist()
    u, u_next = s["u_accept"].double().tolist(), s["u_next"].double().tolist()

    def row(x, i):
        return x[i].double().cpu().numpy().copy()

    paths, counts, nexts = [], [], []
    for r in range(c["R"]):
        a = first[r]
        path, cur = [0], 0
        p, z = row(s["target_probs"], a), 1.0
        for j in range(1, first[r + 1] - a):
            x = tokens[a + j]
            if parents[a + j] != cur or not 0 <= x < V:
                continue
            q = row(s["draft_probs"], a + cur) if c["drafts"] else None
            if p[x] > 0 and u[a + j] * (q[x] if c["drafts"] else 1.0) * z < p[x]:
                path.append(j)
                cur, p, z = j, row(s["target_probs"], a + j), 1.0
            elif c["drafts"]:
                left = np.maximum(p / z - q, 0.0)
                total = math.fsum(left)
                if total > 0:
                    p, z = left, total
            else:
                z -= p[x]
                p[x] = 0.0
        goal = u_next[r] * math.fsum(p)
        at = np.flatnonzero((np.cumsum(p) > goal) & (p > 0))
        left = np.flatnonzero(p > 0)
        nexts.append(int(at[0]) if len(at) else int(left[-1]) if len(left) else -1)
        paths.append(path + [-1] * (T - len(path)))
        counts.append(len(path))
    return tuple(torch.tensor(x, dtype=torch.int32) for x in (paths, counts, nexts))


def _exact_commit(s):
    c = s["case"]
    page, nodes = c["page"], c["nodes"]
    length, path, n_path, table = (s[n].tolist() for n in ("kv_len", "path", "n_path", "page_table"))
    kv_len = torch.tensor([n - nodes + m for n, m in zip(length, n_path)], dtype=torch.int32)
    if c["fmt"] == "fp4":
        ks, vs = [], []
        for r in range(c["R"]):
            k, v = _exact_context(s, r, length[r])
            last = list(range(length[r] - nodes, length[r]))
            source = [length[r] - nodes + x for x in path[r][:n_path[r]]] + last[n_path[r]:]
            ks.append(k[:, source].transpose(0, 1))
            vs.append(v[:, source].transpose(0, 1))
        return torch.cat(ks), torch.cat(vs), kv_len
    pools = []
    for n in ("k_pages", "v_pages"):
        old = s[n].double().flatten(0, 1)
        new = old.clone()
        to, source = [], []
        for r in range(c["R"]):
            at = lambda t: table[r][t // page] * page + t % page  # noqa: E731
            to += [at(length[r] - nodes + j) for j in range(n_path[r])]
            source += [at(length[r] - nodes + path[r][j]) for j in range(n_path[r])]
        new[torch.tensor(to, device="cuda")] = old[torch.tensor(source, device="cuda")]
        pools.append(new.reshape(s[n].shape))
    return pools[0], pools[1], kv_len


def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "verify": _exact_verify, "commit": _exact_commit}[case["kind"]](s)
