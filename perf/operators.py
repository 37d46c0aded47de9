"""The operators of the paged private KV store, as measured cases.

Two operators in two storage formats: rows of new keys and values written into a paged cache with the
position rotation applied on the way ("append"), and decode attention over that cache ("attn").
Formats: bf16 pages [n_pages][page_size][Hkv][D], and 4-bit pages: E2M1 codes with one f16 scale per
(token, KV head, 32 dimensions), 16 tokens of a head to a block of bytes.

`run` computes the plain form with elementary torch operations, or, with `own` set, makes the calls
of the package.  `exact` gives the same results in 64 bits, written apart from both.
"""
import math

import numpy as np
import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_SCALE = 10912.0  # largest f16 whose sixfold is still finite in f16
N_POSITIONS = 40960


# ---- cases ---------------------------------------------------------------------------------------
def _append(name, fmt, R, Hq, Hkv, D, rows, rows_max, ctx, page, rot, interleaved):
    """R requests get rows..rows_max new rows each on top of contexts of up to ctx tokens."""
    return {"name": name, "kind": "append", "fmt": fmt, "R": R, "Hq": Hq, "Hkv": Hkv, "D": D, "rows": rows,
            "rows_max": rows_max, "ctx": ctx, "page": page, "rot": rot, "interleaved": interleaved}


def _attn(name, fmt, R, Hq, Hkv, D, q_len, len_min, len_max, page):
    """R requests of q_len query tokens each over contexts of len_min..len_max tokens."""
    return {"name": name, "kind": "attn", "fmt": fmt, "R": R, "Hq": Hq, "Hkv": Hkv, "D": D, "q_len": q_len,
            "len_min": len_min, "len_max": len_max, "page": page}


def listed():
    return [
        # one new token for each of 64 running requests (the 64-request workload's heads): latency counts
        _append("append bf16 64 tokens", "bf16", 64, 32, 8, 128, 1, 1, 1024, 64, 128, False),
        # prompts of 8 new requests enter the cache, ragged, larger head count
        _append("append bf16 prompts", "bf16", 8, 64, 8, 128, 1024, 3000, 0, 64, 128, False),
        # one new token for each of 1024 requests (the serving workload), 4-bit pages
        _append("append fp4 1024 tokens", "fp4", 1024, 64, 8, 128, 1, 1, 512, 32, 128, False),
        # prompts into 4-bit pages: odd lengths, half of the head rotated, neighbouring pairs
        _append("append fp4 prompts", "fp4", 11, 32, 8, 128, 333, 2001, 77, 16, 64, True),
        # the small workload: 16 requests, one KV head, short contexts
        _attn("attn bf16 16x256 d64", "bf16", 16, 4, 1, 64, 1, 256, 256, 16),
        # the 64-request workload's private contexts
        _attn("attn bf16 64x4096", "bf16", 64, 32, 8, 128, 1, 4096, 4096, 64),
        # ragged contexts of the serving workload, 1K to 32K
        _attn("attn bf16 64x1K-32K", "bf16", 64, 64, 8, 128, 1, 1024, 32768, 128),
        # one request alone, long context: the work is split over the tokens
        _attn("attn fp4 1x8191", "fp4", 1, 32, 8, 128, 1, 8191, 8191, 32),
        _attn("attn fp4 64x4096", "fp4", 64, 32, 8, 128, 1, 4096, 4096, 64),
        # four query tokens a request (speculative decoding), ragged
        _attn("attn fp4 48x4 tokens", "fp4", 48, 32, 8, 128, 4, 777, 6001, 16),
        # the smaller head dimension
        _attn("attn fp4 128x2K d64", "fp4", 128, 16, 4, 64, 1, 1500, 2500, 32),
        _attn("attn fp4 64x1K-32K", "fp4", 64, 64, 8, 128, 1, 1024, 32768, 128),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    fmt = rng.choice(["bf16", "fp4"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if rng.random() < 0.5:
        G = rng.choice([1, 3, 4, 7, 8])
        if rng.random() < 0.5:
            R, rows, rows_max = log(1, 1024), 1, 1
        else:
            R, rows = log(1, 16), log(2, 600)
            rows_max = rows + log(1, 1200)
        rot = rng.choice([D, D, D // 2])
        return {k: v for k, v in _append("", fmt, R, Hkv * G, Hkv, D, rows, rows_max, log(1, 600), page, rot,
                                         rng.random() < 0.4).items() if k != "name"}
    q_len = rng.choice([1, 1, 1, 2, 4]) if D == 128 else 1
    G = rng.choice([1, 2, 3, 4]) if q_len > 1 else rng.choice([1, 2, 4, 5, 8])
    R = log(1, 200)
    most = min(32000, 1000000 // R)
    len_min = log(1, most)
    len_max = min(most, len_min + log(1, most))
    return {k: v for k, v in _attn("", fmt, R, Hkv * G, Hkv, D, q_len, len_min, max(len_min, len_max), page).items()
            if k != "name"}


def _spread(n, lo, hi):
    """n whole numbers spread evenly from lo to hi, the same for every seed."""
    return np.round(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([max(lo, hi)], dtype=np.int64)


def _row_bytes(case):
    D, Hkv = case["D"], case["Hkv"]
    return 4 * D * Hkv if case["fmt"] == "bf16" else (D + D // 8) * Hkv


def work(case):
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    if case["kind"] == "append":
        N = int(_spread(case["R"], case["rows"], case["rows_max"]).sum())
        moved = N * ((2 * Hq + 2 * Hkv) * D * 2 + _row_bytes(case) + 4 * case["rot"] + 4)
        if case["fmt"] == "fp4":
            moved += N * (_row_bytes(case) + 4 * D * Hkv)  # the rows are read back as bf16
        return {"bytes": moved, "flops": N * (Hq + Hkv) * case["rot"] * 3}
    T = int(_spread(case["R"], case["len_min"], case["len_max"]).sum())
    rows = case["R"] * case["q_len"] * Hq
    return {"bytes": T * _row_bytes(case) + rows * (4 * D + 4), "flops": 4 * D * T * Hq * case["q_len"]}


# ---- inputs --------------------------------------------------------------------------------------
def _quantise(x):
    """fp32 [..., D] -> (codes uint8 [..., D] in 0..15, scales f16 [..., D / 32])."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = g.abs().amax(-1)
    six = torch.full((), 6.0, device=x.device)
    s = torch.clamp(amax / six, max=MAX_SCALE).to(torch.float16)
    s = torch.where(torch.isfinite(amax), s, torch.full_like(s, float("nan")))
    t = s.float().unsqueeze(-1)
    a = g.abs()
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


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

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

    rng = np.random.default_rng(int(seed))
    R, Hq, Hkv, D, page = case["R"], case["Hq"], case["Hkv"], case["D"], case["page"]
    if case["kind"] == "append":
        new = _spread(R, case["rows"], case["rows_max"])
        length = new + _spread(R, case["ctx"], 0)  # the longest prompts on the shortest contexts
        mixed = rng.permutation(R)
        new, length = new[mixed], length[mixed]
    else:
        new = np.full(R, case["q_len"], dtype=np.int64)
        length = rng.permutation(_spread(R, case["len_min"], case["len_max"]))
    pages = -(-length // page)
    n_pages = int(pages.sum()) + 3
    order = rng.permutation(n_pages)
    table = np.full((R, int(pages.max())), -1, dtype=np.int32)  # unused entries hold no page
    for r in range(R):
        at = int(pages[:r].sum())
        table[r, :pages[r]] = order[at:at + pages[r]]
    s = {"case": dict(case), "page_table": torch.from_numpy(table).cuda(),
         "kv_len": torch.from_numpy(length.astype(np.int32)).cuda(), "max_len": int(length.max())}
    N = int(new.sum())
    if case["kind"] == "append":
        qkv = fill((N, (Hq + 2 * Hkv) * D), False)  # a projection's output: q, k and v are its columns
        s["q"] = qkv[:, :Hq * D].unflatten(1, (Hq, D))
        s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
        s["v"] = qkv[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
        first = np.concatenate([[0], np.cumsum(new)])
        s["row_start"] = torch.from_numpy(first.astype(np.int32)).cuda()
        # private contexts follow a shared corpus of some thousand tokens
        pos = np.concatenate([np.arange(l - n, l) for l, n in zip(length, new)]) + int(rng.integers(0, 30000))
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        half = case["rot"] // 2
        angle = (torch.arange(N_POSITIONS, device="cuda", dtype=torch.float64).unsqueeze(1)
                 * 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half))
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["uniform"] = bool(case["rows_max"] == 1)
    else:
        s["q"] = fill((N, Hq, D), False)
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
    return s


# ---- the plain forms -----------------------------------------------------------------------------
def _rotate(x, cos, sin, rot, interleaved):
    """x fp32 [N][H][D], cos and sin fp32 [N][rot / 2]: every product and sum rounded once."""
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    c, d = cos.unsqueeze(1), sin.unsqueeze(1)
    lo, hi = a * c - b * d, b * c + a * d
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = lo, hi
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = lo, hi
    return y


def _dequantised(x):
    code, s = _quantise(x)
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=x.device)
    return (lut[code.int()].reshape(*x.shape[:-1], -1, 32) * s.float().unsqueeze(-1)).reshape(x.shape)


def _append_plain(s):
    c = s["case"]
    rot = c["rot"]
    table = s["cos_sin"][s["positions"].long()]
    cos, sin = table[:, :rot // 2], table[:, rot // 2:]
    q_out = _rotate(s["q"].float(), cos, sin, rot, c["interleaved"]).to(torch.bfloat16)
    k = _rotate(s["k"].float(), cos, sin, rot, c["interleaved"])
    v = s["v"].float()
    first = s["row_start"].long()
    row = torch.arange(k.shape[0], device=k.device)
    req = torch.searchsorted(first[1:], row, right=True)
    token = s["kv_len"].long()[req] - (first[req + 1] - row)
    if c["fmt"] == "fp4":
        return q_out, _dequantised(k).to(torch.bfloat16), _dequantised(v).to(torch.bfloat16)
    where = s["page_table"].long()[req, token // c["page"]]
    s["k_pages"][where, token % c["page"]] = k.to(torch.bfloat16)
    s["v_pages"][where, token % c["page"]] = v.to(torch.bfloat16)
    return q_out, s["k_pages"], s["v_pages"]


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


def _attn_plain(s):
    c = s["case"]
    R, Hq, Hkv, D, T, page = c["R"], c["Hq"], c["Hkv"], c["D"], c["q_len"], c["page"]
    G = Hq // Hkv
    table = s["page_table"].long().clamp(min=0)
    if c["fmt"] == "bf16":
        k = s["k_pages"][table].reshape(R, -1, Hkv, D).permute(0, 2, 1, 3).float()
        v = s["v_pages"][table].reshape(R, -1, Hkv, D).permute(0, 2, 1, 3).float()
    else:
        k, v = _unpack_blocks(s["pages4"][table].permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, 18 * D), D)
        k, v = k.reshape(R, Hkv, -1, D), v.reshape(R, Hkv, -1, D)
    q = s["q"].float().reshape(R, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, T * G, D)
    score = q @ k.transpose(-1, -2) * (1.0 / math.sqrt(D))
    token = torch.arange(k.shape[2], device=k.device)
    seen = s["kv_len"].reshape(R, 1) - (T - 1 - torch.arange(T, device=k.device))  # [R][T]
    hidden = (token >= seen.repeat_interleave(G, 1).unsqueeze(-1)).unsqueeze(1)      # [R][1][T G][tokens]
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(-1)
    out = out.reshape(R, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(R * T, Hq, D)
    return out.to(torch.bfloat16), lse.reshape(R, Hkv, T, G).permute(0, 2, 1, 3).reshape(R * T, Hq)


# ---- the package's calls -------------------------------------------------------------------------
def _handle(s):
    """The store over the pages and, for attention, its scratch: made once and kept by a user's program."""
    if "store" not in s:
        from paper_2511_06010_b200 import paged

        c = s["case"]
        if c["fmt"] == "bf16":
            s["store"] = paged.PagedKvStore(k_pages=s["k_pages"], v_pages=s["v_pages"])
        else:
            s["store"] = paged.PagedKvStore(pages4=s["pages4"], page_size=c["page"])
        if c["kind"] == "attn":
            s["attention"] = paged.PagedAttention(c["R"] * c["q_len"], c["Hq"], c["Hkv"], c["D"], s["max_len"],
                                                  fmt=c["fmt"], q_len=c["q_len"])
    return s["store"]


def run(state):
    c = state["case"]
    if not own:
        return _append_plain(state) if c["kind"] == "append" else _attn_plain(state)
    store = _handle(state)
    if c["kind"] == "attn":
        return state["attention"](state["q"], store, state["page_table"], state["kv_len"])
    rows = None if state["uniform"] else state["row_start"]
    q_out = store.append(state["q"], state["k"], state["v"], state["page_table"], state["kv_len"],
                         state["positions"], state["cos_sin"], row_start=rows, interleaved=c["interleaved"])
    if c["fmt"] == "bf16":
        return q_out, store.k_pages, store.v_pages
    k, v = store.gather(state["page_table"], state["kv_len"], state["k"].shape[0], row_start=rows)
    return q_out, k, v


# ---- the definition in 64 bits -------------------------------------------------------------------
def _nearest_e2m1(x):
    """x fp64 [..., D] -> what 4 bits with a scale for each 32 dimensions hold of it (ties to the even code)."""
    g = x.reshape(-1, 32)
    scale = (g.abs().max(1, keepdim=True).values / 6).clamp(max=MAX_SCALE).to(torch.float16).double()
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    a = (g.abs() / torch.where(scale > 0, scale, torch.ones_like(scale))).clamp(max=6.0)
    up = torch.bucketize(a, grid).clamp(max=7)
    down = (up - 1).clamp(min=0)
    mid = (grid[up] + grid[down]) / 2
    pick = torch.where((a > mid) | ((a == mid) & (up % 2 == 0)), up, down)
    pick = torch.where(a == grid[up], up, pick)
    return (grid[pick] * scale * g.sign()).reshape(x.shape)


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


def exact(case, seed):
    s = prepare(case, seed)

    def appended():
        c = s["case"]
        rot, half = c["rot"], c["rot"] // 2
        cs = s["cos_sin"].double()[s["positions"].long()]
        z = torch.complex(cs[:, :half], cs[:, half:]).unsqueeze(1)

        def turned(x):
            x = x.double()
            r = x[..., :rot]
            if c["interleaved"]:
                w = torch.view_as_real(torch.view_as_complex(r.unflatten(-1, (half, 2)).contiguous()) * z).flatten(-2)
            else:
                w = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * z
                w = torch.cat([w.real, w.imag], -1)
            return torch.cat([w, x[..., rot:]], -1)

        q, k, v = turned(s["q"]), turned(s["k"]), s["v"].double()
        if c["fmt"] == "fp4":
            return q, _nearest_e2m1(k), _nearest_e2m1(v)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        first, length, table = s["row_start"].tolist(), s["kv_len"].tolist(), s["page_table"].cpu()
        for r in range(c["R"]):
            n = first[r + 1] - first[r]
            t = torch.arange(length[r] - n, length[r])
            flat = (table[r].long()[t // c["page"]] * c["page"] + t % c["page"]).to(kp.device)
            kp.flatten(0, 1)[flat] = k[first[r]:first[r + 1]]
            vp.flatten(0, 1)[flat] = v[first[r]:first[r + 1]]
        return q, kp, vp

    def attended():
        c = s["case"]
        Hq, Hkv, D, T, page = c["Hq"], c["Hkv"], c["D"], c["q_len"], c["page"]
        G = Hq // Hkv
        out = torch.zeros(c["R"] * T, Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.full((c["R"] * T, Hq), -math.inf, dtype=torch.float64, device="cuda")
        if c["fmt"] == "fp4":
            kbyte, vbyte, kscale, vscale, shift = _byte_map(D)
            value = torch.tensor(E2M1 + tuple(-x for x in E2M1), dtype=torch.float64, device="cuda")
        for r in range(c["R"]):
            n = int(s["kv_len"][r])
            if n == 0:
                continue
            where = s["page_table"][r, :-(-n // page)].long()
            if c["fmt"] == "bf16":
                k = s["k_pages"][where].flatten(0, 1)[:n].double().transpose(0, 1)
                v = s["v_pages"][where].flatten(0, 1)[:n].double().transpose(0, 1)
            else:
                b = s["pages4"][where].transpose(0, 1).flatten(1, 2)  # [Hkv][blocks][bytes]
                f = b.contiguous().view(torch.float16).double()
                k = (value[(b[..., kbyte].int() >> shift) & 15] * f[..., kscale]).reshape(Hkv, -1, D)[:, :n]
                v = (value[(b[..., vbyte].int() >> shift) & 15] * f[..., vscale]).reshape(Hkv, -1, D)[:, :n]
            for i in range(T):
                m = n - (T - 1 - i)
                if m <= 0:
                    continue
                q = s["q"][r * T + i].double().reshape(Hkv, G, D)
                w = torch.einsum("hgd,htd->hgt", q, k[:, :m]) / math.sqrt(D)
                lse[r * T + i] = torch.logsumexp(w, -1).reshape(Hq)
                out[r * T + i] = torch.einsum("hgt,htd->hgd", torch.softmax(w, -1), v[:, :m]).reshape(Hq, D)
        return out, lse

    return appended() if case["kind"] == "append" else attended()
