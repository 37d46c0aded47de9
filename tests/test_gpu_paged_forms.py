"""Forms of the paged attention that the plain cases do not reach: partial slots with several query tokens, the
order of the requests in every instantiation, outlier query dimensions, shared prefixes, padded batches."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    from paper_2511_06010_b200 import binding as M

    M.device_status()
    yield
    torch.cuda.synchronize()
    assert M.device_status() == 0


def _contexts(fmt, D, Hkv, page, lens, gen):
    """Contexts appended into shuffled pages that hold NaN everywhere else; -> store, page table, lengths (GPU)
    and what the store holds of keys and values, [sum(lens)][Hkv][D] in 64 bits."""
    from paper_2511_06010_b200.paged import PagedKvStore

    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 3, generator=gen)
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = order[sum(need[:r]):sum(need[:r]) + n]
    st = PagedKvStore.empty(sum(need) + 3, page, Hkv, D, fmt)
    for pool in (st.k_pages, st.v_pages) if fmt == "bf16" else (st.pages4,):
        pool.view(torch.uint8).fill_(0xFF)
    k, v = (R.make_bf16((sum(lens), Hkv, D), gen) for _ in range(2))
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    st.append(None, k.cuda(), v.cuda(), table.cuda(), length, row_start=first)
    held = [R.to_f64(x) if fmt == "bf16" else R.held32(x.float().numpy()) for x in (k, v)]
    return st, table.cuda(), length, held


def _compare(out, lse, held, lens, q, T, scale, fmt, requests=None):
    """out [B][Hq][D] and lse [B][Hq] (float64, on the host) against the definition."""
    q64 = R.to_f64(q)
    for r in range(len(lens)) if requests is None else requests:
        at, n = sum(lens[:r]), lens[r]
        for i in range(T):
            m, b = max(0, n - (T - 1 - i)), r * T + i
            o, l, o_tol, l_tol = R.attend(q64[b], held[0][at:at + m], held[1][at:at + m], scale, fmt)
            assert (np.abs(out[b] - o) <= o_tol).all(), (r, i, np.abs(out[b] - o).max())
            if m == 0:
                assert np.isneginf(lse[b]).all()
            else:
                assert (np.abs(lse[b] - l) <= l_tol).all(), (r, i)


def _joined(o_part, lse_part):
    """Partial rows [B][Hq][slots][D] and [B][Hq][slots] -> the rows and their lse, in 64 bits."""
    o, l = o_part.double().cpu().numpy(), lse_part.double().cpu().numpy()
    top = l.max(-1, keepdims=True)
    base = np.where(np.isneginf(top), 0.0, top)
    w = np.exp(l - base)
    total = w.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (base + np.log(total))[..., 0]
    return (w[..., None] * o).sum(-2) / np.where(total > 0, total, 1.0), lse


SHAPES = [  # fmt, D, Hq, Hkv, T
    (fmt, D, Hq, Hkv, T)
    for fmt in ("bf16", "fp4")
    for D, Hq, Hkv, T in ((128, 8, 4, 1), (128, 8, 4, 4), (128, 12, 4, 4), (128, 16, 4, 4), (128, 4, 4, 16), (64, 8, 4, 1),
                          (64, 8, 4, 4), (64, 16, 4, 4))
    if fmt == "fp4" or D == 128 or T == 1
]


@pytest.mark.parametrize("fmt,D,Hq,Hkv,T", SHAPES)
@pytest.mark.parametrize("splits", [1, 3])
def test_partial_slots(fmt, D, Hq, Hkv, T, splits):
    """MoskaLayer.unique_paged: the slots behind the shared ones hold the private context's parts, and nothing else is
    touched.  Contexts shorter than the query tokens and empty ones among them."""
    from paper_2511_06010_b200.engine import MoskaLayer

    gen = torch.Generator().manual_seed(61)
    lens = [0, 1, 3, 4, 17, 64, 300, 129, 15, 1000]
    st, table, length, held = _contexts(fmt, D, Hkv, 32, lens, gen)
    B = len(lens) * T
    layer = MoskaLayer(B, Hq, Hkv, D, 4, 128, 2, max(lens), n_unique_splits=splits, q_len=T)
    assert layer.n_slots == 2 + splits
    layer.o_part.fill_(7.0)
    layer.lse_part.fill_(7.0)
    q = R.make_bf16((B, Hq, D), gen)
    layer.unique_paged(q.cuda(), st, table, length)
    assert (layer.o_part[:, :, :2] == 7.0).all() and (layer.lse_part[:, :, :2] == 7.0).all()
    out, lse = _joined(layer.o_part[:, :, 2:], layer.lse_part[:, :, 2:])
    _compare(out, lse, held, lens, q, T, layer.scale, fmt)


@pytest.mark.parametrize("fmt,D,Hq,Hkv,T", SHAPES)
@pytest.mark.parametrize("form", ["final rows", "splits", "slots"])
def test_ragged_contexts_longest_first(fmt, D, Hq, Hkv, T, form):
    """More than 148 CTAs, so that requests are taken longest first: every instantiation, with ties and empty
    contexts."""
    from paper_2511_06010_b200.engine import MoskaLayer
    from paper_2511_06010_b200.paged import PagedAttention

    gen = torch.Generator().manual_seed(62)
    rng = np.random.default_rng(62)
    lens = [int(n) for n in rng.integers(0, 260, 57)] + [16, 16, 0, 1, 259]
    splits = 1 if form == "final rows" else 2
    assert len(lens) * Hkv * splits > 148 and len(lens) <= 128
    st, table, length, held = _contexts(fmt, D, Hkv, 16, lens, gen)
    B = len(lens) * T
    q = R.make_bf16((B, Hq, D), gen)
    if form == "slots":
        layer = MoskaLayer(B, Hq, Hkv, D, 4, 128, 1, max(lens), n_unique_splits=splits, q_len=T)
        layer.o_part.fill_(float("nan"))
        layer.lse_part.fill_(float("nan"))
        layer.unique_paged(q.cuda(), st, table, length)
        out, lse = _joined(layer.o_part[:, :, 1:], layer.lse_part[:, :, 1:])
    else:
        attention = PagedAttention(B, Hq, Hkv, D, max(lens), fmt=fmt, q_len=T, n_unique_splits=splits)
        attention.out.fill_(float("nan"))
        attention.lse.fill_(float("nan"))
        out, lse = (t.double().cpu().numpy() for t in attention(q.cuda(), st, table, length))
    _compare(out, lse, held, lens, q, T, 1.0 / math.sqrt(D), fmt)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("G,T", [(2, 4), (4, 4), (1, 16)])
@pytest.mark.parametrize("splits,two_streams", [(1, False), (3, True)])
def test_decode_step_with_several_query_tokens(fmt, G, T, splits, two_streams):
    from oracle import oracle as O
    from paper_2511_06010_b200 import workloads as W
    from paper_2511_06010_b200.engine import MoskaLayer
    from tests import parity_utils as PU

    lens = [300, 1, 0, 1000, 64, 17, 2, 511]
    Hkv, D, B = 2, 128, len(lens) * T
    gen = torch.Generator().manual_seed(63)
    st, table, length, held = _contexts(fmt, D, Hkv, 64, lens, gen)
    w = W.scaled(W.CONFIGS[1], B=B, Hq=G * Hkv, Hkv=Hkv, C=8, k=3, L=256, unique_len=0)
    sh = W.make_shared_store(w, "cuda")
    q = W.make_queries(w, sh, 0, "cuda")
    layer = MoskaLayer(B, w.Hq, Hkv, D, w.C, w.L, w.k, max(lens), n_unique_splits=splits, q_len=T)
    layer.build_summaries(sh.k_shared)
    out = layer.step_paged(q, sh.k_shared, sh.v_shared, st, table, length, two_streams=two_streams)
    torch.cuda.synchronize()
    o_sh, l_sh = O.shared_partials(q.cpu(), sh.k_shared.cpu(), sh.v_shared.cpu(), layer.topk_idx.cpu().numpy(), layer.scale)
    o_u, l_u = np.zeros((B, w.Hq, D)), np.zeros((B, w.Hq))
    for b in range(B):
        r, i = divmod(b, T)
        at, m = sum(lens[:r]), max(0, lens[r] - (T - 1 - i))
        o_u[b], l_u[b], _, _ = R.attend(R.to_f64(q[b]), held[0][at:at + m], held[1][at:at + m], layer.scale, fmt)
    ref_o, ref_l = O.merge(np.concatenate([o_sh, o_u[:, :, None]], axis=2), np.concatenate([l_sh, l_u[:, :, None]], axis=2))
    PU.check_attention(out.float().cpu().numpy(), ref_o, f"paged step, {fmt}, {T} query tokens")
    PU.check_lse(layer.lse_out.cpu().numpy(), ref_l, "paged step lse")


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("outlier", [2.0 ** 8, 2.0 ** 14])
def test_queries_with_an_outlier_dimension(fmt, outlier):
    """One dimension of the queries far above the others: with keys small there the others still decide.  4-bit
    pages: queries are held in f16 relative to the row's largest, so an element is off by 2^-25 of that at most
    (2^-24 steps), which moves a score by scale 2^-24 max|q| sum|k|."""
    from paper_2511_06010_b200.paged import PagedAttention

    D, Hq, Hkv, lens = 128, 4, 1, [40, 333]
    gen = torch.Generator().manual_seed(64)
    st, table, length, _ = _contexts(fmt, D, Hkv, 16, lens, gen)
    k, v = (R.make_bf16((sum(lens), Hkv, D), gen) for _ in range(2))
    k[..., 32:64] = 0  # (a scale covers 32 dimensions)
    first = torch.tensor([0, 40, 373], dtype=torch.int32).cuda()
    st.append(None, k.cuda(), v.cuda(), table, length, row_start=first)
    held = [R.to_f64(x) if fmt == "bf16" else R.held32(x.float().numpy()) for x in (k, v)]
    q = R.make_bf16((2, Hq, D), gen)
    q[..., 40] = outlier
    attention = PagedAttention(2, Hq, Hkv, D, 333, fmt=fmt, n_unique_splits=1)
    out, lse = (t.double().cpu().numpy() for t in attention(q.cuda(), st, table, length))
    for r, (a, b) in enumerate(((0, 40), (40, 373))):
        o, l, o_tol, l_tol = R.attend(R.to_f64(q[r]), held[0][a:b], held[1][a:b], attention.scale, fmt)
        ds = 0.0 if fmt == "bf16" else attention.scale * 2.0 ** -24 * outlier * np.abs(held[0][a:b]).sum(-1).max()
        o_tol = o_tol + 2 * ds * np.abs(held[1][a:b]).max()
        assert (np.abs(out[r] - o) <= o_tol).all() and (np.abs(lse[r] - l) <= l_tol + ds).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_requests_that_share_the_pages_of_a_prefix(fmt):
    """The same page in several rows of the table, and twice in one; padded request slots without a context between."""
    from paper_2511_06010_b200.paged import PagedAttention

    D, Hq, Hkv, page = 128, 8, 2, 16
    gen = torch.Generator().manual_seed(65)
    st, table, length, held = _contexts(fmt, D, Hkv, page, [64, 33], gen)
    t = table.cpu()
    own, other = t[0, :4].tolist(), t[1, :3].tolist()
    rows = [own, own[:2] + other, [-1] * 5, [own[1]] * 3, [-1] * 5, own[:2] + other]
    lens = [64, 32 + 33, 0, 40, 0, 32 + 20]
    many = torch.full((6, 5), -1, dtype=torch.int32)
    for r, row in enumerate(rows):
        many[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
    q = R.make_bf16((6, Hq, D), gen)
    attention = PagedAttention(6, Hq, Hkv, D, 80, fmt=fmt, n_unique_splits=2)
    out, lse = (x.double().cpu().numpy() for x in
                attention(q.cuda(), st, many.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()))

    def seen(x):
        a, b = x[:64], x[64:]
        return np.concatenate([a, a[:32], b, np.tile(a[16:32], (3, 1, 1))[:40], a[:32], b[:20]])

    _compare(out, lse, [seen(x) for x in held], lens, q, 1, attention.scale, fmt)
