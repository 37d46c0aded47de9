"""GPU parity of the paged private store (append with rotation, read back, attention, decode step), in
bf16 and 4-bit pages, against the plain reference in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu

INACTIVE = 0  # a request slot without a context


@pytest.fixture(autouse=True)
def clean_status():
    from paper_2511_06010_b200 import binding as M

    M.device_status()
    yield
    torch.cuda.synchronize()


def _store(fmt, n_pages, page, Hkv, D, gen, poison=False):
    """A store whose pages hold something everywhere: values that a test can recognise, or NaN."""
    from paper_2511_06010_b200.paged import PagedKvStore

    st = PagedKvStore.empty(n_pages, page, Hkv, D, fmt)
    if fmt == "bf16":
        for t in (st.k_pages, st.v_pages):
            t.fill_(float("nan")) if poison else t.copy_(R.make_bf16(t.shape, gen).cuda())
    else:
        st.pages4.copy_(torch.randint(0, 256, st.pages4.shape, generator=gen, dtype=torch.uint8).cuda())
        if poison:
            st.pages4[..., 16 * D:] = 0xFF  # every scale a NaN
        else:
            st.pages4[..., 16 * D + 1::2] = 0x38  # scales between 0.5 and 1
    return st


def _table(lens, page, gen, spare=2):
    need = [-(-int(n) // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen).tolist()
    table = torch.full((len(lens), max(max(need), 1) + spare), -1, dtype=torch.int32)
    for r, n in enumerate(need):
        for i in range(n):
            table[r, i] = order.pop()
    return table, n_pages


def _pages64(st):
    if st.fmt == "bf16":
        return R.to_f64(st.k_pages), R.to_f64(st.v_pages)
    return R.unpack(st.pages4)


# ---- append --------------------------------------------------------------------------------------
APPENDS = [
    # fmt, D, Hq, Hkv, page, rot, interleaved, new rows of each request, tokens before them
    (fmt, D, Hq, Hkv, page, rot, il, new, before)
    for fmt in ("bf16", "fp4")
    for D, Hq, Hkv, page, rot, il, new, before in (
        (128, 8, 2, 32, 128, False, [1] * 7, [0, 15, 16, 31, 32, 1, 100]),      # one token each
        (64, 6, 2, 16, 64, False, [1, 17, 0, 40, 2], [0, 3, 9, 15, 31]),          # ragged, one request without rows
        (128, 4, 4, 64, 64, True, [33, 1, 5], [0, 63, 130]),                      # half of the head, neighbouring pairs
        (64, 8, 1, 128, 16, False, [100], [0]),                                   # sixteen dimensions
        (128, 7, 1, 16, 0, False, [3, 19], [14, 0]),                              # no rotation
        (128, 24, 8, 32, 128, True, [2, 3], [31, 5]),
    )
]


@pytest.mark.parametrize("fmt,D,Hq,Hkv,page,rot,il,new,before", APPENDS)
def test_append_writes_the_rows_and_nothing_else(fmt, D, Hq, Hkv, page, rot, il, new, before):
    from paper_2511_06010_b200 import binding as M

    gen = torch.Generator().manual_seed(D + Hq + page)
    pad = 3  # rows behind the last request
    n = sum(new)
    lens = [a + b for a, b in zip(new, before)]
    table, n_pages = _table(lens, page, gen)
    st = _store(fmt, n_pages, page, Hkv, D, gen)
    qkv = R.make_bf16((n + pad, (Hq + 2 * Hkv) * D), gen)
    qkv[:, ::7] *= 8
    cuda = qkv.cuda()
    q, k, v = (cuda[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    cs = R.angles(4000, rot) if rot else None
    pos = torch.randint(0, 4000, (n + pad,), generator=gen, dtype=torch.int32)
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    q_out = torch.full((n + pad, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    if fmt == "bf16":
        before_k, before_v = st.k_pages.cpu().clone(), st.v_pages.cpu().clone()
    else:
        before_4 = st.pages4.cpu().numpy().copy()
    out = st.append(q, k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), pos.cuda() if rot else None,
                    cs.cuda() if rot else None, row_start=first.cuda(), interleaved=il, q_out=q_out)
    torch.cuda.synchronize()
    assert M.device_status() == 0 and out is q_out
    table_rows = cs.numpy()[pos.numpy()] if rot else np.zeros((n + pad, 0), np.float32)
    q32, k32, v32 = (t.float().cpu().numpy() for t in (q, k, v))
    rot_q, rot_k = R.rotate32(q32, table_rows, rot, il), R.rotate32(k32, table_rows, rot, il)
    # the operator's own rounding is followed bit for bit ...
    want_q = torch.from_numpy(rot_q[:n]).to(torch.bfloat16)
    assert torch.equal(q_out[:n].cpu(), want_q)
    assert (q_out[n:] == 7.0).all(), "padding rows of q_out were written"
    # ... and is the rotation: bf16 half a step, fp32 two products and a sum (3 roundings of 2^-24 each)
    exact = R.rotate64(q32, table_rows, rot, il)
    room = 3 * 2.0 ** -24 * 2 * np.abs(q32).max(-1, keepdims=True)
    assert (np.abs(R.to_f64(q_out[:n]) - exact[:n]) <= 2.0 ** -8 * np.abs(exact[:n]) + room[:n]).all()
    tokens = [(r, before[r] + i) for r in range(len(new)) for i in range(new[r])]
    if fmt == "bf16":
        for row, (r, t) in enumerate(tokens):
            before_k[table[r, t // page], t % page] = torch.from_numpy(rot_k[row]).to(torch.bfloat16)
            before_v[table[r, t // page], t % page] = torch.from_numpy(v32[row]).to(torch.bfloat16)
        assert torch.equal(st.k_pages.cpu(), before_k) and torch.equal(st.v_pages.cpu(), before_v)
    else:
        kc, ks = R.quantise32(rot_k)
        vc, vs = R.quantise32(v32)
        for row, (r, t) in enumerate(tokens):
            for h in range(Hkv):
                R.pack(before_4, table[r, t // page], t % page, h, kc[row, h], ks[row, h], vc[row, h], vs[row, h])
        assert np.array_equal(st.pages4.cpu().numpy(), before_4)
        # the values held are within half a code step (and the scale's rounding, 2^-11) of the exact ones
        kp, vp = R.unpack(st.pages4)
        exact_k = R.rotate64(k32, table_rows, rot, il)
        for got, ref in ((kp, exact_k), (vp, v32.astype(np.float64))):
            g = np.stack([got[table[r, t // page], t % page] for r, t in tokens]).reshape(n, Hkv, -1, 32)
            e = ref[:n].reshape(n, Hkv, -1, 32)
            s = np.abs(e).max(-1, keepdims=True) / 6
            u = np.abs(e) / s
            half_step = np.where(u < 2, 0.25, np.where(u < 4, 0.5, 1.0)) * s
            assert (np.abs(g - e) <= half_step * (1 + 2.0 ** -10) + 6 * s * 2.0 ** -10).all()
    # reading the rows back gives what is held; padding rows are left alone
    ko, vo = (torch.full((n + pad, Hkv, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st.gather(table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), n + pad, row_start=first.cuda(), k_out=ko, v_out=vo)
    kp, vp = _pages64(st)
    for got, pages in ((ko, kp), (vo, vp)):
        want = torch.from_numpy(np.stack([pages[table[r, t // page], t % page] for r, t in tokens])).to(torch.bfloat16)
        assert torch.equal(got[:n].cpu(), want) and (got[n:] == 5.0).all()
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_append_uniform_rows_inactive_requests_and_keys_only(fmt):
    """q_len rows a request without row_start: contexts shorter than q_len and empty ones are padding."""
    from paper_2511_06010_b200 import binding as M

    gen = torch.Generator().manual_seed(3)
    D, Hkv, page, T = 128, 2, 16, 3
    lens = [0, 2, 3, 17, 1, 64]
    table, n_pages = _table(lens, page, gen)
    st = _store(fmt, n_pages, page, Hkv, D, gen)
    k, v = R.make_bf16((len(lens) * T, Hkv, D), gen).cuda(), R.make_bf16((len(lens) * T, Hkv, D), gen).cuda()
    kb, vb = _pages64(st)
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    assert st.append(None, k, v, table.cuda(), length, q_len=T) is None
    kp, vp = _pages64(st)
    assert M.device_status() == 0
    deq = (lambda x: R.to_f64(x)) if fmt == "bf16" else (lambda x: R.nearest64(R.to_f64(x))[0])
    k64, v64 = deq(k), deq(v)
    for r, n in enumerate(lens):
        for i in range(T):
            t = n - T + i
            if t >= 0:
                kb[table[r, t // page], t % page] = k64[r * T + i]
                vb[table[r, t // page], t % page] = v64[r * T + i]
    assert np.array_equal(kp, kb) and np.array_equal(vp, vb)


def test_append_fp4_special_values():
    """Zeros, values below and above f16's range, infinities and NaN: their 32 dimensions alone are NaN."""
    from paper_2511_06010_b200 import binding as M

    gen = torch.Generator().manual_seed(4)
    D = 128
    k = R.make_bf16((6, 1, D), gen)
    k[0] = 0
    k[1, 0, :32] *= 1e-9   # scale rounds to zero
    k[1, 0, 32:64] *= 1e-6 # a denormal scale
    k[2, 0, 64:96] *= 1e5  # saturates at 6 * 10912
    k[3, 0, 5] = float("inf")
    k[4, 0, 40] = float("nan")
    k[5, 0, 100] = 3e38
    st = _store("fp4", 1, 16, 1, D, gen)
    table, length = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([6], dtype=torch.int32).cuda()
    st.append(None, k.cuda(), k.flip(0).contiguous().cuda(), table, length, row_start=torch.tensor([0, 6], dtype=torch.int32).cuda())
    kp, vp = R.unpack(st.pages4)
    assert M.device_status() == 0
    x = k.float().numpy()
    code, s = R.quantise32(x)
    with np.errstate(invalid="ignore"):
        want = R.E2M1_SIGNED[code] * np.repeat(s.astype(np.float64), 32, axis=-1)
    assert np.array_equal(kp[0, :6], want, equal_nan=True) and np.array_equal(vp[0, :6], want[::-1], equal_nan=True)
    assert np.isnan(want[3, 0, :32]).all() and np.isfinite(want[3, 0, 32:]).all() and np.isnan(want[4, 0, 32:64]).all()
    assert np.isfinite(want[5]).all() and np.abs(want[5]).max() == 6 * 10912.0


# ---- attention -----------------------------------------------------------------------------------
LENS = [0, 1, 15, 16, 17, 31, 33, 64, 127, 128, 129, 300, 2, 517, 1000]
ATTENTIONS = [
    (fmt, D, Hq, Hkv, page, T, splits)
    for fmt in ("bf16", "fp4")
    for D, Hq, Hkv, page, T, splits in (
        (128, 8, 2, 16, 1, 1), (128, 8, 1, 64, 1, 3), (128, 3, 3, 32, 1, 2), (128, 14, 2, 256, 1, 5),
        (64, 4, 1, 16, 1, 1), (64, 16, 2, 64, 1, 4), (128, 8, 4, 32, 4, 1), (128, 8, 2, 16, 4, 3),
        (128, 6, 2, 64, 5, 2), (128, 2, 2, 16, 16, 2), (64, 8, 2, 32, 3, 2),
    ) if fmt == "fp4" or D == 128 or T == 1
]


def _attention_case(fmt, D, Hq, Hkv, page, T, splits, lens, seed=1, poison=True, q_scale=1.0):
    """Contexts written through append into pages that hold NaN everywhere else; queries of T rows."""
    gen = torch.Generator().manual_seed(seed)
    table, n_pages = _table(lens, page, gen)
    st = _store(fmt, n_pages, page, Hkv, D, gen, poison=poison)
    n = sum(lens)
    k, v = R.make_bf16((max(n, 1), Hkv, D), gen), R.make_bf16((max(n, 1), Hkv, D), gen)
    k[..., ::9] *= 4
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    st.append(None, k.cuda(), v.cuda(), table.cuda(), length, row_start=first)
    q = R.make_bf16((len(lens) * T, Hq, D), gen, q_scale)
    return st, table, length, q


def _check(out, lse, st, table, lens, q, T, scale):
    kp, vp = _pages64(st)
    q64, out, lse = R.to_f64(q), R.to_f64(out), lse.double().cpu().numpy()
    for r, n in enumerate(lens):
        for i in range(T):
            m = max(0, n - (T - 1 - i))
            k, v = R.context(kp, vp, table[r].numpy(), m)
            o, l, o_tol, l_tol = R.attend(q64[r * T + i], k, v, scale, st.fmt)
            b = r * T + i
            assert np.isfinite(out[b]).all(), f"request {r} (length {n}), token {i}: not finite"
            worst = (np.abs(out[b] - o) - o_tol).max()
            assert worst <= 0, f"request {r} (length {n}), token {i}: {worst} beyond the bound"
            if m == 0:
                assert np.isneginf(lse[b]).all() and not out[b].any()
            else:
                assert (np.abs(lse[b] - l) <= l_tol).all(), f"request {r}, token {i}: lse {np.abs(lse[b] - l).max()}"


@pytest.mark.parametrize("fmt,D,Hq,Hkv,page,T,splits", ATTENTIONS)
def test_paged_attention_ragged(fmt, D, Hq, Hkv, page, T, splits):
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedAttention

    st, table, length, q = _attention_case(fmt, D, Hq, Hkv, page, T, splits, LENS)
    attention = PagedAttention(len(LENS) * T, Hq, Hkv, D, max(LENS), fmt=fmt, q_len=T, n_unique_splits=splits)
    attention.out.fill_(float("nan"))
    attention.lse.fill_(float("nan"))
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    torch.cuda.synchronize()
    assert M.device_status() == 0
    _check(out, lse, st, table, LENS, q, T, attention.scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("q_scale", [1e-6, 64.0, 3e4])
def test_paged_attention_small_and_large_queries(fmt, q_scale):
    """Queries far from 1: nearly uniform and nearly one-hot softmax."""
    from paper_2511_06010_b200.paged import PagedAttention

    lens = [1, 40, 333]
    st, table, length, q = _attention_case(fmt, 128, 8, 2, 32, 1, 2, lens, seed=5, q_scale=q_scale)
    attention = PagedAttention(len(lens), 8, 2, 128, max(lens), fmt=fmt, n_unique_splits=2)
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    _check(out, lse, st, table, lens, q, 1, attention.scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_nan_behind_a_query_tokens_context_stays_there(fmt):
    """Four query tokens a request, NaN and infinities in the keys and values of the last token: only
    the rows that see it are affected."""
    from paper_2511_06010_b200.paged import PagedAttention

    D, Hq, Hkv, T, page = 128, 4, 1, 4, 16
    lens = [4, 20, 33, 128]
    st, table, length, q = _attention_case(fmt, D, Hq, Hkv, page, T, 1, lens, seed=6)
    attention = PagedAttention(len(lens) * T, Hq, Hkv, D, 128, fmt=fmt, q_len=T, n_unique_splits=2)
    clean = [t.clone() for t in attention(q.cuda(), st, table.cuda(), length)]
    bad = R.make_bf16((len(lens), Hkv, D), torch.Generator().manual_seed(7))
    bad[:, :, 3::32] = float("nan")
    bad[:, :, 4::32] = float("inf")
    st.append(None, bad.cuda(), bad.cuda(), table.cuda(), length)  # over the last token of each
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    torch.cuda.synchronize()
    o, c = out.reshape(len(lens), T, Hq, D), clean[0].reshape(len(lens), T, Hq, D)
    assert torch.equal(o[:, :-1], c[:, :-1])
    assert torch.equal(lse.reshape(len(lens), T, Hq)[:, :-1], clean[1].reshape(len(lens), T, Hq)[:, :-1])
    assert torch.isnan(o[:, -1].float()).all() and torch.isnan(lse.reshape(len(lens), T, Hq)[:, -1]).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_pages_beyond_32_bit_offsets(fmt):
    """A pool whose last pages lie behind 2^32 elements (bf16) and 2^32 bytes (4-bit)."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedAttention, PagedKvStore

    D, Hkv, page = 128, 8, 1024
    token = Hkv * D if fmt == "bf16" else Hkv * 18 * D // 16
    n_pages = (1 << 32) // (token * page) + 3
    st = PagedKvStore.empty(n_pages, page, Hkv, D, fmt)
    lens = [1500, 700]
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, -1]], dtype=torch.int32)
    gen = torch.Generator().manual_seed(8)
    k, v = R.make_bf16((2200, Hkv, D), gen), R.make_bf16((2200, Hkv, D), gen)
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    first = torch.tensor([0, 1500, 2200], dtype=torch.int32).cuda()
    st.append(None, k.cuda(), v.cuda(), table.cuda(), length, row_start=first)
    q = R.make_bf16((2, 16, D), gen)
    attention = PagedAttention(2, 16, Hkv, D, 1500, fmt=fmt)
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    ko, vo = st.gather(table.cuda(), length, 2200, row_start=first)
    assert M.device_status() == 0
    k64, v64 = R.to_f64(ko), R.to_f64(vo)
    if fmt == "bf16":
        assert torch.equal(ko.cpu(), k) and torch.equal(vo.cpu(), v)
    else:
        kq, ks = R.quantise32(k.float().numpy())
        k64 = R.E2M1_SIGNED[kq] * np.repeat(ks.astype(np.float64), 32, axis=-1)
        vq, vs = R.quantise32(v.float().numpy())
        v64 = R.E2M1_SIGNED[vq] * np.repeat(vs.astype(np.float64), 32, axis=-1)
        assert torch.equal(ko.cpu(), torch.from_numpy(k64).to(torch.bfloat16))
    for r, (a, b) in enumerate(((0, 1500), (1500, 2200))):
        o, l, o_tol, l_tol = R.attend(R.to_f64(q[r]), k64[a:b], v64[a:b], attention.scale, fmt)
        assert (np.abs(R.to_f64(out[r]) - o) <= o_tol).all()
        assert (np.abs(lse[r].double().cpu().numpy() - l) <= l_tol).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [5, 6, 33, 64])
def test_many_splits_of_few_and_of_many_rows(fmt, splits):
    """The merge's two forms (a warp or four a row), splits without tokens among them."""
    from paper_2511_06010_b200.paged import PagedAttention

    for R_, Hkv, lens in ((1, 2, [3000]), (3, 1, [70, 0, 2111]), (300, 2, [1 + 3 * i for i in range(300)])):
        Hq = 8 * Hkv
        st, table, length, q = _attention_case(fmt, 128, Hq, Hkv, 64, 1, splits, lens, seed=splits)
        attention = PagedAttention(R_, Hq, Hkv, 128, max(lens), fmt=fmt, n_unique_splits=splits)
        attention.out.fill_(float("nan"))
        out, lse = attention(q.cuda(), st, table.cuda(), length)
        keep = range(0, R_, max(1, R_ // 7))  # the reference of a few requests
        sub = torch.tensor(list(keep))
        _check(out[sub], lse[sub], st, table[sub], [lens[i] for i in keep], q[sub], 1, attention.scale)
        assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("requests", [2, 7, 8, 9, 127, 128, 129])
@pytest.mark.parametrize("kind", ["equal", "ties", "ragged", "one longer"])
def test_order_of_the_requests(fmt, requests, kind):
    """More CTAs than SMs: requests are taken longest first, up to 128 of them; every one exactly once."""
    from paper_2511_06010_b200.paged import PagedAttention

    rng = np.random.default_rng(requests)
    lens = {"equal": [35] * requests, "ties": list(16 * rng.integers(0, 5, requests)), "ragged": list(rng.integers(0, 300, requests)),
            "one longer": [20] * (requests - 1) + [21]}[kind]
    lens = [int(n) for n in lens]
    Hq = Hkv = 4
    splits = 160 // (requests * Hkv) + 1  # more than 148 CTAs
    st, table, length, q = _attention_case(fmt, 128, Hq, Hkv, 16, 1, splits, lens, seed=requests)
    attention = PagedAttention(requests, Hq, Hkv, 128, max(lens), fmt=fmt, n_unique_splits=splits)
    attention.out.fill_(float("nan"))
    attention.lse.fill_(float("nan"))
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    _check(out, lse, st, table, lens, q, 1, attention.scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_bad_lengths_leave_the_order_whole(fmt):
    """A length out of range is reported; every other request still has its own result."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedAttention

    lens = [50 + 3 * (i % 11) for i in range(40)]
    bad = {3: 2**31 - 1, 4: -1, 17: -2**31, 18: 2**31 - 1, 39: 1000}
    st, table, length, q = _attention_case(fmt, 128, 4, 4, 16, 1, 1, lens, poison=False)
    for r, n in bad.items():
        length[r] = n
    attention = PagedAttention(40, 4, 4, 128, 100, fmt=fmt, n_unique_splits=1)
    attention.out.fill_(float("nan"))
    out, lse = attention(q.cuda(), st, table.cuda(), length)
    assert M.device_status() == M.ERR_INVALID_ARG
    good = [r for r in range(40) if r not in bad]
    _check(out[good], lse[good], st, table[good], [lens[r] for r in good], q[good], 1, attention.scale)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_two_streams_at_once(fmt):
    """Two attentions with scratch of their own on two streams, and appends to other requests of the same
    pool beside them: equal to one after the other."""
    from paper_2511_06010_b200.paged import PagedAttention

    lens = [900, 33, 1500, 64]
    st, table, length, q = _attention_case(fmt, 128, 16, 2, 32, 1, 3, [n + 40 for n in lens], seed=21)
    table, q = table.cuda(), q.cuda()
    short = torch.tensor(lens, dtype=torch.int32).cuda()  # tokens behind it are written while it is read
    pair = [PagedAttention(4, 16, 2, 128, 1600, fmt=fmt, n_unique_splits=3) for _ in range(2)]
    want = [t.clone() for t in pair[0](q, st, table, short)]
    rows = R.make_bf16((160, 2, 128), torch.Generator().manual_seed(22)).cuda()
    grown = short + 40
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, attention in zip(streams, pair):
            with torch.cuda.stream(stream):
                attention.out.fill_(0)
                attention(q, st, table, short)
        st.append(None, rows, rows, table, grown, q_len=40, stream=streams[2])
        torch.cuda.synchronize()
        for attention in pair:
            assert torch.equal(attention.out, want[0]) and torch.equal(attention.lse, want[1])


# ---- a run of the operators together ---------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_prompts_then_decode_steps(fmt):
    """Prompts enter, then every step appends a token a request and attends: the page book grows the
    contexts, one request leaves and another takes its pages."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedAttention, PagedKvStore, PageTable

    D, Hq, Hkv, page, rot = 128, 8, 2, 16, 128
    gen = torch.Generator().manual_seed(9)
    st = PagedKvStore.empty(24, page, Hkv, D, fmt)
    book = PageTable(24, page, 3, 12)
    cs = R.angles(500, rot).cuda()
    attention = PagedAttention(3, Hq, Hkv, D, 190, fmt=fmt, n_unique_splits=2)
    history = [[np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))] for _ in range(3)]
    lens = [0, 0, 0]

    def held(x):
        return R.held32(x) if fmt == "fp4" else R.to_f64(torch.from_numpy(x).to(torch.bfloat16))

    def append(new):
        n = sum(new)
        q, k, v = (R.make_bf16((n, h, D), gen) for h in (Hq, Hkv, Hkv))
        pos = np.concatenate([np.arange(l, l + m) for l, m in zip(lens, new)]).astype(np.int32)
        for r, m in enumerate(new):
            lens[r] += m
            book.reserve(r, lens[r])
        length = torch.tensor(lens, dtype=torch.int32).cuda()
        first = None if new == [1] * 3 else torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        q_rot = st.append(q.cuda(), k.cuda(), v.cuda(), book.table(), length, torch.from_numpy(pos).cuda(), cs, row_start=first)
        rows = cs.cpu().numpy()[pos]
        k32, at = R.rotate32(k.float().numpy(), rows, rot, False), 0
        for r, m in enumerate(new):
            history[r][0] = np.concatenate([history[r][0], held(k32[at:at + m])])
            history[r][1] = np.concatenate([history[r][1], held(v[at:at + m].float().numpy())])
            at += m
        return q_rot, length

    append([37, 5, 80])
    for step in range(20):
        if step == 12:  # request 2 leaves, another prompt takes its slot
            book.release(2)
            lens[2], history[2] = 0, [np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))]
            append([0, 0, 131])
        q_rot, length = append([1, 1, 1])
        out, lse = attention(q_rot, st, book.table(), length)
        if step % 6 and step != 19:
            continue
        for r in range(3):
            o, l, o_tol, l_tol = R.attend(R.to_f64(q_rot[r]), *history[r], attention.scale, fmt)
            assert (np.abs(R.to_f64(out[r]) - o) <= o_tol).all(), (step, r)
            assert (np.abs(lse[r].double().cpu().numpy() - l) <= l_tol).all()
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_captured_decode_step_replays_with_new_lengths(fmt):
    """Append and attention in one CUDA graph on a side stream, replayed as the context grows; equal to
    the eager calls bit for bit."""
    from paper_2511_06010_b200.paged import PagedAttention

    D, Hq, Hkv, page, B = 128, 8, 2, 16, 5
    gen = torch.Generator().manual_seed(10)
    lens = [0, 3, 15, 31, 70]
    table, n_pages = _table([n + 6 for n in lens], page, gen)
    st, twin = _store(fmt, n_pages, page, Hkv, D, gen), None
    twin = type(st)(k_pages=st.k_pages.clone(), v_pages=st.v_pages.clone()) if fmt == "bf16" else type(st)(pages4=st.pages4.clone())
    cs = R.angles(200, D).cuda()
    q, k, v = (torch.empty(B, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    length, pos = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    q_rot, table = torch.empty_like(q), table.cuda()
    one, two = (PagedAttention(B, Hq, Hkv, D, 80, fmt=fmt, n_unique_splits=3) for _ in range(2))
    side = torch.cuda.Stream()

    def step(store, attention):
        store.append(q, k, v, table, length, pos, cs, q_out=q_rot)
        return attention(q_rot, store, table, length)

    def inputs(i):
        for t in (q, k, v):
            t.copy_(R.make_bf16(t.shape, torch.Generator().manual_seed(100 + i)))
        length.copy_(torch.tensor([n + i + 1 for n in lens], dtype=torch.int32))
        pos.copy_(length - 1)

    inputs(0)
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(st, one)  # warm-up
        with torch.cuda.graph(graph, stream=side):
            step(st, one)
    torch.cuda.synchronize()
    for i in range(5):
        inputs(i)
        graph.replay()
        want = step(twin, two)
        torch.cuda.synchronize()
        assert torch.equal(one.out, want[0]) and torch.equal(one.lse, want[1]), i
    a, b = (s.pages4 if fmt == "fp4" else s.k_pages for s in (st, twin))
    assert torch.equal(a, b)


# ---- the whole decode step -------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("shared", ["bf16", "fp8"])
@pytest.mark.parametrize("mode", ["one stream", "two streams", "two streams, long", "dense"])
def test_decode_step_with_a_paged_store(fmt, shared, mode):
    from oracle import oracle as O
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200 import workloads as W
    from paper_2511_06010_b200.engine import MoskaLayer
    from tests import parity_utils as PU

    lens = [300, 1, 0, 1000, 64, 17, 129, 511, 20, 77, 5, 900, 33, 640, 256, 4]
    dense = mode == "dense"
    w = W.scaled(W.CONFIGS[1], B=16, C=8, k=8 if dense else 4, L=256, unique_len=0)
    st, table, length, _ = _attention_case(fmt, w.D, w.Hq, w.Hkv, 64, 1, 2, lens, seed=11)
    sh = W.make_shared_store(w, "cuda")
    sf8 = W.quantize_shared_store_fp8(sh) if shared == "fp8" else None
    q = W.make_queries(w, sh, 0, "cuda")
    layer = MoskaLayer(w.B, w.Hq, w.Hkv, w.D, w.C, w.L, w.k, 1000, dense=dense, dense_slots=w.C if dense else None,
                       paged_fmt=fmt)
    layer.build_summaries(sh.k_shared)
    with pytest.raises(ValueError):
        layer.step_paged(q, sh.k_shared, sh.v_shared, st, table[:-1].cuda(), length[:-1])
    out = layer.step_paged(q, sh.k_shared, sh.v_shared, st, table.cuda(), length, two_streams=mode.startswith("two"),
                           unique_tokens=1 << 26 if "long" in mode else 0, sf8=sf8)
    torch.cuda.synchronize()
    assert M.device_status() == 0
    topk = np.tile(np.arange(w.C, dtype=np.int32), (w.B, w.Hkv, 1)) if dense else layer.topk_idx.cpu().numpy()
    if sf8 is None:
        o_sh, l_sh = O.shared_partials(q.cpu(), sh.k_shared.cpu(), sh.v_shared.cpu(), topk, layer.scale)
    else:
        o_sh, l_sh = O.shared_partials_fp8(q.cpu(), sf8.k8.cpu(), sf8.v8.cpu(), sf8.k_scale.cpu(), sf8.v_scale.cpu(), topk, layer.scale)
    kp, vp = _pages64(st)
    o_u, l_u = np.zeros((w.B, w.Hq, w.D)), np.zeros((w.B, w.Hq))
    for b, n in enumerate(lens):
        o_u[b], l_u[b], _, _ = R.attend(R.to_f64(q[b]), *R.context(kp, vp, table[b].numpy(), n), layer.scale, fmt)
    ref_o, ref_l = O.merge(np.concatenate([o_sh, o_u[:, :, None]], axis=2), np.concatenate([l_sh, l_u[:, :, None]], axis=2))
    PU.check_attention(out.float().cpu().numpy(), ref_o, f"paged step, {fmt} pages, {shared} shared, {mode}")
    PU.check_lse(layer.lse_out.cpu().numpy(), ref_l, "paged step lse")


# ---- what only the device can find -----------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_bad_pages_lengths_and_positions_are_reported_and_write_nothing(fmt):
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedAttention

    D, Hq, Hkv, page = 128, 4, 1, 16
    gen = torch.Generator().manual_seed(12)
    st = _store(fmt, 4, page, Hkv, D, gen)
    pools = [st.k_pages, st.v_pages] if fmt == "bf16" else [st.pages4]
    before = [p.clone() for p in pools]
    rows = R.make_bf16((1, Hkv, D), gen).cuda()
    q = R.make_bf16((1, Hq, D), gen).cuda()
    attention = PagedAttention(1, Hq, Hkv, D, 32, fmt=fmt, n_unique_splits=1)
    cs = R.angles(8, D).cuda()
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731

    for entry in (4, -1, 2**31 - 1, -2**31):
        table = ints(0, entry).reshape(1, 2)
        st.append(None, rows, rows, table, ints(17))
        assert M.device_status() == M.ERR_INVALID_ARG
        attention(q, st, table, ints(20))
        assert M.device_status() == M.ERR_INVALID_ARG
        st.gather(table, ints(17), 1)
        assert M.device_status() == M.ERR_INVALID_ARG
        attention(q, st, table, ints(16))  # the bad entry is behind the context
        assert M.device_status() == 0
    table = ints(0, 1).reshape(1, 2)
    for bad in (33, 2**31 - 1, -1, -2**31):
        attention(q, st, table, ints(bad))
        assert M.device_status() == M.ERR_INVALID_ARG
        st.gather(table, ints(bad), 1)
        assert M.device_status() == M.ERR_INVALID_ARG
    st.append(None, rows, rows, table, ints(-5))
    assert M.device_status() == M.ERR_INVALID_ARG
    for p in (8, -1):
        out = torch.full((1, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda")
        st.append(q, rows, rows, table, ints(3), ints(p), cs, q_out=out)
        assert M.device_status() == M.ERR_INVALID_ARG and (out == 3.0).all()
    for n in (33, 2**31 - 1):  # longer than the table row
        st.append(None, rows, rows, table, ints(n))
        assert M.device_status() == M.ERR_INVALID_ARG
    assert all(torch.equal(a, b) for a, b in zip(pools, before))
    # rows that no request has are padding
    st.append(None, rows, rows, table, ints(3), row_start=ints(1, 1))
    assert M.device_status() == 0 and all(torch.equal(a, b) for a, b in zip(pools, before))
