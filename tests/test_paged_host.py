"""Paged private store, without a GPU: refusals of the C ABI, the Python checks, the page book, and the
reference's own consistency."""
import ctypes

import numpy as np
import pytest
import torch

from tests import paged_reference as R

A = 0x10000  # an address aligned to everything asked for; never dereferenced: each call is refused


@pytest.fixture(scope="module")
def M():
    from paper_2511_06010_b200 import build

    build.build()
    from paper_2511_06010_b200 import binding

    return binding


def kv(M, **over):
    f = dict(fmt=M.KV_BF16, page_size=64, n_pages=10, max_pages=4, k_pages=A, v_pages=A, page_table=A, kv_len=A)
    f.update(over)
    return M.paged_kv(**f)


def refused(M, status, call, text=""):
    with pytest.raises(M.MoskaError) as e:
        call()
    assert e.value.status == status and text in M.last_error(), M.last_error()


BAD_STORES = [
    (dict(fmt=2), -1, "format"), (dict(fmt=-1), -1, "format"), (dict(page_size=8), -1, "page_size"),
    (dict(page_size=48), -1, "page_size"), (dict(page_size=65536), -1, "page_size"), (dict(page_size=0), -1, "page_size"),
    (dict(n_pages=0), -1, "n_pages"), (dict(max_pages=0), -1, "max_pages"),
    (dict(page_size=32768, max_pages=1 << 16), -2, "2^30"), (dict(k_pages=None), -1, "NULL"),
    (dict(v_pages=None), -1, "NULL"), (dict(k_pages=A + 8), -1, "aligned"), (dict(page_table=A + 2), -1, "aligned"),
    (dict(kv_len=None), -1, "NULL"), (dict(page_table=None), -1, "NULL"),
]


@pytest.mark.parametrize("over,status,text", BAD_STORES)
def test_bad_stores_are_refused_by_every_call(M, over, status, text):
    s = M.shape(4, 8, 2, 128, 4, 128, 2)
    bad = kv(M, **over)
    refused(M, status, lambda: M.unique_attn_paged(A, bad, A, A, 1.0, s, stream=0), text)
    refused(M, status, lambda: M.paged_attn(A, bad, A, A, 1.0, s, None, stream=0), text)
    refused(M, status, lambda: M.kv_gather_paged(None, 4, A, A, bad, s, stream=0), text)
    refused(M, status, lambda: M.kv_append_paged(A, 1024, A, 256, A, 256, A, A, 10, 128, 0, None, 4, A, bad, s, stream=0), text)
    refused(M, status, lambda: M.decode_step_paged(A, A, A, A, None, None, bad, A, A, A, A, A, A, A, 1.0, s, None, stream=0), text)


def test_pages_beyond_32_bit_arithmetic_are_refused(M):
    wide = M.shape(4, 512, 512, 128, 4, 128, 2)
    refused(M, M.ERR_UNSUPPORTED, lambda: M.paged_attn(A, kv(M, page_size=32768, max_pages=1), A, A, 1.0, wide, None, stream=0), "2^30")


def test_calls_on_the_cpu_are_refused():
    from paper_2511_06010_b200.paged import PagedAttention, PagedKvStore

    st = PagedKvStore.empty(2, 16, 1, 64, device="cpu")
    table, length = torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    k = torch.zeros(1, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: st.append(None, k, k, table, length), lambda: st.gather(table, length, 1),
                 lambda: PagedAttention(1, 1, 1, 64, 1, device="cpu")(k, st, table, length)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_bad_append_arguments_are_refused(M):
    good = dict(q=A, qs=1024, k=A, ks=256, v=A, vs=256, pos=A, cs=A, n=10, rot=128, il=0, rows=None, req=4, out=2 * A)

    def call(D=128, shape=None, **over):
        a = dict(good, **over)
        s = M.shape(**dict(dict(B=4, Hq=8, Hkv=2, D=D, C=1, L=128, k=1), **(shape or {})))
        return lambda: M.kv_append_paged(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["pos"], a["cs"], a["n"], a["rot"],
                                         a["il"], a["rows"], a["req"], a["out"], kv(M), s, stream=0)

    for over in (dict(q=None), dict(out=None), dict(q=A + 2), dict(out=A + 8), dict(qs=1023), dict(qs=1016), dict(ks=248),
                 dict(vs=255), dict(k=None), dict(v=A + 4), dict(rot=8), dict(rot=144), dict(rot=-16), dict(pos=None),
                 dict(cs=A + 8), dict(n=0), dict(req=3), dict(req=0), dict(rows=A + 2)):
        refused(M, M.ERR_INVALID_ARG, call(**over))
    for out in (A + 0x1000, A - 0x1000, A):  # four rows of 2 KB each
        refused(M, M.ERR_INVALID_ARG, call(out=out), "overlaps")
    refused(M, M.ERR_UNSUPPORTED, call(shape=dict(D=96)))
    refused(M, M.ERR_UNSUPPORTED, call(shape=dict(Hq=64)))
    refused(M, M.ERR_INVALID_ARG, call(shape=dict(Hq=9)))
    refused(M, M.ERR_INVALID_ARG, call(shape=dict(q_len=3)))
    refused(M, M.ERR_INVALID_ARG, call(shape=dict(B=-1)))


def test_bad_attention_arguments_are_refused(M):
    s = M.shape(4, 8, 2, 128, 4, 128, 2)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        refused(M, M.ERR_INVALID_ARG, lambda: M.unique_attn_paged(A, kv(M), A, A, scale, s, stream=0), "softmax_scale")
        refused(M, M.ERR_INVALID_ARG, lambda: M.paged_attn(A, kv(M), A, A, scale, s, None, stream=0), "softmax_scale")
    refused(M, M.ERR_INVALID_ARG, lambda: M.unique_attn_paged(A + 2, kv(M), A, A, 1.0, s, stream=0), "aligned")
    refused(M, M.ERR_INVALID_ARG, lambda: M.unique_attn_paged(A, kv(M), A + 4, A, 1.0, s, stream=0), "aligned")
    refused(M, M.ERR_INVALID_ARG, lambda: M.paged_attn(A, kv(M), A + 2, A, 1.0, s, None, stream=0), "aligned")
    refused(M, M.ERR_INVALID_ARG, lambda: M.paged_attn(A, kv(M), A, A + 2, 1.0, s, None, stream=0), "aligned")
    # several query tokens: more than 16 rows a KV head, and the smaller head dimension in bf16
    for fmt in (M.KV_BF16, M.KV_FP4):
        wide = M.shape(8, 32, 4, 128, 4, 128, 2, q_len=4)
        refused(M, M.ERR_UNSUPPORTED, lambda: M.paged_attn(A, kv(M, fmt=fmt), A, A, 1.0, wide, None, stream=0), "q_len")
    small = M.shape(8, 8, 2, 64, 4, 128, 2, q_len=4)
    refused(M, M.ERR_UNSUPPORTED, lambda: M.paged_attn(A, kv(M), A, A, 1.0, small, None, stream=0), "q_len")
    # two splits and more need a workspace
    split = M.shape(4, 8, 2, 128, 4, 128, 2, n_unique_splits=3)
    need = M.paged_attn_workspace_bytes(split)
    assert need >= 4 * 8 * 3 * (128 + 1) * 4
    refused(M, M.ERR_WORKSPACE, lambda: M.paged_attn(A, kv(M), A, A, 1.0, split, None, stream=0))
    ws = type("Ws", (), {"numel": lambda self: need - 1, "element_size": lambda self: 1, "is_contiguous": lambda self: True,
                         "data_ptr": lambda self: A})()
    refused(M, M.ERR_WORKSPACE, lambda: M.paged_attn(A, kv(M), A, A, 1.0, split, ws, stream=0))
    refused(M, M.ERR_INVALID_ARG, lambda: M.decode_step_paged(A, A, A, A, A, None, kv(M), A, A, A, A, A, A, A, 1.0, s, None,
                                                              stream=0), "together")
    assert M.paged_attn_workspace_bytes(s) == 0


def test_pool_sizes_and_splits(M):
    assert M.paged_pool_bytes(M.KV_BF16, 3, 32, 8, 128) == 3 * 32 * 8 * 128 * 2
    assert M.paged_pool_bytes(M.KV_FP4, 3, 32, 8, 128) == 3 * 2 * 8 * 18 * 128
    assert M.paged_pool_bytes(M.KV_FP4, 100000, 1024, 8, 128) == 100000 * 64 * 8 * 18 * 128  # beyond 32 bits
    for bad in ((2, 3, 32, 8, 128), (0, 0, 32, 8, 128), (0, 3, 24, 8, 128), (0, 3, 32, 0, 128), (0, 3, 32, 8, 96)):
        assert M.paged_pool_bytes(*bad) == 0
    for fmt in (M.KV_BF16, M.KV_FP4):
        assert M.default_paged_splits(fmt, 0, 8, 128, 100) == 1 and M.default_paged_splits(fmt, 4, 8, 128, 0) == 1
        assert M.default_paged_splits(fmt, 1000, 8, 128, 500) == 1 and M.default_paged_splits(fmt, 1, 8, 64, 256) == 1
        assert 16 <= M.default_paged_splits(fmt, 1, 8, 128, 8191) <= 32 and M.default_paged_splits(fmt, 1, 1, 128, 1 << 30) == 64
    assert ctypes.sizeof(M.MoskaPagedKv) == 4 * 4 + 4 * 8


def test_store_checks_its_tensors():
    from paper_2511_06010_b200.paged import PagedKvStore

    st = PagedKvStore.empty(4, 32, 2, 128, "fp4", device="cpu")
    assert st.pages4.shape == (4, 2, 2, 18 * 128) and (st.page_size, st.D, st.Hkv) == (32, 128, 2)
    st = PagedKvStore.empty(4, 32, 2, 64, device="cpu")
    assert st.fmt == "bf16" and st.k_pages.shape == (4, 32, 2, 64)
    table, length = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    assert st.kv(table, length).max_pages == 2
    for t, l in ((table.long(), length), (table, length.long()), (table, length[:2]), (table.t(), length)):
        with pytest.raises(ValueError):
            st.kv(t, l)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    for bad in (dict(k=k.float()), dict(k=k[:, :1]), dict(v=k[..., ::2]), dict(q=k.transpose(0, 1)), dict(k=k[:2], v=k[:2]),
                dict(cos_sin=torch.zeros(4, 64)), dict(q_out=k), dict(row_start=torch.zeros(3, dtype=torch.int32))):
        a = dict(dict(q=None, k=k, v=k), **bad)
        with pytest.raises(ValueError):
            st.append(a.pop("q"), a.pop("k"), a.pop("v"), table, length, **a)
    with pytest.raises(ValueError):
        PagedKvStore.empty(4, 24, 2, 64, device="cpu")
    with pytest.raises(ValueError):
        PagedKvStore.empty(4, 32, 2, 64, "fp8", device="cpu")
    with pytest.raises(ValueError):
        PagedKvStore(k_pages=st.k_pages)


def test_page_table_book():
    from paper_2511_06010_b200.paged import PageTable

    t = PageTable(n_pages=6, page_size=16, slots=3, max_pages=4, device="cpu")
    t.reserve(0, 17)
    t.reserve(1, 16)
    t.reserve(1, 5)  # holds enough already
    held = t.table().numpy().copy()
    assert (held[0, :2] >= 0).all() and held[0, 2] == -1 and held[1, 0] >= 0 and (held[2] == -1).all()
    assert len(set(held[held >= 0].tolist())) == 3
    with pytest.raises(RuntimeError):
        t.reserve(2, 64)  # four pages, three left: nothing is taken
    assert len(t.free) == 3 and (t.table().numpy() == held).all()
    with pytest.raises(ValueError):
        t.reserve(2, 65)
    t.release(0)
    t.reserve(2, 64)
    now = t.table().numpy()
    assert (now[0] == -1).all() and len(set(now[now >= 0].tolist())) == 5


def test_reference_blocks_round_trip():
    """Every (token, dimension) has a nibble and every (token, group) a scale of its own in a block, and
    both quantisers agree, ties included."""
    for D in (64, 128):
        kb, vb, ks, vs, sh = R.byte_map(D)
        where = np.concatenate([(2 * kb + sh // 4).ravel(), (2 * vb + sh // 4).ravel()])
        assert sorted(where.tolist()) == list(range(2 * 16 * D))
        scales = set(ks.ravel().tolist()) | set(vs.ravel().tolist())
        assert scales == set(range(16 * D, 18 * D, 2))
        rng = np.random.default_rng(D)
        x = rng.standard_normal((40, D)).astype(np.float32)
        x[0] = 0.0
        x[1] = np.tile(np.array([6, 0.25, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5, -5, 4.99, 5.01, 0.5, -6, 1, 2], np.float32), D // 16)
        code, s = R.quantise32(x)
        y = R.E2M1_SIGNED[code] * np.repeat(s.astype(np.float64), 32, axis=-1)
        want, _ = R.nearest64(x)
        assert np.array_equal(y, want)
        pool = np.zeros((2, 1, 2, 18 * D), np.uint8)
        for slot in range(32):
            R.pack(pool, 1, slot, 0, code[slot], s[slot], code[39 - slot], s[39 - slot])
        k, v = R.unpack(torch.from_numpy(pool))
        assert np.array_equal(k[1, :, 0], y[:32]) and np.array_equal(v[1, :, 0], y[39:7:-1]) and not k[0].any()
