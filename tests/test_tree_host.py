"""Speculative decoding without a GPU: refusals of the C ABI and of the Python calls, and the reference's own
consistency."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import tree_reference as TR

A = 0x10000  # an address aligned to everything asked for; never dereferenced: each call is refused
FAR = [i << 36 for i in range(1, 16)]


@pytest.fixture(scope="module")
def M():
    from paper_2511_06010_b200 import build

    build.build()
    from paper_2511_06010_b200 import binding

    return binding


def kv(M, **over):
    f = dict(fmt=M.KV_BF16, page_size=64, n_pages=10, max_pages=4, k_pages=FAR[0], v_pages=FAR[1], page_table=FAR[2], kv_len=FAR[3])
    f.update(over)
    return M.paged_kv(**f)


def refused(M, status, call, text=""):
    with pytest.raises(M.MoskaError) as e:
        call()
    assert e.value.status == status and text in M.last_error(), M.last_error()


def attn(M, **over):
    a = dict(q=A, kv=kv(M), parents=A, row_start=None, n=4, out=A, lse=A, scale=1.0, s=M.shape(32, 8, 2, 128, 1, 128, 1, q_len=8), ws=None)
    a.update(over)
    return lambda: M.tree_attn(a["q"], a["kv"], a["parents"], a["row_start"], a["n"], a["out"], a["lse"], a["scale"], a["s"], a["ws"],
                               stream=0)


def test_refusals_of_tree_attention(M):
    sh = lambda **k: M.shape(*(dict(dict(B=32, Hq=8, Hkv=2, D=128, C=1, L=128, k=1), **{x: y for x, y in k.items() if x != "q_len" and x != "s"}).values()),  # noqa: E731
                             n_unique_splits=k.get("s", 1), q_len=k.get("q_len", 8))
    for over, status, text in (
            (dict(s=sh(q_len=65)), -1, "nodes"), (dict(s=sh(q_len=-1)), -1, "nodes"), (dict(s=sh(q_len=7)), -1, "must be B"),
            (dict(n=5), -1, "must be B"), (dict(n=0), -1, "n_requests"), (dict(n=-1), -1, "n_requests"), (dict(q=None), -1, "q is NULL"),
            (dict(q=A + 2), -1, "aligned"), (dict(out=None), -1, "out is NULL"), (dict(out=A + 8), -1, "aligned"),
            (dict(lse=A + 2), -1, "aligned"), (dict(parents=A + 1), -1, "parents"), (dict(row_start=A + 2), -1, "row_start"),
            (dict(scale=0.0), -1, "softmax_scale"), (dict(scale=float("nan")), -1, "softmax_scale"),
            (dict(scale=float("inf")), -1, "softmax_scale"), (dict(s=sh(s=0)), -1, "n_unique_splits"), (dict(s=sh(s=2)), -3, "workspace"),
            (dict(s=sh(Hq=18)), -2, "G ="), (dict(s=sh(D=96)), -2, "D ="), (dict(s=sh(Hq=9)), -1, "multiple"),
            (dict(kv=kv(M, page_size=24)), -1, "page_size"), (dict(kv=kv(M, fmt=3)), -1, "format"),
            (dict(kv=kv(M, kv_len=None)), -1, "NULL")):
        refused(M, status, attn(M, **over), text)


def test_refusals_of_the_step_over_trees(M):
    s = M.shape(32, 8, 2, 128, 4, 128, 2, q_len=8)
    step = lambda **k: lambda: M.decode_step_tree(A, A, A, A, k.get("ks"), None, k.get("kv", kv(M)), k.get("up", A), A, A, A, A, A, A, A,  # noqa: E731
                                                  k.get("scale", 1.0), k.get("s", s), None, stream=0)
    refused(M, -1, step(s=M.shape(66, 8, 2, 128, 4, 128, 2, q_len=66)), "nodes")
    refused(M, -1, step(ks=A), "together")
    refused(M, -1, step(scale=-1.0), "softmax_scale")
    refused(M, -1, step(up=A + 2), "parents")
    refused(M, -1, step(kv=kv(M, n_pages=0)), "n_pages")
    part = lambda **k: lambda: M.unique_attn_tree(k.get("q", A), kv(M), A, k.get("o", A), k.get("l", A), k.get("scale", 1.0), k.get("s", s), stream=0)  # noqa: E731
    refused(M, -1, part(s=M.shape(66, 8, 2, 128, 4, 128, 2, q_len=66)), "nodes")
    refused(M, -1, part(q=None), "q is NULL")
    refused(M, -1, part(o=A + 4), "o_part")
    refused(M, -1, part(l=None), "lse_part")
    refused(M, -1, part(scale=0.0), "softmax_scale")


def test_refusals_of_verification(M):
    good = dict(t=FAR[0], ts=100, d=FAR[1], ds=100, type=0, V=100, tokens=FAR[2], parents=FAR[3], u=FAR[4], un=FAR[5], rs=None, n=4,
                nodes=8, B=32, path=FAR[6], n_path=FAR[7], nxt=FAR[8])

    def call(**over):
        a = dict(good, **over)
        return lambda: M.verify_tree(a["t"], a["ts"], a["d"], a["ds"], a["type"], a["V"], a["tokens"], a["parents"], a["u"], a["un"],
                                     a["rs"], a["n"], a["nodes"], a["B"], a["path"], a["n_path"], a["nxt"], stream=0)

    for over, text in ((dict(type=2), "prob_type"), (dict(V=0), "V ="), (dict(V=2**30 + 1), "V ="), (dict(nodes=65), "nodes"),
                       (dict(nodes=-1), "nodes"), (dict(n=3), "must be B"), (dict(n=0), "n_requests"), (dict(t=None), "target_probs is NULL"),
                       (dict(t=A + 2), "aligned"), (dict(d=A + 1, type=1), "draft_probs"), (dict(ts=99), "hold a row"),
                       (dict(ds=99), "hold a row"), (dict(tokens=None), "tokens"), (dict(parents=None), "parents"), (dict(u=None), "u_accept"),
                       (dict(un=None), "u_next"), (dict(path=None), "path"), (dict(n_path=None), "n_path"), (dict(nxt=A + 2), "next_token"),
                       (dict(rs=A + 1), "row_start"), (dict(path=FAR[0] + 31 * 400), "path overlaps target_probs"),
                       (dict(n_path=FAR[6] + 4 * 31), "path overlaps n_path"), (dict(nxt=FAR[2] + 4 * 31), "next_token overlaps tokens"),
                       (dict(nxt=FAR[5]), "next_token overlaps u_next"), (dict(n_path=FAR[1]), "n_path overlaps draft_probs")):
        refused(M, -1, call(**over), text)


def test_refusals_of_commit(M):
    s = M.shape(32, 2, 2, 128, 1, 128, 1, q_len=8)

    def call(**over):
        a = dict(dict(path=FAR[4], stride=8, n_path=FAR[5], rs=None, n=4, to=FAR[6], kv=kv(M), s=s), **over)
        return lambda: M.kv_commit_paged(a["path"], a["stride"], a["n_path"], a["rs"], a["n"], a["to"], a["kv"], a["s"], stream=0)

    pool = M.paged_pool_bytes(M.KV_BF16, 10, 64, 2, 128)
    for over, status, text in (
            (dict(path=None), -1, "path"), (dict(stride=0), -1, "path_stride"), (dict(n_path=None), -1, "n_path"), (dict(to=None), -1, "kv_len_out"),
            (dict(n=5), -1, "must be B"), (dict(s=M.shape(65, 2, 2, 128, 1, 128, 1, q_len=65)), -1, "nodes"),
            (dict(s=M.shape(32, 2, 2, 100, 1, 128, 1, q_len=8)), -2, "D ="), (dict(kv=kv(M, max_pages=0)), -1, "max_pages"),
            (dict(to=FAR[3]), -1, "kv_len_out overlaps kv_len"), (dict(to=FAR[4] + 4 * 31), -1, "kv_len_out overlaps path"),
            (dict(to=FAR[2]), -1, "kv_len_out overlaps page_table"), (dict(to=FAR[0] + pool - 4), -1, "kv_len_out overlaps k_pages"),
            (dict(path=FAR[1] + pool - 4), -1, "path overlaps v_pages"), (dict(kv=kv(M, v_pages=FAR[0])), -1, "overlaps")):
        refused(M, status, call(**over), text)


def test_sizes_and_splits(M):
    s = M.shape(35, 8, 2, 128, 1, 128, 1, n_unique_splits=3, q_len=8)  # rows need no multiple of the largest tree
    assert M.tree_attn_workspace_bytes(s) >= 35 * 8 * 3 * 129 * 4
    s.n_unique_splits = 1
    assert M.tree_attn_workspace_bytes(s) == 0
    assert M.default_tree_splits(1, 8, 32, 8, 100000) > 1
    assert M.default_tree_splits(1, 8, 32, 8, 8) == 1
    assert M.default_tree_splits(1000, 64, 64, 8, 32768) >= 1
    assert M.default_tree_splits(0, 8, 32, 8, 8) == M.default_tree_splits(1, 8, 72, 8, 8) == 1
    assert M.default_tree_splits(1, 64, 4, 1, 1 << 30) <= 64


def test_python_checks(M):
    from paper_2511_06010_b200 import speculative
    from paper_2511_06010_b200.paged import PagedKvStore

    with pytest.raises(ValueError, match="max_nodes"):
        speculative.TreeAttention(8, 8, 2, 128, 100, 1, 65, device="cpu")
    with pytest.raises(ValueError, match="max_nodes"):
        speculative.TreeAttention(8, 8, 2, 128, 100, 1, 0, device="cpu")
    st = PagedKvStore.empty(4, 16, 2, 128, "bf16", device="cpu")
    at = speculative.TreeAttention(12, 8, 2, 128, 32, 2, 6, device="cpu", n_unique_splits=1)
    table, length = torch.zeros(2, 2, dtype=torch.int32), torch.full((2,), 20, dtype=torch.int32)
    q, up = torch.zeros(12, 8, 128, dtype=torch.bfloat16), torch.zeros(12, dtype=torch.int32)
    for call, text in (
            (lambda: at(q[:11], st, table, length, up), "q:"), (lambda: at(q.float(), st, table, length, up), "q:"),
            (lambda: at(q, st, table, length, up.long()), "parents"), (lambda: at(q, st, table, length, up[:5]), "parents"),
            (lambda: at(q, st, table[:1], length[:1], up), "page-table rows"), (lambda: at(q, st, table, length[:1], up), "kv_len"),
            (lambda: at(q, st, table, length, up, row_start=torch.zeros(2, dtype=torch.int32)), "row_start"),
            (lambda: at(q, PagedKvStore.empty(4, 16, 2, 128, "fp4", device="cpu"), table, length, up), "format"),
            (lambda: at(q, st, table, length, up), "not on a GPU")):
        with pytest.raises(ValueError, match=text):
            call()
    path, n_path = torch.zeros(2, 6, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for call, text in (
            (lambda: st.commit(table, length, path.long(), n_path, 6), "path"), (lambda: st.commit(table, length, path[:1], n_path, 6), "path"),
            (lambda: st.commit(table, length, path, n_path[:1], 6), "n_path"), (lambda: st.commit(table, length, path, n_path, 65), "max_nodes"),
            (lambda: st.commit(table, length, path, n_path, 0), "max_nodes"),
            (lambda: st.commit(table, length, path, n_path, 6, kv_len_out=n_path.float()), "kv_len_out"),
            (lambda: st.commit(table, length, path, n_path, 6, row_start=n_path), "row_start"),
            (lambda: st.commit(table, length, path, n_path, 6), "not on a GPU")):
        with pytest.raises(ValueError, match=text):
            call()
    p = torch.zeros(12, 50)
    u, un = torch.zeros(12), torch.zeros(2)
    for call, text in (
            (lambda: speculative.verify(p.half(), up, up, u, un), "target_probs"), (lambda: speculative.verify(p[0], up, up, u, un), "target_probs"),
            (lambda: speculative.verify(p, up, up, u, un, draft_probs=p.bfloat16()), "draft_probs"),
            (lambda: speculative.verify(p, up, up, u, un, draft_probs=p[:, :49]), "draft_probs"),
            (lambda: speculative.verify(p.t().contiguous().t(), up, up, u, un), "neighbours"),
            (lambda: speculative.verify(p[:1].expand(12, 50), up, up, u, un), "overlap"),
            (lambda: speculative.verify(p, up[:5], up, u, un), "tokens"), (lambda: speculative.verify(p, up, up.long(), u, un), "parents"),
            (lambda: speculative.verify(p, up, up, u.double(), un), "u_accept"), (lambda: speculative.verify(p, up, up, u, un.double()), "u_next"),
            (lambda: speculative.verify(p, up, up, u, un, max_nodes=5), "give row_start"),
            (lambda: speculative.verify(p, up, up, u, un, row_start=torch.zeros(3, dtype=torch.int32)), "max_nodes"),
            (lambda: speculative.verify(p, up, up, u, un, out=(path.long(), n_path, n_path)), "path"),
            (lambda: speculative.verify(p, up, up, u, un), "not on a GPU")):
        with pytest.raises(ValueError, match=text):
            call()


def test_the_reference_walk_keeps_the_targets_distribution():
    """Three drafts under the root, drawn from q: the emitted token's distribution, by exact enumeration, is p."""
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.2, 0.7, 0.1])
    target, draft = np.tile(p, (3, 1)), np.tile(q, (3, 1))
    n = 40  # midpoints of n intervals for each of the three random numbers
    mid = (np.arange(n) + 0.5) / n
    got = np.zeros(3)
    for a in range(3):
        for b in range(3):
            for u1 in mid:
                for u2 in mid:
                    for u3 in mid:
                        path, nxt = TR.verify(target, draft, [0, a, b], [-1, 0, 0], [0, u1, u2], u3)
                        got[[0, a, b][path[1]] if len(path) > 1 else nxt] += q[a] * q[b] / n ** 3
    assert np.abs(got - p).max() < 3.0 / n  # one interval of each number


def test_the_reference_attention_of_a_chain_is_the_paged_reference():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((4, 64)), rng.standard_normal((30, 2, 64)), rng.standard_normal((30, 2, 64))
    sees = TR.visible(np.arange(-1, 4), 30)
    assert [len(s) for s in sees] == [26, 27, 28, 29, 30]
    for s in sees:
        a, b = TR.attend(q, k[s], v[s], 0.125, "bf16"), R.attend(q, k[:len(s)], v[:len(s)], 0.125, "bf16")
        assert all(np.array_equal(x, y) for x, y in zip(a, b))
    assert TR.visible(np.array([-1, 0, 0, 2]), 3) == [[], [0], [1], [1, 2]]
    assert TR.visible(np.array([-1, 0]), 0) == [[], []]


def test_overlaps_of_tree_attention(M):
    """Results and workspace apart from one another and from what is read (bytes of the batch: q and out 65536, lse 1024)."""
    apart = dict(q=FAR[4], out=FAR[5], lse=FAR[6], parents=FAR[7])
    for over, text in (
            (dict(out=FAR[4] + 65536 - 16), "out"), (dict(lse=FAR[5] + 65536 - 4), "lse_out"), (dict(lse=FAR[4] + 4), "lse_out"),
            (dict(lse=FAR[7] + 124), "parents"), (dict(out=FAR[0] + 16), "k_pages"), (dict(lse=FAR[1]), "v_pages"),
            (dict(lse=FAR[3] + 12), "kv_len"), (dict(out=FAR[2] + 48), "page_table"), (dict(row_start=FAR[6] + 1020), "row_start")):
        refused(M, -1, attn(M, **{**apart, **over}), text)
