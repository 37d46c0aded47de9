"""Keeping accepted paths in a paged store: bytes of the moved rows and of everything else; and the operators of a
speculative step together."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import tree_reference as TR

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    from paper_2511_06010_b200 import binding as M

    M.device_status()
    yield
    torch.cuda.synchronize()


def filled(fmt, n_pages, page, Hkv, D, seed=0):
    from paper_2511_06010_b200.paged import PagedKvStore

    gen = torch.Generator().manual_seed(seed)
    st = PagedKvStore.empty(n_pages, page, Hkv, D, fmt)
    for t in ([st.k_pages, st.v_pages] if fmt == "bf16" else [st.pages4]):
        bits = torch.randint(0, 256, (t.numel() * t.element_size(),), generator=gen, dtype=torch.uint8)
        t.view(torch.uint8).view(-1).copy_(bits)  # any bits at all: NaN patterns too
    return st


def token_bytes(st):
    """Every token's bytes as a list of arrays [n_pages][page_size][bytes] that share the pools' memory (numpy)."""
    if st.fmt == "bf16":
        return [t.view(torch.uint8).cpu().numpy().reshape(st.n_pages, st.page_size, -1) for t in (st.k_pages, st.v_pages)]
    p = st.pages4.cpu().numpy()  # [n_pages][Hkv][blocks][18 D]
    D = st.D
    kb, vb, ks, vs, _ = R.byte_map(D)
    parts = []
    for t in range(16):
        at = np.unique(np.concatenate([kb[t], vb[t], ks[t], ks[t] + 1, vs[t], vs[t] + 1]))
        assert len(at) == 18 * D // 16
        # in the order of what they mean: the codes by dimension, then the scales
        at = np.concatenate([kb[t, ::2], vb[t, ::2], ks[t, ::32], ks[t, ::32] + 1, vs[t, ::32], vs[t, ::32] + 1])
        parts.append(p[..., at])
    x = np.stack(parts, 3)  # [n_pages][Hkv][blocks][16][bytes]
    return [x.transpose(0, 2, 3, 1, 4).reshape(st.n_pages, st.page_size, -1).copy()]


def expected(before, table, lens, nodes, path, n_path, page):
    want = [b.copy() for b in before]
    for r, T in enumerate(nodes):
        c = lens[r] - T
        if c < 0:
            continue
        for w, b in zip(want, before):
            for j in range(n_path[r]):
                s, d = c + path[r][j], c + j
                w[table[r][d // page], d % page] = b[table[r][s // page], s % page]
    return want


CASES = [
    # D, Hkv, page, lengths, nodes, paths
    (128, 2, 16, [40, 16, 9], [8, 8, 8], [[0, 2, 3, 7], [0, 1, 2], [0]]),           # sources that are places of others
    (64, 3, 32, [64, 33], [33, 33], [list(range(0, 33, 2)), list(range(33))]),
    (128, 8, 64, [64, 200, 129], [64, 64, 64], [list(range(1, 64)), list(range(64)), [63]]),  # 63 rows by one
    (64, 1, 16, [20, 17], [4, 4], [[], [3]]),
    (128, 1, 128, [300] * 5, [20] * 5, [[0, 5, 9], [0, 19], [0, 1, 2, 3, 18], [7], []]),
]


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hkv,page,lens,nodes,paths", CASES)
def test_rows_move_and_nothing_else_changes(fmt, D, Hkv, page, lens, nodes, paths):
    from paper_2511_06010_b200 import binding as M

    rng = np.random.default_rng(D + page)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    order = list(rng.permutation(n_pages))
    table = np.full((len(lens), max(need)), -1, dtype=np.int32)
    for r, m in enumerate(need):
        for i in range(m):
            table[r, i] = order.pop()
    st = filled(fmt, n_pages, page, Hkv, D)
    before = token_bytes(st)
    path = np.full((len(lens), max(nodes)), 1 << 20, dtype=np.int32)  # entries behind the path are not read
    for r, p in enumerate(paths):
        path[r, :len(p)] = p
    n_path = [len(p) for p in paths]
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    new = st.commit(torch.from_numpy(table).cuda(), length, torch.from_numpy(path).cuda(),
                    torch.tensor(n_path, dtype=torch.int32).cuda(), nodes[0])
    assert new.tolist() == [n - t + m for n, t, m in zip(lens, nodes, n_path)] and length.tolist() == lens
    for got, want in zip(token_bytes(st), expected(before, table, lens, nodes, path, n_path, page)):
        assert np.array_equal(got, want)
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_ragged_trees_padding_and_bad_paths(fmt):
    """Requests of different trees and without a context; paths that are none are reported and their rows left."""
    from paper_2511_06010_b200 import binding as M

    page, lens, nodes = 16, [30, 0, 3, 25, 40], [7, 5, 6, 0, 12]
    table = np.arange(15, dtype=np.int32).reshape(5, 3)
    start = torch.tensor(np.concatenate([[0], np.cumsum(nodes)]), dtype=torch.int32).cuda()
    good = [[0, 3, 6], [0, 1], [0, 4], [], [0, 2, 11]]
    bad = {"descending": [0, 3, 2], "twice": [0, 4, 4], "behind the tree": [0, 3, 12], "negative": [-1, 2, 3], "too many": None,
           "fewer than none": None}
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    for what in [None] + list(bad):
        st = filled(fmt, 15, page, 2, 128, seed=3)
        before = token_bytes(st)
        path = np.full((5, 12), -1, dtype=np.int32)
        for r, p in enumerate(good):
            path[r, :len(p)] = p
        n_path = [len(p) for p in good]
        done = list(n_path)
        want_len = [30 - 7 + 3, 0, 3, 25, 40 - 12 + 3]
        if what is not None:
            if bad[what] is None:
                n_path[4] = 13 if what == "too many" else -1
            else:
                path[4, :3] = bad[what]
            done[4], want_len[4] = 0, 40
        new = st.commit(torch.from_numpy(table).cuda(), length, torch.from_numpy(path).cuda(),
                        torch.tensor(n_path, dtype=torch.int32).cuda(), 12, row_start=start)
        assert M.device_status() == (0 if what is None else M.ERR_INVALID_ARG)
        assert new.tolist() == want_len, what
        for got, want in zip(token_bytes(st), expected(before, table, lens, nodes, path, done, page)):
            assert np.array_equal(got, want), what


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_a_page_outside_the_pool_is_reported(fmt):
    from paper_2511_06010_b200 import binding as M

    st = filled(fmt, 4, 16, 2, 64)
    before = token_bytes(st)
    table = torch.tensor([[0, 4], [2, -1]], dtype=torch.int32).cuda()
    length = torch.tensor([20, 16], dtype=torch.int32).cuda()
    path = torch.tensor([[0, 5], [0, 3]], dtype=torch.int32).cuda()
    new = st.commit(table, length, path, torch.tensor([2, 2], dtype=torch.int32).cuda(), 6)
    assert M.device_status() == M.ERR_INVALID_ARG
    assert new.tolist() == [20, 12]  # the first request is left as it was
    for got, want in zip(token_bytes(st), expected(before, table.cpu().numpy(), [20, 16], [6, 6], [[], [0, 3]], [0, 2], 16)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_speculative_steps_together(fmt):
    """Several steps of append, attention, verification and commit, captured in one graph: the kept rows are those that
    a list of the accepted tokens' rows holds, and attention over them is the reference's."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200 import speculative
    from paper_2511_06010_b200.paged import PagedKvStore, PageTable

    Rn, T, Hq, Hkv, D, V, page = 3, 10, 8, 2, 128, 40, 16
    rng = np.random.default_rng(12)
    st = PagedKvStore.empty(60, page, Hkv, D, fmt)
    book = PageTable(60, page, Rn, 12)
    gen = torch.Generator().manual_seed(13)
    kv_len = torch.tensor([5, 0, 33], dtype=torch.int32).cuda()
    kept = []
    for r, n in enumerate(kv_len.tolist()):
        book.reserve(r, 180)
        kept.append([R.make_bf16((n, Hkv, D), gen), R.make_bf16((n, Hkv, D), gen)])
    rows = [torch.cat([kept[r][i] for r in range(Rn)]).cuda() for i in range(2)]
    st.append(None, *rows, book.table(), kv_len, row_start=torch.tensor([0, 5, 5, 38], dtype=torch.int32).cuda())
    attention = speculative.TreeAttention(Rn * T, Hq, Hkv, D, 180, Rn, T, fmt=fmt)
    # the step's buffers, as a graph has them
    q, k, v = (torch.zeros(Rn * T, h, D, dtype=torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    parents, tokens, positions = (torch.zeros(Rn * T, dtype=torch.int32).cuda() for _ in range(3))
    target, draft = (torch.full((Rn * T, V), 1.0 / V).cuda() for _ in range(2))
    u, un = torch.zeros(Rn * T).cuda(), torch.zeros(Rn).cuda()
    with_tree, q_rot = torch.zeros_like(kv_len), torch.zeros_like(q)
    cos_sin = R.angles(256, 64).cuda()
    out = [torch.zeros(Rn, T, dtype=torch.int32).cuda(), torch.zeros_like(kv_len), torch.zeros_like(kv_len)]
    after = torch.zeros_like(kv_len)

    def step():
        torch.add(kv_len, T, out=with_tree)
        st.append(q, k, v, book.table(), with_tree, positions, cos_sin, q_len=T, q_out=q_rot)
        attention(q_rot, st, book.table(), with_tree, parents)
        speculative.verify(target, tokens, parents, u, un, draft_probs=draft, out=out)
        st.commit(book.table(), with_tree, out[0], out[1], T, kv_len_out=after)
        kv_len.copy_(after)

    start = kv_len.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    kv_len.copy_(start)
    for _ in range(6):
        before = kv_len.tolist()
        trees = [TR.random_tree(rng, T) for _ in range(Rn)]
        parents.copy_(torch.from_numpy(np.concatenate(trees)))
        depth = [TR.ancestors(t).sum(1) - 1 for t in trees]
        positions.copy_(torch.from_numpy(np.concatenate([b + d for b, d in zip(before, depth)]).astype(np.int32)))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen))
        for t in (target, draft):
            t.copy_(torch.softmax(2 * torch.randn(t.shape, generator=gen), 1))
        tokens.copy_(torch.randint(0, V, tokens.shape, generator=gen))
        u.copy_(torch.rand(u.shape, generator=gen) * 0.5)
        un.copy_(torch.rand(un.shape, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        assert M.device_status() == 0
        pos, cs = positions.cpu().numpy(), cos_sin.cpu().numpy()
        k32, q32 = (R.rotate32(t.float().cpu().numpy(), cs[pos], 64, False) for t in (k, q))
        assert torch.equal(q_rot.cpu(), torch.from_numpy(q32).to(torch.bfloat16))
        as_held = (lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()) if fmt == "bf16" else R.held32
        new_k, new_v = as_held(k32), as_held(v.float().cpu().numpy())
        for r in range(Rn):
            s = slice(r * T, (r + 1) * T)
            want, token = TR.verify(target[s].double().cpu().numpy(), draft[s].double().cpu().numpy(), tokens[s].tolist(), trees[r],
                                    u[s].tolist(), float(un[r]))
            assert out[0][r].tolist() == want + [-1] * (T - len(want)) and int(out[1][r]) == len(want) and int(out[2][r]) == token
            assert int(kv_len[r]) == before[r] + len(want)
            old = [as_held(x.float().numpy()) if isinstance(x, torch.Tensor) else x for x in kept[r]]
            seen = TR.ancestors(trees[r])
            for i in range(0, T, 3):
                see = np.flatnonzero(seen[i])
                o, l, o_tol, l_tol = TR.attend(R.to_f64(q_rot[r * T + i]), np.concatenate([old[0], new_k[s][see]]),
                                               np.concatenate([old[1], new_v[s][see]]), attention.scale, fmt)
                assert (np.abs(R.to_f64(attention.out[r * T + i]) - o) <= o_tol).all()
                assert (np.abs(attention.lse[r * T + i].double().cpu().numpy() - l) <= l_tol).all()
            kept[r] = [np.concatenate([old[0], new_k[s][want]]), np.concatenate([old[1], new_v[s][want]])]
    lens = kv_len.tolist()
    first = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()
    ko, vo = st.gather(book.table(), kv_len, sum(lens), row_start=first)
    for got, i in ((ko, 0), (vo, 1)):
        assert torch.equal(got.cpu(), torch.from_numpy(np.concatenate([kept[r][i] for r in range(Rn)])).to(torch.bfloat16))
