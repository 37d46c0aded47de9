"""GPU parity of attention for drafted trees over paged contexts, against the plain reference in 64 bits."""
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


def case(fmt, D, Hq, Hkv, page, lens, nodes, seed=0, width=3, scale=1.0, pad=0, max_nodes=None, splits=None):
    """Contexts of random values in a pool that holds NaN everywhere else; trees of the given sizes."""
    from paper_2511_06010_b200.paged import PagedKvStore
    from paper_2511_06010_b200.speculative import TreeAttention

    gen = torch.Generator().manual_seed(1000 * D + 10 * Hq + seed)
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    order = list(rng.permutation(n_pages))
    table = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32)
    for r, m in enumerate(need):
        for i in range(m):
            table[r, i] = int(order.pop())
    st = PagedKvStore.empty(n_pages, page, Hkv, D, fmt)
    if fmt == "bf16":
        st.k_pages.fill_(float("nan"))
        st.v_pages.fill_(float("nan"))
    else:
        st.pages4.fill_(0xFF)
    total = sum(lens)
    k, v = R.make_bf16((max(total, 1), Hkv, D), gen), R.make_bf16((max(total, 1), Hkv, D), gen)
    k[..., ::16] *= 4
    first = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32)
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    if total:
        st.append(None, k[:total].cuda(), v[:total].cuda(), table.cuda(), length, row_start=first.cuda())
    rows = sum(nodes) + pad
    parents = np.concatenate([TR.random_tree(rng, t, width) for t in nodes if t] + [np.full(pad, 7, np.int32)])
    c = dict(fmt=fmt, lens=lens, nodes=nodes, table=table.cuda(), length=length, store=st, parents=parents,
             up=torch.from_numpy(parents.astype(np.int32)).cuda(), q=(scale * R.make_bf16((rows, Hq, D), gen)).bfloat16(),
             start=torch.tensor(np.concatenate([[0], np.cumsum(nodes)]), dtype=torch.int32).cuda(), rows=rows)
    c["attention"] = TreeAttention(rows, Hq, Hkv, D, max(max(lens), 1), len(lens), max_nodes or max(max(nodes), 1), fmt=fmt,
                                   n_unique_splits=splits)
    c["attention"].out.fill_(float("nan"))
    c["attention"].lse.fill_(float("nan"))
    return c


def held(c):
    """The contexts' keys and values in 64 bits."""
    st = c["store"]
    k, v = (R.to_f64(st.k_pages), R.to_f64(st.v_pages)) if st.fmt == "bf16" else R.unpack(st.pages4)
    return [R.context(k, v, c["table"][r].cpu().numpy(), n) for r, n in enumerate(c["lens"])]


def check(c, out, lse, only=None):
    out, lse, at = R.to_f64(out), lse.double().cpu().numpy(), 0
    contexts = held(c)
    for r, T in enumerate(c["nodes"]):
        sees = TR.visible(c["parents"][at:at + T], c["lens"][r])
        k, v = contexts[r]
        for i in range(T):
            if only is None or only(r, i):
                o, l, o_tol, l_tol = TR.attend(R.to_f64(c["q"][at + i]), k[sees[i]], v[sees[i]], c["attention"].scale, c["fmt"])
                assert (np.abs(out[at + i] - o) <= o_tol).all(), (r, i, np.abs(out[at + i] - o).max(), o_tol.max())
                assert (np.abs(np.where(np.isinf(l) & (l == lse[at + i]), 0, lse[at + i] - np.where(np.isinf(l), 0, l))) <= l_tol).all(), \
                    (r, i, lse[at + i], l)
        at += T


SHAPES = [
    # D, Hq, Hkv, page, lengths, nodes, splits
    (128, 8, 2, 32, [8], [8], None),                                  # nothing but the tree
    (128, 8, 2, 16, [1, 2, 17, 128, 129], [1, 1, 1, 1, 1], 1),        # one node: decode
    (128, 16, 2, 64, [64, 65, 200], [64, 64, 64], 1),                 # the largest trees, 512 rows a head
    (64, 16, 2, 16, [127, 128, 130, 300], [33, 33, 33, 33], 1),       # trees across tile borders
    (128, 7, 1, 128, [300, 40, 257], [20, 20, 20], 2),                # G that does not divide a tile
    (64, 12, 4, 32, [500, 77], [5, 5], 3),
    (128, 5, 1, 16, [1000], [13], 7),                                 # many splits of one request
    (64, 6, 2, 256, [700, 1300], [11, 11], 64),                       # splits without tokens
    (128, 24, 8, 16, [90, 16, 33], [9, 9, 9], None),
    (64, 1, 1, 16, [64], [64], 1),
    (128, 64, 8, 128, [700], [60], None),
]


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,Hkv,page,lens,nodes,splits", SHAPES)
def test_trees_match_the_reference(fmt, D, Hq, Hkv, page, lens, nodes, splits):
    from paper_2511_06010_b200 import binding as M

    c = case(fmt, D, Hq, Hkv, page, lens, nodes, splits=splits, seed=len(lens))
    out, lse = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"])
    check(c, out, lse)
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_ragged_trees_and_padding_rows(fmt, splits, D):
    """Trees of different sizes, requests without nodes, without a context or with one shorter than their tree."""
    from paper_2511_06010_b200 import binding as M

    lens, nodes = [40, 0, 300, 5, 64, 150], [3, 6, 31, 9, 0, 64]
    c = case(fmt, D, 8, 2, 32, lens, nodes, seed=5, pad=4, splits=splits)
    at = c["attention"]
    at.out.fill_(3.0)
    at.lse.fill_(5.0)
    out, lse = at(c["q"].cuda(), c["store"], c["table"], c["length"], c["up"], row_start=c["start"])
    check(c, out, lse)
    assert (out[-4:] == 3.0).all() and (lse[-4:] == 5.0).all()
    assert (out[3:9] == 0).all() and (lse[3:9] == -float("inf")).all()  # no context
    assert (out[40:44] == 0).all() and (lse[40:44] == -float("inf")).all()  # nodes whose token is negative
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [4, 1])
def test_what_a_node_does_not_see_has_no_influence(fmt, D, G):
    """Infinities and NaN in the keys and values of nodes: rows that do not see them are as without them, bit for
    bit; the others are not finite."""
    lens, nodes = [200, 131], [40, 40]
    c = case(fmt, D, 2 * G, 2, 16, lens, nodes, seed=3)
    out, lse = (x.clone() for x in c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"]))
    check(c, out, lse)
    Hkv, bad = 2, {7: float("nan"), 21: float("inf"), 39: -float("inf")}
    touched = np.zeros((2, 40), dtype=bool)
    k, v = c["store"].gather(c["table"], c["length"], 80, q_len=40)
    for r in range(2):
        for j, x in bad.items():
            v[40 * r + j, 1, 5] = x  # one element of one head
            touched[r] |= TR.ancestors(c["parents"][40 * r:40 * r + 40])[:, j]
    c["store"].append(None, k, v, c["table"], c["length"], q_len=40)
    out2, lse2 = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"])
    keep = torch.from_numpy(~touched.reshape(-1)).cuda()
    assert torch.equal(out2[keep], out[keep]) and torch.equal(lse2[keep], lse[keep])
    assert torch.equal(out2[:, :G], out[:, :G])  # the other head's rows
    spoilt = slice(5, 6) if fmt == "bf16" else slice(0, 32)  # in 4 bits all that shares the scale
    assert not torch.isfinite(out2[~keep][:, G:, spoilt]).any()
    rest = out2[~keep][:, G:].clone()
    rest[..., spoilt] = 0
    assert torch.isfinite(rest).all()
    k[7, 0] = float("nan")  # a key: every score of that node
    c["store"].append(None, k, v, c["table"], c["length"], q_len=40)
    out3, _ = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"])
    sees = torch.from_numpy(TR.ancestors(c["parents"][:40])[:, 7]).cuda()
    assert torch.isnan(out3[:40][sees][:, :G]).all() and torch.equal(out3[:40][~sees][:, :G], out[:40][~sees][:, :G])


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("nodes", [17, 14, 5])
def test_large_scores(fmt, nodes):
    """Scores of hundreds: probabilities that underflow, a maximum that moves by more than any of them."""
    c = case(fmt, 128, 8, 2, 64, [900, 401], [nodes, nodes], seed=9, scale=24.0)
    out, lse = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"])
    check(c, out, lse)


@pytest.mark.parametrize("fmt,Hq,q_len", [("bf16", 8, 4), ("fp4", 4, 16), ("fp4", 8, 3)])
def test_chains_are_what_paged_attention_gives(fmt, Hq, q_len):
    from paper_2511_06010_b200.paged import PagedAttention

    lens = [300, 77, 1030]
    c = case(fmt, 128, Hq, Hq // 4 if Hq > 4 else 4, 32, lens, [q_len] * 3, seed=2)
    chain = np.concatenate([np.arange(-1, q_len - 1)] * 3).astype(np.int32)
    c["parents"] = chain
    for parents in (None, torch.from_numpy(chain).cuda()):
        out, lse = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], parents)
        check(c, out, lse)
    other, other_lse = PagedAttention(c["rows"], Hq, c["store"].Hkv, 128, max(lens), fmt=fmt, q_len=q_len)(
        c["q"].cuda(), c["store"], c["table"], c["length"])
    assert (other.float() - out.float()).abs().max() < 0.05 and (other_lse - lse).abs().max() < 0.02


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_bad_parents_tables_and_rows_are_reported(fmt):
    """A parent that does not come before its child counts as none; bad pages, lengths and row ranges raise the status
    word and leave other requests' results as they are."""
    from paper_2511_06010_b200 import binding as M

    c = case(fmt, 128, 8, 2, 32, [90, 60, 75], [12, 12, 12], seed=4)
    q, up = c["q"].cuda(), c["up"].clone()
    up[3], up[13], up[20] = 3, -2, 11
    out, lse = c["attention"](q, c["store"], c["table"], c["length"], up)
    assert M.device_status() == M.ERR_INVALID_ARG
    c["parents"] = c["parents"].copy()
    c["parents"][[3, 13, 20]] = -1
    check(c, out, lse)
    table = c["table"].clone()
    table[1, 0] = 10**6
    out, lse = c["attention"](q, c["store"], table, c["length"], c["up"])
    assert M.device_status() == M.ERR_INVALID_ARG
    c = case(fmt, 128, 8, 2, 32, [90, 60, 75], [12, 12, 12], seed=4)
    length = c["length"].clone()
    length[1] = 2**31 - 1
    out, lse = c["attention"](q, c["store"], c["table"], length, c["up"])
    assert M.device_status() == M.ERR_INVALID_ARG
    check(c, out, lse, only=lambda r, i: r != 1)
    for start in ([0, 12, 24, 37], [0, -5, 24, 36], [0, 30, 24, 36]):
        c["attention"](q, c["store"], c["table"], c["length"], c["up"], row_start=torch.tensor(start, dtype=torch.int32).cuda())
        assert M.device_status() == M.ERR_INVALID_ARG
    c["attention"](q, c["store"], c["table"], c["length"], c["up"], row_start=c["start"])
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_another_stream_and_a_captured_graph(fmt):
    c = case(fmt, 128, 16, 2, 32, [700, 350], [24, 24], seed=6, splits=3)
    q, at = c["q"].cuda(), c["attention"]
    want = [x.clone() for x in at(q, c["store"], c["table"], c["length"], c["up"])]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    at.out.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    at(q, c["store"], c["table"], c["length"], c["up"], stream=side)
    side.synchronize()
    assert torch.equal(at.out, want[0]) and torch.equal(at.lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at(q, c["store"], c["table"], c["length"], c["up"])
    q.zero_()
    graph.replay()
    q.copy_(c["q"])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(at.out, want[0]) and torch.equal(at.lse, want[1])


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_pages_beyond_32_bit_offsets(fmt):
    """A pool of more than 4 GB of elements, contexts in its last pages."""
    from paper_2511_06010_b200.paged import PagedKvStore

    D, Hkv, page = 128, 8, 1024
    token = Hkv * D if fmt == "bf16" else Hkv * 18 * D // 16
    n_pages = (1 << 32) // (token * page) + 3
    c = case(fmt, D, 16, Hkv, page, [1500, 700], [20, 20], seed=8)
    big = PagedKvStore.empty(n_pages, page, Hkv, D, fmt)
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, -1]], dtype=torch.int32).cuda()
    for to, at in ((n_pages - 1, c["table"][0, 0]), (0, c["table"][0, 1]), (n_pages - 2, c["table"][1, 0])):
        for name in ("k_pages", "v_pages") if fmt == "bf16" else ("pages4",):
            getattr(big, name)[to] = getattr(c["store"], name)[int(at)]
    out, lse = c["attention"](c["q"].cuda(), big, table, c["length"], c["up"])
    check(c, out, lse)


def _layer_case(fmt, two_streams, dense):
    from paper_2511_06010_b200 import workloads as W
    from paper_2511_06010_b200.engine import MoskaLayer

    T, n = 12, 4
    w = W.scaled(W.CONFIGS[1], B=n * T, C=8, k=2, unique_len=256)
    c = case(fmt, w.D, w.Hq, w.Hkv, 64, [256, 40, 0, 333], [T] * n, seed=11)
    sh = W.make_shared_store(w, "cuda")
    q = W.make_queries(w, sh, 0, "cuda")
    layer = MoskaLayer(w.B, w.Hq, w.Hkv, w.D, w.C, w.L, w.k, 333, q_len=T, paged_fmt=fmt, dense=dense)
    layer.build_summaries(sh.k_shared)
    return w, c, sh, q, layer


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("two_streams", [False, True])
@pytest.mark.parametrize("dense", [False, True])
def test_the_layers_step_over_trees(fmt, two_streams, dense):
    """Shared chunks, seen whole by every node, and the tree's private context, merged."""
    from paper_2511_06010_b200 import binding as M

    w, c, sh, q, layer = _layer_case(fmt, two_streams, dense)
    out = layer.step_paged(q, sh.k_shared, sh.v_shared, c["store"], c["table"], c["length"], two_streams=two_streams, parents=c["up"])
    torch.cuda.synchronize()
    assert M.device_status() == 0
    ks, vs = R.to_f64(sh.k_shared), R.to_f64(sh.v_shared)  # [Hkv][C][L][D]
    contexts, got, G = held(c), R.to_f64(out), w.Hq // w.Hkv
    got_lse = layer.lse_out.double().cpu().numpy()
    for b in range(0, w.B, 5):
        r, i = b // 12, b % 12
        see = TR.visible(c["parents"][12 * r:12 * r + 12], c["lens"][r])[i]
        for h in range(w.Hkv):
            chunks = range(w.C) if dense else layer.topk_idx[b, h].tolist()
            k = np.concatenate([ks[h, x] for x in chunks] + [contexts[r][0][see, h]])[:, None]
            v = np.concatenate([vs[h, x] for x in chunks] + [contexts[r][1][see, h]])[:, None]
            o, l, o_tol, l_tol = TR.attend(R.to_f64(q[b, h * G:(h + 1) * G]), k, v, layer.scale, fmt)
            # the shared part's probabilities are bf16 whatever the private format
            o_tol = o_tol + R.attend(R.to_f64(q[b, h * G:(h + 1) * G]), k, v, layer.scale, "bf16")[2]
            assert (np.abs(got[b, h * G:(h + 1) * G] - o) <= o_tol).all()
            assert (np.abs(got_lse[b, h * G:(h + 1) * G] - l) <= l_tol + 2.0 ** -18).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_stage_of_the_layer_for_trees(fmt):
    """unique_paged with parents fills the private slots with what the step merges."""
    w, c, sh, q, layer = _layer_case(fmt, False, False)
    layer.unique_paged(q, c["store"], c["table"], c["length"], parents=c["up"])
    n = layer.shape.n_unique_splits
    lse = torch.logsumexp(layer.lse_part[..., -n:].double(), -1)
    weight = torch.exp(layer.lse_part[..., -n:].double() - lse.unsqueeze(-1)).nan_to_num(0.0)
    out = (layer.o_part[..., -n:, :].double() * weight.unsqueeze(-1)).sum(-2)
    c["q"] = q.cpu()
    check(c, out.float(), lse.float())
