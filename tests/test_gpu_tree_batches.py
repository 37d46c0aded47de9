"""Attention of drafted trees over batches and contexts at the ends of their ranges: how the work is cut among the SMs must
not show in the results."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import tree_reference as TR
from tests.test_gpu_tree import case, check, clean_status  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


def run(c, **kw):
    out, lse = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"], **kw)
    return out.clone(), lse.clone()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [1, 2, None])
def test_many_requests(fmt, splits):
    """More requests than a CTA has threads, of all small sizes, some without nodes or a context, the last ones too."""
    from paper_2511_06010_b200 import binding as M

    rng = np.random.default_rng(1)
    n = 700
    lens = [int(x) for x in rng.integers(0, 200, n)]
    nodes = [int(x) for x in rng.integers(0, 20, n)]
    nodes[-3:], nodes[300:310], lens[5:8] = [0] * 3, [0] * 10, [0] * 3
    c = case(fmt, 64, 16, 2, 16, lens, nodes, seed=1, pad=3, splits=splits)
    out, lse = run(c, row_start=c["start"])
    assert M.device_status() == 0
    check(c, out, lse, only=lambda r, i: r < 10 or r % 23 == 0 or r > n - 6)
    assert torch.isnan(out[-3:]).all() and not torch.isnan(out[:-3]).any()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,nodes", [(64, 64, 40), (128, 16, 9)])
def test_long_parts(fmt, D, Hq, nodes):
    """Enough tiles that every SM walks many units, whose ends count on the line too: the same rows whatever a context may
    be cut into (each part's probabilities and result rounded on their own: twice the bounds of one)."""
    lens = [int(x) for x in np.random.default_rng(2).integers(700, 3200, 30)]
    c = case(fmt, D, Hq, 8, 32, lens, [nodes] * 30, seed=2)
    out, lse = run(c)
    check(c, out, lse, only=lambda r, i: r % 10 == 0 and i % 13 == 0)
    for splits in (1, 2, 3):
        from paper_2511_06010_b200.speculative import TreeAttention

        c["attention"] = TreeAttention(c["rows"], Hq, 8, D, max(lens), 30, nodes, fmt=fmt, n_unique_splits=splits)
        other, other_lse = run(c)
        check(c, other, other_lse, only=lambda r, i: r == 20 and i % 13 == 0)
        # values are at most about 5: probabilities are off by half a step of their type, results by half a step of bf16
        assert (other.float() - out.float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -8) * 5
        assert (other_lse - lse).abs().max() <= 2.0 ** -12


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [1, 2, 5, 64])
@pytest.mark.parametrize("T,Hq", [(20, 16), (7, 8), (1, 2)])
def test_slots_of_the_layer(fmt, splits, T, Hq):
    """The layer's partial slots for any number of them, long and short contexts in one batch."""
    from paper_2511_06010_b200.engine import MoskaLayer

    lens = [2000, 30, 0, 700]
    c = case(fmt, 128, Hq, 2, 64, lens, [T] * 4, seed=7)
    layer = MoskaLayer(c["rows"], Hq, 2, 128, 1, 128, 1, max(lens), q_len=T, paged_fmt=fmt, n_unique_splits=splits)
    layer.o_part.fill_(float("nan"))
    layer.lse_part.fill_(float("nan"))
    layer.unique_paged(c["q"].cuda(), c["store"], c["table"], c["length"], parents=c["up"])
    part, o = layer.lse_part[..., -splits:].double(), layer.o_part[..., -splits:, :].double()
    assert not torch.isnan(part).any() and not torch.isnan(o).any()
    lse = torch.logsumexp(part, -1)
    weight = torch.exp(part - lse.unsqueeze(-1)).nan_to_num(0.0)
    check(c, (o * weight.unsqueeze(-1)).sum(-2).float(), lse.float(), only=lambda r, i: i % 4 == 0)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_graphs_that_share_a_workspace_and_calls_at_once(fmt):
    c = case(fmt, 128, 16, 2, 32, [900, 350, 1500], [24] * 3, seed=6)
    at, q = c["attention"], c["q"].cuda()
    p = -q
    want = [x for y in (q, p) for x in (t.clone() for t in at(y, c["store"], c["table"], c["length"], c["up"]))]
    graphs = []
    for x in (q, p):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            at(x, c["store"], c["table"], c["length"], c["up"])
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(at.out, want[2 * i]) and torch.equal(at.lse, want[2 * i + 1])
    from paper_2511_06010_b200.speculative import TreeAttention

    others = [TreeAttention(c["rows"], 16, 2, 128, 1500, 3, 24, fmt=fmt) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for a, s, x in zip(others, streams, (q, p)):
            a(x, c["store"], c["table"], c["length"], c["up"], stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(others[i].out, want[2 * i]) and torch.equal(others[i].lse, want[2 * i + 1])


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("length", [20_000_001, 2 ** 30])  # the longest that a table row may have
def test_contexts_of_millions_of_tokens(fmt, length):
    """One page stands for all committed ones, so that a token's weight is how often it is seen."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedKvStore
    from paper_2511_06010_b200.speculative import TreeAttention

    D, Hq, page, T = 64, 2, 32768, 5
    gen = torch.Generator().manual_seed(5)
    pages = -(-length // page)
    table = torch.zeros(1, pages, dtype=torch.int32)
    table[0, -1] = 1
    last = length - (pages - 1) * page  # tokens of the last page, the tree among them
    st = PagedKvStore.empty(2, page, 1, D, fmt)
    k, v = R.make_bf16((page + last, 1, D), gen), R.make_bf16((page + last, 1, D), gen)
    st.append(None, k.cuda(), v.cuda(), torch.tensor([[0, 1]], dtype=torch.int32).cuda(),
              torch.tensor([page + last], dtype=torch.int32).cuda(), row_start=torch.tensor([0, page + last], dtype=torch.int32).cuda())
    q = R.make_bf16((T, Hq, D), gen)
    parents = np.array([-1, 0, 0, 1, 3], dtype=np.int32)
    at = TreeAttention(T, Hq, 1, D, length, 1, T, fmt=fmt)
    out, lse = at(q.cuda(), st, table.cuda(), torch.tensor([length], dtype=torch.int32).cuda(), torch.from_numpy(parents).cuda())
    assert M.device_status() == 0
    kk, vv = (R.to_f64(st.k_pages), R.to_f64(st.v_pages)) if fmt == "bf16" else R.unpack(st.pages4)
    kk, vv = R.context(kk, vv, np.array([0, 1]), page + last)
    times = np.concatenate([np.full(page, pages - 1.0), np.ones(last)])
    sees = TR.visible(parents, page + last)
    # sums in 32 bits: a part is at most a 63rd of the context here (of many parts, equal ones), its row sum a chain of an
    # addition a step of 64 tokens and group, its result one of an addition 16 tokens, each off by 2^-24 or, cut off, 2^-23
    part = length / 63 if length > 2 ** 28 else length / 100
    for i in range(T):
        o, l, o_tol, l_tol = TR.attend(R.to_f64(q[i]), kk[sees[i]], vv[sees[i]], at.scale, fmt)
        s = np.einsum("hd,td->ht", R.to_f64(q[i]), kk[sees[i], 0]) * at.scale + np.log(times[sees[i]])
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        l = np.log(p.sum(-1)) + top[:, 0]
        o = (p / p.sum(-1, keepdims=True)) @ vv[sees[i], 0]
        mass = (p / p.sum(-1, keepdims=True)) @ np.abs(vv[sees[i], 0])
        assert (np.abs(lse[i].double().cpu().numpy() - l) <= l_tol + part / 128 * 2.0 ** -24 + 2.0 ** -20).all()
        assert (np.abs(R.to_f64(out[i]) - o) <= 2 * o_tol + part / 16 * 2.0 ** -23 * mass).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("most", [1, 8, 16])
def test_small_ragged_trees(fmt, splits, D, most):
    """Trees of few rows, ragged, without nodes or a context, or with a context shorter than the tree."""
    from paper_2511_06010_b200 import binding as M

    lens = [40, 0, 700, 5, 64, 257]
    nodes = [min(most, x) for x in (3, 6, most, 9, 0, 5)]
    c = case(fmt, D, 8, 2, 32, lens, nodes, seed=5, pad=4, splits=splits, max_nodes=most)
    out, lse = run(c, row_start=c["start"])
    check(c, out, lse)
    assert torch.isnan(out[-4:]).all() and torch.isnan(lse[-4:]).all()
    assert M.device_status() == 0
