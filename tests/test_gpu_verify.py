"""Verification of drafted tokens on the GPU: every answer is a whole number and equal to the plain reference's."""
import numpy as np
import pytest
import torch

from tests import tree_reference as TR

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    from paper_2511_06010_b200 import binding as M

    M.device_status()
    yield
    torch.cuda.synchronize()


def make(rng, nodes, V, width=3, peak=3.0, drafts=True, dtype=torch.float32, pad=0):
    B = sum(nodes)
    logits = peak * rng.standard_normal((B + pad, V))
    p = np.exp(logits - logits.max(1, keepdims=True))
    d = np.exp(logits + rng.standard_normal(logits.shape))
    target = torch.from_numpy(p / p.sum(1, keepdims=True)).to(dtype)
    draft = torch.from_numpy(d / d.sum(1, keepdims=True)).to(dtype)
    parents = np.concatenate([TR.random_tree(rng, t, width) for t in nodes if t] + [np.full(pad, 9, np.int32)])
    first = np.concatenate([[0], np.cumsum(nodes)])
    tokens = np.zeros(B + pad, dtype=np.int32)
    for r, t in enumerate(nodes):
        for j in range(t):
            row = draft[first[r] + max(0, parents[first[r] + j])].double().numpy()
            tokens[first[r] + j] = rng.choice(V, p=row / row.sum())
    u = rng.random(B + pad).astype(np.float32)
    return dict(target=target, draft=draft if drafts else None, parents=parents.astype(np.int32), tokens=tokens, u=u,
                un=rng.random(len(nodes)).astype(np.float32), first=first.astype(np.int32), nodes=nodes)


def run(c, uniform=False, **more):
    from paper_2511_06010_b200 import speculative

    dev = lambda x: None if x is None else (x if isinstance(x, torch.Tensor) else torch.from_numpy(x)).cuda()  # noqa: E731
    return speculative.verify(c.get("target_dev", dev(c["target"])), dev(c["tokens"]), dev(c["parents"]), dev(c["u"]), dev(c["un"]),
                              draft_probs=c.get("draft_dev", dev(c["draft"])), row_start=None if uniform else dev(c["first"]),
                              max_nodes=max(max(c["nodes"]), 1), **more)


def check(c, got):
    path, n_path, nxt = (x.cpu().numpy() for x in got)
    target = c["target"].double().numpy()
    draft = None if c["draft"] is None else c["draft"].double().numpy()
    for r, t in enumerate(c["nodes"]):
        s = slice(int(c["first"][r]), int(c["first"][r]) + t)
        want, token = TR.verify(target[s], None if draft is None else draft[s], c["tokens"][s], c["parents"][s], c["u"][s], c["un"][r])
        assert n_path[r] == len(want) and list(path[r][:len(want)]) == want and (path[r][len(want):] == -1).all(), (r, want, path[r])
        assert nxt[r] == token, (r, token, nxt[r])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 1000, 4099, 32000, 50257])
def test_walks_match_the_reference(V, drafts, dtype):
    from paper_2511_06010_b200 import binding as M

    rng = np.random.default_rng(V)
    nodes = [5, 1, 12, 0, 33, 2] if V < 30000 else [6, 9]
    c = make(rng, nodes, V, drafts=drafts, dtype=dtype, pad=2, peak=3.0 if V < 100 else 5.0)
    check(c, run(c))
    assert M.device_status() == 0


@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("requests", [1, 3, 40, 200, 700])
def test_batches_and_wide_trees(requests, drafts):
    """Many requests, 64 nodes, one parent for all of them (63 tests at a node) or a chain."""
    rng = np.random.default_rng(requests)
    c = make(rng, [64 if requests < 100 else 8] * requests, 300, drafts=drafts, peak=1.0)
    for r in range(requests):
        s = slice(int(c["first"][r]) + 1, int(c["first"][r + 1]))
        if r % 3 == 0:
            c["parents"][s] = 0
            c["u"][s] = 1 - 2.0 ** -24 * (1 + rng.integers(0, 8))  # nearly always rejected
        elif r % 3 == 1:
            c["parents"][s] = np.arange(s.stop - s.start)
            c["u"][s] *= 0.3
    check(c, run(c, uniform=True))


@pytest.mark.parametrize("drafts", [True, False])
def test_borders(drafts):
    """Probabilities that are powers of two, random numbers on the borders between tokens, 0 and the largest below 1."""
    V, R = 64, 300
    rng = np.random.default_rng(1)
    c = make(rng, [3] * R, V, drafts=drafts)
    c["target"] = torch.full((3 * R, V), 1.0 / V)
    c["target"][::2] = torch.where(torch.arange(V) % 2 == 0, 2.0 / V, 0.0)
    if drafts:
        c["draft"] = torch.full((3 * R, V), 1.0 / V)
    c["tokens"] = rng.integers(0, V, 3 * R).astype(np.int32)
    c["u"] = rng.choice([0.0, 0.25, 0.5, 1 - 2.0 ** -24], 3 * R).astype(np.float32)
    c["un"] = np.where(np.arange(R) % 3 == 0, (np.arange(R) % V) / V, rng.choice([0.0, 1 - 2.0 ** -24], R)).astype(np.float32)
    check(c, run(c, uniform=True))


def test_odd_probabilities():
    """Rows of zeros, negative entries, NaN, all of the mass on one token, drafts equal to the target, the same token
    twice under one parent, tokens outside the vocabulary."""
    V = 100
    rng = np.random.default_rng(2)
    c = make(rng, [6] * 12, V)
    t, d = c["target"], c["draft"]
    t[0:6] = 0
    t[6:12, ::3] = -1.0
    t[12:18, 50:] = float("nan")
    t[18:24] = 0
    t[18:24, 37] = 1.0
    d[24:30] = t[24:30]
    c["u"][24:30] = 1.0  # (outside [0, 1): a test that fails although p = q, so that nothing is left)
    d[30:36] = 0
    d[36:42, 10:] = float("nan")
    c["parents"][43:48] = 0
    c["tokens"][43:48] = c["tokens"][43]
    c["u"][43:48] = 0.999
    c["tokens"][49:54] = [-1, V, 2**31 - 1, -2**31, 3]
    t[54:60] *= 5.0  # not normalised
    check(c, run(c, uniform=True))
    c["draft"] = None
    check(c, run(c, uniform=True))


@pytest.mark.parametrize("offset,pad", [(0, 3), (1, 0), (3, 5), (0, 4)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_lie_apart_and_unaligned(offset, pad, dtype):
    rng = np.random.default_rng(3)
    V = 1003
    c = make(rng, [9, 4, 7], V, dtype=dtype)
    for name in ("target", "draft"):
        wide = torch.full((20 * (V + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
        shift = offset if name == "target" else 0  # differently aligned
        view = wide[shift:shift + 20 * (V + pad)].view(20, V + pad)[:, :V]
        view.copy_(c[name])
        c[name + "_dev"] = view
    check(c, run(c))


def test_bad_rows_and_parents_are_reported():
    from paper_2511_06010_b200 import binding as M

    rng = np.random.default_rng(4)
    c = make(rng, [5, 5, 5], 50)
    c["parents"][[2, 8]] = [2, -7]
    got = run(c)
    assert M.device_status() == M.ERR_INVALID_ARG
    c["parents"][[2, 8]] = -1  # never tried
    check(c, got)
    good = c["first"].copy()
    for start in ([0, 5, 10, 16], [0, 5, -1, 15], [0, 9, 10, 15]):
        c["first"] = np.array(start, dtype=np.int32)
        run(c)
        assert M.device_status() == M.ERR_INVALID_ARG
    c["first"] = good
    check(c, run(c))


def test_the_emitted_tokens_follow_the_target():
    """The first token behind the root, accepted or drawn, is distributed as the target, whatever the draft: 40000 walks
    over five tokens, counts within five standard deviations."""
    from paper_2511_06010_b200 import speculative

    R, V = 40000, 5
    gen = torch.Generator().manual_seed(5)
    p, q = torch.tensor([0.1, 0.4, 0.05, 0.25, 0.2]), torch.tensor([0.3, 0.1, 0.3, 0.1, 0.2])
    parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32).repeat(R).cuda()
    target, draft = (x.expand(4 * R, V).contiguous().cuda() for x in (p, q))
    tokens = torch.multinomial(q.expand(4 * R, V), 1, generator=gen).squeeze(1).int().cuda()
    u, un = torch.rand(4 * R, generator=gen).cuda(), torch.rand(R, generator=gen).cuda()
    path, n_path, nxt = speculative.verify(target, tokens, parents, u, un, draft_probs=draft, max_nodes=4)
    first = torch.where(n_path > 1, tokens.view(R, 4).gather(1, path[:, 1:2].long().clamp(min=0)).squeeze(1), nxt)
    count = torch.bincount(first.long(), minlength=V).double().cpu()
    assert ((count - R * p).abs() < 5 * (R * p * (1 - p)).sqrt()).all(), count / R
    assert 0.3 < float((n_path > 1).double().mean()) < 1.0


def test_given_results_another_stream_and_a_captured_graph():
    rng = np.random.default_rng(6)
    c = make(rng, [16] * 5, 2000)
    from paper_2511_06010_b200 import speculative

    args = [c["target"].cuda()] + [torch.from_numpy(c[n]).cuda() for n in ("tokens", "parents", "u", "un")]
    draft = c["draft"].cuda()
    want = [x.clone() for x in speculative.verify(*args, draft_probs=draft)]
    check(c, want)
    out = [torch.empty_like(x) for x in want]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = speculative.verify(*args, draft_probs=draft, out=out, stream=side)
    side.synchronize()
    assert all(g.data_ptr() == o.data_ptr() and torch.equal(o, w) for g, o, w in zip(got, out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        speculative.verify(*args, draft_probs=draft, out=out)
    for o in out:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(out, want))
