"""Attention of drafted trees where its arithmetic is near its limits."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import tree_reference as TR
from tests.test_gpu_paged_numerics import _filled, _held, clean_status  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


def chain(T):
    return np.arange(-1, T - 1, dtype=np.int32)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,T", [(128, 1, 1), (128, 4, 8), (128, 4, 16), (128, 8, 16), (64, 8, 20), (64, 2, 3)])
@pytest.mark.parametrize("where", ["first", "last"])
def test_many_small_probabilities_beside_a_few_large_ones(fmt, D, Hq, T, where):
    """Four tokens 2^26.5 times as probable as each of 2^18 others, in the first or the last 64 committed tokens and 16 apart, so
    that each part of a row meets one: the others' values are still there.

    Bound.  Weights are rounded to 16 bits: bf16 half a step, 2^-8 of a weight.  f16 holds weights relative to a reference of
    at most 2^-7 of the largest: half its smallest step there, 2^-25 2^-7 of the largest, for every token; above that
    half a step, 2^-11.  The scores' own error (2^-21 of 18.4 and the exponential's 2^-22): below 2^-16 of a weight.
    The product adds to its fp32 sums once for 16 tokens: each time at most 2^-23 of the sum (it may cut off), the row sum
    2^-24 no more often.  The output's rounding: 2^-8."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.speculative import TreeAttention

    n = (1 << 18) + 7
    k, v = torch.zeros(n, 1, D, dtype=torch.bfloat16), torch.ones(n, 1, D, dtype=torch.bfloat16)
    peak = [16 * i + 3 for i in range(4)] if where == "first" else [n - T - 90 + 16 * i for i in range(4)]
    k[peak] = 26.5 * np.log(2.0) / np.sqrt(D)
    v[peak] = 0
    st, table, length = _filled(fmt, k, v, [n], page=256)
    attention = TreeAttention(T, Hq, 1, D, n, 1, T, fmt=fmt, n_unique_splits=1)
    out, lse = attention(torch.ones(T, Hq, D, dtype=torch.bfloat16, device="cuda"), st, table, length, torch.from_numpy(chain(T)).cuda())
    assert M.device_status() == 0
    score = _held(k[peak[0]], fmt).sum() * attention.scale
    p, adds = np.exp(-score), -(-n // 16)
    for i in range(T):
        others = n - (T - 1 - i) - 4
        total = 4 + others * p
        want = others * p / total
        lost = 0.0 if fmt == "bf16" else others * 2.0 ** -32 / total
        tol = lost + want * ((2.0 ** -8 if fmt == "bf16" else 2.0 ** -11) + 2.0 ** -16 + 1.5 * adds * 2.0 ** -23)
        tol += 2.0 ** -8 * (want + tol)
        got = R.to_f64(out[i])
        assert (np.abs(got - want) <= tol).all(), (i, np.abs(got - want).max(), want, tol)
        assert (np.abs(lse[i].double().cpu().numpy() - (score + np.log(total))) <= 2.0 ** -18 * score + adds * 2.0 ** -24).all()


def with_scales(D, page, lens, T, gen, key_scales, value_scales, value_codes=16):
    """A 4-bit store of random codes whose tokens' scales are drawn from the given ones; tables and lengths.  Value codes are
    below value_codes or its negatives."""
    from paper_2511_06010_b200.paged import PagedKvStore

    need = [-(-n // page) for n in lens]
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = torch.arange(sum(need[:r]), sum(need[:r]) + n)
    st = PagedKvStore.empty(sum(need), page, 2, D, "fp4")
    code = torch.randint(0, 256, st.pages4.shape, generator=gen, dtype=torch.uint8)
    if value_codes < 16:
        low = torch.randint(0, value_codes, (2, *st.pages4.shape[:-1], 8 * D), generator=gen, dtype=torch.uint8)
        sign = torch.randint(0, 2, low.shape, generator=gen, dtype=torch.uint8) * 8
        code[..., 8 * D:16 * D] = (low[0] + sign[0]) | (low[1] + sign[1]) << 4
    for at, scales in ((16 * D, key_scales), (17 * D, value_scales)):
        pick = torch.randint(0, len(scales), (*st.pages4.shape[:-1], D // 2), generator=gen)
        code[..., at:at + D] = torch.tensor(scales, dtype=torch.float16)[pick].view(torch.uint8).reshape(*st.pages4.shape[:-1], D)
    st.pages4.copy_(code)
    return st, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()


def check(st, table, lens, T, parents, q, attention, out, lse):
    k64, v64 = R.unpack(st.pages4)
    for r, n in enumerate(lens):
        k, v = R.context(k64, v64, table[r].cpu().numpy(), n)
        sees = TR.visible(parents[r * T:(r + 1) * T], n)
        for i in range(T):
            o, l, o_tol, l_tol = R.attend(R.to_f64(q[r * T + i]), k[sees[i]], v[sees[i]], attention.scale, "fp4")
            assert (np.abs(R.to_f64(out[r * T + i]) - o) <= o_tol).all(), (r, i)
            assert (np.abs(lse[r * T + i].double().cpu().numpy() - l) <= l_tol).all(), (r, i, lse[r * T + i], l)


FORMS = [(64, 8, 7), (128, 8, 5), (128, 8, 13), (64, 2, 40), (128, 16, 20)]  # D, Hq (of 2 KV heads), nodes


@pytest.mark.parametrize("D,Hq,T", FORMS)
@pytest.mark.parametrize("scales,q_scale", [([10912.0, 10920.0, 20000.0, 65504.0], 2.0 ** -17), ([1.0, 30000.0, 2.0 ** -24], 2.0 ** -15),
                                            ([2.0 ** -24, 3 * 2.0 ** -24, 1000 * 2.0 ** -24, 2.0 ** -14], 2.0 ** 13)])
@pytest.mark.parametrize("splits", [1, 3])
def test_key_scales_of_any_size(D, Hq, T, scales, q_scale, splits):
    """Scales larger than appends write, whose products with a code no f16 number holds, and the smallest there are."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.speculative import TreeAttention

    gen, rng, lens = torch.Generator().manual_seed(D + T), np.random.default_rng(T), [50, 300, 130]
    st, table, length = with_scales(D, 16, lens, T, gen, scales, [0.5, 1.0, 1.25])
    parents = np.concatenate([TR.random_tree(rng, T) for _ in lens])
    q = R.make_bf16((len(lens) * T, Hq, D), gen, q_scale)
    attention = TreeAttention(len(lens) * T, Hq, 2, D, max(lens), len(lens), T, fmt="fp4", n_unique_splits=splits)
    out, lse = attention(q.cuda(), st, table, length, torch.from_numpy(parents).cuda())
    assert M.device_status() == 0
    check(st, table, lens, T, parents, q, attention, out, lse)


@pytest.mark.parametrize("D,Hq,T", FORMS)
@pytest.mark.parametrize("splits", [1, 3])
def test_value_scales_above_what_appends_write(D, Hq, T, splits):
    """Where the product is finite, a value counts with its probability like any other, drafted tokens' too; one that is not
    spoils its own dimensions of the rows that see it, and nothing else."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.speculative import TreeAttention

    gen, rng, lens = torch.Generator().manual_seed(D + T + 1), np.random.default_rng(T + 1), [50, 300, 130]
    st, table, length = with_scales(D, 16, lens, T, gen, [0.25, 0.125], [1.0, 10920.0, 20000.0], value_codes=6)  # 3 at most
    parents = np.concatenate([TR.random_tree(rng, T) for _ in lens])
    q, up = R.make_bf16((len(lens) * T, Hq, D), gen), torch.from_numpy(parents).cuda()
    attention = TreeAttention(len(lens) * T, Hq, 2, D, max(lens), len(lens), T, fmt="fp4", n_unique_splits=splits)
    out, lse = (x.clone() for x in attention(q.cuda(), st, table, length, up))
    assert M.device_status() == 0
    check(st, table, lens, T, parents, q, attention, out, lse)
    j = T // 2  # a node of the second request: its value 120000 in four dimensions of the second head
    token = lens[1] - T + j
    pool = st.pages4.cpu().numpy()
    _, vb, _, vs, _ = R.byte_map(D)
    block, t = pool[int(table[1, token // 16]), 1, 0], token % 16
    block[vb[t, :4]] = 0x77
    block[vs[t, 0]:vs[t, 0] + 2] = np.array([20000.0], dtype=np.float16).view(np.uint8)
    st.pages4.copy_(torch.from_numpy(pool))
    out2, lse2 = attention(q.cuda(), st, table, length, up)
    sees = torch.zeros(len(lens) * T, dtype=torch.bool)
    sees[T:2 * T] = torch.from_numpy(TR.ancestors(parents[T:2 * T])[:, j])
    half = Hq // 2
    assert torch.equal(out2[~sees], out[~sees]) and torch.equal(out2[:, :half], out[:, :half]) and torch.equal(lse2, lse)
    assert not torch.isfinite(out2[sees][:, half:, :4]).any() and torch.isfinite(out2[sees][:, half:, 4:]).all()
    k, v = R.context(*R.unpack(st.pages4), table[1].cpu().numpy(), lens[1])
    seen = TR.visible(parents[T:2 * T], lens[1])
    for i in np.flatnonzero(sees[T:2 * T].numpy()):
        o, _, o_tol, _ = R.attend(R.to_f64(q[T + i]), k[seen[i]], v[seen[i]], attention.scale, "fp4")
        assert (np.abs(R.to_f64(out2[T + i]) - o) <= o_tol)[half:, 4:].all(), i


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,T", [(128, 4, 5), (64, 8, 16), (128, 2, 24)])
@pytest.mark.parametrize("scale", [1e-45, 1e-40, 1e-8, 0.125])
@pytest.mark.parametrize("q_scale", [0.0, 1e-38, 1e-30])
def test_zero_and_tiny_query_rows_with_small_softmax_scales(fmt, D, Hq, T, scale, q_scale):
    """A hidden token has weight 0 whatever the row's scores are multiplied with."""
    from paper_2511_06010_b200.speculative import TreeAttention

    gen, rng, lens = torch.Generator().manual_seed(41), np.random.default_rng(41), [T, 40, 200, 333]
    k, v = (R.make_bf16((sum(lens), 1, D), gen) for _ in range(2))
    st, table, length = _filled(fmt, k, v, lens)
    parents = np.concatenate([TR.random_tree(rng, T) for _ in lens])
    q = R.make_bf16((len(lens) * T, Hq, D), gen, q_scale)
    attention = TreeAttention(len(lens) * T, Hq, 1, D, max(lens), len(lens), T, fmt=fmt, n_unique_splits=2)
    attention.scale = scale
    out, lse = attention(q.cuda(), st, table, length, torch.from_numpy(parents).cuda())
    k64, v64, at = _held(k, fmt), _held(v, fmt), 0
    for r, n in enumerate(lens):
        sees = TR.visible(parents[r * T:(r + 1) * T], n)
        for i in range(T):
            o, l, o_tol, l_tol = R.attend(R.to_f64(q[r * T + i]), k64[at:at + n][sees[i]], v64[at:at + n][sees[i]], scale, fmt)
            assert (np.abs(R.to_f64(out[r * T + i]) - o) <= o_tol).all(), (r, i)
            assert (np.abs(lse[r * T + i].double().cpu().numpy() - l) <= l_tol).all(), (r, i)
        at += n


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("nodes", [3, 24])
@pytest.mark.parametrize("scale", [64.0, 3e38])
def test_the_largest_query_rows_and_softmax_scales_on_keys_of_zero(fmt, nodes, scale):
    """Scores of exactly 0: the mean of the values, however large the row and the softmax scale are."""
    from paper_2511_06010_b200.speculative import TreeAttention

    lens, D = [nodes, 64, 130], 128
    gen = torch.Generator().manual_seed(42)
    v = R.make_bf16((sum(lens), 1, D), gen)
    st, table, length = _filled(fmt, torch.zeros_like(v), v, lens)
    q = torch.full((3 * nodes, 4, D), 2.0 ** 126, dtype=torch.bfloat16)
    attention = TreeAttention(3 * nodes, 4, 1, D, max(lens), 3, nodes, fmt=fmt, n_unique_splits=1)
    attention.scale = scale
    out, lse = attention(q.cuda(), st, table, length)  # chains
    v64, at = _held(v, fmt), 0
    for r, n in enumerate(lens):
        for i in range(nodes):
            m = n - nodes + 1 + i
            o, l, o_tol, l_tol = R.attend(np.zeros((4, D)), np.zeros((m, 1, D)), v64[at:at + m], 1.0, fmt)
            row = r * nodes + i
            assert (np.abs(R.to_f64(out[row]) - o) <= o_tol).all() and (np.abs(lse[row].double().cpu().numpy() - l) <= l_tol).all()
        at += n
