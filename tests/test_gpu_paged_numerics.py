"""Attention over pages where the arithmetic is near its limits: query rows and softmax scales at the ends of
fp32's range, long contexts whose weight lies in many small probabilities."""
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


def _filled(fmt, k, v, lens, page=32):
    """A store holding the rows k, v [sum(lens)][Hkv][D] (bf16, CPU) of contexts one after another; -> store,
    page table and lengths on the GPU."""
    from paper_2511_06010_b200.paged import PagedKvStore

    need = [-(-n // page) for n in lens]
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = torch.arange(sum(need[:r]), sum(need[:r]) + n)
    st = PagedKvStore.empty(sum(need), page, k.shape[1], k.shape[2], fmt)
    for pool in (st.k_pages, st.v_pages) if fmt == "bf16" else (st.pages4,):
        pool.view(torch.uint8).fill_(0xFF)  # behind the contexts: NaN everywhere
    length = torch.tensor(lens, dtype=torch.int32).cuda()
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    st.append(None, k.cuda(), v.cuda(), table.cuda(), length, row_start=first)
    return st, table.cuda(), length


def _held(x, fmt):
    return R.to_f64(x) if fmt == "bf16" else R.held32(x.float().numpy())


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,T", [(128, 4, 1), (128, 4, 4), (64, 4, 1)])
@pytest.mark.parametrize("scale", [1e-40, 1e-8, 0.125])
@pytest.mark.parametrize("q_scale", [0.0, 1e-38, 1e-30])
def test_zero_and_tiny_query_rows_with_small_softmax_scales(fmt, D, Hq, T, scale, q_scale):
    """A hidden token has weight 0 whatever the row's scores are multiplied with."""
    from paper_2511_06010_b200.paged import PagedAttention

    lens = [4, 21, 63, 200, 333]
    gen = torch.Generator().manual_seed(31)
    k, v = (R.make_bf16((sum(lens), 1, D), gen) for _ in range(2))
    st, table, length = _filled(fmt, k, v, lens)
    q = R.make_bf16((len(lens) * T, Hq, D), gen, q_scale)
    attention = PagedAttention(len(lens) * T, Hq, 1, D, max(lens), fmt=fmt, q_len=T, n_unique_splits=2)
    attention.scale = scale
    out, lse = attention(q.cuda(), st, table, length)
    k64, v64, at = _held(k, fmt), _held(v, fmt), 0
    for r, n in enumerate(lens):
        for i in range(T):
            m = n - (T - 1 - i)
            o, l, o_tol, l_tol = R.attend(R.to_f64(q[r * T + i]), k64[at:at + m], v64[at:at + m], scale, fmt)
            assert (np.abs(R.to_f64(out[r * T + i]) - o) <= o_tol).all(), (r, i)
            assert (np.abs(lse[r * T + i].double().cpu().numpy() - l) <= l_tol).all(), (r, i)
        at += n


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_the_largest_query_rows_on_keys_of_zero(fmt):
    """Scores of exactly 0: the mean of the values, however large the row and the softmax scale are."""
    from paper_2511_06010_b200.paged import PagedAttention

    lens, D = [5, 64, 130], 128
    gen = torch.Generator().manual_seed(32)
    v = R.make_bf16((sum(lens), 1, D), gen)
    st, table, length = _filled(fmt, torch.zeros_like(v), v, lens)
    q = torch.full((3, 2, D), 2.0 ** 126, dtype=torch.bfloat16)
    attention = PagedAttention(3, 2, 1, D, max(lens), fmt=fmt, n_unique_splits=1)
    attention.scale = 64.0
    out, lse = attention(q.cuda(), st, table, length)
    v64, at = _held(v, fmt), 0
    for r, n in enumerate(lens):
        o, l, o_tol, l_tol = R.attend(np.zeros((2, D)), np.zeros((n, 1, D)), v64[at:at + n], 1.0, fmt)
        assert (np.abs(R.to_f64(out[r]) - o) <= o_tol).all() and (np.abs(lse[r].double().cpu().numpy() - l) <= l_tol).all()
        at += n


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,T", [(128, 1, 1), (128, 4, 4), (64, 8, 1)])
@pytest.mark.parametrize("where", ["first", "last"])
def test_many_small_probabilities_beside_a_few_large_ones(fmt, D, Hq, T, where):
    """Four tokens 2^26.5 times as probable as each of 2^18 others (one in every unit of the first or the last
    pass, so that every warp meets one): the others' values are still there.

    Bound.  Weights are rounded to 16 bits: bf16 half a step, 2^-8 of a weight.  f16 holds weights relative to
    a reference at most 2^-7 of the largest: half its smallest step there, 2^-25 2^-7 of the largest, for
    every token; above that half a step, 2^-11.  The scores' own error (2^-21 of 18.4 and the exponential's
    2^-22): below 2^-16 of a weight.  A warp adds to its fp32 sums once for 64 tokens: each time at most 2^-23 of
    the sum in the product (the MMA may cut off), 2^-24 in the row sum.  The output's rounding: 2^-8."""
    from paper_2511_06010_b200.paged import PagedAttention

    n = (1 << 18) + 7
    k, v = torch.zeros(n, 1, D, dtype=torch.bfloat16), torch.ones(n, 1, D, dtype=torch.bfloat16)
    peak = [64 * i + 3 for i in range(4)] if where == "first" else [n - T - 40 - 64 * i for i in range(4)]
    k[peak] = 26.5 * np.log(2.0) / np.sqrt(D)
    v[peak] = 0
    st, table, length = _filled(fmt, k, v, [n], page=256)
    attention = PagedAttention(T, Hq, 1, D, n, fmt=fmt, q_len=T, n_unique_splits=1)
    out, lse = attention(torch.ones(T, Hq, D, dtype=torch.bfloat16, device="cuda"), st, table, length)
    score = _held(k[peak[0]], fmt).sum() * attention.scale
    p, adds = np.exp(-score), -(-n // 64)
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
