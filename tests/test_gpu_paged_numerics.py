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
