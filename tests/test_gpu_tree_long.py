"""Attention of drafted trees over contexts of hundreds of millions of tokens, with sums that fp32 holds exactly."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests import tree_reference as TR
from tests.test_gpu_tree import clean_status  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("length,splits", [(2 ** 30, None), (2 ** 29 + 77, 1), (20_000_001, None)])
def test_contexts_of_hundreds_of_millions_of_tokens(fmt, length, splits):
    """Two pages stand for the two halves of the committed tokens, with values of 2 and of 4 in one of 64 tokens, 0 in the others,
    and keys of 0.  In one part the walk takes seconds.

    Bounds.  All probabilities are one power of two, so such a token adds 2 or 4 times that to the product, a step of 64 tokens 64
    times it to the row sum of its group (16 times to that of a part of a row), and every sum is a whole number below 2^24
    of those: exact.  What is left: in the result the division and the joins of parts, whose weights cancel (2^-18), and its
    rounding, 2^-8; in lse the logarithms and their sums, a few steps of 2^-19 for numbers of 16 to 32."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedKvStore
    from paper_2511_06010_b200.speculative import TreeAttention

    D, Hq, page, T = 64, 2, 32768, 5
    gen = torch.Generator().manual_seed(6)
    pages = -(-length // page)
    last = length - (pages - 1) * page  # tokens of the last page, the tree among them
    half = (pages - 1) // 2
    table = torch.cat([torch.zeros(half), torch.ones(pages - 1 - half), torch.full((1,), 2)]).to(torch.int32).reshape(1, -1)
    st = PagedKvStore.empty(3, page, 1, D, fmt)
    sign = (torch.randint(0, 2, (D,), generator=gen) * 2 - 1).to(torch.bfloat16)
    v = torch.zeros(2 * page + last, 1, D, dtype=torch.bfloat16)
    some = torch.arange(page) % 64 == 0
    v[:page][some] = 2 * sign
    v[page:2 * page][some] = 4 * sign
    for x in (v[:page], v[page:2 * page]):  # (a 6 in each group of 32 dimensions: 4 bits hold 2 and 4 with a scale of 1)
        x[:, 0, ::32][some] = 6.0
    lens = torch.tensor([2 * page + last], dtype=torch.int32).cuda()
    st.append(None, torch.zeros_like(v).cuda(), v.cuda(), torch.tensor([[0, 1, 2]], dtype=torch.int32).cuda(), lens,
              row_start=torch.tensor([0, 2 * page + last], dtype=torch.int32).cuda())
    q = R.make_bf16((T, Hq, D), gen)
    parents = np.array([-1, 0, 0, 1, 3], dtype=np.int32)
    at = TreeAttention(T, Hq, 1, D, length, 1, T, fmt=fmt, n_unique_splits=splits)
    out, lse = at(q.cuda(), st, table.cuda(), torch.tensor([length], dtype=torch.int32).cuda(), torch.from_numpy(parents).cuda())
    assert M.device_status() == 0
    n = length - T + TR.ancestors(parents).sum(1)
    want = (half * 2.0 + (pages - 1 - half) * 4.0) * (page // 64) * sign.double().numpy() / n[:, None]
    rest = np.arange(D) % 32 != 0
    got = R.to_f64(out)
    tol = np.abs(want) * (2.0 ** -8 + 2.0 ** -18)
    assert (tol < np.abs(want) / 100).all()
    assert (np.abs(got - want[:, None]) <= tol[:, None])[..., rest].all(), np.abs(got - want[:, None])[..., rest].max()
    assert (np.abs(lse.double().cpu().numpy() - np.log(n)[:, None]) <= 2.0 ** -17).all()
