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
