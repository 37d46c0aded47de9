"""Keeping accepted paths where a request's rows or its length are none: nothing of it moves."""
import numpy as np
import pytest
import torch

from tests.test_gpu_commit import clean_status, expected, filled, token_bytes  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

LENS, NODES, PATHS = [30, 26, 40], [7, 9, 12], [[0, 3, 6], [0, 2, 8], [0, 5, 11]]


def commit(st, table, length, start, B, kv_len_out):
    """By the C entry point, with the batch's number of rows."""
    from paper_2511_06010_b200 import binding as M

    path = np.full((3, 12), -1, dtype=np.int32)
    for r, p in enumerate(PATHS):
        path[r, :len(p)] = p
    s = M.shape(B, 2, 2, st.D, 1, 128, 1, q_len=12)
    M.kv_commit_paged(torch.from_numpy(path).cuda(), 12, torch.tensor([3, 3, 3], dtype=torch.int32).cuda(), start, 3, kv_len_out,
                      st.kv(table, length), s)


def check(fmt, length, start, B, done):
    """`done`: the requests that are moved; the others keep their bytes and lengths, and the error is reported."""
    from paper_2511_06010_b200 import binding as M

    st = filled(fmt, 9, 16, 2, 128, seed=4)
    before, table = token_bytes(st), np.arange(9, dtype=np.int32).reshape(3, 3)
    out = torch.full((3,), 77, dtype=torch.int32).cuda()
    commit(st, torch.from_numpy(table).cuda(), torch.tensor(length, dtype=torch.int32).cuda(),
           torch.tensor(start, dtype=torch.int32).cuda(), B, out)
    assert M.device_status() == (0 if len(done) == 3 else M.ERR_INVALID_ARG)
    assert out.tolist() == [LENS[r] - NODES[r] + 3 if r in done else length[r] for r in range(3)]
    n_path = [3 if r in done else 0 for r in range(3)]
    for got, want in zip(token_bytes(st), expected(before, table, LENS, NODES, PATHS, n_path, 16)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("start,B,done", [([0, 7, 16, 28], 28, [0, 1, 2]),
                                          ([0, 7, 16, 29], 29, [0, 1]),     # 13 nodes of 12
                                          ([0, 7, 16, 80], 100, [0, 1]),    # more than any tree has
                                          ([0, 7, 16, 28], 27, [0, 1]),     # behind the batch
                                          ([-1, 6, 15, 27], 28, [1, 2]),    # before it
                                          ([7, 0, 9, 21], 28, [1, 2])])     # descending
def test_bad_row_ranges(fmt, start, B, done):
    check(fmt, LENS, start, B, done)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("bad", [49, 1000, 2 ** 31 - 1, -1, -(2 ** 31)])
def test_bad_lengths(fmt, bad):
    check(fmt, [LENS[0], bad, LENS[2]], [0, 7, 16, 28], 28, [0, 2])
