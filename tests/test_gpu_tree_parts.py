"""Attention of drafted trees: parts that a context may be cut into, and repeated calls."""
import pytest
import torch

from tests.test_gpu_tree import case, check, clean_status  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [148, 10 ** 6, 2 ** 31 - 1])
def test_more_parts_than_there_are(fmt, splits):
    c = case(fmt, 128, 16, 2, 32, [900, 35, 2500], [24] * 3, seed=14, splits=splits)
    out, lse = c["attention"](c["q"].cuda(), c["store"], c["table"], c["length"], c["up"])
    check(c, out, lse, only=lambda r, i: i % 5 == 0)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("D,Hq,nodes", [(128, 64, 60), (64, 16, 20), (128, 32, 8)])
def test_the_same_call_gives_the_same_bits(fmt, D, Hq, nodes):
    """No order of CTAs, warps or atomics shows."""
    lens = [3000, 1700, 900, 64 + nodes, 2048]
    c = case(fmt, D, Hq, 8 if Hq > 16 else 4, 64, lens, [nodes] * 5, seed=15)
    q = c["q"].cuda()
    first = [x.clone() for x in c["attention"](q, c["store"], c["table"], c["length"], c["up"])]
    for _ in range(20):
        c["attention"].out.fill_(7.0)
        out, lse = c["attention"](q, c["store"], c["table"], c["length"], c["up"])
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
