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


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("dense", [False, True])
def test_a_step_filled_up_with_nodes_that_none_sees(fmt, dense):
    """Smaller trees in a step of larger ones: a request's rows are what they are without the others' fill, and the step is the
    same with a second stream."""
    from paper_2511_06010_b200 import binding as M
    from tests.test_gpu_tree import _layer_case

    w, c, sh, q, layer = _layer_case(fmt, False, dense)
    up = c["up"].view(-1, 12).clone()
    up[:, 7:] = -1  # five nodes of fill
    parents = up.reshape(-1).contiguous()
    step = lambda table, length, two: layer.step_paged(q, sh.k_shared, sh.v_shared, c["store"], table, length,  # noqa: E731
                                                       two_streams=two, parents=parents).clone()
    out = step(c["table"], c["length"], False)
    assert torch.equal(step(c["table"], c["length"], True), out)
    if fmt == "bf16":  # other rows in the places of the fill
        for r, n in ((0, 256), (1, 40), (3, 333)):
            for t in range(n - 5, n):
                page = int(c["table"][r, t // 64])
                c["store"].k_pages[page, t % 64] = float("inf")
                c["store"].v_pages[page, t % 64] = float("nan")
    else:
        gen = torch.Generator().manual_seed(3)
        k, v = (100 * torch.randn(20, w.Hkv, w.D, generator=gen).bfloat16().cuda() for _ in range(2))
        c["store"].append(None, k, v, c["table"], c["length"], q_len=5)
    again = step(c["table"], c["length"], False)
    assert torch.equal(again.view(-1, 12, w.Hq, w.D)[:, :7], out.view(-1, 12, w.Hq, w.D)[:, :7])
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_the_step_over_a_shared_store_in_fp8(fmt):
    """What its stages give one by one."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200 import workloads as W
    from tests.test_gpu_tree import _layer_case

    w, c, sh, q, layer = _layer_case(fmt, False, True)
    sf8 = W.quantize_shared_store_fp8(sh)
    out = layer.step_paged(q, None, None, c["store"], c["table"], c["length"], sf8=sf8, parents=c["up"]).clone()
    layer.o_part.fill_(float("nan"))
    layer.lse_part.fill_(float("nan"))
    layer.unique_paged(q, c["store"], c["table"], c["length"], parents=c["up"])
    layer.shared_fp8(q, sf8)
    layer.merge()
    assert torch.equal(layer.out, out) and torch.isfinite(out).all()
    other = layer.step_paged(q, sh.k_shared, sh.v_shared, c["store"], c["table"], c["length"], parents=c["up"])
    assert not torch.equal(other, out)  # (the bf16 store)
    assert M.device_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("splits", [1, 64])
def test_no_lse_and_rows_before_the_first_request(fmt, splits):
    """lse_out may be NULL; rows before row_start[0] are padding like those behind the last request."""
    from paper_2511_06010_b200 import binding as M

    lens, nodes = [700, 90, 300], [20, 5, 11]
    c = case(fmt, 128, 16, 2, 32, lens, nodes, seed=16, splits=splits)
    at, q, up = c["attention"], c["q"].cuda(), c["up"]
    want = [x.clone() for x in at(q, c["store"], c["table"], c["length"], up, row_start=c["start"])]
    check(c, *want, only=lambda r, i: i % 4 == 0)
    kv = c["store"].kv(c["table"], c["length"])
    at.out.fill_(5.0)
    M.tree_attn(q, kv, up, c["start"], 3, at.out, None, at.scale, at.shape, at.ws)
    assert torch.equal(at.out, want[0])
    pad = 6
    q2, up2 = torch.cat([q.new_full((pad, 16, 128), float("nan")), q]), torch.cat([up.new_full((pad,), 99), up])
    out, lse = q2.new_full(q2.shape, 3.0), torch.full((pad + c["rows"], 16), 4.0, device="cuda")
    s = M.shape(pad + c["rows"], 16, 2, 128, 1, 128, 1, n_unique_splits=splits, q_len=20)
    M.tree_attn(q2, kv, up2, c["start"] + pad, 3, out, lse, at.scale, s, at.ws)
    assert torch.equal(out[pad:], want[0]) and torch.equal(lse[pad:], want[1])
    assert (out[:pad] == 3.0).all() and (lse[:pad] == 4.0).all()
    assert M.device_status() == 0
