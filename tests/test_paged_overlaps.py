"""Buffers of a paged append or gather that overlap are refused (addresses are never dereferenced here: every call
is refused); neighbours in one allocation are not."""
import pytest
import torch

Q, K, V, OUT, KP, VP, A = (i << 32 for i in range(1, 8))  # far from one another
HQ, HKV, D, B, PAGE, PAGES = 8, 2, 128, 4, 64, 10
Q_ROW, KV_ROW = HQ * D * 2, HKV * D * 2  # bytes
POOL = {0: PAGES * PAGE * KV_ROW, 1: PAGES * HKV * PAGE // 16 * 18 * D}


@pytest.fixture(scope="module")
def M():
    from paper_2511_06010_b200 import build

    build.build()
    from paper_2511_06010_b200 import binding

    return binding


def _refused(M, call, text):
    with pytest.raises(M.MoskaError) as e:
        call()
    assert e.value.status == M.ERR_INVALID_ARG and text in M.last_error(), M.last_error()


def _cases(fmt):
    """(argument, address, message): one buffer at the first or at the last piece of another."""
    wide = (HQ + 2 * HKV) * D * 2  # bytes between rows of q, k and v
    span = {Q: 3 * wide + Q_ROW, K: 3 * wide + KV_ROW, V: 3 * wide + KV_ROW, OUT: B * Q_ROW, KP: POOL[fmt], VP: POOL[fmt]}
    names = {Q: "q", K: "k", V: "v", OUT: "q_out", KP: "k_pages", VP: "v_pages"}
    for moved, others in ((OUT, (Q, K, V, KP, VP)), (Q, (KP, VP)), (K, (KP, VP)), (V, (KP, VP)), (KP, (VP,))):
        for other in others:
            if VP in (moved, other) and fmt == 1:
                continue
            for at in (other, other + span[other] - 16, other - span[moved] + 16):
                yield names[moved], at, f"{names[moved]} overlaps {names[other]}"


@pytest.mark.parametrize("fmt", [0, 1])
def test_overlapping_buffers_of_append_are_refused(M, fmt):
    s = M.shape(B, HQ, HKV, D, 1, 128, 1)
    stride = (HQ + 2 * HKV) * D
    for name, at, text in _cases(fmt):
        a = dict(dict(q=Q, k=K, v=V, q_out=OUT, k_pages=KP, v_pages=VP), **{name: at})
        kv = M.paged_kv(fmt, PAGE, PAGES, 4, a["k_pages"], a["v_pages"], A, A)
        _refused(M, lambda: M.kv_append_paged(a["q"], stride, a["k"], stride, a["v"], stride, A, A, 10, D, 0, None, B, a["q_out"],
                                              kv, s, stream=0), text)


@pytest.mark.parametrize("fmt", [0, 1])
def test_overlapping_buffers_of_gather_are_refused(M, fmt):
    s = M.shape(B, HKV, HKV, D, 1, 128, 1)
    kv = M.paged_kv(fmt, PAGE, PAGES, 4, KP, VP, A, A)
    rows = B * KV_ROW
    for k, v, text in ((K, K, "k_out overlaps v_out"), (K, K + rows - 16, "k_out overlaps v_out"),
                       (K + rows - 16, K, "k_out overlaps v_out"), (KP + POOL[fmt] - 16, V, "k_out overlaps k_pages"),
                       (K, KP + 16, "v_out overlaps k_pages"), (K, KP - rows + 16, "v_out overlaps k_pages")):
        _refused(M, lambda: M.kv_gather_paged(None, B, k, v, kv, s, stream=0), text)
    if fmt == 0:
        for k, v, text in ((VP, V, "k_out overlaps v_pages"), (K, VP + POOL[0] - 16, "v_out overlaps v_pages")):
            _refused(M, lambda: M.kv_gather_paged(None, B, k, v, kv, s, stream=0), text)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_neighbours_in_one_allocation_are_taken(fmt):
    """q_out, the projection's rows, both results of gather and the pools one behind the other, nothing between."""
    from paper_2511_06010_b200 import binding as M
    from paper_2511_06010_b200.paged import PagedKvStore

    page, pages = 16, 3
    pool = pages * page * HKV * D if fmt == "bf16" else pages * HKV * 18 * D // 2  # in bf16 elements
    sizes = [B * HQ * D, B * (HQ + 2 * HKV) * D, B * HKV * D, B * HKV * D, pool] + ([pool] if fmt == "bf16" else [])
    memory = torch.zeros(sum(sizes), dtype=torch.bfloat16, device="cuda")
    q_out, qkv, ko, vo, *pools = torch.split(memory, sizes)
    qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(51)))
    q_out, ko, vo = q_out.view(B, HQ, D), ko.view(B, HKV, D), vo.view(B, HKV, D)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.view(B, -1).split([HQ * D, HKV * D, HKV * D], 1))
    if fmt == "bf16":
        st = PagedKvStore(*(p.view(pages, page, HKV, D) for p in pools))
    else:
        st = PagedKvStore(pages4=pools[0].view(torch.uint8).view(pages, HKV, 1, 18 * D))
    table, length = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.full((1,), B, dtype=torch.int32).cuda()
    before = qkv.clone()
    st.append(q, k, v, table, length, q_len=B, q_out=q_out)
    st.gather(table, length, B, q_len=B, k_out=ko, v_out=vo)
    assert M.device_status() == 0 and torch.equal(q_out, q) and torch.equal(qkv, before)
    if fmt == "bf16":
        assert torch.equal(ko, k) and torch.equal(vo, v)
    else:
        from tests import paged_reference as R

        assert torch.equal(ko.cpu(), torch.from_numpy(R.held32(k.float().cpu().numpy())).to(torch.bfloat16))
    with pytest.raises(M.MoskaError):
        st.gather(table, length, B, q_len=B, k_out=ko, v_out=ko)
    with pytest.raises(M.MoskaError):
        st.append(q, k, v, table, length, q_len=B, q_out=memory[B * HQ * D - 8:][:B * HQ * D].view(B, HQ, D))
