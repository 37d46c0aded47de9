"""Calls on a stream that is not the current one: what memory they may use, and when it may be used again."""
import gc

import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu

BUSY = 40_000_000  # clock cycles: some 20 ms that a stream is kept busy for


@pytest.fixture(autouse=True)
def clean_status():
    from paper_2511_06010_b200 import binding as M

    gc.collect()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    M.device_status()
    yield
    torch.cuda.synchronize()
    assert M.device_status() == 0


def _case(fmt, R_=3, T=64, Hq=16, Hkv=2, D=128, page=32):
    """A store and rows for it, T to each of R_ requests; results of some hundred KB."""
    from paper_2511_06010_b200.paged import PagedKvStore

    gen = torch.Generator().manual_seed(41)
    pages = -(-T // page)
    st = PagedKvStore.empty(R_ * pages, page, Hkv, D, fmt)
    table = torch.arange(R_ * pages, dtype=torch.int32).reshape(R_, pages).cuda()
    length = torch.full((R_,), T, dtype=torch.int32).cuda()
    q, k, v = (R.make_bf16((R_ * T, h, D), gen).cuda() for h in (Hq, Hkv, Hkv))
    return st, table, length, q, k, v


def _freed_while_in_use(like):
    """The address of a block that torch's current stream has been given back but is still going to write to."""
    torch.cuda._sleep(BUSY)
    t = torch.empty_like(like)
    t.fill_(3.0)
    return t.data_ptr()


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_results_made_on_another_stream_are_not_memory_of_the_current_one(fmt, raw):
    st, table, length, q, k, v = _case(fmt)
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    want = st.append(q, k, v, table, length, q_len=64)
    want_kv = st.gather(table, length, k.shape[0], q_len=64)
    torch.cuda.synchronize()
    in_use = [_freed_while_in_use(q)]
    got = st.append(q, k, v, table, length, q_len=64, stream=stream)
    assert got.data_ptr() not in in_use and torch.cuda.current_stream() != side
    in_use += [_freed_while_in_use(k) for _ in range(2)]
    got_kv = st.gather(table, length, k.shape[0], q_len=64, stream=stream)
    assert not {t.data_ptr() for t in got_kv} & set(in_use)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(got_kv, want_kv))


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_what_a_call_on_another_stream_uses_may_be_dropped(fmt):
    """Results and inputs dropped while the stream is busy: their memory is not handed out before it is done."""
    st, table, length, q, k, v = _case(fmt)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    inputs = [t.clone() for t in (q, k, v, table, length)]
    torch.cuda.current_stream().synchronize()
    used = {t.data_ptr() for t in inputs}
    out = st.append(*inputs, q_len=64, stream=side)
    pair = st.gather(inputs[3], inputs[4], k.shape[0], q_len=64, stream=side)
    used |= {t.data_ptr() for t in (out, *pair)}
    del inputs, out, pair
    fresh = [torch.empty_like(t) for t in (q, q, k, k, k, k, v, table, length)]
    assert not side.query(), "the stream was done too early to show anything"
    assert not used & {t.data_ptr() for t in fresh}
    torch.cuda.synchronize()


def test_the_callers_stream_may_go_on_with_a_result_and_drop_it():
    """The memory of a result belongs to the stream that wrote it: that stream gets it back only when the one
    that the call was made from is done with it."""
    st, table, length, q, k, v = _case("bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = st.append(q, k, v, table, length, q_len=64, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(BUSY)
    copy = out.clone()
    address = out.data_ptr()
    del out
    with torch.cuda.stream(side):
        fresh = [torch.empty_like(q) for _ in range(4)]
    assert not torch.cuda.current_stream().query(), "the stream was done too early to show anything"
    assert address not in {t.data_ptr() for t in fresh}
    torch.cuda.synchronize()
    assert torch.equal(copy, q)  # no rotation: a copy of the queries


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_an_attention_dropped_while_it_runs_on_another_stream(fmt):
    from paper_2511_06010_b200.paged import PagedAttention

    st, table, length, q, k, v = _case(fmt)
    st.append(None, k, v, table, length, q_len=64)
    rows = q[:3].contiguous()
    side = torch.cuda.Stream()
    attention = PagedAttention(3, 16, 2, 128, 64, fmt=fmt, n_unique_splits=2)
    want = [t.clone() for t in attention(rows, st, table, length)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    out, lse = attention(rows, st, table, length, stream=side)
    like = [torch.empty_like(t, device="meta") for t in (attention.ws, attention.out, attention.lse)]
    used = {t.data_ptr() for t in (attention.ws, attention.out, attention.lse)}
    kept = (out, lse)
    del attention, out, lse
    fresh = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in like for _ in range(3)]
    assert not side.query() and not used & {t.data_ptr() for t in fresh}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_buffers_of_new_objects_are_not_in_use_any_more():
    """A store or an attention is ready for every stream: nothing queued before may still write to its memory."""
    from paper_2511_06010_b200.paged import PagedAttention, PagedKvStore, PageTable

    for make in (lambda: PagedAttention(3, 16, 2, 128, 64, n_unique_splits=2), lambda: PagedKvStore.empty(4, 16, 2, 128),
                 lambda: PagedKvStore.empty(4, 16, 2, 128, "fp4"), lambda: PageTable(4, 16, 2, 2)):
        torch.cuda._sleep(BUSY)
        assert not torch.cuda.current_stream().query()
        make()
        assert torch.cuda.current_stream().query()


def test_capture_with_a_stream_of_its_own():
    """A call on a stream that a capture has forked to: results are allocated inside the graph."""
    st, table, length, q, k, v = _case("bf16")
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    st.append(q, k, v, table, length, q_len=64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        out = st.append(q, k, v, table, length, q_len=64, stream=side)
        main.wait_stream(side)
        twice = out + out
    k2 = torch.randn_like(k)
    k.copy_(k2)
    q.neg_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(twice, q + q)
    ko, _ = st.gather(table, length, k.shape[0], q_len=64)
    assert torch.equal(ko, k2)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_a_page_table_changes_behind_the_calls_that_read_it(fmt, raw):
    """Calls queued on a stream still find the pages of their time when the book is changed and brought up to date
    there, and calls that follow find the new ones."""
    from paper_2511_06010_b200.paged import PagedAttention, PagedKvStore, PageTable

    gen = torch.Generator().manual_seed(42)
    Hq, Hkv, D, page, T = 16, 2, 128, 16, 64
    st = PagedKvStore.empty(12, page, Hkv, D, fmt)
    book = PageTable(12, page, 2, 4)
    assert (book.table(0) == -1).all()
    book.reserve(0, 1)
    assert (book.table(0).cpu().numpy() == book.host).all()  # 0: the default stream's address
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    length = torch.tensor([T, T], dtype=torch.int32).cuda()
    k, v, k2, v2 = (R.make_bf16((2 * T, Hkv, D), gen).cuda() for _ in range(4))
    q = R.make_bf16((2, Hq, D), gen).cuda()
    one, two = (PagedAttention(2, Hq, Hkv, D, T, fmt=fmt, n_unique_splits=2) for _ in range(2))
    for slot in (0, 1):
        book.reserve(slot, T)
    st.append(None, k, v, book.table(), length, q_len=T)
    first = [t.clone() for t in one(q, st, book.table(), length)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    out = one(q, st, book.table(), length, stream=stream)
    old = book.host.copy()
    book.release(0)                        # ... while that waits: other pages, or none
    book.release(1)
    book.reserve(0, T)
    assert book.table(stream) is book.device_table
    assert torch.equal(out[0], first[0]) and torch.equal(out[1], first[1])
    book.reserve(1, T)
    new = book.table(stream)
    st.append(None, k2, v2, new, length, q_len=T, stream=stream)
    out2 = two(q, st, book.table(stream), length, stream=stream)
    torch.cuda.synchronize()
    assert (book.device_table.cpu().numpy() == book.host).all() and (old != book.host).any()
    fresh = PagedKvStore.empty(12, page, Hkv, D, fmt)
    straight = torch.arange(8, dtype=torch.int32).reshape(2, 4).cuda()
    fresh.append(None, k2, v2, straight, length, q_len=T)
    want = one(q, fresh, straight, length)
    assert torch.equal(out2[0], want[0]) and torch.equal(out2[1], want[1])
