"""The cache in 4 bits beside pages that were handed back, counts that only the device knows, rows that are not seen, other streams and ranges that are refused."""
import numpy as np
import pytest
import torch

from tests import reference_q4 as ref
from tests.test_gpu_q4 import Case, as_bits, every_third, from_bits, normal, numbers
from tests.test_gpu_q4_sizes import check, expected

pytestmark = pytest.mark.gpu


# ---- chunks whose bf16 rows are gone ---------------------------------------------------------------------------------------------------

def stale_copies(st):
    """4-bit pages that look like good ones: an earlier owner's"""
    st.kv4_pages.fill_(0x11)


def test_discarded_chunks_handed_back_before_packing():
    """nothing that gated attention reads is missing: no error; whoever reads the discarded chunks all the same gets NaN"""
    case = Case(n=700, W=60, listed=9, keep=every_third, packed=0, Hkv=3, G=2, max_tokens=800)
    st = case.st
    stale_copies(st)
    _, count = st.reclaim_pages(0, 0, 9, mode="discarded")
    st.pack_chunks(0, 0, 9)
    torch.cuda.synchronize()
    gone = 9 * 3 - sum(len(k) for k in case.kept)
    assert int(count) == gone and st.poll_status() == 0 and st.packed_chunks(0) == 9
    case.packed = 9
    q = normal((1, 1, 6, 128), 5)
    check(case, q, dense=False)
    for got, rows in zip(st.unpack_chunks(0, 0, 9), (case.K, case.V)):
        got, want = numbers(got), ref.quantise(as_bits(rows)[:, :576])[0]
        for s in range(3):
            for t in range(9):
                at = s, slice(64 * t, 64 * t + 64)
                if t in case.kept[s]:
                    assert (np.abs(got[at] - want[at]) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want[at]) + 2.0 ** -134).all()
                else:
                    assert np.isnan(got[at]).all()
    assert torch.isnan(st.decode_attn_q4(0, q, dense=True)).all()      # every sequence misses a chunk
    assert st.poll_status() == 0
    st.append(0, normal((3, 64, 128), 20), normal((3, 64, 128), 21))      # and further on, with the chunks behind them
    st.pack_chunks(0, 9, 10)
    torch.cuda.synchronize()
    assert st.poll_status() == 0 and st.packed_chunks(0) == 10


@pytest.mark.parametrize("listed", [0, 9])
def test_a_chunk_that_is_wanted_and_gone_is_flagged(listed):
    case = Case(n=700, W=60, listed=listed, keep=lambda s, t: t != 1, packed=0, Hkv=2)
    st = case.st
    stale_copies(st)
    st.page_table[0, 1, 4] = -1
    st.pack_chunks(0, 0, 9)
    torch.cuda.synchronize()
    assert st.poll_status() == -3
    case.packed = 9
    q = normal((1, 1, 2, 128), 5)
    for dense in (False, True):
        got = numbers(st.decode_attn_q4(0, q, dense=dense))[0, 0]
        assert np.isnan(got[1]).all()
        want, _, bound, _ = expected(case, numbers(q), dense, sequences=(0,))
        assert (np.abs(got[0] - want[0, 0, 0]) <= bound[0, 0, 0]).all()
    k, v = st.unpack_chunks(0, 4, 5)
    assert torch.isnan(k[1]).all() and torch.isnan(v[1]).all() and torch.isfinite(k[0]).all() and torch.isfinite(v[0]).all()


def test_a_page_that_is_out_of_range_is_flagged_even_if_discarded():
    case = Case(n=700, W=60, listed=9, keep=lambda s, t: t != 1, packed=0)
    st = case.st
    st.page_table[0, 0, 1] = 1 << 30
    st.pack_chunks(0, 0, 9)
    torch.cuda.synchronize()
    assert st.poll_status() == -3


def test_replayed_packing_keeps_the_copies_of_chunks_handed_back():
    case = Case(n=700, W=60, packed=0)
    st = case.st
    stale_copies(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.pack_chunks(0, 0, 8)
    graph.replay()
    st.reclaim_pages(0, 2, 5, mode="packed")
    torch.cuda.synchronize()
    assert st.poll_status() == 0
    case.packed = 8
    q = normal((1, 1, 2, 128), 5)
    check(case, q)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert st.poll_status() == -3
    check(case, q)
    assert st.packed_chunks(0) == 8


# ---- counts that the host has not heard of ---------------------------------------------------------------------------------------------

def test_bf16_pages_stay_where_the_device_holds_no_copy():
    """packing that was captured and never ran, and a replayed kvE_set_len: the only copy of a chunk is not handed back"""
    case = Case(n=700, W=60, packed=0)
    st, table = case.st, case.st.page_table.clone()
    q = normal((1, 1, 2, 128), 5)
    torch.cuda.synchronize()
    pack, cut = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(pack):
        st.pack_chunks(0, 0, 9)
    _, count = st.reclaim_pages(0, 0, 9, mode="packed")
    torch.cuda.synchronize()
    assert int(count) == 0 and torch.equal(st.page_table, table) and st.poll_status() == -3
    check(case, q)
    pack.replay()
    case.packed = 9
    check(case, q)
    with torch.cuda.graph(cut):
        st.set_len(0, 300)
    st.set_len(0, 700)
    st.adopt_device_state(0)
    st.pack_chunks(0, 0, 9)
    cut.replay()                                            # the device: chunks 0 to 3, the host: nine
    free, count = st.reclaim_pages(0, 0, 9, mode="packed")
    torch.cuda.synchronize()
    assert int(count) == 8 and (st.page_table[0, :, :4] == -1).all() and torch.equal(st.page_table[0, :, 4:], table[0, :, 4:])
    assert sorted(free[:8].tolist()) == sorted(table[0, :, :4].flatten().tolist())
    assert st.poll_status() == -3


def test_bf16_pages_stay_where_there_is_no_4_bit_page():
    case = Case(n=700, W=60, packed=0)
    st, table = case.st, case.st.page_table.clone()
    for bad in (-1, 1 << 30):
        st.page_table4[0, 1, 2] = bad
        st.pack_chunks(0, 0, 9)
        torch.cuda.synchronize()
        assert st.poll_status() == -3
        _, count = st.reclaim_pages(0, 2, 3, mode="packed")
        torch.cuda.synchronize()
        assert int(count) == (1 if bad == -1 else 0) and st.poll_status() == -3
        assert st.page_table[0, 0, 2] == -1 and st.page_table[0, 1, 2] == table[0, 1, 2]


def test_unpacking_what_the_device_does_not_hold_is_flagged():
    case = Case(n=700, W=60, packed=0)
    st = case.st
    stale_copies(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.pack_chunks(0, 0, 9)
    out = [torch.full((2, 9 * 64, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    st.unpack_chunks(0, 0, 9, *out)
    torch.cuda.synchronize()
    assert st.poll_status() == -3 and all((x == 9.0).all() for x in out)
    graph.replay()
    st.unpack_chunks(0, 0, 9, *out)
    torch.cuda.synchronize()
    assert st.poll_status() == 0
    want = ref.quantise(as_bits(case.V)[:, :576])[0]
    assert (np.abs(numbers(out[1]) - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want) + 2.0 ** -134).all()


# ---- rows that are not seen ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,G", [(4, 1), (7, 1), (2, 2), (16, 1), (7, 4), (5, 8)])
@pytest.mark.parametrize("n", [40, 333, 700])
def test_causal_blocks_with_rows_that_are_not_finite(T, G, n):
    """keys and values of a token are nothing to the tokens in front of it"""
    K, V = as_bits(normal((2, n, 128), 2)).copy(), as_bits(normal((2, n, 128), 3)).copy()
    V[0, n - 1, 5], V[0, n - 1, 70] = 0x7F80, 0x7FC0
    K[1, n - 1] = 0x7FC0
    V[1, n - T // 2, :] = 0xFF80
    case = Case(n=n, W=60, T=T, G=G, K=from_bits(K), V=from_bits(V))
    q = normal((1, T, 2 * G, 128), 4)
    got = numbers(case.st.decode_attn_q4(0, q, dense=True, causal=True))
    assert case.st.poll_status() == 0
    want, _, bound, _ = expected(case, numbers(q), True, True)
    for s, first in ((0, T - 1), (1, T - T // 2)):          # the first token that sees one of them
        heads = slice(s * G, s * G + G)
        seen = got[0, :first, heads]
        assert seen.size and (np.abs(seen - want[0, :first, heads]) <= bound[0, :first, heads]).all()
    assert np.isposinf(got[0, T - 1, :G, 5]).all() and np.isnan(got[0, T - 1, :G, 70]).all()
    assert np.isfinite(np.delete(got[0, T - 1, :G], [5, 70], axis=-1)).all()
    assert np.isnan(got[0, T - 1, G:]).all()
    if T // 2 > 1:
        assert np.isneginf(got[0, T - T // 2:T - 1, G:]).all()


# ---- results on another stream ---------------------------------------------------------------------------------------------------------

def freed_block(shape):
    """the address of a block that the current stream has just given back"""
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    return t.data_ptr()


@pytest.mark.parametrize("native", [True, False])
def test_results_of_a_call_on_another_stream_are_that_streams(native, monkeypatch):
    """a block that the current stream has given back may still be in use there: a call on another stream does not take it for its result"""
    from paper_2509_21354_b200 import binding as b
    case = Case(B=2, Hkv=2, n=700, W=60, max_tokens=800)
    if not native:
        monkeypatch.setattr(b, "_bind", None)
    st, side, rope = case.st, torch.cuda.Stream(), b.Rope()
    q = normal((2, 1, 4, 128), 1)[:, :, :2].contiguous()
    k, v = normal((2, 1, 2, 128), 2), normal((2, 1, 2, 128), 3)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    ways = [((2, 1, 2, 128), lambda: [st.decode_attn_q4(0, q, dense=True, stream=side)]),
            ((2, 1, 2, 128), lambda: [st.append_rope(0, q, k, v, rope, stream=side)[0]]),
            ((2, 1, 2, 128), lambda: [st.append_rope_next(0, q, k, v, rope, stream=side)]),
            ((4, 64, 128), lambda: list(st.unpack_chunks(0, 1, 2, stream=side)))]
    for shape, call in ways:
        was = freed_block(shape)
        again = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        assert again.data_ptr() == was                      # (the allocator hands the block out again at once)
        del again
        results = call()
        assert all(r.data_ptr() != was for r in results)
        torch.cuda.synchronize()
        plain = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        assert plain.data_ptr() == was                      # it was there to be taken
        del plain, results
    assert st.poll_status() == 0


def test_results_of_the_other_calls_on_another_stream():
    from paper_2509_21354_b200 import binding as b
    st, side = b.Store(B=2, H=2, C_=64, W=60, max_tokens=800, d_g=64, max_query_tokens=4), torch.cuda.Stream()
    st.append(0, normal((4, 700, 128), 1), normal((4, 700, 128), 2))
    one = lambda i: normal((4, 128), i)
    rows = [one(i) for i in range(3)]
    block = normal((2, 3, 2, 128), 6)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    ways = [((4, 128), lambda: st.decode_attn(0, rows[0], stream=side)), ((4, 128), lambda: st.decode_attn_dense(0, rows[0], stream=side)),
            ((4, 128), lambda: st.decode_step(0, *rows, stream=side)), ((2, 3, 2, 128), lambda: st.decode_attn_block(0, block, dense=True, stream=side))]
    for shape, call in ways:
        was = freed_block(shape)
        result = call()
        assert result.shape == shape and result.data_ptr() != was
        torch.cuda.synchronize()
        assert freed_block(shape) == was
        del result
    # the count is a zero that the call's own stream wrote, not one that may come behind its result
    busy = torch.zeros(1 << 28, device="cuda")
    for _ in range(20):
        busy.add_(1.0)
    _, count = st.reclaim_pages(0, 0, 0, stream=side)
    side.synchronize()
    assert int(count) == 0 and st.poll_status() == 0


# ---- ranges that are refused -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("native", [True, False])
def test_ranges_of_chunks_to_unpack(native, monkeypatch):
    from paper_2509_21354_b200 import binding as b
    case = Case(n=700, W=60)
    if not native:
        monkeypatch.setattr(b, "_bind", None)
    st = case.st
    for lo, hi, rc in ((2, 1, -1), (-1, 2, -1), (-2, -1, -1), (0, 11, -4), (11, 11, -4), (0, 1 << 20, -4), (0, 1 << 40, -4), (10, 1 << 31, -4)):
        with pytest.raises(b.KveError) as e:
            st.unpack_chunks(0, lo, hi)
        assert e.value.rc == rc
    for at in (0, 4, 10):
        k, v = st.unpack_chunks(0, at, at)
        assert k.shape == v.shape == (2, 0, 128)
    with pytest.raises(b.KveError):
        b.Store(B=1, H=1, C_=64, W=0, max_tokens=128, d_g=64).unpack_chunks(0, 0, 0)
    assert st.unpack_chunks(0, 0, 10)[0].shape == (2, 640, 128) and st.poll_status() == 0
