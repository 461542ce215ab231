"""kvE_append_rope / kvE_append_rope_next against the 64-bit restatement: axes, layouts, strides, far positions, graph replay, refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import reference_q4 as ref

pytestmark = pytest.mark.gpu


def store(B, Hkv, G, C_=64, max_tokens=256, **kw):
    from paper_2509_21354_b200 import binding as b
    return b.Store(B=B, H=Hkv, Hq=Hkv * G, C_=C_, W=0, max_tokens=max_tokens, d_g=64, **kw)


def normal(shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def projections(B, n, Hq, Hkv, seed, fused):
    """q, k, v [B, n, heads, 128]: parts of one tensor, or tensors whose heads come first in memory"""
    if fused:
        return normal((B, n, Hq + 2 * Hkv, 128), seed).split([Hq, Hkv, Hkv], dim=2)
    return tuple(normal((B, h, n, 128), seed + i).transpose(1, 2) for i, h in enumerate((Hq, Hkv, Hkv)))


def numbers(t):
    return t.float().cpu().numpy().astype(np.float64)


def stored(st, n0, n, layer=0):
    """rows n0 .. n0 + n of every sequence as the pages hold them: [B, n, Hkv, 128], keys and values"""
    table = st.page_table[layer].cpu().numpy()
    rows = []
    for pages in (st.k_pages, st.v_pages):
        p = numbers(pages)
        rows.append(np.stack([[p[table[s, i // st.C], i % st.C] for i in range(n0, n0 + n)] for s in range(st.S)]).reshape(st.B, st.H, n, 128).transpose(0, 2, 1, 3))
    return rows


def check_turned(got, x, positions, rope):
    """one bf16 rounding (half a step: 2^-8) of numbers computed in fp32: the angle in turns off by 2^-25 at most (6.2832 * 2^-25 rad),
    sincospif within 2 units in the last place (2^-23), three roundings of products and sum (3 * 2^-24); at positions up to 2^31 the angles
    in 64 bits, here and there, are themselves off by 2^31 * 2 pi * 2^-53 * 2 = 2^-18.3 / 4: together below 2^-19 (|a| + |b|)"""
    axis, freq = np.array(list(rope.c.axis)), np.array(list(rope.c.inv_freq))
    adjacent = rope.c.layout == 1
    want = ref.turn(x, positions, axis, freq, adjacent)
    a = np.abs(x)
    size = np.repeat(a[..., 0::2] + a[..., 1::2], 2, axis=-1) if adjacent else np.concatenate([a[..., :64] + a[..., 64:]] * 2, axis=-1)
    bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())


CASES = [  # B, Hkv, G, n0, n, sections, layout, fused, first position
    (1, 1, 1, 0, 1, (64,), "halves", True, 0),
    (1, 1, 1, 5, 1, (64,), "adjacent", True, 123456789),
    (2, 3, 1, 0, 7, (64,), "halves", False, -50),
    (1, 8, 4, 63, 2, (16, 24, 24), "halves", True, 2000000),
    (3, 2, 7, 10, 33, (16, 24, 24), "adjacent", False, 17),
    (2, 5, 2, 1, 130, (20, 30), "halves", True, 0),            # the last 14 pairs stay as they are
    (1, 1, 1, 0, 200, (10, 10, 20, 24), "adjacent", True, 1000),
    (2, 32, 1, 100, 9, (64,), "halves", True, 2 ** 31 - 20),
]


@pytest.mark.parametrize("B,Hkv,G,n0,n,sections,layout,fused,first", CASES)
@pytest.mark.parametrize("form", ["host", "device"])
def test_rope_append(B, Hkv, G, n0, n, sections, layout, fused, first, form):
    from paper_2509_21354_b200 import binding as b
    st = store(B, Hkv, G, C_=24 if B == 3 else 64, page_perm="random", seed=3)
    st.k_pages.fill_(7.0)
    st.v_pages.fill_(7.0)
    if n0:
        st.append(0, *(normal((st.S, n0, 128), 90 + i) for i in range(2)))
    before = stored(st, 0, n0)
    rope = b.Rope(sections, layout=layout)
    q, k, v = projections(B, n, Hkv * G, Hkv, 1, fused)
    rng = np.random.default_rng(4)
    positions = rng.integers(first, min(first + 5000, 2 ** 31 - 1), size=(B, n, len(sections)), dtype=np.int64)
    pos = torch.from_numpy(positions.astype(np.int32)).cuda()
    if form == "host":
        out, ready = st.append_rope(0, q, k, v, rope, positions=pos)
        assert ready == (n0 + n) // st.C
    else:
        out = st.append_rope_next(0, q, k, v, rope, positions=pos)
    torch.cuda.synchronize()
    assert st.poll_status() == 0 and st.layer_state(0)["n_tokens"] == n0 + n and (st.seq_len == n0 + n).all()
    check_turned(numbers(out), numbers(q), positions, rope)
    got_k, got_v = stored(st, n0, n)
    check_turned(got_k, numbers(k), positions, rope)
    assert np.array_equal(got_v, numbers(v))
    for x, y in zip(stored(st, 0, n0), before):
        assert np.array_equal(x, y)
    if n0 + n < st.max_tokens:      # what lies behind the last token is left alone
        for x in stored(st, n0 + n, min(3, st.max_tokens - n0 - n)):
            assert (x == 7.0).all()


@pytest.mark.parametrize("Hkv,G,n", [(1, 1, 16600), (1, 7, 9100)])
def test_many_tokens_of_few_heads(Hkv, G, n):
    """as many tokens a CTA as there are"""
    from paper_2509_21354_b200 import binding as b
    st = store(2, Hkv, G, max_tokens=n + 3, page_perm="random", seed=5)
    rope = b.Rope((40, 24))
    q, k, v = projections(2, n, Hkv * G, Hkv, 6, True)
    positions = np.random.default_rng(7).integers(0, 100000, size=(2, n, 2), dtype=np.int64)
    out, _ = st.append_rope(0, q, k, v, rope, positions=torch.from_numpy(positions.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    assert st.poll_status() == 0
    check_turned(numbers(out), numbers(q), positions, rope)
    got_k, got_v = stored(st, 0, n)
    check_turned(got_k, numbers(k), positions, rope)
    assert np.array_equal(got_v, numbers(v))


@pytest.mark.parametrize("form", ["host", "device"])
def test_positions_default_to_the_index_and_q_may_be_missing(form):
    from paper_2509_21354_b200 import binding as b
    st = store(2, 2, 1)
    rope = b.Rope((32, 32))
    call = (lambda *a, **kw: st.append_rope(*a, **kw)[0]) if form == "host" else st.append_rope_next
    _, k, v = projections(2, 5, 2, 2, 1, True)
    assert call(0, None, k, v, rope) is None
    q, k, v = projections(2, 3, 2, 2, 2, True)
    out = call(0, q, k, v, rope)
    index = np.broadcast_to(np.arange(5, 8)[None, :, None], (2, 3, 2))
    check_turned(numbers(out), numbers(q), index, rope)
    check_turned(stored(st, 5, 3)[0], numbers(k), index, rope)


def test_q_in_place_and_other_layers_and_streams():
    from paper_2509_21354_b200 import binding as b
    st = store(2, 4, 2, n_layers=3)
    rope = b.Rope()
    q = normal((2, 6, 8, 128), 1)
    _, k, v = projections(2, 6, 8, 4, 2, True)
    x = numbers(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    st.append_rope(1, q, k, v, rope, q_out=q, stream=side)
    side.synchronize()
    index = np.broadcast_to(np.arange(6)[None, :, None], (2, 6, 1))
    check_turned(numbers(q), x, index, rope)
    check_turned(stored(st, 0, 6, layer=1)[0], numbers(k), index, rope)
    assert [st.layer_state(i)["n_tokens"] for i in range(3)] == [0, 6, 0]


def test_zero_frequency_leaves_a_pair_and_zero_tokens_do_nothing():
    from paper_2509_21354_b200 import binding as b
    st = store(1, 1, 1)
    rope = b.Rope(inv_freq=[0.0] * 64)
    q, k, v = projections(1, 4, 1, 1, 1, True)
    pos = torch.full((1, 4, 1), 12345, dtype=torch.int32, device="cuda")
    out, _ = st.append_rope(0, q, k, v, rope, positions=pos)
    assert torch.equal(out, q) and np.array_equal(stored(st, 0, 4)[0], numbers(k))
    empty = [t[:, :0] for t in (q, k, v)]
    st.append_rope(0, *empty, rope)
    assert st.layer_state(0)["n_tokens"] == 4


def test_replayed_from_a_graph():
    from paper_2509_21354_b200 import binding as b
    st = store(2, 4, 2)
    rope = b.Rope((16, 24, 24))
    q, k, v = (t.contiguous() for t in projections(2, 1, 8, 4, 1, True))
    pos = torch.zeros((2, 1, 3), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    st.append_rope_next(0, q, k, v, rope, positions=pos, q_out=out)      # (warm-up)
    st.set_len(0, 0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.append_rope_next(0, q, k, v, rope, positions=pos, q_out=out, n_reserve=100)
    st.set_len(0, 0)
    for i in range(70):
        new = [normal(t.shape, 100 + 3 * i + j) for j, t in enumerate((q, k, v))]
        for t, x in zip((q, k, v), new):
            t.copy_(x)
        at = np.array([[[i, 2 * i, 1000 - i]], [[7 * i, i * i, 3]]])
        pos.copy_(torch.from_numpy(at.astype(np.int32)))
        g.replay()
        torch.cuda.synchronize()
        if i % 23 == 0 or i == 69:
            check_turned(numbers(out), numbers(new[0]), at, rope)
            kk, vv = stored(st, i, 1)
            check_turned(kk, numbers(new[1]), at, rope)
            assert np.array_equal(vv, numbers(new[2]))
    assert (st.seq_len == 70).all()
    st.adopt_device_state(0)
    assert st.layer_state(0)["n_tokens"] == 70


def test_full_cache_and_missing_pages_are_flagged():
    from paper_2509_21354_b200 import binding as b
    st = store(1, 2, 1, max_tokens=64)
    rope = b.Rope()
    q, k, v = projections(1, 3, 2, 2, 1, True)
    st.set_len(0, 62)
    with pytest.raises(b.KveError) as e:
        st.append_rope(0, q, k, v, rope)
    assert e.value.rc == -3
    st.set_len(0, 60)
    st.seq_len.fill_(62)      # as after replays that the host has not heard of
    before = st.k_pages.clone()
    st.append_rope_next(0, q, k, v, rope)
    torch.cuda.synchronize()
    assert st.poll_status() == -3 and torch.equal(st.k_pages, before) and (st.seq_len == 62).all()
    st.set_len(0, 0)
    st.page_table[0, 1, 0] = -1
    st.append_rope(0, q, k, v, rope)
    torch.cuda.synchronize()
    assert st.poll_status() == -3
    assert np.array_equal(numbers(st.v_pages)[0, :3], numbers(v)[0, :, 0])      # the other sequence has its rows


def test_refusals():
    from paper_2509_21354_b200 import binding as b
    st = store(1, 2, 1)
    rope = b.Rope()
    q, k, v = (t.contiguous() for t in projections(1, 3, 2, 2, 1, True))
    lib, out = st.lib, torch.empty_like(q)
    rows = lambda t, off=0, step=0: b.kvE_rows(t.data_ptr() + off, t.stride(0), t.stride(1) + step, t.stride(2))

    def call(q_=rows(q), k_=rows(k), v_=rows(v), n=3, r=rope.c, o=out.data_ptr(), layer=0):
        ref_ = lambda x: None if x is None else C.byref(x)
        return lib.kvE_append_rope(st.handle, layer, ref_(q_), ref_(k_), ref_(v_), None, n, ref_(r), o, None, None)

    def changed(**kw):
        c = b.kvE_rope.from_buffer_copy(rope.c)
        for name, value in kw.items():
            setattr(c, name, value)
        return c
    bad_axis = changed()
    bad_axis.axis[63] = 1
    assert call(k_=None) == call(v_=None) == call(r=None) == call(layer=1) == call(layer=-1) == call(n=-1) == -1
    assert call(k_=rows(k, off=2)) == call(v_=rows(v, step=4)) == call(q_=rows(q, off=8)) == call(o=out.data_ptr() + 2) == -1
    assert call(q_=None) == call(o=None) == -1                       # q and q_out come together
    assert call(r=changed(n_axes=0)) == call(r=changed(n_axes=5)) == call(r=changed(layout=2)) == call(r=bad_axis) == -1
    assert call(n=257) == -3
    assert st.layer_state(0)["n_tokens"] == 0
    assert call(q_=None, o=None) == 0
    with pytest.raises(AssertionError):
        st.append_rope(0, q.float(), k, v, rope)
    with pytest.raises(AssertionError):
        st.append_rope(0, q, k, v, rope, positions=torch.zeros((1, 3, 2), dtype=torch.int32, device="cuda"))
