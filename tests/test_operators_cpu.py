"""Rotary append and the cache in 4 bits, as far as they go without a GPU: struct layouts, sizes, refusals that need no device."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2509_21354_b200 import binding as b
from tests import reference_q4 as ref


def config(**kw):
    base = dict(B=2, Hq=8, Hkv=4, d=128, C=64, W=64, max_tokens=1024, n_layers=1, agg=0, d_sum=0, d_g=64, attend=0)
    return b.kvE_config(**{**base, **kw})


def test_struct_layouts():
    assert C.sizeof(b.kvE_rope) == 4 + 4 + 64 + 64 * 8
    assert C.sizeof(b.kvE_rows) == 4 * 8
    assert C.sizeof(b.kvE_q4_buffers) == 6 * 8


def test_q4_workspace_and_geometry():
    lib = b.load_library()
    size = lambda t=1, **kw: lib.kvE_q4_workspace_bytes(C.byref(config(**kw)), t)
    assert size() > 0
    assert size(t=8) > size()                       # more query rows, larger records
    assert size(C=48) > 0 and size(C=16) > 0
    assert size(C=24) == 0 and size(C=8) == 0       # not whole units of 16 rows
    assert size(t=0) == 0 and size(t=-1) == 0
    assert size(t=64) > 0 and size(t=65) == 0       # 2 heads a KV head: 128 query rows at most
    assert size(d=64) == 0


def test_calls_without_a_handle_are_refused():
    lib = b.load_library()
    rope, rows, n = b.Rope().c, b.kvE_rows(), C.c_int(0)
    assert lib.kvE_append_rope(None, 0, None, C.byref(rows), C.byref(rows), None, 1, C.byref(rope), None, None, None) == -1
    assert lib.kvE_append_rope_next(None, 0, None, C.byref(rows), C.byref(rows), None, 1, 0, C.byref(rope), None, None) == -1
    assert lib.kvE_attach_q4(None, None) == -1
    assert lib.kvE_pack_chunks(None, 0, 0, 1, None) == -1
    assert lib.kvE_unpack_chunks(None, 0, 0, 1, None, None, None) == -1
    assert lib.kvE_packed_chunks(None, 0, C.byref(n)) == -1
    assert lib.kvE_decode_attn_q4(None, 0, None, 1, 0, 0, None, None, 0.1, None) == -1


def test_rope_object():
    r = b.Rope((16, 24, 24), theta=500.0, layout="adjacent")
    assert r.n_axes == 3 and r.c.layout == 1
    assert list(r.c.axis) == [0] * 16 + [1] * 24 + [2] * 24
    assert np.allclose(list(r.c.inv_freq), 500.0 ** (-np.arange(64) / 64.0), rtol=1e-14)
    part = b.Rope((8, 8))                           # the other pairs are not turned
    assert list(part.c.inv_freq)[16:] == [0.0] * 48 and part.c.inv_freq[15] > 0
    dealt = b.Rope(axis=[j % 3 for j in range(64)], inv_freq=[0.5] * 64)
    assert dealt.n_axes == 3 and list(dealt.c.inv_freq) == [0.5] * 64
    for bad in (dict(sections=(40, 40)), dict(sections=(10,) * 5), dict(axis=[0] * 63), dict(axis=[4] * 64), dict(axis=[-1] + [0] * 63)):
        with pytest.raises(ValueError):
            b.Rope(**bad)


def test_reference_quantisation_by_hand():
    """the tests' own reference: borders, ties, constant groups"""
    x = np.zeros((1, 128))
    x[0, :64] = np.arange(64) % 16                  # 0..15: scale 1, codes are the numbers
    x[0, 64:] = -2.5
    values, scale, low = ref.quantise(ref.bits(x))
    assert np.array_equal(values[0], x[0]) and scale[0].tolist() == [1.0, 0.0] and low[0].tolist() == [0.0, -2.5]
    x[0, :3] = [0.5, 1.5, 2.5625]                   # on a border: the lower code; just above: the upper
    assert ref.quantise(ref.bits(x))[0][0, :3].tolist() == [0.0, 1.0, 3.0]
    x[0, 0] = np.inf
    values, _, _ = ref.quantise(ref.bits(x))
    assert np.isnan(values[0, :64]).all() and np.array_equal(values[0, 64:], x[0, 64:])


def test_operators_do_not_run_without_cuda():
    if torch.cuda.is_available():
        pytest.skip("CUDA present")
    with pytest.raises(RuntimeError):
        b.Store(B=1, H=1, C_=64, W=0, max_tokens=128, d_g=64).attach_q4()
