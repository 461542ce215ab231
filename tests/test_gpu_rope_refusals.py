"""Rotary positions that kvE_append_rope refuses, beyond those of tests/test_gpu_rope.py."""
import pytest
import torch

from tests.test_gpu_rope import normal, store

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("form", ["append_rope", "append_rope_next"])
def test_frequencies_that_are_not_finite(form, bad):
    """they would put NaN into the cache"""
    from paper_2509_21354_b200 import binding as b
    st = store(1, 2, 1)
    q, k, v = (normal((1, 3, 2, 128), i) for i in range(3))
    with pytest.raises(b.KveError) as e:
        getattr(st, form)(0, q, k, v, b.Rope(inv_freq=[1.0] * 63 + [bad]))
    assert e.value.rc == -1 and st.layer_state(0)["n_tokens"] == 0
    torch.cuda.synchronize()
    assert (st.seq_len == 0).all() and st.poll_status() == 0
    getattr(st, form)(0, q, k, v, b.Rope(inv_freq=[1.0] * 64))
