"""Attention over 4 bits with values of very different sizes in one sequence, against the 64-bit restatement: rows much larger than the rest
whose weight is next to nothing, query rows that disagree about which rows matter, sums next to the end of the declared range."""
import numpy as np
import pytest
import torch

from tests import reference_q4 as ref
from tests.test_gpu_q4 import Case, as_bits, from_bits, numbers

pytestmark = pytest.mark.gpu


def expected(case, q, dense=False, causal=False, sequences=None):
    """out, lse, the bound of |out - want| and that of |lse - want|, of the sequences named (others NaN).  The bound, per number of the result:
      2^-8 |want|: its bf16 rounding;
      2^-11 sum p c s: a packed row's weight times scale is one fp16 number, off by half a step, relative to its share c s beyond the lowest number;
      2^-21 * 15 * rows * (largest p s): where that number is not a normal fp16 one it is off by 2^-25, and the factor in front keeps the largest
        at 2^-4 or more;
      2^-16 sum p |v|, with |low| + c s for a packed row: bf16 rows' weights are two bf16 planes (2^-17 at most), ex2 within 2 units of 2^-23, and
        fp32 sums: a warp's chain of additions has fewer than 2^6 links here, each off by 2^-24;
      2 dl sum p |v|: the logits, off by dl (16 steps of 2^-23 relative to sum |q| (max |k| + 16 scales) times scale: eight MMAs with their last
        bits cut off, two halves, scale and offset), move numerator and denominator;
      2^-76: what the largest factor (2^56) leaves of the smallest rows;
    all sums over the rows that the query row sees, relative to the sum of p; packed groups are judged by scales of their own."""
    st, c, n = case.st, case.st.C, case.n
    B, T, Hq, _ = q.shape
    G, cut = Hq // st.H, case.packed * c
    out, bound = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, dlse = np.full(q.shape[:3], np.nan), np.full(q.shape[:3], np.nan)
    Kb, Vb = as_bits(case.K), as_bits(case.V)
    for s in range(st.S) if sequences is None else sequences:
        kq, ks, _ = ref.quantise(Kb[s, :cut])
        vq, vs, vl = ref.quantise(Vb[s, :cut])
        K, V = np.concatenate([kq, ref.number(Kb[s, cut:])]), np.concatenate([vq, ref.number(Vb[s, cut:])])
        low, scale = (np.repeat(x, 64, axis=-1) for x in (vl, vs))      # [cut, 128]
        seen = np.ones(n, bool)
        if not dense:
            seen[:case.listed * c] = False
            for t in case.kept[s]:
                seen[t * c:t * c + c] = True
        b_, h = divmod(s, st.H)
        for t in range(T):
            see = seen & (np.arange(n) <= n - T + t) if causal else seen
            for head in range(h * G, h * G + G):
                row = q[b_, t, head]
                o, l, _ = ref.attend(row[None], K, V, see[None])
                at = b_, t, head
                out[at], lse[at] = o[0], l[0]
                reach = np.abs(row).sum() * (np.abs(K[see]).max(initial=0.0) + (16 * ks.max() if cut else 0.0))
                dl = 2.0 ** -19 * reach * ref.SCALE
                dlse[at] = dl + 2.0 ** -21 * (1 + abs(l[0]))
                p = np.where(see, np.exp(np.where(see, K @ row * ref.SCALE, -np.inf) - l[0]), 0.0)[:, None]
                with np.errstate(invalid="ignore"):
                    sizes = np.concatenate([np.abs(low) + np.abs(vq - low), np.abs(V[cut:])])
                    used = (p != 0)[:, 0]
                    M = (p[used] * sizes[used]).sum(0)
                    u4 = used[:cut]
                    A = (p[:cut][u4] * np.abs(vq - low)[u4]).sum(0)
                    top = (p[:cut][u4] * scale[u4]).max(0, initial=0.0)
                bound[at] = 2.0 ** -8 * np.abs(o[0]) + 2.0 ** -11 * A + 2.0 ** -21 * 15 * cut * top + (2.0 ** -16 + 2 * dl) * M + 2.0 ** -76
    return out, lse, bound, dlse


def check(case, q, dense=True, causal=False, sequences=None):
    st = case.st
    lse = torch.full(q.shape[:3], 5.0, dtype=torch.float32, device="cuda")
    got = st.decode_attn_q4(case.layer, q, dense=dense, causal=causal, lse=lse)
    torch.cuda.synchronize()
    assert st.poll_status() == 0
    want, want_lse, bound, dlse = expected(case, numbers(q), dense, causal, sequences)
    got, lse = numbers(got), lse.cpu().numpy().astype(np.float64)
    if sequences is None:
        assert np.isfinite(want).all()
    ok = np.isfinite(want)
    assert np.isfinite(got[ok]).all()
    err = np.abs(got - want)[ok] / bound[ok]
    assert err.max() <= 1.0, err.max()
    ok = np.isfinite(want_lse)
    assert (np.abs(lse - want_lse)[ok] <= dlse[ok]).all()


def signed_queries(B, T, Hq, signs, seed):
    """q near +-1: rows of keys near -5 get weights of e^-56, or all of the weight"""
    rng = np.random.default_rng(seed)
    q = (1 + 0.1 * rng.standard_normal((B, T, Hq, 128))) * np.asarray(signs)[np.arange(T * Hq) % len(signs)].reshape(1, T, Hq, 1)
    return from_bits(ref.bits(q.astype(np.float32)))


def with_outliers(S, n, rows, size, seed):
    """keys of size 0.1, values of size 1; the rows named have keys of -5 and values of size 2^size"""
    rng = np.random.default_rng(seed)
    K, V = 0.1 * rng.standard_normal((S, n, 128)), rng.standard_normal((S, n, 128))
    K[:, rows] = -5.0
    V[:, rows] *= 2.0 ** size
    return from_bits(ref.bits(K.astype(np.float32))), from_bits(ref.bits(V.astype(np.float32)))


WHERE = {"front": [0], "behind": [639], "both": [0, 1, 638, 639], "every chunk": list(range(7, 640, 64)), "whole chunk": list(range(128, 192))}


@pytest.mark.parametrize("G", [1, 3, 8, 16])
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("size", [12, 24, 30, 50])
def test_large_values_of_little_weight(G, where, size):
    """they must not cost the others their bits"""
    K, V = with_outliers(2, 700, WHERE[where], size, G)
    case = Case(n=700, W=60, G=G, K=K, V=V)
    check(case, signed_queries(1, 1, 2 * G, [1], 3))


@pytest.mark.parametrize("G,T", [(2, 1), (4, 1), (7, 1), (8, 1), (16, 1), (5, 4)])
@pytest.mark.parametrize("size", [30, -30])
def test_query_rows_that_disagree_about_what_matters(G, T, size):
    """the large (or small) rows have all of the weight of every other query row, and none of the rest's"""
    K, V = with_outliers(2, 700, WHERE["every chunk"], size, G)
    case = Case(n=700, W=60, G=G, T=T, K=K, V=V)
    check(case, signed_queries(1, T, 2 * G, [1, -1], 4))


@pytest.mark.parametrize("G", [1, 8, 16])
def test_large_values_of_little_weight_in_long_runs(G):
    """CTAs that go through whole sequences, and through more than one: a factor that sinks must rise again"""
    rows = [0, 1, 2] + list(range(500, 564)) + [1439]
    K, V = with_outliers(160, 1500, rows, 30, 5)
    case = Case(B=80, Hkv=2, n=1500, W=60, G=G, K=K, V=V)
    check(case, signed_queries(80, 1, 2 * G, [1, -1, 1], 6), sequences=(0, 77, 158, 159))


@pytest.mark.parametrize("G", [1, 8, 16])
def test_weights_that_rise_along_the_sequence(G):
    """first rows with large scales and all the weight there is so far, then ones whose logits pass them by 0 to 80"""
    rng = np.random.default_rng(8)
    for rise in (5.0, 30.0, 80.0):
        K, V = 0.1 * rng.standard_normal((2, 700, 128)), rng.standard_normal((2, 700, 128))
        K += np.linspace(0, rise / (128 * ref.SCALE), 700)[None, :, None]
        V *= np.exp2(np.linspace(30, 0, 700))[None, :, None]
        case = Case(n=700, W=60, G=G, K=from_bits(ref.bits(K.astype(np.float32))), V=from_bits(ref.bits(V.astype(np.float32))))
        check(case, signed_queries(1, 1, 2 * G, [1, -1], 9))


# ---- the end of the declared range ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G", [1, 8, 16])
@pytest.mark.parametrize("packed", [0, 1, None])
@pytest.mark.parametrize("size", [59, -59])
def test_sums_of_the_largest_and_smallest_values(G, packed, size):
    """equal logits and values of one sign, between 2^58 and 2^60 (or 2^-60 and 2^-58), dozens of rows a warp: in bf16 only, in both forms, nearly
    all in 4 bits"""
    rng = np.random.default_rng(10)
    V = rng.uniform(0.5, 1.99, (160, 700, 128)) * 2.0 ** size
    K = np.zeros((160, 700, 128), np.float32)
    K[:, 300:] = 0.45      # logits of 5.1 in the later rows: below what raises the reference, so their weights are above 1
    case = Case(B=80, Hkv=2, n=700, W=30, G=G, packed=packed, K=from_bits(ref.bits(K)), V=from_bits(ref.bits(V.astype(np.float32))))
    check(case, signed_queries(80, 1, 2 * G, [1], 11), sequences=(0, 77, 158, 159))
