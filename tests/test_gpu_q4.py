"""The cache in 4 bits (kvE_pack_chunks, kvE_unpack_chunks) and attention over it (kvE_decode_attn_q4) against the 64-bit restatement."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import reference_q4 as ref

pytestmark = pytest.mark.gpu


def normal(shape, seed, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def as_bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def from_bits(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)


def numbers(t):
    return t.float().cpu().numpy().astype(np.float64)


class Case:
    """A store with n tokens, chunks [0, packed) in 4 bits, a keep list over [0, listed) that keeps `keep` (a function of sequence and chunk)."""

    def __init__(self, B=1, Hkv=2, G=1, n=300, C_=64, W=64, T=1, packed=None, listed=0, keep=None, seed=0, n_layers=1, layer=0, K=None, V=None, max_tokens=None):
        from paper_2509_21354_b200 import binding as b
        self.b, self.layer, self.T, self.n = b, layer, T, n
        self.st = st = b.Store(B=B, H=Hkv, Hq=Hkv * G, C_=C_, W=W, max_tokens=max_tokens or max(n, 1) + 40, d_g=64, n_layers=n_layers, page_perm="random", seed=seed)
        st.attach_q4(max_query_tokens=T, page_perm="random", seed=seed + 1)
        # whatever is read although it should not be shows
        st.k_pages.fill_(float("nan"))
        st.v_pages.fill_(float("nan"))
        st.kv4_pages.fill_(0xFF)
        self.stale = max(0, n - W) // C_
        self.packed = self.stale if packed is None else packed
        self.K = normal((st.S, n, 128), seed + 2) if K is None else K
        self.V = normal((st.S, n, 128), seed + 3) if V is None else V
        if n:
            st.append(layer, self.K, self.V)
        self.listed, self.kept = listed, [[] for _ in range(st.S)]
        if listed:
            rng = np.random.default_rng(seed)
            weight = lambda *shape: rng.standard_normal(shape).astype(np.float32) / 16
            lstm = b.LstmWeights(dict(W_ih=weight(256, 256), W_hh=weight(256, 64), b_ih=weight(256), b_hh=weight(256), w_s=weight(64), b_s=0.0))
            st.summarize_chunks(layer, 0, listed)
            st.gate(layer, 0, listed, lstm)
            flags = np.array([[1.0 if keep(s, t) else 0.0 for t in range(listed)] for s in range(st.S)], np.float32)
            st.scores[layer, :, :listed] = torch.from_numpy(flags).cuda()
            st.compact(layer, 0.5)
            self.kept = [[t for t in range(listed) if keep(s, t)] for s in range(st.S)]
        if self.packed:
            st.pack_chunks(layer, 0, self.packed)

    def want(self, q, dense, causal):
        """q: numbers [B, T, Hq, 128] -> out, lse, spread, largest |k| + 16 scales (per output row)"""
        st, c, n = self.st, self.st.C, self.n
        B, T, Hq, _ = q.shape
        G = Hq // st.H
        out, lse, spread, reach = np.zeros(q.shape), np.zeros(q.shape[:3]), np.zeros(q.shape), np.zeros(q.shape[:3])
        Kb, Vb = as_bits(self.K), as_bits(self.V)
        for s in range(st.S):
            cut = self.packed * c
            kq, ks, _ = ref.quantise(Kb[s, :cut])
            vq, vs, _ = ref.quantise(Vb[s, :cut])
            K, V = np.concatenate([kq, ref.number(Kb[s, cut:])]), np.concatenate([vq, ref.number(Vb[s, cut:])])
            seen = np.ones(n, bool)
            if not dense:
                seen[:self.listed * c] = False
                for t in self.kept[s]:
                    seen[t * c:t * c + c] = True
            b_, h = divmod(s, st.H)
            heads = slice(h * G, h * G + G)
            for t in range(T):
                see = seen & (np.arange(n) <= n - T + t) if causal else seen
                rows = q[b_, t, heads]
                o, l, sp = ref.attend(rows, K, V, np.broadcast_to(see, (G, n)))
                out[b_, t, heads], lse[b_, t, heads] = o, l
                spread[b_, t, heads] = sp + (16 * vs.max() if cut else 0.0)
                sizes = np.abs(K[see & np.isfinite(K).all(-1)])      # (an infinite number's logit is not computed to any precision)
                reach[b_, t, heads] = np.abs(rows).sum(-1) * ((sizes.max() if sizes.size else 0.0) + (16 * np.nanmax(ks) if cut else 0.0))
        return out, lse, spread, reach

    def check(self, q=None, dense=False, causal=False, seed=7, **kw):
        st = self.st
        q = normal((st.B, self.T, st.Hq, 128), seed) if q is None else q
        lse = torch.full(q.shape[:3], 5.0, dtype=torch.float32, device="cuda")
        out = torch.full_like(q, 5.0)
        st.decode_attn_q4(self.layer, q, dense=dense, causal=causal, out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        assert st.poll_status() == 0
        self.compare(out, lse, *self.want(numbers(q), dense, causal))
        return q, out, lse

    def compare(self, out, lse, want, want_lse, spread, reach):
        """Logits: sums of 128 products in fp32, in the tensor core with its last bits cut off, of q with numbers up to |k| + 16 s: off by
        16 steps of 2^-23 relative to sum |q| (max |k| + 16 s) times scale at most (eight MMAs, two halves, scale and offset).  Weights: two
        bf16 planes (2^-17), ex2 of 2 units in the last place, times values of up to |v| + 16 s.  One bf16 rounding: 2^-8."""
        got, got_lse = numbers(out), lse.cpu().numpy().astype(np.float64)
        dl = 2.0 ** -19 * reach * ref.SCALE
        bound = 2.0 ** -8 * np.abs(want) + (2 * dl[..., None] + 2.0 ** -16) * spread + 1e-30
        bad = np.isnan(want)
        assert np.array_equal(np.isnan(got), bad)
        err = np.where(bad, 0.0, np.abs(got - want))
        assert (err <= np.where(bad, 1.0, bound)).all(), float(np.nanmax(err / bound))
        inf = np.isinf(want_lse)
        assert np.array_equal(got_lse[inf], want_lse[inf])
        ok = ~inf & ~np.isnan(want_lse)
        assert (np.abs(got_lse[ok] - want_lse[ok]) <= dl[ok] + 2.0 ** -21 * (1 + np.abs(want_lse[ok]))).all()
        # and as a whole: a bf16 rounding is 2^-8 / sqrt(3) rms of the value at most
        w = want[~bad]
        if w.size >= 4096 and np.any(w):
            assert np.sqrt(np.mean(err[~bad] ** 2)) <= 1.05 * 2.0 ** -8 / np.sqrt(3) * np.sqrt(np.mean(w ** 2))


# ---- the rows themselves ---------------------------------------------------------------------------------------------------------------

def awkward_rows(S, n, seed):
    """bf16 bits [S, n, 128]: rows of every sort (normal, constant, ties, tiny, huge, one outlier, infinities and NaN)"""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((S, n, 128)).astype(np.float32)
    kinds = rng.integers(0, 10, size=(S, n))
    x[kinds == 1] = 0.0
    x[kinds == 2] = 3.25
    x[kinds == 3] = rng.integers(-15, 16, size=x[kinds == 3].shape) * 0.5            # ties everywhere
    x[kinds == 4] *= 1e-30
    x[kinds == 5] *= 1e30
    x[kinds == 6, 5] = 100.0
    x[kinds == 7] = rng.integers(0, 31, size=x[kinds == 7].shape) / 2.0               # scale 1, numbers on the borders
    x[kinds == 8] = 1000.0 + rng.integers(0, 3, size=x[kinds == 8].shape) * 8
    x[kinds == 9] *= np.exp2(rng.integers(-120, 100, size=x[kinds == 9].shape)).astype(np.float32)
    return ref.bits(x)


@pytest.mark.parametrize("B,Hkv,C_,chunks,W", [(1, 1, 16, 1, 0), (2, 3, 48, 5, 7), (1, 2, 64, 3, 64), (2, 1, 256, 2, 10), (1, 1, 1024, 1, 0), (3, 2, 32, 9, 100)])
def test_pack_and_unpack_every_code(B, Hkv, C_, chunks, W):
    S, n = B * Hkv, chunks * C_ + W
    K, V = awkward_rows(S, n, 1), awkward_rows(S, n, 2)
    case = Case(B=B, Hkv=Hkv, n=n, C_=C_, W=W, K=from_bits(K), V=from_bits(V))
    assert case.packed == chunks and case.st.packed_chunks(0) == chunks
    for lo, hi in {(0, chunks), (chunks - 1, chunks), (0, 1), (chunks // 2, chunks)}:
        for got, rows in zip(case.st.unpack_chunks(0, lo, hi), (K, V)):
            want = ref.quantise(rows[:, lo * C_:hi * C_])[0]
            got = numbers(got)
            # the value low + c s in 64 bits, fp32 rounding of the sum (2^-24), one bf16 rounding
            bound = (2.0 ** -8 + 2.0 ** -23) * np.abs(want) + 2.0 ** -134
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(got), nan)
            assert (np.abs(got - want)[~nan] <= bound[~nan]).all()
    assert case.st.poll_status() == 0


def test_pack_infinities_and_nan_stay_in_their_group():
    K = awkward_rows(2, 64, 3)
    K[0, 3, 10], K[1, 20, 100], K[1, 21, 64] = 0x7F80, 0x7FC0, 0xFF80
    case = Case(Hkv=2, n=64, C_=16, W=0, K=from_bits(K), V=from_bits(K))
    for got in case.st.unpack_chunks(0, 0, 4):
        nan = np.isnan(numbers(got))
        want = np.zeros_like(nan)
        want[0, 3, :64] = want[1, 20, 64:] = want[1, 21, 64:] = True
        assert np.array_equal(nan, want)


def test_pack_the_whole_range_of_bf16():
    """groups whose numbers lie further apart than fp32 reaches, beside ordinary ones, and numbers of the smallest sizes there are"""
    rng = np.random.default_rng(11)
    x = rng.standard_normal((2, 128, 128)).astype(np.float32)
    top = ref.number(np.uint16(0x7F7F))
    x[0, ::2] = rng.uniform(-1, 1, size=(64, 128)) * top
    x[0, 0, 3], x[0, 0, 4], x[0, 0, 64:] = top, -top, 1.0
    x[0, 2, :64] = rng.integers(-15, 16, size=64) * np.exp2(123.0)         # on the borders
    x[1, ::4] = np.exp2(rng.integers(-133, 128, size=(32, 128))) * rng.choice([-1.0, 1.0], size=(32, 128))
    x[1, 1] *= np.exp2(-133.0)
    K, V = ref.bits(x), ref.bits(x[::-1])
    case = Case(Hkv=2, n=128, C_=64, W=0, K=from_bits(K), V=from_bits(V))
    for got, rows in zip(case.st.unpack_chunks(0, 0, 2), (K, V)):
        want, got = ref.quantise(rows)[0], numbers(got)
        over = np.abs(want) >= 2.0 ** 128 * (1 - 2.0 ** -9)                # rounded to bf16 that is an infinity
        assert np.array_equal(got[over], np.sign(want[over]) * np.inf)
        # as above: 64 bits, fp32 rounding of the sum, one bf16 rounding
        assert (np.abs(got - want)[~over] <= ((2.0 ** -8 + 2.0 ** -23) * np.abs(want) + 2.0 ** -134)[~over]).all()
    assert case.st.poll_status() == 0


def test_scale_is_rounded_once():
    """groups whose (largest - smallest) / 15 lies next to the middle of two bf16 numbers"""
    rng = np.random.default_rng(5)
    x = np.zeros((1, 64, 128), np.float32)
    ends = ref.number(ref.bits(np.exp2(rng.uniform(-3, 3, size=(200000, 2))) * [1, -1]))
    quotient = (ends[:, 0] - ends[:, 1]) / 15.0
    near = np.abs(quotient / np.exp2(np.floor(np.log2(quotient)) - 8) % 1.0 - 0.0)
    mid = np.abs((quotient / np.exp2(np.floor(np.log2(quotient)) - 7)) % 1.0 - 0.5)
    pick = ends[np.argsort(mid)[:128]]
    assert near.size and mid.min() < 1e-3
    x[0, :, 0], x[0, :, 1], x[0, :, 64], x[0, :, 65] = pick[:64, 0], pick[:64, 1], pick[64:, 0], pick[64:, 1]
    K = ref.bits(x)
    case = Case(Hkv=1, n=64, C_=64, W=0, K=from_bits(K), V=from_bits(K))
    want = ref.quantise(K)[0]
    for got in case.st.unpack_chunks(0, 0, 1):
        assert (np.abs(numbers(got) - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want)).all()


# ---- attention --------------------------------------------------------------------------------------------------------------------------

every_third = lambda s, t: (s + t) % 3 == 0
CASES = [  # what the store holds, what is asked for
    (dict(n=1, W=64), {}),
    (dict(n=63, W=64), {}),
    (dict(n=64, W=0), {}),                                                             # everything in 4 bits
    (dict(n=16, C_=16, W=0), {}),
    (dict(n=300), {}),
    (dict(n=300), dict(dense=True)),
    (dict(n=1000, C_=48, W=5, B=2, Hkv=3), dict(dense=True)),                          # tiles of 32 and 16 rows
    (dict(n=2100, C_=1024, W=3), dict(dense=True)),
    (dict(n=777, C_=16, W=0, Hkv=5), dict(dense=True)),
    (dict(n=1500, C_=32, W=100, G=4, B=2), dict(dense=True)),
    (dict(n=1500, C_=32, W=100, G=5, B=2), dict(dense=True)),
    (dict(n=900, C_=64, W=10, G=8), dict(dense=True)),
    (dict(n=900, C_=64, W=10, G=3, T=4), dict(dense=True)),                            # 12 query rows
    (dict(n=900, C_=64, W=10, G=1, T=16), dict(dense=True, causal=True)),
    (dict(n=900, C_=64, W=30, G=4, T=7), dict(dense=True, causal=True)),
    (dict(n=900, C_=128, W=128, G=8, T=16, B=2), dict(dense=True, causal=True)),        # 128 query rows: four groups
    (dict(n=700, C_=64, W=40, G=7, T=5), dict(dense=True)),                            # 35 query rows: two groups, the second with 3
    (dict(n=5, C_=64, W=64, T=5, G=2), dict(causal=True)),                             # a block that is the whole cache
    (dict(n=1100, W=64, listed=16, keep=every_third, Hkv=4), {}),
    (dict(n=1100, W=64, listed=16, keep=every_third, Hkv=4), dict(dense=True)),        # the list does not matter
    (dict(n=1100, W=64, listed=16, keep=every_third, packed=9, Hkv=4, G=2), {}),       # kept chunks in 4 bits and in bf16
    (dict(n=1100, W=64, listed=16, keep=every_third, packed=0), {}),                   # nothing in 4 bits
    (dict(n=1100, W=64, listed=7, keep=every_third, packed=14, G=4, T=2), dict(causal=True)),      # chunks behind the list in 4 bits
    (dict(n=640, C_=32, W=0, listed=20, keep=lambda s, t: False), {}),                 # nothing is left: 0 and -inf
    (dict(n=640, C_=32, W=0, listed=20, keep=lambda s, t: s == 1 and t == 19, Hkv=3, G=8), {}),    # one sequence has a chunk
    (dict(n=640, C_=32, W=3, listed=19, keep=lambda s, t: True, Hkv=3, G=6, T=3), dict(causal=True)),
    (dict(n=20000, C_=64, W=100, Hkv=1, G=2), dict(dense=True)),                       # cut along the sequence
    (dict(n=20011, C_=128, W=1000, Hkv=2, G=4, listed=100, keep=lambda s, t: t % 2 == s), {}),
    (dict(n=200, C_=16, W=4, B=40, Hkv=16), dict(dense=True)),                         # many sequences
    (dict(n=70, C_=16, W=4, B=100, Hkv=3, G=2, listed=4, keep=lambda s, t: (s * 7 + t) % 4 < s % 4), {}),      # CTAs that go from one to the next, with few rows and none kept
    (dict(n=333, C_=64, W=30, B=20, Hkv=8, G=7, listed=4, keep=every_third), {}),
    (dict(n=333, C_=32, W=30, B=20, Hkv=8, G=3, T=4), dict(dense=True, causal=True)),
    (dict(n=90, C_=16, W=40, B=6, Hkv=30, G=1, T=40), dict(dense=True, causal=True)),  # 40 query rows: three groups
    (dict(n=3, C_=16, W=1, B=200, Hkv=1, G=1), {}),
]


@pytest.mark.parametrize("held,asked", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention(held, asked):
    Case(**held).check(**asked)


@pytest.mark.parametrize("T", [1, 3])
def test_empty_cache(T):
    case = Case(n=0, T=T)
    _, out, lse = case.check()
    assert (out == 0).all() and torch.isinf(lse).all()
    case.check(dense=True)


def test_large_logits_and_offsets():
    """keys whose logits spread over hundreds, with an offset that all of them share"""
    rng = np.random.default_rng(3)
    K = ref.bits((20 * rng.standard_normal((2, 700, 128)) + 50 * rng.standard_normal((2, 1, 128))).astype(np.float32))
    case = Case(n=700, W=50, K=from_bits(K))
    case.check(dense=True)
    rising = ref.bits((np.linspace(0, 8, 700)[None, :, None] * np.ones((2, 1, 128))).astype(np.float32))      # the largest logit comes last
    case = Case(n=700, W=50, K=from_bits(rising))
    case.check(q=torch.ones((1, 1, 2, 128), dtype=torch.bfloat16, device="cuda"), dense=True)


@pytest.mark.parametrize("G", [1, 8, 16])
@pytest.mark.parametrize("sizes", [(1e-12, 1e-12), (1e12, 1e12), (1e-9, 1e9), (1e9, 1e-9)])
def test_values_of_any_size(G, sizes):
    """packed values, and bf16 ones beside them, of other sizes than 1; scales that grow and shrink along the sequence"""
    rng = np.random.default_rng(5)
    V = rng.standard_normal((2, 700, 128))
    V[:, :640] *= sizes[0] * np.exp2(rng.integers(-6, 7, size=(2, 10, 1))).repeat(64, axis=1)
    V[:, 640:] *= sizes[1]
    V[:, :, 64:] *= 1e-3
    case = Case(n=700, W=60, G=G, V=from_bits(ref.bits(V.astype(np.float32))))
    case.check(dense=True)


def test_queries_of_any_size():
    """each query row has a power of two of its own"""
    case = Case(n=500, G=4, B=1, Hkv=2)
    q = normal((1, 1, 8, 128), 3)
    q = (q.float() * torch.tensor([1e-20, 1.0, 1e4, 1e-3, 3e-39, 0.0, 1e2, 1e-8], device="cuda").view(1, 1, 8, 1)).to(torch.bfloat16)
    q[0, 0, 1, 5:] *= 1e-6
    case.check(q=q, dense=True)


def test_infinite_and_nan_rows():
    """a NaN row in the bf16 part, or in 4 bits, makes the sequences that see it NaN; logits of -inf have weight 0"""
    K = as_bits(normal((2, 300, 128), 2)).copy()
    K[0, 290, 5] = 0x7FC0
    case = Case(n=300, K=from_bits(K))
    q = normal((1, 1, 2, 128), 7)
    out = numbers(case.st.decode_attn_q4(0, q, dense=True))
    assert np.isnan(out[0, 0, 0]).all() and np.isfinite(out[0, 0, 1]).all()
    K = as_bits(normal((2, 300, 128), 2)).copy()
    K[1, 10, 77] = 0x7F80
    case = Case(n=300, K=from_bits(K))
    out = numbers(case.st.decode_attn_q4(0, q, dense=True))
    assert np.isfinite(out[0, 0, 0]).all() and np.isnan(out[0, 0, 1]).all()
    K = as_bits(normal((2, 60, 128), 2)).copy()
    K[:, ::2, 0] = 0xFF80                                   # logits of -inf where q's number is positive
    q = normal((1, 1, 2, 128), 8)
    q[..., 0] = 1.0
    case = Case(n=60, K=from_bits(K))
    case.check(q=q)
    K[:, :, 0] = 0xFF80
    case = Case(n=60, K=from_bits(K))
    _, out, lse = case.check(q=q)
    assert (out == 0).all() and torch.isinf(lse).all()


def test_scale_and_missing_lse():
    case = Case(n=500, G=2, B=2)
    q = normal((2, 1, 4, 128), 3)
    a = case.st.decode_attn_q4(0, q, scale=0.0)
    want = case.want(numbers(q) * 0.0, False, False)[0]
    assert np.abs(numbers(a) - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-4


# ---- as it is used ------------------------------------------------------------------------------------------------------------------------

def test_rows_of_packed_chunks_are_not_read_in_bf16():
    """pages handed back after packing: same result"""
    case = Case(n=700, W=64, listed=8, keep=every_third, Hkv=3, G=4)
    st = case.st
    q = normal((1, 1, 12, 128), 3)
    want = {d: st.decode_attn_q4(0, q, dense=d) for d in (False, True)}
    free, count = st.reclaim_pages(0, 0, case.packed, mode="packed")
    torch.cuda.synchronize()
    assert int(count) == 3 * case.packed and (st.page_table[0, :, :case.packed] == -1).all()
    st.k_pages[free[:int(count)].long()] = float("nan")
    for d in (False, True):
        assert torch.equal(st.decode_attn_q4(0, q, dense=d), want[d])
    assert st.poll_status() == 0
    st.pack_chunks(0, 0, 1)                                 # its rows are gone: flagged, the copy stays
    torch.cuda.synchronize()
    assert st.poll_status() == -3
    assert torch.equal(st.decode_attn_q4(0, q, dense=True), want[True])


def test_rolling_back_into_packed_chunks():
    case = Case(n=700, W=64)
    st = case.st
    assert st.packed_chunks(0) == 9
    k, v = st.unpack_chunks(0, 4, 5)
    st.set_len(0, 4 * 64 + 10)
    assert st.packed_chunks(0) == 4
    case.n, case.packed = 266, 4
    case.K, case.V = case.K[:, :266], case.V[:, :266]
    case.check(dense=True)
    st.set_len(0, 256)                                      # the chunk's rows as they were kept, and others behind them
    st.append(0, k, v)
    more = [normal((2, 100, 128), 50 + i) for i in range(2)]
    st.append(0, *more)
    case.n, case.K, case.V = 420, torch.cat([case.K[:, :256], k, more[0]], 1), torch.cat([case.V[:, :256], v, more[1]], 1)
    case.check(dense=True)
    st.pack_chunks(0, 4, 5)
    case.packed = 5
    case.check(dense=True)
    st.set_len(0, 0)
    assert st.packed_chunks(0) == 0


def test_lengths_and_packing_replayed_on_another_state():
    """a captured kvE_set_len lowers what the device holds packed at replay time; captured packing names no chunk without rows"""
    case = Case(n=200, W=64, packed=0, max_tokens=740)
    st = case.st
    torch.cuda.synchronize()
    cut, pack = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(cut):
        st.set_len(0, 130)
    st.adopt_device_state(0)
    st.append(0, normal((2, 500, 128), 80), normal((2, 500, 128), 81))
    st.pack_chunks(0, 0, 9)
    torch.cuda.synchronize()
    with torch.cuda.graph(pack):
        st.pack_chunks(0, 0, 9)
    cut.replay()
    st.adopt_device_state(0)
    assert st.packed_chunks(0) == 2

    def put(n, seed):
        more = [normal((2, n, 128), seed + i) for i in range(2)]
        st.append(0, *more)
        case.K, case.V, case.n = torch.cat([case.K, more[0]], 1), torch.cat([case.V, more[1]], 1), case.n + n
    case.K, case.V, case.n, case.packed = case.K[:, :130], case.V[:, :130], 130, 2
    put(400, 82)
    case.check(dense=True)
    pack.replay()
    st.adopt_device_state(0)
    assert st.packed_chunks(0) == 8
    case.packed = 8
    case.check(dense=True)
    put(100, 84)
    case.check(dense=True)


def test_pages_whose_offsets_pass_32_bits():
    from paper_2509_21354_b200 import binding as b
    chunks, C_, n, G = 16600, 1024, 2100, 2                # numbers and 4-bit bytes of the pool both pass 2^31
    far = np.arange(chunks, dtype=np.int32)[::-1]
    st = b.Store(B=1, H=1, Hq=G, C_=C_, W=20, max_tokens=chunks * C_, d_g=64, page_perm=far)
    st.attach_q4(page_perm=far)
    q, k, v = normal((1, n, G, 128), 1), normal((1, n, 1, 128), 2), normal((1, n, 1, 128), 3)
    turned, _ = st.append_rope(0, q, k, v, b.Rope((0, 64)), positions=torch.zeros((1, n, 2), dtype=torch.int32, device="cuda"))      # (an angle of 0)
    assert torch.equal(turned, q)
    st.pack_chunks(0, 0, 2)
    K, V = as_bits(k)[0, :, 0], as_bits(v)[0, :, 0]
    kq, vq = ref.quantise(K[:2048])[0], ref.quantise(V[:2048])[0]
    for got, want in zip(st.unpack_chunks(0, 0, 2), (kq, vq)):
        assert (np.abs(numbers(got)[0] - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want) + 2.0 ** -134).all()
    out = st.decode_attn_q4(0, q[:, -1:].contiguous(), dense=True)
    assert st.poll_status() == 0
    want, _, spread = ref.attend(numbers(q)[0, -1], np.concatenate([kq, ref.number(K[2048:])]), np.concatenate([vq, ref.number(V[2048:])]), np.ones((G, n), bool))
    assert (np.abs(numbers(out)[0, 0] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -13 * spread).all()      # (Case.compare's bound with logits of this size)


def test_two_graphs_of_one_handle_in_turn():
    """launches of different shapes share the records and counters of the workspace"""
    case = Case(B=2, Hkv=3, G=4, n=1500, T=5)
    st = case.st
    calls = []
    for T, causal in ((1, False), (5, True), (3, False)):
        q = normal((2, T, 12, 128), 60 + T)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
        run = lambda q=q, out=out, lse=lse, causal=causal: st.decode_attn_q4(0, q, dense=True, causal=causal, out=out, lse=lse)
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        calls.append((graph, out, lse, out.clone(), lse.clone(), q))      # (q: the graph reads it)
    for i in (0, 1, 2, 1, 0, 2, 2, 0):
        calls[i][1].fill_(7.0)
        calls[i][0].replay()
    torch.cuda.synchronize()
    assert st.poll_status() == 0
    for _, out, lse, want, want_lse, _ in calls:
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_layers_are_apart():
    case = Case(n=500, n_layers=3, layer=1, Hkv=2)
    st = case.st
    assert [st.packed_chunks(i) for i in range(3)] == [0, 6, 0]
    st.append(2, *(normal((2, 90, 128), i) for i in range(2)))
    case.check(dense=True)
    q = normal((1, 1, 2, 128), 1)
    assert (st.decode_attn_q4(0, q) == 0).all()
    assert (st.kv4_pages[st.page_table4[0].flatten().long()] == 0xFF).all()


def test_a_decode_loop_from_a_graph():
    """rotary append, then attention over the packed history, replayed; the host packs in between"""
    from paper_2509_21354_b200 import binding as b
    B, Hkv, G = 2, 2, 4
    case = Case(B=B, Hkv=Hkv, G=G, n=200, C_=32, W=40, max_tokens=400)
    st, rope = case.st, b.Rope((16, 24, 24))
    q, k, v = normal((B, 1, Hkv * G, 128), 1), normal((B, 1, Hkv, 128), 2), normal((B, 1, Hkv, 128), 3)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty((B, 1, Hkv * G), dtype=torch.float32, device="cuda")

    def step(reserve):
        st.append_rope_next(0, q, k, v, rope, q_out=turned, n_reserve=reserve)
        st.decode_attn_q4(0, turned, dense=True, out=out, lse=lse)
    step(0)
    st.set_len(0, 200)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(150)
    st.set_len(0, 200)
    axis, freq = np.array(list(rope.c.axis)), np.array(list(rope.c.inv_freq))
    for i in range(130):
        for j, t in enumerate((q, k, v)):
            t.copy_(normal(t.shape, 1000 + 3 * i + j))
        g.replay()
        at = np.full((B, 1, 3), 200 + i)
        row = [ref.turn(numbers(k), at, axis, freq, False), numbers(v)]
        # the stored key row, as the device rounded it
        table = st.page_table[0].cpu().numpy()
        n = 200 + i
        stored = torch.stack([st.k_pages[table[s, n // 32], n % 32] for s in range(st.S)])[:, None]
        assert np.abs(numbers(stored).reshape(B, Hkv, 128) - row[0][:, 0]).max() <= 2.0 ** -8 * np.abs(row[0]).max() + 1e-5
        case.K, case.V, case.n = torch.cat([case.K, stored], 1), torch.cat([case.V, v.reshape(st.S, 1, 128)], 1), n + 1
        if i in (0, 31, 77, 129):
            torch.cuda.synchronize()
            case.compare(out, lse, *case.want(numbers(turned), True, False))
        if i == 60:
            st.adopt_device_state(0)
            done = (case.n - 40) // 32
            st.pack_chunks(0, case.packed, done)
            case.packed = done
    assert st.poll_status() == 0


def test_triggers_and_packing_together():
    """gated decoding: after every trigger the chunk that left the window is packed"""
    from paper_2509_21354_b200 import binding as b
    case = Case(n=300, C_=32, W=40, listed=8, keep=lambda s, t: t % 2 == 0, Hkv=2, G=1, max_tokens=500)
    st = case.st
    rng = np.random.default_rng(1)
    weight = lambda *shape: rng.standard_normal(shape).astype(np.float32) / 16
    lstm = b.LstmWeights(dict(W_ih=weight(256, 256), W_hh=weight(256, 64), b_ih=weight(256), b_hh=weight(256), w_s=weight(64), b_s=0.0))
    for i in range(70):
        k, v = normal((2, 1, 128), 600 + i), normal((2, 1, 128), 800 + i)
        ready = st.append(0, k, v)
        case.K, case.V, case.n = torch.cat([case.K, k], 1), torch.cat([case.V, v], 1), case.n + 1
        if ready:
            t = case.listed
            st.summarize_chunks(0, t, t + 1)
            st.gate_next(0, lstm, 0.5)
            st.pack_chunks(0, t, t + 1)
            torch.cuda.synchronize()
            case.listed = case.packed = t + 1
            case.kept = [st.keep_idx[0, s, :int(st.keep_cnt[0, s])].tolist() for s in range(2)]
        if ready or i % 20 == 0:
            case.check(seed=i)
    assert case.listed == 10


def test_another_stream_and_two_handles():
    side = torch.cuda.Stream()
    cases = [Case(n=3000, Hkv=2, G=4, seed=10 * i) for i in range(2)]
    q = normal((1, 1, 8, 128), 3)
    want = [c.st.decode_attn_q4(0, q, dense=True) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(side):
            a = cases[0].st.decode_attn_q4(0, q, dense=True)
        z = cases[1].st.decode_attn_q4(0, q, dense=True)
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(z, want[1])


def test_same_bits_every_time():
    case = Case(n=30000, Hkv=2, G=4, C_=64, W=200)
    q = normal((1, 1, 8, 128), 3)
    first = case.st.decode_attn_q4(0, q, dense=True)
    for _ in range(10):
        assert torch.equal(case.st.decode_attn_q4(0, q, dense=True), first)


def test_bad_pages_are_flagged_and_skipped():
    case = Case(n=700, W=64, Hkv=2)
    st, q = case.st, normal((1, 1, 2, 128), 3)
    want = st.decode_attn_q4(0, q, dense=True)
    for table, chunk in ((st.page_table4, 3), (st.page_table, 10)):
        for bad in (-1, 1 << 30):
            good = int(table[0, 0, chunk])
            table[0, 0, chunk] = bad
            got = st.decode_attn_q4(0, q, dense=True)
            torch.cuda.synchronize()
            assert st.poll_status() == -3 and torch.equal(got[0, 0, 1], want[0, 0, 1])
            table[0, 0, chunk] = good
    st.page_table4[0, 1, 2] = -1
    k = [torch.full((2, 64, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    st.unpack_chunks(0, 2, 3, *k)
    torch.cuda.synchronize()
    assert st.poll_status() == -3 and (k[0][1] == 9.0).all() and not (k[0][0] == 9.0).any()
    assert torch.equal(st.decode_attn_q4(0, q, dense=True)[0, 0, 0], want[0, 0, 0]) and st.poll_status() == -3


def test_refusals():
    from paper_2509_21354_b200 import binding as b
    case = Case(n=300, T=2, G=2, Hkv=1)
    st, lib, h = case.st, case.st.lib, case.st.handle
    q = normal((1, 2, 2, 128), 1)
    out = torch.empty_like(q)
    go = lambda q_=q.data_ptr(), t=2, dense=0, causal=0, o=out.data_ptr(), layer=0: lib.kvE_decode_attn_q4(h, layer, q_, t, dense, causal, o, None, 0.1, None)
    assert go() == 0
    assert go(q_=None) == go(o=None) == go(t=0) == go(t=-1) == go(layer=1) == go(layer=-1) == go(q_=q.data_ptr() + 2) == go(o=out.data_ptr() + 8) == -1
    assert go(t=3) == -3
    assert lib.kvE_pack_chunks(h, 0, -1, 0, None) == lib.kvE_pack_chunks(h, 0, 2, 1, None) == lib.kvE_pack_chunks(h, 1, 0, 1, None) == -1
    assert lib.kvE_pack_chunks(h, 0, 0, 4, None) == -4                      # the window stays in bf16
    assert lib.kvE_pack_chunks(h, 0, 3, 3, None) == 0
    st.set_len(0, 100)
    assert st.packed_chunks(0) == 1 and lib.kvE_pack_chunks(h, 0, 2, 3, None) == -4
    st.set_len(0, 300)
    assert lib.kvE_pack_chunks(h, 0, 2, 3, None) == -4                      # no gaps
    k = torch.empty((1, 64, 128), dtype=torch.bfloat16, device="cuda")
    unpack = lambda lo, hi, ko=k.data_ptr(), vo=k.data_ptr(): lib.kvE_unpack_chunks(h, 0, lo, hi, ko, vo, None)
    assert unpack(0, 2) == unpack(1, 2) == -4
    assert unpack(-1, 1) == unpack(1, 0) == unpack(0, 1, ko=None) == unpack(0, 1, vo=k.data_ptr() + 2) == -1
    assert unpack(0, 1) == 0 and unpack(1, 1) == 0
    free, count = torch.empty(8, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    assert lib.kvE_reclaim_pages(h, 0, 0, 2, 2, free.data_ptr(), 8, count.data_ptr(), None) == -4
    assert lib.kvE_reclaim_pages(h, 0, 0, 1, 3, free.data_ptr(), 8, count.data_ptr(), None) == -1
    # a causal block needs rows of its own behind the packed chunks
    tight = Case(n=65, C_=64, W=1, T=3, G=1)
    q3 = normal((1, 3, 2, 128), 1)
    with pytest.raises(b.KveError) as e:
        tight.st.decode_attn_q4(0, q3, causal=True)
    assert e.value.rc == -4
    tight.check(q=q3)
    # without 4-bit pages
    bare = b.Store(B=1, H=1, C_=64, W=0, max_tokens=128, d_g=64)
    q1 = normal((1, 1, 1, 128), 1)
    for call in (lambda: bare.decode_attn_q4(0, q1), lambda: bare.pack_chunks(0, 0, 0), lambda: bare.unpack_chunks(0, 0, 1)):
        with pytest.raises(b.KveError) as e:
            call()
        assert e.value.rc == -4
    for C_, t in ((24, 1), (64, 129), (64, 0)):
        with pytest.raises(b.KveError):
            b.Store(B=1, H=1, C_=C_, W=0, max_tokens=128, d_g=64).attach_q4(max_query_tokens=t)
    with pytest.raises(AssertionError):
        case.st.decode_attn_q4(0, q.float())
    with pytest.raises(AssertionError):
        case.st.decode_attn_q4(0, q[:, :, :1])
    # attach: buffers are checked before they are taken
    buf = lambda **kw: C.byref(b.kvE_q4_buffers(**{**dict(kv4_pages=st.kv4_pages.data_ptr(), n_pages4=4, page_table4=st.page_table4.data_ptr(),
                                                        max_query_tokens=1, workspace=(st.q4_workspace.data_ptr() + 255) // 256 * 256, workspace_bytes=st.q4_workspace.numel() - 256), **kw}))
    attach = lambda **kw: lib.kvE_attach_q4(h, buf(**kw))
    assert attach(kv4_pages=None) == attach(kv4_pages=st.kv4_pages.data_ptr() + 4) == attach(n_pages4=0) == attach(page_table4=None) == attach(workspace=None) == -1
    assert attach(workspace_bytes=10) == -3 and attach(max_query_tokens=100) == -2 and attach(max_query_tokens=0) == -1
    assert st.packed_chunks(0) == 1


def test_attaching_again_starts_empty():
    case = Case(n=300)
    assert case.st.packed_chunks(0) == 3
    old = case.st.kv4_pages
    case.st.attach_q4()
    assert case.st.packed_chunks(0) == 0 and case.st.kv4_pages.data_ptr() != old.data_ptr()
    case.packed = 0
    case.check(dense=True)


def test_profile_names():
    case = Case(n=300)
    case.st.profile(True)
    case.st.pack_chunks(0, 0, 3)
    case.st.decode_attn_q4(0, normal((1, 1, 2, 128), 1))
    us = case.st.profile_read()
    assert us["pack"] > 0 and us["attn_q4"] > 0 and us["attn"] is None
