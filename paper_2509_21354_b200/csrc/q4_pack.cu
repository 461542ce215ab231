// kvE_pack_chunks / kvE_unpack_chunks: completed chunks to 4 bits and back (format: q4.cuh).
//
// HBM-bound in principle: a row is read (256 bytes) and its 72 bytes written.  A warp takes a unit of 16 rows; its loads are all in flight
// before the first row is looked at.  Eight lanes hold a group: largest and smallest number in packed bf16 steps, then the codes in
// packed fp32 pairs.
//
// The codes are those of the real numbers, not of fp32 rounding: with bf16 input, numbers that lie on a border are not rare
// (x - low and s have few bits: one number in 250 of a normal distribution).  rint((x - low) / s (1 - 2^-13)) is the code or one less, as the
// quotient's own relative error is below 2^-21 and it is 15 1/16 at most, and the remainder x - low - c s says which: x - low is rounded up, so that it is above a border
// (which fp32 holds) exactly where the real difference is, and the remainder of that is exact.
#include <type_traits>

#include "q4.cuh"

namespace kve {

constexpr int PK_WARPS = 8;
constexpr float PK_SHY = 1.f - 0x1p-13f;      // 1 / scale is taken that much smaller
constexpr int PK_PITCH = 20;      // words of a row of values on their way between lanes: the four lanes of a column read different banks

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// a b + c of two pairs, rounded up
__device__ __forceinline__ float2 fma2_up(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rp.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// bf16 bits of (high - low) / 15, rounded once; NaN where a number of the group is not finite
__device__ __forceinline__ uint32_t q4_scale_bits(float high, float low) {
  // within 4 units in the last place; the halves cannot overflow
  float f = (high * 0.5f - low * 0.5f) * (2.f / 15.f);
  if (!(f < INFINITY)) return 0x7fffu;
  uint32_t u = __float_as_uint(f);
  if (abs((int)(u & 0xffffu) - 0x8000) <= 8 || f < 1e-30f) {      // next to the middle of two bf16 numbers, or short of bits: from 64 bits
    const double q = ((double)high - (double)low) / 15.0;
    f = __double2float_rz(q);
    u = __float_as_uint(f) | ((double)f != q ? 1u : 0u);           // (rounding to odd: the second rounding sees which side the rest is on)
  }
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// The codes of eight numbers of a group (c[i]: whole numbers 0..15).  ANY: scales may be so small that 1 / scale overflows, or so large that largest - low does: such
// groups are taken times a power of two (exact: bf16 numbers keep 16 bits to spare at either end).
template <bool ANY>
__device__ __forceinline__ void q4_codes(const uint4& x, float scale, float low, float inv, float (&c)[8]) {
  const float up = !ANY ? 1.f : (scale < 0x1p-60f ? 0x1p64f : (scale > 0x1p120f ? 0x1p-8f : 1.f));
  const float s = ANY ? scale * up : scale, half = 0.5f * s;      // (scale 0: the codes do not matter)
  if (ANY) inv = s > 0.f ? __frcp_rn(s) * PK_SHY : 0.f;
  const float2 up2 = make_float2(up, up), off = make_float2(-low * up, -low * up), inv2 = make_float2(inv, inv), neg_s = make_float2(-s, -s);
  const float2 magic = make_float2(0x1.8p23f, 0x1.8p23f), unmagic = make_float2(-0x1.8p23f, -0x1.8p23f);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 t = fma2_up(make_float2(bf16lo(w[e]), bf16hi(w[e])), up2, off);      // x - low
    float2 n = add2(fma2(t, inv2, magic), unmagic);                                   // the code, or one less
    const float2 r = fma2(n, neg_s, t);
    if (r.x > half) n.x += 1.f;
    if (r.y > half) n.y += 1.f;
    c[2 * e] = n.x;
    c[2 * e + 1] = n.y;
  }
}
// four codes, 4 bits each, in the low half of a word
__device__ __forceinline__ uint32_t q4_half(float c0, float c1, float c2, float c3) {
  return __float_as_uint(fmaf(fmaf(c3, 16.f, c2), 256.f, fmaf(c1, 16.f, c0)) + 8388608.f);
}

// the keep list covers chunk t of sequence s and leaves it out: gated attention does not come to it
__device__ __forceinline__ bool discarded(const LayerView& v, int s, int t) {
  if (t >= *v.n_listed) return false;
  const int32_t* kept = v.keep_idx + (long long)s * v.max_chunks;
  int lo = 0, hi = v.keep_cnt[s];
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (kept[mid] < t) lo = mid + 1; else hi = mid;
  }
  return lo == v.keep_cnt[s] || kept[lo] != t;
}

__global__ void __launch_bounds__(PK_WARPS * 32) kve_pack_kernel(LayerView v, Q4Pages p, int t0, int n_chunks, int n_units, FastDiv by_units, FastDiv by_chunks,
                                                                 int32_t* ticket) {
  __shared__ uint32_t codes[PK_WARPS][Q4_UNIT_ROWS * PK_PITCH];
  __shared__ int had_packed;
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int rows = 0, arrived = 0;
  if (threadIdx.x == 0) {
    rows = v.seq_len[0];
    had_packed = *reinterpret_cast<const volatile int32_t*>(v.n_packed);
  }
  const int item = blockIdx.x * PK_WARPS + warp;
  const bool live = item < n_units;
  const int per_chunk = v.C / Q4_UNIT_ROWS;
  const bool is_v = item & 1;
  const int x = (int)by_units.div((uint32_t)(item >> 1)), unit = (item >> 1) - x * per_chunk;
  const int s = (int)by_chunks.div((uint32_t)x), t = t0 + x - s * n_chunks;
  const long long at = (long long)s * v.max_chunks + t, page = live ? v.page_table[at] : -1, page4 = live ? p.table[at] : -1;
  const bool source = page >= 0 && page < v.n_pages, target = page4 >= 0 && page4 < p.n_pages, whole = source && target;
  const int half = lane >> 4, l16 = lane & 15;
  uint8_t* dst = p.kv + (page4 * per_chunk + unit) * Q4_PAIR_BYTES + (is_v ? Q4_UNIT_BYTES : 0);
  uint4 row[8];
  if (whole) {
    const uint4* src = reinterpret_cast<const uint4*>((is_v ? v.v_pages : v.k_pages) + (page * v.C + unit * Q4_UNIT_ROWS) * D) + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) row[i] = __ldcs(src + i * 32);      // rows 2 i + half
  }
  // The count of packed chunks goes up when every CTA has read it: a chunk that was not packed before and whose rows are gone has no copy that could stay.
  __syncthreads();
  if (threadIdx.x == 0) arrived = atomicAdd(ticket, 1);      // (no fence: the barrier has waited for the read, which is all that the last one's write must not pass)
  auto count = [&]() {      // (the ticket has come back by the time the rows have)
    if (threadIdx.x != 0 || arrived != (int)gridDim.x - 1) return;
    const int now = min(t0 + n_chunks, rows / v.C);      // (a replay may find another length, or fewer chunks packed: none is named that has no rows, no gap left)
    if (had_packed >= t0 && now > had_packed) *v.n_packed = now;
    *ticket = 0;      // clean for the next launch
  };
  if (!live) {
    count();
    return;
  }
  if (!whole) {      // (warp by warp)
    if (!source && target && t >= had_packed)      // 16 rows of two groups that stand for NaN, not for what the page held before
      *reinterpret_cast<uint32_t*>(dst + Q4_CODE_BYTES + lane * 4) = 0x7fff7fffu;
    if (lane == 0 && !(page == -1 && target && discarded(v, s, t))) set_status(v.status, ERR_CAPACITY);
    count();
    return;
  }
  // (largest, -smallest) of this lane's part of row 2 i + half; then of the whole group, lane by lane: lane 8 g + i has group g of the rows 2 i and 2 i + 1
  uint32_t m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4& r = row[i];
    const uint32_t mx = max2_nan(max2_nan(r.x, r.y), max2_nan(r.z, r.w)), mn = min2_nan(min2_nan(r.x, r.y), min2_nan(r.z, r.w)) ^ 0x80008000u;
    m[i] = max2_nan(__byte_perm(mx, mn, 0x5410), __byte_perm(mx, mn, 0x7632));
  }
#pragma unroll
  for (int o = 4; o >= 1; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const uint32_t keep = upper ? m[i + o] : m[i], give = upper ? m[i] : m[i + o];
      m[i] = max2_nan(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  const uint32_t sb = q4_scale_bits(bf16lo(m[0]), -bf16hi(m[0])), head = sb | (sb == 0x7fffu ? 0x7fff0000u : (m[0] & 0xffff0000u) ^ 0x80000000u);
  const float my_scale = __uint_as_float(sb << 16), my_inv = my_scale > 0.f ? __frcp_rn(my_scale) * PK_SHY : 0.f;
  *reinterpret_cast<uint32_t*>(dst + Q4_CODE_BYTES + (2 * (lane & 7) + half) * 8 + ((lane >> 3) & 1) * 4) = head;
  auto encode = [&](auto any) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int from = (lane & 24) | i, line = 2 * i + half;
      const uint32_t g = __shfl_sync(0xffffffffu, head, from);
      const float inv = __shfl_sync(0xffffffffu, my_inv, from);
      float c[8];
      q4_codes<decltype(any)::value>(row[i], bf16lo(g), bf16hi(g), inv, c);
      if (is_v) {
        codes[warp][line * PK_PITCH + l16] = __byte_perm(q4_half(c[0], c[1], c[2], c[3]), q4_half(c[4], c[5], c[6], c[7]), 0x5410);
      } else {
        const uint32_t w = __byte_perm(q4_half(c[0], c[2], c[4], c[6]), q4_half(c[1], c[3], c[5], c[7]), 0x5410);
        *reinterpret_cast<uint32_t*>(dst + line * 64 + (l16 & 3) * 16 + (l16 >> 2) * 4) = w;
      }
    }
  };
  if (__any_sync(0xffffffffu, my_scale > 0.f && (my_scale < 0x1p-100f || my_scale > 0x1p120f))) encode(std::true_type());
  else encode(std::false_type());
  if (is_v) {
    __syncwarp();
    const int g8 = lane >> 2, t4 = lane & 3;
    const uint32_t* cw = codes[warp] + 2 * t4 * PK_PITCH + g8;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4] = {cw[8 * h], cw[8 * PK_PITCH + 8 * h], cw[PK_PITCH + 8 * h], cw[9 * PK_PITCH + 8 * h]};
      transpose_bytes(w);
      *reinterpret_cast<uint4*>(dst + h * 512 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  count();
}

__global__ void __launch_bounds__(PK_WARPS * 32) kve_unpack_kernel(LayerView v, Q4Pages p, int t0, int n_chunks, int n_units, FastDiv by_units, FastDiv by_chunks,
                                                                   uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out) {
  __shared__ uint32_t codes[PK_WARPS][Q4_UNIT_ROWS * PK_PITCH];
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int item = blockIdx.x * PK_WARPS + warp;
  if (item >= n_units) return;
  const int per_chunk = v.C / Q4_UNIT_ROWS;
  const bool is_v = item & 1;
  const int x = (int)by_units.div((uint32_t)(item >> 1)), unit = (item >> 1) - x * per_chunk;
  const int s = (int)by_chunks.div((uint32_t)x), t = t0 + x - s * n_chunks;
  const long long page4 = p.table[(long long)s * v.max_chunks + t];
  if (page4 < 0 || page4 >= p.n_pages || t >= *v.n_packed) {      // (packing that was captured and has not run is in the host's count already)
    if (lane == 0) set_status(v.status, ERR_CAPACITY);
    return;
  }
  const int half = lane >> 4, l16 = lane & 15;
  const uint8_t* src = p.kv + (page4 * per_chunk + unit) * Q4_PAIR_BYTES + (is_v ? Q4_UNIT_BYTES : 0);
  uint4* dst = reinterpret_cast<uint4*>((is_v ? v_out : k_out) + ((long long)x * v.C + unit * Q4_UNIT_ROWS) * D) + lane;
  uint32_t* cw = codes[warp];
  // keys: lane (row, t) has the words j = 0..3, numbers 32 j + 8 t .. + 7: word 4 j + t of the row;
  // values: back to a word per row and eight numbers, natural order
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 q = __ldcs(reinterpret_cast<const uint4*>(src + h * 512 + lane * 16));
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
    const int g8 = lane >> 2, t4 = lane & 3;
    if (is_v) {
      transpose_bytes(w);
      uint32_t* o = cw + 2 * t4 * PK_PITCH + g8 + 8 * h;
      o[0] = w[0]; o[8 * PK_PITCH] = w[1]; o[PK_PITCH] = w[2]; o[9 * PK_PITCH] = w[3];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) cw[(h * 8 + g8) * PK_PITCH + 4 * j + t4] = w[j];
    }
  }
  const uint2 head = __ldcs(reinterpret_cast<const uint2*>(src + Q4_CODE_BYTES + (lane & 15) * 8));      // lanes 0-15: a row each
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int line = 2 * i + half;
    const uint32_t sx = __shfl_sync(0xffffffffu, head.x, line), sy = __shfl_sync(0xffffffffu, head.y, line), sl = l16 < 8 ? sx : sy;
    const float scale = bf16lo(sl), low = bf16hi(sl);
    const uint32_t w = cw[line * PK_PITCH + l16];
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {      // numbers 2 e, 2 e + 1 (their product with the scale is exact)
      const uint32_t a = (w >> (is_v ? 8 * e : 4 * e)) & 15u, b = (w >> (is_v ? 8 * e + 4 : 16 + 4 * e)) & 15u;
      o[e] = pack_bf16x2(fmaf((float)a, scale, low), fmaf((float)b, scale, low));
    }
    __stcs(dst + i * 32, make_uint4(o[0], o[1], o[2], o[3]));
  }
}

static unsigned pack_grid(const LayerView& v, int chunks, int& n_units, FastDiv& by_units, FastDiv& by_chunks) {
  const int per_chunk = v.C / Q4_UNIT_ROWS;
  n_units = v.S * chunks * per_chunk * 2;
  by_units = fast_div((uint32_t)per_chunk);
  by_chunks = fast_div((uint32_t)chunks);
  return (unsigned)((n_units + PK_WARPS - 1) / PK_WARPS);
}

cudaError_t launch_pack(const LayerView& v, const Q4Pages& p, int t0, int t1, int32_t* ticket, cudaStream_t st) {
  int n_units;
  FastDiv by_units, by_chunks;
  const unsigned grid = pack_grid(v, t1 - t0, n_units, by_units, by_chunks);
  return launch_pdl(kve_pack_kernel, dim3(grid), dim3(PK_WARPS * 32), 0, st, v, p, t0, t1 - t0, n_units, by_units, by_chunks, ticket);
}

cudaError_t launch_unpack(const LayerView& v, const Q4Pages& p, int t0, int t1, void* k_out, void* v_out, cudaStream_t st) {
  int n_units;
  FastDiv by_units, by_chunks;
  const unsigned grid = pack_grid(v, t1 - t0, n_units, by_units, by_chunks);
  return launch_pdl(kve_unpack_kernel, dim3(grid), dim3(PK_WARPS * 32), 0, st, v, p, t0, t1 - t0, n_units, by_units, by_chunks,
                    static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out));
}

}  // namespace kve
