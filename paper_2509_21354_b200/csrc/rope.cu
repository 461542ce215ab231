// kvE_append_rope / kvE_append_rope_next: rotary positions on several axes (time, height, width, ...) turned into q and k while k and
// v go to the tail of every sequence's pages.
//
// Pair j of a row turns by phi_j = pos[axis_j] inv_freq_j:  (a, b) -> (a cos - b sin, b cos + a sin), in fp32, rounded to bf16 once.
// The angle is reduced in 64 bits: inv_freq comes in turns, whole turns are taken off pos * turns exactly, and what is left (half a
// turn at most) goes to sincospif in 32.  In 32 bits alone a position of 10^6 leaves an angle off by 0.06.
//
// HBM-bound: (Hq + 2 Hkv) rows of 256 bytes a token are read and written once.  All heads of a token share its 64 angles, so a CTA
// takes whole tokens: its first threads work out the angles while the first rows are on their way, the rest is one pass.  A thread holds
// 16 numbers of one row (two 16-byte pieces, 64 numbers apart), whose pairs it has whole in either layout; eight threads a row.
#include <type_traits>

#include "common.cuh"
#include "kernels.h"

namespace kve {

constexpr int RP_THREADS = 256;
constexpr int RP_CTAS = 6;                    // per SM (8 x 4096 tokens of 96 rows: 254 us; 5 of them 264, 4 281, 8 301)
constexpr int RP_ROWS = RP_THREADS / 8;       // rows under way at a time
constexpr int RP_MAX_TOKENS = 16;             // tokens of one CTA (few heads)
constexpr int RP_TABLE = 8 * 9;               // (cos, sin) of pair 8 x + e at 9 x + e: eight threads read different banks

struct RopeArgs : RopeCall {
  int n_tokens, tokens_per_cta;      // B n_new; of one CTA
  FastDiv by_rows, by_new, by_c;
};

// NEXT: at the length the device holds, which the last CTA advances (as kve_append_next_kernel does)
template <bool NEXT>
__global__ void __launch_bounds__(RP_THREADS, RP_CTAS) kve_append_rope_kernel(LayerView v, RopeArgs a) {
  __shared__ float2 table[RP_MAX_TOKENS][RP_TABLE];
  __shared__ int last;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, x = tid & 7;
  const int tok0 = blockIdx.x * a.tokens_per_cta, n_tok = min(a.tokens_per_cta, a.n_tokens - tok0);
  const int rows = a.Hq + 2 * v.H, n_items = n_tok * rows;
  const int off_a = 8 * x, off_b = 64 + 8 * x;      // the thread's two pieces of a row (adjacent pairs too: side by side they made half of every 32-byte sector a load of its own, 254 -> 264 us)

  // a row under way: its numbers, its token, where it goes (null: nowhere), whether it turns
  struct Row { uint4 lo, hi; uint16_t* dst; int tok; bool turns; };
  auto fetch = [&](int item) {
    Row r;
    r.dst = nullptr;
    r.tok = 0;
    r.turns = false;
    if (item >= n_items) return r;
    r.tok = (int)a.by_rows.div((uint32_t)item);
    const int row = item - r.tok * rows, t = tok0 + r.tok;
    const int b = (int)a.by_new.div((uint32_t)t), i = t - b * a.n_new;
    const int kind = row < a.Hq ? 0 : (row < a.Hq + v.H ? 1 : 2), h = kind == 0 ? row : row - a.Hq - (kind == 2 ? v.H : 0);
    r.turns = kind != 2;
    const uint16_t* base = kind == 0 ? a.q.data : (kind == 1 ? a.k.data : a.v.data);
    const long long stride_b = kind == 0 ? a.q.stride_b : (kind == 1 ? a.k.stride_b : a.v.stride_b);
    const long long stride_t = kind == 0 ? a.q.stride_t : (kind == 1 ? a.k.stride_t : a.v.stride_t);
    const long long stride_h = kind == 0 ? a.q.stride_h : (kind == 1 ? a.k.stride_h : a.v.stride_h);
    const uint16_t* p = base + b * stride_b + i * stride_t + h * stride_h;
    r.lo = *reinterpret_cast<const uint4*>(p + off_a);      // (not the read-only path: q may be turned in place)
    r.hi = *reinterpret_cast<const uint4*>(p + off_b);
    if (kind == 0) {
      r.dst = a.q_out + ((long long)t * a.Hq + h) * D;
      return r;
    }
    const int n0 = NEXT ? *reinterpret_cast<const volatile int32_t*>(v.seq_len + b) : a.pos0;
    if (n0 < 0 || n0 > v.max_tokens - a.n_new) {      // no room: nothing is stored (NEXT: flagged by the last CTA)
      if (!NEXT) set_status(v.status, ERR_CAPACITY);
      return r;
    }
    const int pos = n0 + i, chunk = (int)a.by_c.div((uint32_t)pos);
    const long long page = v.page_table[((long long)b * v.H + h) * v.max_chunks + chunk];
    if (page < 0 || page >= v.n_pages) { set_status(v.status, ERR_CAPACITY); return r; }
    r.dst = (kind == 1 ? v.k_pages : v.v_pages) + (page * v.C + (pos - chunk * v.C)) * D;
    return r;
  };

  Row cur = fetch(tid >> 3);
  // Angles: warp w has the pairs 8 w .. 8 w + 7, eight lanes a token.  (The launch's arrays are read at fixed places only.)
  {
    const int w = tid >> 5, e = tid & 7;
    double turns = 0.0;
    int axis = 0;
    auto pick = [&](auto first) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (e == j) { turns = a.turns[decltype(first)::value + j]; axis = a.axis[decltype(first)::value + j]; }
    };
    switch (w) {
      case 0: pick(std::integral_constant<int, 0>()); break;
      case 1: pick(std::integral_constant<int, 8>()); break;
      case 2: pick(std::integral_constant<int, 16>()); break;
      case 3: pick(std::integral_constant<int, 24>()); break;
      case 4: pick(std::integral_constant<int, 32>()); break;
      case 5: pick(std::integral_constant<int, 40>()); break;
      case 6: pick(std::integral_constant<int, 48>()); break;
      default: pick(std::integral_constant<int, 56>()); break;
    }
    for (int tok = (tid & 31) >> 3; tok < n_tok; tok += 4) {
      const int t = tok0 + tok;
      int pos;
      if (a.positions != nullptr) {
        pos = a.positions[(long long)t * a.n_axes + axis];
      } else {
        const int b = (int)a.by_new.div((uint32_t)t);
        pos = (NEXT ? *reinterpret_cast<const volatile int32_t*>(v.seq_len + b) : a.pos0) + t - b * a.n_new;
      }
      const double x_turns = (double)pos * turns;
      float sn, cs;
      sincospif(2.f * (float)(x_turns - rint(x_turns)), &sn, &cs);
      table[tok][w * 9 + e] = make_float2(cs, sn);
    }
  }
  __syncthreads();

  for (int item = tid >> 3; item < n_items; item += RP_ROWS) {
    const Row nxt = fetch(item + RP_ROWS);
    if (cur.dst != nullptr) {
      uint4 lo = cur.lo, hi = cur.hi;
      if (cur.turns) {
        const float2* cs = table[cur.tok] + (a.adjacent ? (x >> 1) * 9 + (x & 1) * 4 : x * 9);      // of pairs 8 x .. 8 x + 7; adjacent: of 4 x .. + 3, those of the second piece 32 pairs on
        uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        if (a.adjacent) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 f = cs[e < 4 ? e : 4 * 9 + e - 4];
            const float p = bf16lo(w[e]), q = bf16hi(w[e]);
            w[e] = pack_bf16x2(p * f.x - q * f.y, q * f.x + p * f.y);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = cs[2 * e], g = cs[2 * e + 1];
            const float p0 = bf16lo(w[e]), p1 = bf16hi(w[e]), q0 = bf16lo(w[4 + e]), q1 = bf16hi(w[4 + e]);
            w[e] = pack_bf16x2(p0 * f.x - q0 * f.y, p1 * g.x - q1 * g.y);
            w[4 + e] = pack_bf16x2(q0 * f.x + p0 * f.y, q1 * g.x + p1 * g.y);
          }
        }
        lo = make_uint4(w[0], w[1], w[2], w[3]);
        hi = make_uint4(w[4], w[5], w[6], w[7]);
      }
      *reinterpret_cast<uint4*>(cur.dst + off_a) = lo;
      *reinterpret_cast<uint4*>(cur.dst + off_b) = hi;
    }
    cur = nxt;
  }

  if constexpr (!NEXT) {
    if (blockIdx.x == 0)
      for (int b = tid; b < v.B; b += RP_THREADS) v.seq_len[b] = a.pos0 + a.n_new;
  } else {
    // every CTA has read the old lengths: the last to arrive advances them
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1 ? 1 : 0;
    __syncthreads();
    if (!last) return;
    for (int b = tid; b < v.B; b += RP_THREADS) {
      const int n = v.seq_len[b];
      if (n < 0 || n > v.max_tokens - a.n_new) set_status(v.status, ERR_CAPACITY);
      else v.seq_len[b] = n + a.n_new;
    }
    if (tid == 0) *a.ticket = 0;      // clean for the next launch
  }
}

cudaError_t launch_append_rope(const LayerView& v, const RopeCall& call, bool next, cudaStream_t st) {
  const int rows = call.Hq + 2 * v.H;
  RopeArgs a;
  static_cast<RopeCall&>(a) = call;
  a.n_tokens = v.B * a.n_new;
  // one pass of the CTA, or one token; with tokens for two full waves, six passes (the rows of one pass are fetched while the ones before are turned and stored, and the
  // angles of a few tokens take as long as those of one).  8 x 4096 tokens of 96 rows: 254 us, with three passes 260, with twelve 262; 16 x 4096 of 9 rows 58, with three 60; of 6 and
  // 12 rows 45 and 70, with three passes as with six.  At the device's length 293, 54 (6 rows), 67, 81: a CTA waits for its stores before it takes its ticket
  int per = RP_ROWS / rows, most = a.n_tokens / (2 * RP_CTAS * sm_count());
  const int want = (6 * RP_ROWS + rows - 1) / rows;
  if (most > want) most = want;
  per = per < most ? most : per;
  per = per < 1 ? 1 : (per > RP_MAX_TOKENS ? RP_MAX_TOKENS : per);
  a.tokens_per_cta = per;
  a.by_rows = fast_div((uint32_t)rows); a.by_new = fast_div((uint32_t)a.n_new); a.by_c = fast_div((uint32_t)v.C);
  const unsigned grid = (unsigned)((a.n_tokens + per - 1) / per);
  return next ? launch_pdl(kve_append_rope_kernel<true>, dim3(grid), dim3(RP_THREADS), 0, st, v, a)
              : launch_pdl(kve_append_rope_kernel<false>, dim3(grid), dim3(RP_THREADS), 0, st, v, a);
}

}  // namespace kve
