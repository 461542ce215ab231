// Decode attention over a history held in 4 bits (kvE_decode_attn_q4):
//   out = softmax(q K'^T * scale) V',  rows of K', V' = [chunks held in 4 bits ; chunks and recent rows in bf16]
// for T x G query rows per KV head (T query tokens, G query heads a KV head).
//
// HBM is the floor: 144 bytes a packed row, 512 a bf16 row, each read once per group of query rows.  At 144 bytes a row the SM has ~100
// cycles for 16 rows, so what has to be small is the number of instructions per code:
//  * the codes lie in the pages in the order of the MMA operands (q4.cuh): eight of them are one 32-bit word of one lane, and become four
//    operand registers (fp16 numbers c 2^-24 and c 2^-20) in five logic instructions.  The powers of two go into q, into the softmax's scale and into
//    the result; scale and lowest number of a group are applied to the sums (keys: per row and group to the logit) or to the weights (values:
//    p s per group of 64 dims).  q enters as fp16 as well, times a power of two that puts its largest number at 2^14: exact but for numbers 2^25 below that.
//  * all products are m16n8k16 MMAs.  Three forms, by the query rows of a CTA (q4_attn_shape), because the tensor core takes 16 rows by 8 columns whether they are used or not:
//      1 to 4 rows: the cache on the M side (keys: 16 rows; values, transposed: 16 dims), the queries in the eight columns: the four rows twice, once for either group of 64
//        dims (q is zero in the other half; the weights have the group's scale), so that a lane has to do with one group only: half of the scales, weights and conversions.
//        16 sequences x 32 heads x 16512 rows, half of the chunks kept: 156 us (when both were built: 160, with the rows once in eight columns 170).
//      5 to 8 rows: the same, a row a column.  128 sequences x 8320 rows: 41 us (when both were built: 43, with the queries on the M side 65).
//        In both the logits' accumulator becomes the weights' operand through movmatrix, in registers.
//      9 to 16 rows: the queries on the M side, where the logits' accumulator is the weights' operand as it stands.  The lowest numbers' share of a logit, minus the
//        reference, is a product too, of three bf16 planes.  128 sequences x 8320 rows, 16 rows: 66 us (as two blocks of columns of the form above 72).
//  * the weights p s F of packed rows are fp16: 11 bits, off by half a step (2^-11 of the weight) at most, for half the MMAs of two planes.  What a weight multiplies is
//    c s, up to 15 steps above the lowest number, so for values around 0 its rounding counts a few times: normal values make 5e-4 (relative, rms) of it before the result is
//    rounded to bf16 (1.6e-3), 1.7e-3 with both.  F, a power of two per warp, query row and group, keeps them between what fp16 overflows at and where it runs out of
//    bits (qa_factor).  bf16 rows take their weights as two bf16 planes.
//  * a tile's products with the values are summed from zero and added to the accumulator by ordinary additions: the tensor core cuts off what lies below
//    the last bit of its accumulator at every step, always in one direction.
//  * the reference of the softmax is raised only when a logit passes it by more than 2^8 (a vote), not at every tile.
//  * a consumer warp is on its own: a ring of stages and a softmax state in registers for the whole sequence.  A tile is 32 packed rows or 8 bf16 rows: about as
//    many bytes, so that equal counts are equal work.  Two producer warps ask for all of them, a lane per consumer (done by the consumers themselves that was a
//    sixth of all instructions); a planner warp looks them up ahead, 32 side by side, into a table in shared memory.
//  * every sequence is cut into k equal parts, and a CTA of one resident wave takes a contiguous run of them: all CTAs have about the same number of
//    tiles, whatever the sequences.  At the end of a sequence a consumer leaves its state in shared memory and goes on; the merger warp folds the states.
// More than 16 query rows: groups of 16 in neighbouring CTAs, which go through the same rows at the same time (HBM reads them once).
// A CTA with a whole sequence writes the result, others a record; the last CTA of a sequence to finish merges the records.
// Every wait is bounded; on give-up the status word gets KVE_ERR_TIMEOUT.
#include <type_traits>

#include "q4.cuh"

namespace kve {

constexpr int QA_TILE_BYTES = 2 * Q4_PAIR_BYTES;             // two units of keys and values
constexpr int QA_V_OFF = 2 * Q4_UNIT_BYTES;                  // bf16 rows: values behind the keys
constexpr int QA_ROWS4 = 2 * Q4_UNIT_ROWS, QA_ROWS16 = 8;    // rows of a tile of either kind
static_assert(QA_ROWS16 * ROW_BYTES <= QA_V_OFF, "eight bf16 rows fit a stage");
constexpr float QA_SLACK = 8.f;                              // by how much (log2) a logit may pass the softmax reference
constexpr float QA_TOP = 128.f;                              // most that scale times factor may be: with weights of up to 2^QA_SLACK their product stays below fp16's 2^16
constexpr int QA_F_MOST = 56;                                // exponent of the largest factor, and of the first: sums of 2^23 bf16 rows of |v| = 2^60, at weights of 2^QA_SLACK, stay finite times F 2^-20
constexpr int QA_PLAN = 128;                                 // tiles looked up ahead of the copies
constexpr int QA_NEW = 1 << 16, QA_FLUSH = 2 << 16, QA_END = 4 << 16;          // first, last tile of a sequence for this warp; nothing comes after it

struct Q4AttnArgs {
  LayerView v;
  Q4Pages p;
  FastDiv by_g, by_h, by_k;                 // by G, by KV heads, by k
  FastDiv by_tiles4, by_tiles16;            // by the tiles of a chunk of either kind
  int dense, T, G, causal, k, groups;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  float scale;
  float* partials;      // the record of (sequence s, group, run c) at (s + c) groups + group: [query rows of a CTA][132]
  int32_t* counters;    // [S][groups], zero between launches
};

// COLS_: query rows of a CTA, 4, 8 or 16
template <int COLS_> struct QaShape {
  static constexpr int COLS = COLS_;
  static constexpr bool MANY = COLS == 16;
  static constexpr int QROWS = MANY ? 16 : 8;                // rows of fp16 queries (four of them twice)
  static constexpr int CW = MANY ? 8 : 12;                   // consumer warps
  static constexpr int PRODUCERS = 2, PLANNER = CW + PRODUCERS, MERGER = PLANNER + 1, WARPS = MERGER + 1;
  static constexpr int STAGES = 3;                           // per consumer
  static constexpr int OFF_STATE = CW * STAGES * QA_TILE_BYTES;                          // [consumers][query rows][132]: behind the ring
  static constexpr int OFF_Q = OFF_STATE + CW * COLS * ATTN_PARTIAL_FLOATS * 4;          // [2][query rows][128] bf16; the same as fp16; what undoes their powers of two: [2][query rows]
  static constexpr int OFF_QH = OFF_Q + 2 * COLS * ROW_BYTES;
  static constexpr int OFF_UNDO = OFF_QH + 2 * QROWS * ROW_BYTES;
  static constexpr int OFF_SUMS = OFF_UNDO + 2 * COLS * 4;   // MANY: sums of the query rows over the groups, times scale: [2][query rows][2]
  static constexpr int OFF_INFO = OFF_SUMS + (MANY ? 2 * COLS * 8 : 0);      // [consumers][stages] int4: the tile's entry of the table
  static constexpr int OFF_PLAN = OFF_INFO + CW * STAGES * 16;      // [QA_PLAN] int4: tiles looked up
  static constexpr int OFF_BAR = OFF_PLAN + QA_PLAN * 16;
  static constexpr int SMEM = OFF_BAR + (2 * CW * STAGES + 3) * 8 + 16 + (CW + 2) * 4;
  static_assert(OFF_INFO % 16 == 0 && OFF_BAR % 8 == 0 && SMEM <= 227 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ int load_now(const int32_t* p) { return *reinterpret_cast<const volatile int32_t*>(p); }
__device__ __forceinline__ float2 f16_pair(uint32_t w) {
  float2 d;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(d.x), "=f"(d.y) : "r"(w));
  return d;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// MMAs that start from zero, or go on with a sum (not volatile, unlike the one in common.cuh: the compiler may move them past one another)
#define QA_MMA(NAME, TYPES)                                                                                                                        \
  __device__ __forceinline__ void NAME##_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {                                \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPES ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"                             \
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));               \
  }                                                                                                                                              \
  __device__ __forceinline__ void NAME##_next(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {                                 \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPES ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"                                 \
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));                         \
  }
QA_MMA(mma_f16, "f16.f16")
QA_MMA(mma_bf16, "bf16.bf16")
#undef QA_MMA
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}

// which halves of a bf16 pair are an infinity or a NaN, as a mask of bits
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u); }
// word i of four (i known at compile time)
__device__ __forceinline__ uint32_t word_of(const uint4& w, int i) { return i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w)); }
// folds a state (accumulator, reference, sum) into one with reference `top`
__device__ __forceinline__ void fold(const float* st, float top, float& sum, float4& o, int lane) {
  const float m = st[128], f = m == -INFINITY ? 0.f : exp2f(m - top);
  const float4 x = *reinterpret_cast<const float4*>(st + lane * 4);
  sum = fmaf(st[129], f, sum);
  o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
}
// The power of two that a query row's fp16 weights of a group are taken times, from now on.  now: its exponent so far; raw: the largest scale in the tile; most: the largest
// weight times scale so far; f: what a raised reference leaves of earlier weights.  Scales like the tile's are to fit with a weight of 2^QA_SLACK (to 2^7), so that rows like
// these do not ask again.  But a scale whose row has next to no weight must not take the bits of the others: `most` keeps 2^-3, whose fp16 numbers are normal down to 2^-11
// of it.  (The tile's own weights fit either way; a tile with a scale beyond 2^7 over the factor asks again.)  Without a raised reference the factor only sinks.
__device__ __forceinline__ int qa_exponent(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }      // 2^e <= x; 0: -127; not finite: 128
__device__ __forceinline__ float qa_power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ int qa_factor(int now, float raw, float most, float f) {
  const int er = qa_exponent(raw), fit = max(6 - er, -3 - qa_exponent(most));
  const int up = min(now - qa_exponent(f), now + 100);
  return max(min(min(up, QA_F_MOST), min(fit, 125 - er)), -118);      // (scale times factor stays finite)
}
// a warp writes query row rr of sequence s
__device__ __forceinline__ void write_row(const Q4AttnArgs& a, int s, int rr, float4 o, float top, float sum, int lane) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (no row, or weights of 0 only: 0; NaN stays)
  const int t = (int)a.by_g.div((uint32_t)rr), g = rr - t * a.G, b = (int)a.by_h.div((uint32_t)s), h = s - b * a.v.H;
  const long long at = (((long long)b * a.T + t) * a.v.H + h) * a.G + g;
  *reinterpret_cast<uint2*>(a.out + at * D + lane * 4) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994530942f;
}

// CTA c of P takes parts [c I / P, (c + 1) I / P) (32-bit arithmetic: the host keeps I P below 2^32)
__device__ __forceinline__ uint32_t qa_begin(uint32_t c, uint32_t I, uint32_t P) { return (c * I) / P; }
__device__ __forceinline__ uint32_t qa_owner(uint32_t x, uint32_t I, uint32_t P) { return ((x + 1u) * P - 1u) / I; }

template <int COLS>
__global__ void __launch_bounds__(QaShape<COLS>::WARPS * 32, 1) kve_decode_attn_q4_kernel(Q4AttnArgs a) {
  using Shape = QaShape<COLS>;
  constexpr int STAGES = Shape::STAGES, CW = Shape::CW, WARPS = Shape::WARPS;
  constexpr bool MANY = Shape::MANY, DUO = COLS == 4;
  extern __shared__ __align__(128) unsigned char smem[];
  const LayerView& v = a.v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + Shape::OFF_BAR);      // [consumers][stages]
  uint64_t* empty = full + CW * STAGES;
  uint64_t* left = empty + CW * STAGES;      // all consumers have left their state of a sequence
  uint64_t* merged = left + 1;               // which has been folded, and the query rows of the sequence after the next brought
  uint64_t* fetched = merged + 1;            // the query rows of the first two sequences are there
  int* flags = reinterpret_cast<int*>(fetched + 1);      // at the end: records of the first and of the last sequence, where this CTA merges them
  volatile int* progress = flags + 4;                    // [consumers] the entry of the table that each will need next; behind them: entries there are; tokens stored
  int4* plan = reinterpret_cast<int4*>(smem + Shape::OFF_PLAN);
  int4* infos = reinterpret_cast<int4*>(smem + Shape::OFF_INFO);
  float* states = reinterpret_cast<float*>(smem + Shape::OFF_STATE);
  const int R = a.T * a.G;
  const float sl2 = a.scale * 1.44269504088896340736f;      // logits in log2 units

  pdl_launch_dependents();
  for (int i = threadIdx.x; i < 2 * CW * STAGES; i += WARPS * 32) mbar_init(&full[i], 1);
  if (threadIdx.x == 0) {
    mbar_init(left, CW);
    mbar_init(merged, 1);
    mbar_init(fetched, 1);
    progress[CW] = 0;
  }
  if (threadIdx.x < CW) progress[threadIdx.x] = threadIdx.x;
  mbar_fence_init();
  // the run of this CTA: parts i0 .. i1 - 1 of the sequences x0 .. x1, for one group of query rows
  const uint32_t uk = (uint32_t)a.k, n_items = (uint32_t)v.S * uk, P = gridDim.x / (uint32_t)a.groups;
  const int run = (int)(blockIdx.x / (uint32_t)a.groups), group = (int)blockIdx.x - run * a.groups;
  const int row0 = group * COLS, n_rows = min(R - row0, COLS);      // its query rows
  const uint32_t i0 = qa_begin((uint32_t)run, n_items, P), i1 = qa_begin((uint32_t)run + 1u, n_items, P);
  const int x0 = (int)a.by_k.div(i0), x1 = (int)a.by_k.div(i1 - 1u);      // (i0 < i1: there are no more runs than parts)
  __syncthreads();
  pdl_wait();

  // ---- a warp brings the query rows of sequence s into slot `slot`: bf16, and fp16 times a power of two ----
  auto fetch_queries = [&](int s, int slot) {
    uint32_t* Qh = reinterpret_cast<uint32_t*>(smem + Shape::OFF_QH) + slot * Shape::QROWS * 64;
    uint32_t* Qb = reinterpret_cast<uint32_t*>(smem + Shape::OFF_Q) + slot * COLS * 64;
    float* q_undo = reinterpret_cast<float*>(smem + Shape::OFF_UNDO) + slot * COLS;
    const int b = (int)a.by_h.div((uint32_t)s), h = s - b * v.H, piece = lane & 15;
#pragma unroll 4
    for (int c = lane >> 4; c < COLS; c += 2) {      // column c of the MMAs is query row row0 + c; rows that do not exist are zeros.  Half a warp a row
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (c < n_rows) {
        const int t = (int)a.by_g.div((uint32_t)(row0 + c)), gq = row0 + c - t * a.G;
        w = __ldcg(reinterpret_cast<const uint4*>(a.q + ((((long long)b * a.T + t) * v.H + h) * a.G + gq) * D + piece * 8));
      }
      const uint32_t word[4] = {w.x, w.y, w.z, w.w};
      // where pair e of the piece lies: row by row, or (MANY) as the operand registers of the eight products along a row, four of each lane
      auto place = [&](int e) { return MANY ? (((piece >> 2) * 2 + (e >> 1)) * 32 + (c & 7) * 4 + (piece & 3)) * 4 + (c >> 3) + 2 * (e & 1) : c * 64 + piece * 4 + e; };
#pragma unroll
      for (int e = 0; e < 4; ++e) Qb[place(e)] = word[e];
      float most = 0.f;      // of the finite ones
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = fabsf(bf16lo(word[e])), q = fabsf(bf16hi(word[e]));
        most = fmaxf(most, fmaxf(p < INFINITY ? p : 0.f, q < INFINITY ? q : 0.f));
      }
#pragma unroll
      for (int o = 1; o <= 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      const int power = most > 0.f ? min(max(14 - ((int)(__float_as_uint(most) >> 23) - 127), -100), 120) : 0;
      const float up = __uint_as_float((uint32_t)(127 + power) << 23);
#pragma unroll
      for (int e = 0; e < 4; ++e) {      // odd pairs meet codes that are 2^4 times as large
        const float f = e & 1 ? up * 0.0625f : up;
        const uint32_t w16 = pack_f16x2(bf16lo(word[e]) * f, bf16hi(word[e]) * f);
        if constexpr (DUO) {
          Qh[c * 64 + piece * 4 + e] = piece < 8 ? w16 : 0u;
          Qh[(c + 4) * 64 + piece * 4 + e] = piece < 8 ? 0u : w16;
        } else {
          Qh[place(e)] = w16;
        }
      }
      if (piece == 0) q_undo[c] = __uint_as_float((uint32_t)(127 - power) << 23);
    }
  };
  // one CTA has all parts of sequence x
  auto whole = [&](int x) { return qa_owner((uint32_t)x * uk, n_items, P) == qa_owner((uint32_t)(x + 1) * uk - 1u, n_items, P); };
  // folds the consumers' states of query row r of sequence x: the result, or a record
  auto fold_states = [&](int x, int r) {
    const float* st = states + r * ATTN_PARTIAL_FLOATS;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < CW; ++w) top = fmaxf(top, st[w * COLS * ATTN_PARTIAL_FLOATS + 128]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < CW; ++w) fold(st + w * COLS * ATTN_PARTIAL_FLOATS, top, sum, o, lane);
    if (whole(x)) {
      write_row(a, x, row0 + r, o, top, sum, lane);
    } else {
      float* rec = a.partials + (((long long)(x + run) * a.groups + group) * COLS + r) * ATTN_PARTIAL_FLOATS;
      *reinterpret_cast<float4*>(rec + lane * 4) = o;
      if (lane == 0) { rec[128] = top; rec[129] = sum; }
    }
  };

  if (warp == Shape::PLANNER) {
    // ================= planner: looks up tiles, 32 side by side =================
    const int len = load_now(v.seq_len), dev_packed = load_now(v.n_packed), dev_listed = a.dense ? 0 : load_now(v.n_listed);
    int dev_kept = a.dense ? 0 : load_now(v.keep_cnt + x0);      // (all four on their way together)
    const int n = min(max(len, 0), v.max_tokens), complete = n / v.C;
    const int packed = min(max(dev_packed, 0), complete), listed = min(max(dev_listed, 0), complete);
    if (lane == 0) progress[CW + 1] = n;
    const int per4 = (v.C + QA_ROWS4 - 1) / QA_ROWS4, per16 = v.C / QA_ROWS16;
    const int c_tail = max(listed, packed), tail = n - c_tail * v.C;      // the rest in bf16: first chunk, rows
    if (a.causal && tail < a.T && lane == 0) set_status(v.status, ERR_CAPACITY);      // (a replay that outgrew its capture: the block's first tokens have no rows of their own any more)
    // The table's entries are numbered through; entry i is consumer i % CW's.  A sequence has at least CW of them, so that every consumer learns of it.
    int x = x0, j = 0, j_end = 0, pos_in = 0, n_entries = 0;      // sequence being looked up; its next tile and last; entries it has so far, and will have
    int e0 = 0, e1 = 0, e2 = 0, kept4 = 0;                        // in tiles: kept chunks in 4 bits up to e0; chunks behind the keep list in 4 bits up to e1; kept chunks in bf16 up to e2; the rest in bf16
    int planned = 0;
    auto enter = [&]() {
      const long long sb = (long long)x * v.max_chunks;
      const int kept = min(max(dev_kept, 0), listed);
      if (!a.dense && x < x1) dev_kept = load_now(v.keep_cnt + x + 1);      // the next one's
      kept4 = kept;      // kept chunks that are packed: the list ascends
      if (packed < listed) {
        int lo = 0, hi = kept;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (__ldcg(v.keep_idx + sb + mid) < packed) lo = mid + 1; else hi = mid;
        }
        kept4 = lo;
      }
      e0 = kept4 * per4;
      e1 = e0 + max(packed - listed, 0) * per4;
      e2 = e1 + (kept - kept4) * per16;
      const int total = e2 + (tail + QA_ROWS16 - 1) / QA_ROWS16;
      const uint32_t p_lo = x == x0 ? i0 - (uint32_t)x * uk : 0u, p_hi = x == x1 ? i1 - (uint32_t)x * uk : uk;
      j = (int)((long long)p_lo * total / a.k);
      j_end = (int)((long long)p_hi * total / a.k);
      pos_in = 0;
      n_entries = max(j_end - j, CW);
    };
    // the next entries, up to 32 of one sequence, a lane each
    auto look_up = [&]() {
      const int jj = j + lane, at = pos_in + lane, count = min(32, n_entries - pos_in);
      int4 e = make_int4(0, 0, 0, 0);      // page; first row in it, flags above; rows (negative: bf16 ones; 0: none); position of the first row
      if (jj < j_end) {
        const long long sb = (long long)x * v.max_chunks;
        const int of = jj < e0 ? jj : (jj < e1 ? jj - e0 : (jj < e2 ? jj - e1 : jj - e2));      // in its list
        const bool in4 = jj < e1;
        const int nth = (int)(in4 ? a.by_tiles4 : a.by_tiles16).div((uint32_t)of), within = of - nth * (in4 ? per4 : per16);
        int chunk;
        if (jj < e0) chunk = __ldcg(v.keep_idx + sb + nth);
        else if (jj < e1) chunk = listed + nth;
        else if (jj < e2) chunk = __ldcg(v.keep_idx + sb + kept4 + nth);
        else chunk = c_tail + nth;
        int page = chunk >= 0 && chunk < v.max_chunks ? __ldcg((in4 ? a.p.table : v.page_table) + sb + chunk) : -1;
        if (page < 0 || page >= (in4 ? a.p.n_pages : (long long)v.n_pages)) { set_status(v.status, ERR_CAPACITY); page = 0; }
        e.x = page;
        e.y = within * (in4 ? QA_ROWS4 : QA_ROWS16);
        e.z = in4 ? min(QA_ROWS4, v.C - e.y) : -(jj < e2 ? QA_ROWS16 : min(QA_ROWS16, tail - of * QA_ROWS16));
        e.w = chunk * v.C + e.y;
      }
      const bool last = at + CW >= n_entries;
      e.y |= (at < CW ? QA_NEW : 0) | (last ? QA_FLUSH : 0) | (last && x == x1 ? QA_END : 0);
      if (lane < count) plan[(planned + lane) % QA_PLAN] = e;
      planned += count;
      pos_in += count;
      j += count;
      if (pos_in == n_entries && ++x <= x1) enter();
      __syncwarp();
    };
    enter();
    for (int idle = 0; x <= x1;) {
      // room for 32 more: entries that all have come past
      if (planned + 32 - (int)__reduce_min_sync(0xffffffffu, lane < CW ? (unsigned)progress[lane] : 0xffffffffu) <= QA_PLAN) {
        look_up();
        __threadfence_block();
        __syncwarp();
        if (lane == 0) progress[CW] = planned;
        idle = 0;
      } else {
        __nanosleep(200);
        if (++idle > (1 << 20)) {
          if (lane == 0) set_status(v.status, ERR_TIMEOUT);
          break;
        }
      }
    }
  } else if (warp >= CW && warp < Shape::PLANNER) {
    // ================= producers: a lane fills the ring of a consumer =================
    const int w = (warp - CW) * (CW / Shape::PRODUCERS) + lane;      // that consumer
    uint64_t *my_full = full + w * STAGES, *my_empty = empty + w * STAGES;
    int pushed = 0, entry = w, idle = 0;      // tiles asked for; the next one's entry
    const bool mine = lane < CW / Shape::PRODUCERS;
    bool active = mine;
    while (__any_sync(0xffffffffu, active)) {
      const int stage = pushed % STAGES, round = pushed / STAGES;
      const bool ready = active && entry < progress[CW] && (round == 0 || mbar_test_wait(&my_empty[stage], (uint32_t)(round - 1) & 1u));
      if (ready) {
        __threadfence_block();
        const int4 e = plan[entry % QA_PLAN];
        infos[w * STAGES + stage] = e;
        if (e.z != 0) {
          unsigned char* dst = smem + (w * STAGES + stage) * QA_TILE_BYTES;
          const bool in4 = e.z > 0;
          const long long row = (long long)e.x * v.C + (e.y & 0xffff);
          if (in4) {
            const uint32_t bytes = (uint32_t)e.z * (Q4_PAIR_BYTES / Q4_UNIT_ROWS);
            mbar_arrive_expect_tx(&my_full[stage], bytes);      // release: whoever sees the phase sees the description
            bulk_g2s(dst, a.p.kv + row * (Q4_PAIR_BYTES / Q4_UNIT_ROWS), bytes, &my_full[stage]);
          } else {
            const uint32_t bytes = (uint32_t)-e.z * ROW_BYTES;
            mbar_arrive_expect_tx(&my_full[stage], 2 * bytes);
            bulk_g2s(dst, v.k_pages + row * D, bytes, &my_full[stage]);
            bulk_g2s(dst + QA_V_OFF, v.v_pages + row * D, bytes, &my_full[stage]);
          }
        } else {
          mbar_arrive(&my_full[stage]);
        }
        ++pushed;
        entry += CW;
        __threadfence_block();
        progress[w] = active && (e.y & QA_END) ? 0x7fffffff : entry;      // (the planner may write over what this lane has read)
        active = (e.y & QA_END) == 0;
      }
      if (__any_sync(0xffffffffu, ready)) {
        idle = 0;
      } else {
        if (pushed > 0) __nanosleep(100);
        if (++idle > (1 << 20)) {
          if (lane == 0) set_status(v.status, ERR_TIMEOUT);
          break;
        }
      }
    }
    // nobody leaves with copies under way: their consumers see all of them land, unless one has given up
    if (mine) ring_drain<STAGES>(my_full, pushed);
  } else if (warp == Shape::MERGER) {
    // ================= merger: brings query rows, folds the states of all sequences but the last =================
    fetch_queries(x0, 0);
    if (x1 > x0) fetch_queries(x0 + 1, 1);
    __syncwarp();
    if (lane == 0) mbar_arrive(fetched);
    for (int x = x0; x < x1; ++x) {
      if (!mbar_wait_bounded(left, (uint32_t)(x - x0) & 1u)) {
        if (lane == 0) set_status(v.status, ERR_TIMEOUT);
        break;
      }
      for (int r = 0; r < n_rows; ++r) fold_states(x, r);
      __syncwarp();
      if (x + 2 <= x1) fetch_queries(x + 2, (x - x0) & 1);
      __threadfence_block();
      __syncwarp();
      if (lane == 0) mbar_arrive(merged);
    }
  } else {
    // ================= consumers =================
    // goes through this warp's tiles: start(slot) at the first of a sequence, packed rows, bf16 rows, leave() at the last
    auto consume = [&](auto&& start, auto&& packed_rows, auto&& bf16_rows, auto&& leave) {
      uint64_t *my_full = full + warp * STAGES, *my_empty = empty + warp * STAGES;
      int nth = 0, stage = 0;      // sequences begun; stage of the next tile
      uint32_t phase = 0;
      bool ok = mbar_wait_bounded(fetched, 0);
      if (!ok && lane == 0) set_status(v.status, ERR_TIMEOUT);
      while (ok) {
        if (!mbar_wait_bounded(&my_full[stage], phase)) {
          if (lane == 0) set_status(v.status, ERR_TIMEOUT);
          break;
        }
        const unsigned char* base = smem + (warp * STAGES + stage) * QA_TILE_BYTES;
        const int4 what = infos[warp * STAGES + stage];
        if (what.y & QA_NEW) {      // its query rows were brought when the sequence two before it was merged, which this warp has waited for
          start(nth & 1);
          ++nth;
        }
        if (what.z > 0) packed_rows(what.z, base);
        else if (what.z < 0) bf16_rows(-what.z, what.w, base);
        __syncwarp();
        if (lane == 0) mbar_arrive(&my_empty[stage]);
        if (what.y & QA_FLUSH) {
          // the states of the sequence before are done with
          if (nth >= 2 && !mbar_wait_bounded(merged, (uint32_t)(nth - 2) & 1u)) {
            if (lane == 0) set_status(v.status, ERR_TIMEOUT);
            break;
          }
          leave();
          if (what.y & QA_END) break;
          if (lane == 0) mbar_arrive(left);      // release
        }
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
    };
    // A causal block's newest rows, which not all query rows see: a product with a weight of 0 would still make NaN of a value that is not finite.  Whether the tile of
    // `rows` bf16 rows from position pos has any of those ...
    auto hides = [&](int rows, int pos, const unsigned char* base) {
      if (!a.causal || pos + rows - 1 <= progress[CW + 1] - a.T) return false;
      uint32_t any = 0u;
      if (g8 < rows)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(base + QA_V_OFF + g8 * ROW_BYTES + i * 64 + t4 * 16);
          any |= not_finite(w.x) | not_finite(w.y) | not_finite(w.z) | not_finite(w.w);
        }
      return (bool)__any_sync(0xffffffffu, any != 0u);
    };
    // ... and when every lane has added those that its query rows see, zeros in their place
    auto clear = [&](int rows, const unsigned char* base) {
      __syncwarp();
      if (g8 < rows)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4* p = reinterpret_cast<uint4*>(const_cast<unsigned char*>(base) + QA_V_OFF + g8 * ROW_BYTES + i * 64 + t4 * 16);
          const uint4 w = *p;
          *p = make_uint4(w.x & ~not_finite(w.x), w.y & ~not_finite(w.y), w.z & ~not_finite(w.z), w.w & ~not_finite(w.w));
        }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (the stage is filled by a bulk copy again)
      __syncwarp();
    };
    if constexpr (!MANY) {
      // ---- up to eight query rows: the cache on the M side, the queries in the columns.  Up to four (DUO): rows 0 to 3 twice, where the products with packed keys and
      // values have group 0 in the columns below 4 and group 1 in those from 4 on ----
      constexpr int NT = 1, NG = DUO ? 1 : 2;      // groups that a lane has to do with
      const uint16_t *Qh = nullptr, *Qb = nullptr;      // its query rows, as fp16 and as bf16
      // column nt 8 + g8: the numbers 32 j + 8 t4 .. + 7, as fp16 (from shared memory every time)
      auto q_half = [&](int nt, int j) { return *reinterpret_cast<const uint4*>(Qh + (nt * 8 + g8) * D + 32 * j + 8 * t4); };
      float undo[NT][2], qsum[NT][NG][2];     // per column 2 t4, 2 t4 + 1: what takes q's power of two off a sum of codes (2^-24) and makes it a log2 logit; sums of q over the groups
      auto row_of = [&](int nt, int c) { return nt * 8 + (DUO ? c & 3 : c); };      // the query row of a column
      auto last_pos = [&](int nt, int x) {    // causal: the last position a column sees
        return a.causal ? progress[CW + 1] - a.T + (int)a.by_g.div((uint32_t)min(row0 + row_of(nt, 2 * t4 + x), R - 1)) : 0x7fffffff;
      };

      float acc[NT][8][4];           // [m]: dims d = 64 (m / 4) + 8 g8 + 2 (m % 4) and d + 1, columns 2 t4 and 2 t4 + 1: (d, c), (d, c + 1), times F 2^-24; (d + 1, c), (d + 1, c + 1), times F 2^-20
      float l[NT][2], zs[NT][NG][2]; // this lane's rows' share, per column: sum of weights; of weights times what code 0 stands for
      // per column: the softmax's reference (0 until there is one), and what a logit may exceed it by (-inf until there is one)
      float ref[NT][2], over_by[NT][2];
      float F[NG][2];  // weight factors of the columns; a scale with s F > 2^7 asks for another
      // the largest weight times scale that column c has had in a tile that was looked at (in what the records do not use of the state, for the rare case alone)
      auto most_of = [&](int nt, int g, int c) { return states + (warp * COLS + row_of(nt, 2 * t4 + c)) * ATTN_PARTIAL_FLOATS + 130 + (DUO ? t4 >> 1 : g); };
      // a fresh state, and the query rows in slot `slot`
      auto start = [&](int slot) {
        Qh = reinterpret_cast<const uint16_t*>(smem + Shape::OFF_QH) + slot * Shape::QROWS * D;
        Qb = reinterpret_cast<const uint16_t*>(smem + Shape::OFF_Q) + slot * COLS * D;
        const float* q_undo = reinterpret_cast<const float*>(smem + Shape::OFF_UNDO) + slot * COLS;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float sum[NG] = {};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint4 w = q_half(nt, j);
            const float2 e0 = f16_pair(w.x), e1 = f16_pair(w.y), e2 = f16_pair(w.z), e3 = f16_pair(w.w);
            sum[DUO ? 0 : j >> 1] += (e0.x + e0.y) + (e2.x + e2.y) + 16.f * ((e1.x + e1.y) + (e3.x + e3.y));
          }
          const float off = q_undo[row_of(nt, g8)] * sl2;
#pragma unroll
          for (int h = 0; h < NG; ++h) {
            float y = sum[h];
            y += __shfl_xor_sync(0xffffffffu, y, 1);
            y += __shfl_xor_sync(0xffffffffu, y, 2);      // of column g8, in its four lanes
            y *= off;
            qsum[nt][h][0] = __shfl_sync(0xffffffffu, y, 8 * t4);
            qsum[nt][h][1] = __shfl_sync(0xffffffffu, y, 8 * t4 + 4);
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            undo[nt][c] = q_undo[row_of(nt, 2 * t4 + c)] * 0x1p12f * sl2 * 0x1p12f;
            ref[nt][c] = 0.f; over_by[nt][c] = -INFINITY; l[nt][c] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) { zs[nt][g][c] = 0.f; F[g][c] = qa_power(QA_F_MOST); }
          }
#pragma unroll
          for (int m = 0; m < 8; ++m)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[nt][m][y] = 0.f;
        }
      };

      // Logits minus reference (log2 units; of each of this lane's rows: c, c + 1) to weights in place.  s: the largest scale of
      // these rows in either group; scale(row, group): theirs one by one.  Raises the reference and changes the factors where it has to.
      auto weigh = [&](auto& x, float s0, float s1, auto&& scale) {
        constexpr int N = (int)(sizeof(x[0]) / sizeof(float));
        bool over = false;
#pragma unroll
        for (int g = 0; g < NG; ++g) over |= (g ? s1 : s0) * fmaxf(F[g][0], F[g][1]) > QA_TOP;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < N; ++i) over |= x[nt][i] > over_by[nt][i & 1];
        if (__any_sync(0xffffffffu, over)) {
          float raw[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            raw[g] = g ? s1 : s0;
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) raw[g] = fmaxf(raw[g], __shfl_xor_sync(0xffffffffu, raw[g], o));
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float top = x[nt][c];
#pragma unroll
              for (int i = c + 2; i < N; i += 2) top = fmaxf(top, x[nt][i]);
#pragma unroll
              for (int o = 4; o <= 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
              const bool first = over_by[nt][c] == -INFINITY;
              const float to = ref[nt][c] + (first ? (top == -INFINITY ? 0.f : top) : fmaxf(top, 0.f)), up = to - ref[nt][c];
              const float f = first ? 1.f : ex2_fast(-up);
              if (top != -INFINITY) over_by[nt][c] = QA_SLACK;
              ref[nt][c] = to;
#pragma unroll
              for (int i = c; i < N; i += 2) x[nt][i] -= up;
              l[nt][c] *= f;
#pragma unroll
              for (int m = 0; m < 8; ++m) { acc[nt][m][c] *= f; acc[nt][m][2 + c] *= f; }
#pragma unroll
              for (int g = 0; g < NG; ++g) {
                zs[nt][g][c] *= f;
                float ps = 0.f;      // the tile's largest weight times scale
#pragma unroll
                for (int i = c; i < N; i += 2) ps = fmaxf(ps, ex2_fast(x[nt][i]) * scale(i >> 1, g));
#pragma unroll
                for (int o = 4; o <= 16; o <<= 1) ps = fmaxf(ps, __shfl_xor_sync(0xffffffffu, ps, o));
                float* at = most_of(nt, g, c);
                const float most = first ? ps : fmaxf(*at * f, ps);
                const int was = qa_exponent(F[g][c]), now = qa_factor(was, raw[g], most, f);
                const float by = qa_power(max(now - was, -127));
                __syncwarp();
                *at = most;      // (the lanes of a column write the same)
                F[g][c] = qa_power(now);
#pragma unroll
                for (int m = 0; m < (DUO ? 8 : 4); ++m) { acc[nt][4 * g + m][c] *= by; acc[nt][4 * g + m][2 + c] *= by; }      // (DUO: what the lane holds of the other group's dims is nobody's)
              }
            }
          __syncwarp();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            x[nt][i] = ex2_fast(x[nt][i]);
            l[nt][i & 1] += x[nt][i];
          }
      };

      auto add_to = [](float (&sum)[4], const float (&d)[4], float2 f01, float2 f23) {
        const float2 p = fma2(make_float2(d[0], d[1]), f01, make_float2(sum[0], sum[1])), q = fma2(make_float2(d[2], d[3]), f23, make_float2(sum[2], sum[3]));
        sum[0] = p.x; sum[1] = p.y; sum[2] = q.x; sum[3] = q.y;
      };
      // a tile of packed rows, UNITS times 16
      auto packed_rows = [&](auto units, const unsigned char* base) {
        constexpr int UNITS = decltype(units)::value;
        float x[NT][4 * UNITS];
        uint32_t va[UNITS][NG], vc[UNITS][NG];      // scale and lowest number of the rows g8 and g8 + 8, values
        {
          float d[UNITS][NT][2][4];      // two chains: the groups; DUO: even and odd words
          uint4 ka[UNITS], kc[UNITS];
#pragma unroll
          for (int u = 0; u < UNITS; ++u) {
            ka[u] = *reinterpret_cast<const uint4*>(base + u * Q4_PAIR_BYTES + lane * 16);
            kc[u] = *reinterpret_cast<const uint4*>(base + u * Q4_PAIR_BYTES + 512 + lane * 16);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t pa[UNITS][4], pc[UNITS][4];
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
              q4_spread(word_of(ka[u], j), pa[u]);
              q4_spread(word_of(kc[u], j), pc[u]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint4 qw = q_half(nt, j);
#pragma unroll
              for (int u = 0; u < UNITS; ++u) {
                const uint32_t A0[4] = {pa[u][0], pc[u][0], pa[u][1], pc[u][1]}, A1[4] = {pa[u][2], pc[u][2], pa[u][3], pc[u][3]};
                float(&to)[4] = d[u][nt][DUO ? j & 1 : j >> 1];
                if (DUO ? j < 2 : (j & 1) == 0) mma_f16_first(to, A0, qw.x, qw.y);
                else mma_f16_next(to, A0, qw.x, qw.y);
                mma_f16_next(to, A1, qw.z, qw.w);
              }
            }
          }
          // x = low + s c: the sum over a group is s (what the MMAs give) + low (sum of q)
#pragma unroll
          for (int u = 0; u < UNITS; ++u) {
            const unsigned char* kh = base + u * Q4_PAIR_BYTES + Q4_CODE_BYTES + g8 * 8;
            const unsigned char* vh = kh + Q4_UNIT_BYTES;
            if constexpr (DUO) {
              // a lane has the sum of its own group; the other group's is in the lane t4 ^ 2
              const int of = (t4 >> 1) * 4;
              const uint32_t ha = *reinterpret_cast<const uint32_t*>(kh + of), hc = *reinterpret_cast<const uint32_t*>(kh + 64 + of);
              const float sa = bf16lo(ha), sc = bf16lo(hc), la = bf16hi(ha), lc = bf16hi(hc);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const float(&y)[2][4] = d[u][0];
                const float half_ref = -0.5f * ref[0][c];
                const float p = fmaf((y[0][c] + y[1][c]) * sa, undo[0][c], fmaf(la, qsum[0][0][c], half_ref));
                const float q = fmaf((y[0][2 + c] + y[1][2 + c]) * sc, undo[0][c], fmaf(lc, qsum[0][0][c], half_ref));
                x[0][4 * u + c] = p + __shfl_xor_sync(0xffffffffu, p, 2);
                x[0][4 * u + 2 + c] = q + __shfl_xor_sync(0xffffffffu, q, 2);
              }
              va[u][0] = *reinterpret_cast<const uint32_t*>(vh + of);
              vc[u][0] = *reinterpret_cast<const uint32_t*>(vh + 64 + of);
            } else {
              const uint2 ha = *reinterpret_cast<const uint2*>(kh), hc = *reinterpret_cast<const uint2*>(kh + 64), wa = *reinterpret_cast<const uint2*>(vh), wc = *reinterpret_cast<const uint2*>(vh + 64);
              const float sa0 = bf16lo(ha.x), sa1 = bf16lo(ha.y), sc0 = bf16lo(hc.x), sc1 = bf16lo(hc.y);
              const float la0 = bf16hi(ha.x), la1 = bf16hi(ha.y), lc0 = bf16hi(hc.x), lc1 = bf16hi(hc.y);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const float(&y)[2][4] = d[u][nt];
                  x[nt][4 * u + c] = fmaf(fmaf(y[0][c], sa0, y[1][c] * sa1), undo[nt][c], fmaf(la0, qsum[nt][0][c], fmaf(la1, qsum[nt][NG - 1][c], -ref[nt][c])));
                  x[nt][4 * u + 2 + c] = fmaf(fmaf(y[0][2 + c], sc0, y[1][2 + c] * sc1), undo[nt][c], fmaf(lc0, qsum[nt][0][c], fmaf(lc1, qsum[nt][NG - 1][c], -ref[nt][c])));
                }
              va[u][0] = wa.x; va[u][NG - 1] = wa.y;
              vc[u][0] = wc.x; vc[u][NG - 1] = wc.y;
            }
          }
        }
        float most[NG] = {};
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
          for (int g = 0; g < NG; ++g) most[g] = fmaxf(most[g], fmaxf(bf16lo(va[u][g]), bf16lo(vc[u][g])));
        weigh(x, most[0], most[NG - 1], [&](int row, int g) { return bf16lo(row & 1 ? vc[row >> 1][g] : va[row >> 1][g]); });
        uint32_t b[NG][UNITS][NT][2];      // weights times scale: MMA operands
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int u = 0; u < UNITS; ++u) {
            const float s_a = bf16lo(va[u][g]), s_c = bf16lo(vc[u][g]);
            const float2 F2 = make_float2(F[g][0], F[g][1]), f_a = mul2(make_float2(s_a, s_a), F2), f_c = mul2(make_float2(s_c, s_c), F2);
            const float l_a = bf16hi(va[u][g]), l_c = bf16hi(vc[u][g]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float* p = &x[nt][4 * u];
              const float2 w_a = mul2(make_float2(p[0], p[1]), f_a), w_c = mul2(make_float2(p[2], p[3]), f_c);
              b[g][u][nt][0] = transpose_8x8(pack_f16x2(w_a.x, w_a.y));
              b[g][u][nt][1] = transpose_8x8(pack_f16x2(w_c.x, w_c.y));
#pragma unroll
              for (int c = 0; c < 2; ++c) zs[nt][g][c] = fmaf(p[c], l_a, fmaf(p[2 + c], l_c, zs[nt][g][c]));
            }
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int g = DUO ? 0 : h;
          uint4 vw[UNITS];
#pragma unroll
          for (int u = 0; u < UNITS; ++u) vw[u] = *reinterpret_cast<const uint4*>(base + u * Q4_PAIR_BYTES + Q4_UNIT_BYTES + h * 512 + lane * 16);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            float d[NT][4];
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
              uint32_t A[4];
              q4_spread(word_of(vw[u], m), A);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (u == 0) mma_f16_first(d[nt], A, b[g][u][nt][0], b[g][u][nt][1]);
                else mma_f16_next(d[nt], A, b[g][u][nt][0], b[g][u][nt][1]);
              }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) add_to(acc[nt][4 * h + m], d[nt], make_float2(1.f, 1.f), make_float2(1.f, 1.f));
          }
        }
      };

      // a tile of `rows` <= 8 bf16 rows, the first at position pos
      auto bf16_rows = [&](int rows, int pos, const unsigned char* base) {
        if (hides(rows, pos, base)) {
#pragma unroll 1
          for (int j = 0; j < rows; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 w = *reinterpret_cast<const uint4*>(base + QA_V_OFF + j * ROW_BYTES + h * 128 + g8 * 16);
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                const uint32_t v2 = word_of(w, m), bad = not_finite(v2);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int c = 0; c < 2; ++c) {
                    if (pos + j > last_pos(nt, c)) continue;
                    if (bad & 0xffffu) acc[nt][4 * h + m][c] += bf16lo(v2);
                    if (bad >> 16) acc[nt][4 * h + m][2 + c] += bf16hi(v2);
                  }
              }
            }
          clear(rows, base);
        }
        float x[NT][2];
        {
          float d[NT][2][4];
          const uint4* kr = reinterpret_cast<const uint4*>(base + g8 * ROW_BYTES) + t4;
#pragma unroll
          for (int jw = 0; jw < 4; ++jw) {
            const uint4 kw = kr[4 * jw];
            const uint32_t A0[4] = {kw.x, 0u, kw.y, 0u}, A1[4] = {kw.z, 0u, kw.w, 0u};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint4 qw = *reinterpret_cast<const uint4*>(Qb + row_of(nt, g8) * D + 32 * jw + 8 * t4);
              if ((jw & 1) == 0) mma_bf16_first(d[nt][jw >> 1], A0, qw.x, qw.y);
              else mma_bf16_next(d[nt][jw >> 1], A0, qw.x, qw.y);
              mma_bf16_next(d[nt][jw >> 1], A1, qw.z, qw.w);
            }
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) x[nt][c] = fmaf(d[nt][0][c] + d[nt][1][c], sl2, -ref[nt][c]);
          if (rows < QA_ROWS16 || a.causal) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c)
                if (g8 >= rows || pos + g8 > last_pos(nt, c)) x[nt][c] = -INFINITY;
          }
        }
        uint4 e[2], o[2];      // this lane's numbers of the rows 2 t4 and 2 t4 + 1
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          e[h] = *reinterpret_cast<const uint4*>(base + QA_V_OFF + 2 * t4 * ROW_BYTES + h * 128 + g8 * 16);
          o[h] = *reinterpret_cast<const uint4*>(base + QA_V_OFF + (2 * t4 + 1) * ROW_BYTES + h * 128 + g8 * 16);
        }
        if (rows < QA_ROWS16) {      // what an earlier tile left there may be anything
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (2 * t4 >= rows) e[h] = make_uint4(0u, 0u, 0u, 0u);
            if (2 * t4 + 1 >= rows) o[h] = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        weigh(x, 0.f, 0.f, [](int, int) { return 0.f; });
        // both planes of the weights in one MMA: rows 0-7 of its contraction have the first, rows 8-15, the same rows again, the second
        uint32_t b[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint32_t hi = pack_bf16x2(x[nt][0], x[nt][1]);
          b[nt][0] = transpose_8x8(hi);
          b[nt][1] = transpose_8x8(pack_bf16x2(x[nt][0] - bf16lo(hi), x[nt][1] - bf16hi(hi)));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t ew[4] = {e[h].x, e[h].y, e[h].z, e[h].w}, ow[4] = {o[h].x, o[h].y, o[h].z, o[h].w};
          const float(&f)[2] = F[DUO ? 0 : h];
          const float2 f01 = make_float2(f[0] * 0x1p-24f, f[1] * 0x1p-24f), f23 = make_float2(f[0] * 0x1p-20f, f[1] * 0x1p-20f);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const uint32_t a0 = __byte_perm(ew[m], ow[m], 0x5410), a1 = __byte_perm(ew[m], ow[m], 0x7632);
            const uint32_t A[4] = {a0, a1, a0, a1};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float d[4];
              mma_bf16_first(d, A, b[nt][0], b[nt][1]);
              add_to(acc[nt][4 * h + m], d, f01, f23);
            }
          }
        }
      };

      // leaves the state of the sequence in shared memory
      auto leave = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) {
              l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], o);
#pragma unroll
              for (int g = 0; g < NG; ++g) zs[nt][g][c] += __shfl_xor_sync(0xffffffffu, zs[nt][g][c], o);
            }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float* st = states + (warp * COLS + row_of(nt, 2 * t4 + c)) * ATTN_PARTIAL_FLOATS;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              const float zv = zs[nt][g][c], un = 1.f / F[g][c];
              float* o = st + 64 * (DUO ? t4 >> 1 : g) + 8 * g8;
              float y[8];
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                const float even = DUO && t4 >= 2 ? acc[nt][4 + m][c] : acc[nt][4 * g + m][c], odd = DUO && t4 >= 2 ? acc[nt][4 + m][2 + c] : acc[nt][4 * g + m][2 + c];
                y[2 * m] = fmaf(even * un, 0x1p24f, zv);      // (in this order: sums of large values times 2^24 may pass what fp32 holds)
                y[2 * m + 1] = fmaf(odd * un, 0x1p20f, zv);
              }
              *reinterpret_cast<float4*>(o) = make_float4(y[0], y[1], y[2], y[3]);
              *reinterpret_cast<float4*>(o + 4) = make_float4(y[4], y[5], y[6], y[7]);
            }
            if (g8 == 0 && (!DUO || t4 < 2)) { st[128] = over_by[nt][c] == -INFINITY ? -INFINITY : ref[nt][c]; st[129] = l[nt][c]; }
          }
        __syncwarp();
      };

      consume(start, [&](int rows, const unsigned char* base) {
        if (rows == QA_ROWS4) packed_rows(std::integral_constant<int, 2>(), base);
        else packed_rows(std::integral_constant<int, 1>(), base);      // (the end of a chunk that is not a multiple of 32)
      }, bf16_rows, leave);
    } else {
      // ---- up to sixteen query rows: the queries on the M side of both products, so that the logits' accumulator is the weights' operand as it stands.  A lane has the
      // query rows g8 and g8 + 8 and two keys of every eight ----
      const uint4 *Qh = nullptr, *Qb = nullptr;      // query rows, as fp16 and as bf16: operands of the eight products along a row
      float acc[16][4];          // [8 h + 2 m + e]: rows g8 and g8 + 8, dims d = 64 h + 8 c + 2 m + e of the columns c = 2 t4, 2 t4 + 1; times F 2^-24 (e = 0), F 2^-20 (e = 1)
      float undo[2], l[2], zs[2][2], ref[2], over_by[2];      // per row, as in the other form; zs: [row][group]
      uint32_t F[2];             // [group]: the factors of both rows, as bf16
      auto most_of = [&](int r, int h) { return states + (warp * COLS + g8 + 8 * r) * ATTN_PARTIAL_FLOATS + 130 + h; };
      // The share of a logit that does not come from codes, low_0 (sum of q over group 0) + low_1 (of group 1) - reference, is a product as well: bf16 planes of the three
      // fp32 numbers of a query row (eight bits each, exact) against low_0 three times, low_1 three times, -1 three times.  This lane's part of the first operand:
      uint32_t la[4];
      float* qsum = nullptr;     // of the rows in use: [row][group], log2 units (used in the rare case only; all warps write the same)
      auto planes_of = [&](float y, uint32_t (&w)[3]) {      // bf16 bits of y = w0 + w1 + w2
        uint32_t p[3];
        split3_pair(y, 0.f, p);
#pragma unroll
        for (int i = 0; i < 3; ++i) w[i] = p[i] & 0xffffu;
      };
      auto set_rest = [&]() {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          uint32_t p0[3], p1[3], pr[3];
          planes_of(qsum[2 * (g8 + 8 * r)], p0);
          planes_of(qsum[2 * (g8 + 8 * r) + 1], p1);
          planes_of(ref[r], pr);
          // columns of the contraction: 0-2 q of group 0, 3-5 of group 1, 6-8 the reference; a lane has 2 t4, 2 t4 + 1 and 2 t4 + 8, 2 t4 + 9
          la[r] = t4 == 0 ? p0[0] | p0[1] << 16 : (t4 == 1 ? p0[2] | p1[0] << 16 : (t4 == 2 ? p1[1] | p1[2] << 16 : pr[0] | pr[1] << 16));
          la[2 + r] = t4 == 0 ? pr[2] : 0u;
        }
      };
      // the other operand for the key that the two words are of: low_0 and low_1 in their upper halves
      const uint32_t pick = t4 == 0 ? 0x3232u : (t4 == 1 ? 0x7632u : 0x7676u), minus_one = t4 == 0 ? 0xbf80u : 0u;
      auto rest_of = [&](uint2 w) { return t4 == 3 ? 0xbf80bf80u : __byte_perm(w.x, w.y, pick); };
      auto last_pos = [&](int r) { return a.causal ? progress[CW + 1] - a.T + (int)a.by_g.div((uint32_t)min(row0 + g8 + 8 * r, R - 1)) : 0x7fffffff; };

      auto start = [&](int slot) {
        Qh = reinterpret_cast<const uint4*>(smem + Shape::OFF_QH) + slot * 256 + lane;
        Qb = reinterpret_cast<const uint4*>(smem + Shape::OFF_Q) + slot * 256 + lane;
        const float* q_undo = reinterpret_cast<const float*>(smem + Shape::OFF_UNDO) + slot * 16;
        qsum = reinterpret_cast<float*>(smem + Shape::OFF_SUMS) + slot * 32;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float off = q_undo[g8 + 8 * r] * sl2;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 w = Qh[(4 * h + i) * 32];
              const float2 e0 = f16_pair(r ? w.y : w.x), e1 = f16_pair(r ? w.w : w.z);
              y += (e0.x + e0.y) + 16.f * (e1.x + e1.y);
            }
            y += __shfl_xor_sync(0xffffffffu, y, 1);
            y += __shfl_xor_sync(0xffffffffu, y, 2);
            qsum[2 * (g8 + 8 * r) + h] = y * off;
            F[h] = (uint32_t)(127 + QA_F_MOST) * 0x00800080u;
          }
          undo[r] = off * 0x1p12f * 0x1p12f;
          ref[r] = 0.f; over_by[r] = -INFINITY; l[r] = 0.f; zs[r][0] = zs[r][1] = 0.f;
        }
        set_rest();
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) acc[i][y] = 0.f;
      };

      // logits minus reference to weights in place, [8 keys each][row g8: two keys; row g8 + 8: two keys]; s0, s1: the largest scales of this lane's keys;
      // scale(i, k, group): that of key k of the i-th eight
      auto weigh = [&](auto& x, float s0, float s1, auto&& scale) {
        constexpr int N = (int)(sizeof(x) / sizeof(x[0]));
        bool over = s0 * fmaxf(bf16lo(F[0]), bf16hi(F[0])) > QA_TOP || s1 * fmaxf(bf16lo(F[1]), bf16hi(F[1])) > QA_TOP;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) over |= x[i][y] > over_by[y >> 1];
        if (__any_sync(0xffffffffu, over)) {
          float raw[2] = {s0, s1};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            raw[h] = fmaxf(raw[h], __shfl_xor_sync(0xffffffffu, raw[h], 1));
            raw[h] = fmaxf(raw[h], __shfl_xor_sync(0xffffffffu, raw[h], 2));
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, fmaxf(x[i][2 * r], x[i][2 * r + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool first = over_by[r] == -INFINITY;
            const float to = ref[r] + (first ? (top == -INFINITY ? 0.f : top) : fmaxf(top, 0.f)), up = to - ref[r];
            const float f = first ? 1.f : ex2_fast(-up);
            if (top != -INFINITY) over_by[r] = QA_SLACK;
            ref[r] = to;
#pragma unroll
            for (int i = 0; i < N; ++i) { x[i][2 * r] -= up; x[i][2 * r + 1] -= up; }
            l[r] *= f; zs[r][0] *= f; zs[r][1] *= f;
#pragma unroll
            for (int i = 0; i < 16; ++i) { acc[i][2 * r] *= f; acc[i][2 * r + 1] *= f; }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float ps = 0.f;      // the tile's largest weight times scale
#pragma unroll
              for (int i = 0; i < N; ++i) ps = fmaxf(ps, fmaxf(ex2_fast(x[i][2 * r]) * scale(i, 0, h), ex2_fast(x[i][2 * r + 1]) * scale(i, 1, h)));
              ps = fmaxf(ps, __shfl_xor_sync(0xffffffffu, ps, 1));
              ps = fmaxf(ps, __shfl_xor_sync(0xffffffffu, ps, 2));
              float* at = most_of(r, h);
              const float most = first ? ps : fmaxf(*at * f, ps);
              const int was = qa_exponent(r ? bf16hi(F[h]) : bf16lo(F[h])), now = qa_factor(was, raw[h], most, f);
              const float by = qa_power(max(now - was, -127));
              __syncwarp();
              *at = most;      // (the lanes of a row write the same)
              F[h] = __byte_perm(F[h], __float_as_uint(qa_power(now)), r ? 0x7610 : 0x3276);
#pragma unroll
              for (int i = 0; i < 8; ++i) { acc[8 * h + i][2 * r] *= by; acc[8 * h + i][2 * r + 1] *= by; }
            }
          }
          __syncwarp();
          set_rest();
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            x[i][y] = ex2_fast(x[i][y]);
            l[y >> 1] += x[i][y];
          }
      };
      auto add_to = [](float (&sum)[4], const float (&d)[4], float by0, float by1) {      // times the factors of the rows g8 and g8 + 8
        const float2 p = fma2(make_float2(d[0], d[1]), make_float2(by0, by0), make_float2(sum[0], sum[1])), q = fma2(make_float2(d[2], d[3]), make_float2(by1, by1), make_float2(sum[2], sum[3]));
        sum[0] = p.x; sum[1] = p.y; sum[2] = q.x; sum[3] = q.y;
      };

      // 32 packed rows, or 16 (the end of a chunk that is not a multiple of 32: what lies in the second unit is of an earlier tile)
      auto packed_rows = [&](int rows, const unsigned char* base) {
        float x[4][4];             // [eight keys each]
        {
          float d[4][2][4];        // [eight keys][group]
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint4 q0 = Qh[2 * j * 32], q1 = Qh[(2 * j + 1) * 32];
            const uint32_t A0[4] = {q0.x, q0.y, q0.z, q0.w}, A1[4] = {q1.x, q1.y, q1.z, q1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t b[4];
              q4_spread(*reinterpret_cast<const uint32_t*>(base + (i >> 1) * Q4_PAIR_BYTES + (i & 1) * 512 + lane * 16 + 4 * j), b);
              if ((j & 1) == 0) mma_f16_first(d[i][j >> 1], A0, b[0], b[1]);
              else mma_f16_next(d[i][j >> 1], A0, b[0], b[1]);
              mma_f16_next(d[i][j >> 1], A1, b[2], b[3]);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned char* heads = base + (i >> 1) * Q4_PAIR_BYTES + Q4_CODE_BYTES + (i & 1) * 64;
            const uint4 w = *reinterpret_cast<const uint4*>(heads + 16 * t4);      // the keys 2 t4 and 2 t4 + 1: scale and lowest number of both groups
            const float s0a = bf16lo(w.x), s1a = bf16lo(w.y), s0b = bf16lo(w.z), s1b = bf16lo(w.w);
            float rest[4];
            mma_bf16_first(rest, la, rest_of(*reinterpret_cast<const uint2*>(heads + 8 * g8)), minus_one);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              x[i][2 * r] = fmaf(fmaf(d[i][0][2 * r], s0a, d[i][1][2 * r] * s1a), undo[r], rest[2 * r]);
              x[i][2 * r + 1] = fmaf(fmaf(d[i][0][2 * r + 1], s0b, d[i][1][2 * r + 1] * s1b), undo[r], rest[2 * r + 1]);
            }
          }
        }
        const bool whole = rows == QA_ROWS4;
        if (!whole) {
#pragma unroll
          for (int i = 2; i < 4; ++i) x[i][0] = x[i][1] = x[i][2] = x[i][3] = -INFINITY;
        }
        // scale and lowest number of both groups of the keys 2 t4 and 2 t4 + 1 of the i-th eight, values (from shared memory every time)
        auto head = [&](int i) {
          return i >= 2 && !whole ? make_uint4(0u, 0u, 0u, 0u)
                                  : *reinterpret_cast<const uint4*>(base + (i >> 1) * Q4_PAIR_BYTES + Q4_UNIT_BYTES + Q4_CODE_BYTES + (i & 1) * 64 + 16 * t4);
        };
        uint32_t most0 = 0u, most1 = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 w = head(i);
          most0 = max_bf16x2(most0, max_bf16x2(w.x, w.z));
          most1 = max_bf16x2(most1, max_bf16x2(w.y, w.w));
        }
        weigh(x, bf16lo(most0), bf16lo(most1), [&](int i, int k, int h) { const uint4 w = head(i); return bf16lo(k ? (h ? w.w : w.z) : (h ? w.y : w.x)); });
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 F2 = make_float2(bf16lo(F[h]), bf16hi(F[h]));
          uint32_t A[2][4];        // weights times scale
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 vh = head(i);
            const uint32_t wa = h ? vh.y : vh.x, wb = h ? vh.w : vh.z;
            const float sa = bf16lo(wa), sb = bf16lo(wb), lo_a = bf16hi(wa), lo_b = bf16hi(wb);
            const float2 fa = mul2(make_float2(sa, sa), F2), fb = mul2(make_float2(sb, sb), F2);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              A[i >> 1][2 * (i & 1) + r] = pack_f16x2(x[i][2 * r] * (r ? fa.y : fa.x), x[i][2 * r + 1] * (r ? fb.y : fb.x));
              zs[r][h] = fmaf(x[i][2 * r], lo_a, fmaf(x[i][2 * r + 1], lo_b, zs[r][h]));
            }
          }
          const uint4 v0 = *reinterpret_cast<const uint4*>(base + Q4_UNIT_BYTES + h * 512 + lane * 16), v1 = *reinterpret_cast<const uint4*>(base + Q4_PAIR_BYTES + Q4_UNIT_BYTES + h * 512 + lane * 16);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            uint32_t b0[4], b1[4];
            q4_spread(word_of(v0, m), b0);
            q4_spread(word_of(v1, m), b1);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float d[4];
              mma_f16_first(d, A[0], b0[e], b0[2 + e]);
              mma_f16_next(d, A[1], b1[e], b1[2 + e]);
              add_to(acc[8 * h + 2 * m + e], d, 1.f, 1.f);
            }
          }
        }
      };

      // `rows` <= 8 bf16 rows, the first at position pos
      auto bf16_rows = [&](int rows, int pos, const unsigned char* base) {
        if (hides(rows, pos, base)) {
#pragma unroll 1
          for (int j = 0; j < rows; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const uint4 w = *reinterpret_cast<const uint4*>(base + QA_V_OFF + j * ROW_BYTES + h * 128 + (2 * t4 + c) * 16);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                  const uint32_t v2 = word_of(w, m), bad = not_finite(v2);
#pragma unroll
                  for (int r = 0; r < 2; ++r) {
                    if (pos + j > last_pos(r)) continue;
                    if (bad & 0xffffu) acc[8 * h + 2 * m][2 * r + c] += bf16lo(v2);
                    if (bad >> 16) acc[8 * h + 2 * m + 1][2 * r + c] += bf16hi(v2);
                  }
                }
              }
          clear(rows, base);
        }
        float d[2][4], x[1][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 q0 = Qb[2 * j * 32], q1 = Qb[(2 * j + 1) * 32];
          const uint4 kw = *reinterpret_cast<const uint4*>(base + g8 * ROW_BYTES + 64 * j + 16 * t4);
          const uint32_t A0[4] = {q0.x, q0.y, q0.z, q0.w}, A1[4] = {q1.x, q1.y, q1.z, q1.w};
          if ((j & 1) == 0) mma_bf16_first(d[j >> 1], A0, kw.x, kw.y);
          else mma_bf16_next(d[j >> 1], A0, kw.x, kw.y);
          mma_bf16_next(d[j >> 1], A1, kw.z, kw.w);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) x[0][y] = fmaf(d[0][y] + d[1][y], sl2, -ref[y >> 1]);
        if (rows < QA_ROWS16 || a.causal) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int key = 2 * t4 + (y & 1);
            if (key >= rows || pos + key > last_pos(y >> 1)) x[0][y] = -INFINITY;
          }
        }
        weigh(x, 0.f, 0.f, [](int, int, int) { return 0.f; });
        // both planes of the weights in one product: rows 0-7 of its contraction have the first, rows 8-15, the same keys again, the second
        uint32_t A[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          A[r] = pack_bf16x2(x[0][2 * r], x[0][2 * r + 1]);
          A[2 + r] = pack_bf16x2(x[0][2 * r] - bf16lo(A[r]), x[0][2 * r + 1] - bf16hi(A[r]));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 e = *reinterpret_cast<const uint4*>(base + QA_V_OFF + 2 * t4 * ROW_BYTES + h * 128 + g8 * 16), o = *reinterpret_cast<const uint4*>(base + QA_V_OFF + (2 * t4 + 1) * ROW_BYTES + h * 128 + g8 * 16);
          if (2 * t4 >= rows) e = make_uint4(0u, 0u, 0u, 0u);      // what an earlier tile left there may be anything
          if (2 * t4 + 1 >= rows) o = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t b = __byte_perm(word_of(e, m), word_of(o, m), y ? 0x7632 : 0x5410);
              float t[4];
              mma_bf16_first(t, A, b, b);
              add_to(acc[8 * h + 2 * m + y], t, bf16lo(F[h]) * (y ? 0x1p-20f : 0x1p-24f), bf16hi(F[h]) * (y ? 0x1p-20f : 0x1p-24f));
            }
        }
      };

      auto leave = [&]() {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int o = 1; o <= 2; o <<= 1) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
            zs[r][0] += __shfl_xor_sync(0xffffffffu, zs[r][0], o);
            zs[r][1] += __shfl_xor_sync(0xffffffffu, zs[r][1], o);
          }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float* st = states + (warp * COLS + g8 + 8 * r) * ATTN_PARTIAL_FLOATS;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float un = 1.f / (r ? bf16hi(F[h]) : bf16lo(F[h]));
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float y[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = fmaf(acc[8 * h + i][2 * r + c] * un, i & 1 ? 0x1p20f : 0x1p24f, zs[r][h]);
              float* o = st + 64 * h + 8 * (2 * t4 + c);
              *reinterpret_cast<float4*>(o) = make_float4(y[0], y[1], y[2], y[3]);
              *reinterpret_cast<float4*>(o + 4) = make_float4(y[4], y[5], y[6], y[7]);
            }
          }
          if (t4 == 0) { st[128] = over_by[r] == -INFINITY ? -INFINITY : ref[r]; st[129] = l[r]; }
        }
        __syncwarp();
      };

      consume(start, packed_rows, bf16_rows, leave);
    }
  }

  // ---- the last sequence's states, by all warps; then sequences of which other CTAs have parts: the first and the last of this run ----
  __syncthreads();
  for (int r = warp; r < n_rows; r += WARPS) fold_states(x1, r);
  if (whole(x0) && whole(x1)) return;
  __syncthreads();
  // The ticket is an acquire-release atomic at device scope, taken when all warps have written their records: it publishes them, and makes those of the other
  // CTAs visible to this one's warps once they have synchronised again.
  if (threadIdx.x < 2) {
    const int x = threadIdx.x ? x1 : x0;
    const int parts = (int)(qa_owner((uint32_t)(x + 1) * uk - 1u, n_items, P) - qa_owner((uint32_t)x * uk, n_items, P)) + 1;
    int mine = 0;
    if (parts > 1 && (threadIdx.x == 0 || x1 > x0)) {
      int arrived;
      asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(arrived) : "l"(a.counters + x * a.groups + group) : "memory");
      if (arrived == parts - 1) {
        mine = parts;
        a.counters[x * a.groups + group] = 0;      // clean for the next launch
      }
    }
    flags[threadIdx.x] = mine;
  }
  __syncthreads();
  for (int e = 0; e < 2; ++e) {
    const int parts = flags[e], x = e ? x1 : x0;
    if (parts == 0) continue;
    const float* recs = a.partials + ((long long)(x + (int)qa_owner((uint32_t)x * uk, n_items, P)) * a.groups + group) * COLS * ATTN_PARTIAL_FLOATS;
    const long long stride = (long long)a.groups * COLS * ATTN_PARTIAL_FLOATS;      // from run to run
    // several warps share the records of a row where there are fewer rows than warps; a record is one trip to L2
    const int per_row = n_rows >= WARPS ? 1 : WARPS / n_rows;
    for (int y = warp; y < n_rows * per_row; y += WARPS) {
      const int r = y / per_row, sub = y - r * per_row;
      const float* rec = recs + r * ATTN_PARTIAL_FLOATS;
      float top = -INFINITY, sum = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p0 = sub; p0 < parts; p0 += 4 * per_row) {
        float m[4], l[4];
        float4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = p0 + i * per_row;
          const float* st = rec + (p < parts ? p : p0) * stride;
          m[i] = __ldcg(st + 128); l[i] = __ldcg(st + 129);
          w[i] = __ldcg(reinterpret_cast<const float4*>(st + lane * 4));
        }
        float to = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) to = fmaxf(to, m[i]);
        const float f0 = top == -INFINITY ? 0.f : exp2f(top - to);
        sum *= f0; o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
        top = to;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (p0 + i * per_row >= parts) continue;
          const float f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - top);
          sum = fmaf(l[i], f, sum);
          o.x = fmaf(w[i].x, f, o.x); o.y = fmaf(w[i].y, f, o.y); o.z = fmaf(w[i].z, f, o.z); o.w = fmaf(w[i].w, f, o.w);
        }
      }
      if (per_row == 1) {
        write_row(a, x, row0 + r, o, top, sum, lane);
      } else {
        float* st = states + y * ATTN_PARTIAL_FLOATS;
        *reinterpret_cast<float4*>(st + lane * 4) = o;
        if (lane == 0) { st[128] = top; st[129] = sum; }
      }
    }
    if (per_row > 1) {
      __syncthreads();
      for (int r = warp; r < n_rows; r += WARPS) {
        const float* st = states + r * per_row * ATTN_PARTIAL_FLOATS;
        float top = -INFINITY, sum = 0.f;
        for (int sub = 0; sub < per_row; ++sub) top = fmaxf(top, st[sub * ATTN_PARTIAL_FLOATS + 128]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int sub = 0; sub < per_row; ++sub) fold(st + sub * ATTN_PARTIAL_FLOATS, top, sum, o, lane);
        write_row(a, x, row0 + r, o, top, sum, lane);
      }
    }
    __syncthreads();
  }
}

Q4AttnShape q4_attn_shape(int rows) {
  const int cols = rows <= 4 ? 4 : (rows <= 8 ? 8 : 16);
  return {cols, (rows + cols - 1) / cols};
}

cudaError_t launch_attn_q4(const LayerView& v, const Q4Pages& p, bool dense, int T, int G, bool causal, int parts_per_seq, int runs, const void* q, void* out,
                           float* lse, float scale, float* partials, int32_t* counters, cudaStream_t st) {
  const Q4AttnShape shape = q4_attn_shape(T * G);
  Q4AttnArgs a;
  a.v = v; a.p = p;
  a.by_g = fast_div((uint32_t)G); a.by_h = fast_div((uint32_t)v.H); a.by_k = fast_div((uint32_t)parts_per_seq);
  a.by_tiles4 = fast_div((uint32_t)((v.C + QA_ROWS4 - 1) / QA_ROWS4));
  a.by_tiles16 = fast_div((uint32_t)(v.C / QA_ROWS16));
  a.dense = dense ? 1 : 0; a.T = T; a.G = G; a.causal = causal ? 1 : 0; a.k = parts_per_seq; a.groups = shape.groups;
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse = lse; a.scale = scale;
  a.partials = partials; a.counters = counters;
  auto launch = [&](auto kernel, DeviceFlags& opted, int warps, int smem) {
    const cudaError_t e = smem_opt_in(opted, kernel, smem);
    return e != cudaSuccess ? e : launch_pdl(kernel, dim3((unsigned)(runs * shape.groups)), dim3((unsigned)warps * 32), (size_t)smem, st, a);
  };
  static DeviceFlags f4, f8, f16;
  switch (shape.cols) {
    case 4: return launch(kve_decode_attn_q4_kernel<4>, f4, QaShape<4>::WARPS, QaShape<4>::SMEM);
    case 8: return launch(kve_decode_attn_q4_kernel<8>, f8, QaShape<8>::WARPS, QaShape<8>::SMEM);
    default: return launch(kve_decode_attn_q4_kernel<16>, f16, QaShape<16>::WARPS, QaShape<16>::SMEM);
  }
}

}  // namespace kve
