// Decode attention over a history held in 4 bits (kvE_decode_attn_q4):
//   out = softmax(q K'^T * scale) V',  rows of K', V' = [chunks held in 4 bits ; chunks and recent rows in bf16]
// for T x G query rows per KV head (T query tokens, G query heads a KV head).
//
// HBM is the floor: 144 bytes a packed row, 512 a bf16 row, each read once per group of query rows.  At 144 bytes a row the SM has ~100
// cycles for 16 rows, so what has to be small is the number of instructions per code:
//  * the codes lie in the pages in the order of the MMA operands (q4.cuh): eight of them are one 32-bit word of one lane, and become four
//    operand registers in seven instructions.  They enter the products as 1 + c / 16, exactly; scale and lowest number of a group
//    are applied to the sums (keys: per row and group to the logit) or to the weights (values: p s per group of 64 dims).
//  * both products are m16n8k16 MMAs with the cache on the M side (keys: 16 rows; values, transposed: 16 dims) and the queries in the
//    eight columns.  The weights p s enter as two bf16 planes (16 bits); with up to four query rows the planes take four columns each
//    and cost one MMA.  The logits' accumulator becomes the weights' operand through movmatrix, in registers.
//  * a warp is on its own: it has a ring of stages in shared memory, asks for its tiles by bulk copies (one lane), waits for them and
//    keeps its softmax state in registers.  No barrier between warps before the end.  A tile is 32 packed rows or 8 bf16 rows: about as many
//    bytes, so that equal counts are equal work.
//  * the reference of the softmax is raised only when a logit passes it by more than 2^8 (a vote), not at every tile.
// A sequence's tiles are cut into `splits` equal parts, a CTA each; the last CTA of a sequence to finish merges the records.
#include "q4.cuh"

namespace kve {

constexpr int QA_WARPS = 8;
constexpr int QA_TILE_BYTES = 4 * Q4_UNIT_BYTES;             // two units of keys, two of values
constexpr int QA_V_OFF = 2 * Q4_UNIT_BYTES;                  // values behind the keys
constexpr int QA_ROWS4 = 2 * Q4_UNIT_ROWS, QA_ROWS16 = 8;    // rows of a tile of either kind
// bf16 rows are spread out in the stage so that the lanes' reads meet different banks
__device__ __forceinline__ constexpr int qa_k_row(int r) { return (r >> 1) * 576 + (r & 1) * 320; }
__device__ __forceinline__ constexpr int qa_v_row(int r) { return QA_V_OFF + r * 272; }
static_assert(qa_k_row(7) + ROW_BYTES <= QA_V_OFF && qa_v_row(7) + ROW_BYTES <= QA_TILE_BYTES, "eight bf16 rows fit a stage");
constexpr float QA_SLACK = 8.f;                              // by how much (log2) a logit may pass the softmax reference

struct Q4AttnArgs {
  LayerView v;
  Q4Pages p;
  FastDiv by_g, by_tiles4, by_tiles16;      // by G; by the tiles of a chunk of either kind
  int dense, T, G, causal, splits;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  float scale;
  float* partials;      // [S][splits][T G][132]
  int32_t* counters;    // [row groups][S]
};

template <int NT> struct QaShape {
  static constexpr int COLS = 8 * NT;                        // query rows of a CTA
  static constexpr int STAGES = NT == 1 ? 3 : 5;
  static constexpr int CTAS = NT == 1 ? 2 : 1;               // per SM
  static constexpr int RING = QA_WARPS * STAGES * QA_TILE_BYTES;
  static constexpr int MERGE = QA_WARPS * COLS * ATTN_PARTIAL_FLOATS * 4;      // the warps' states, in place of the ring
  static constexpr int OFF_Q = RING > MERGE ? RING : MERGE;  // query rows, bf16
  static constexpr int OFF_BAR = OFF_Q + COLS * ROW_BYTES;
  static constexpr int SMEM = OFF_BAR + QA_WARPS * STAGES * 8 + 16;
};

// a tile as one lane knows it: where its rows lie (byte offset in the 4-bit pool, or element offset in the bf16 pool), how many, of which kind
struct QaTile { long long at; int rows, kind; };

__device__ __forceinline__ void mma_bf16_1688(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(b0));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// NT: column tiles of eight query rows; SPLIT (NT == 1): up to four query rows, their weights' two planes side by side in the columns
template <int NT, bool SPLIT>
__global__ void __launch_bounds__(QA_WARPS * 32, QaShape<NT>::CTAS) kve_decode_attn_q4_kernel(Q4AttnArgs a) {
  using Shape = QaShape<NT>;
  constexpr int STAGES = Shape::STAGES;
  constexpr int PER_GROUP = SPLIT ? 4 : Shape::COLS;      // query rows of this CTA
  extern __shared__ __align__(128) unsigned char smem[];
  uint16_t* Qs = reinterpret_cast<uint16_t*>(smem + Shape::OFF_Q);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Shape::OFF_BAR);
  int* flag = reinterpret_cast<int*>(bars + QA_WARPS * STAGES);
  const LayerView& v = a.v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
  const int part = blockIdx.x, s = blockIdx.y, z = blockIdx.z;
  const int R = a.T * a.G, row0 = z * PER_GROUP, n_rows = min(R - row0, PER_GROUP);
  uint64_t* full = bars + warp * STAGES;
  unsigned char* ring = smem + warp * STAGES * QA_TILE_BYTES;

  pdl_launch_dependents();
  if (lane < STAGES) mbar_init(&full[lane], 1);
  mbar_fence_init();
  __syncwarp();
  pdl_wait();

  // ---- the lists: kept chunks in 4 bits, chunks behind the keep list in 4 bits, kept chunks in bf16, the rest in bf16 ----
  const int n = min(max(*reinterpret_cast<const volatile int32_t*>(v.seq_len), 0), v.max_tokens);
  const int packed = min(max(*reinterpret_cast<const volatile int32_t*>(v.n_packed), 0), n / v.C);
  const int listed = a.dense ? 0 : min(max(*reinterpret_cast<const volatile int32_t*>(v.n_listed), 0), n / v.C);
  const long long sb = (long long)s * v.max_chunks;
  const int kept = a.dense ? 0 : min(max(*reinterpret_cast<const volatile int32_t*>(v.keep_cnt + s), 0), listed);
  int kept4 = kept;      // kept chunks that are packed: the list ascends
  if (packed < listed) {
    int lo = 0, hi = kept;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (__ldcg(v.keep_idx + sb + mid) < packed) lo = mid + 1; else hi = mid;
    }
    kept4 = lo;
  }
  const int c_tail = max(listed, packed), tail = n - c_tail * v.C;
  const int per4 = (v.C + QA_ROWS4 - 1) / QA_ROWS4, per16 = v.C / QA_ROWS16;
  const int e0 = kept4 * per4, e1 = e0 + max(packed - listed, 0) * per4, e2 = e1 + (kept - kept4) * per16, total = e2 + (tail + QA_ROWS16 - 1) / QA_ROWS16;
  const int j0 = (int)((long long)part * total / a.splits), j1 = (int)((long long)(part + 1) * total / a.splits);
  const int mine = max(0, (j1 - j0 - warp + QA_WARPS - 1) / QA_WARPS);      // tiles of this warp: j0 + warp, + 8, ...
  if (a.causal && tail < a.T && threadIdx.x == 0) set_status(v.status, ERR_CAPACITY);      // (a replay that outgrew its capture: the block's first tokens have no rows of their own any more)

  // Where the tile this lane looks after lies.  In two steps, so that no look-up is waited for: the chunk, then its page.
  auto chunk_of = [&](int i) -> int {      // i: index among this warp's tiles; -1: none
    if (i >= mine) return -1;
    const int j = j0 + warp + i * QA_WARPS;
    if (j < e0) return __ldcg(v.keep_idx + sb + (int)a.by_tiles4.div((uint32_t)j));
    if (j < e1) return listed + (int)a.by_tiles4.div((uint32_t)(j - e0));
    if (j < e2) return __ldcg(v.keep_idx + sb + kept4 + (int)a.by_tiles16.div((uint32_t)(j - e1)));
    return c_tail + (int)a.by_tiles16.div((uint32_t)(j - e2));
  };
  auto page_of = [&](int i, int chunk) -> int {
    if (i >= mine || chunk < 0 || chunk >= v.max_chunks) return -1;
    return __ldcg((j0 + warp + i * QA_WARPS < e1 ? a.p.table : v.page_table) + sb + chunk);
  };
  auto tile_of = [&](int i, int page) -> QaTile {
    QaTile t;
    t.at = 0; t.rows = 0; t.kind = 0;
    if (i >= mine) return t;
    const int j = j0 + warp + i * QA_WARPS;
    t.kind = j < e1 ? 0 : 1;
    if (t.kind == 0) {
      const int jj = j < e0 ? j : j - e0, within = jj - (int)a.by_tiles4.div((uint32_t)jj) * per4;
      t.rows = min(QA_ROWS4, v.C - within * QA_ROWS4);
      if (page < 0 || page >= a.p.n_pages) { set_status(v.status, ERR_CAPACITY); page = 0; }
      t.at = ((long long)page * v.C + within * QA_ROWS4) * (Q4_UNIT_BYTES / Q4_UNIT_ROWS);
    } else {
      const int jj = j < e2 ? j - e1 : j - e2, within = jj - (int)a.by_tiles16.div((uint32_t)jj) * per16;
      t.rows = j < e2 ? QA_ROWS16 : min(QA_ROWS16, tail - jj * QA_ROWS16);
      if (page < 0 || page >= v.n_pages) { set_status(v.status, ERR_CAPACITY); page = 0; }
      t.at = ((long long)page * v.C + within * QA_ROWS16) * D;
    }
    return t;
  };
  const int chunk0 = chunk_of(lane);
  QaTile cur = tile_of(lane, page_of(lane, chunk0));
  int next_chunk = -1, next_page = -1;      // of the tile 32 on
  // asks for tile i; i runs through 0, 1, 2, ...
  auto issue = [&](int i) {
    const int l = i & 31, stage = i % STAGES;
    if (l == 0 && i > 0) cur = tile_of(i + lane, next_page);
    if (l == 8) next_chunk = chunk_of((i & ~31) + 32 + lane);
    if (l == 20) next_page = page_of((i & ~31) + 32 + lane, next_chunk);
    unsigned char* dst = ring + stage * QA_TILE_BYTES;
    const int kind = __shfl_sync(0xffffffffu, cur.kind, l), rows = __shfl_sync(0xffffffffu, cur.rows, l);
    const long long at = __shfl_sync(0xffffffffu, cur.at, l);
    if (kind == 0) {
      if (lane == 0) {
        const uint32_t bytes = (uint32_t)rows * (Q4_UNIT_BYTES / Q4_UNIT_ROWS);
        mbar_arrive_expect_tx(&full[stage], 2 * bytes);
        bulk_g2s(dst, a.p.k + at, bytes, &full[stage]);
        bulk_g2s(dst + QA_V_OFF, a.p.v + at, bytes, &full[stage]);
      }
    } else {
      if (lane == 0) mbar_arrive_expect_tx(&full[stage], (uint32_t)rows * 2 * ROW_BYTES);
      __syncwarp();
      const int r = lane & 7;
      if (lane < 16 && r < rows) {
        if (lane < 8) bulk_g2s(dst + qa_k_row(r), v.k_pages + at + r * D, ROW_BYTES, &full[stage]);
        else bulk_g2s(dst + qa_v_row(r), v.v_pages + at + r * D, ROW_BYTES, &full[stage]);
      }
    }
  };
  for (int i = 0; i < STAGES && i < mine; ++i) issue(i);

  // ---- query rows: operand fragments, and the sums of their two halves ----
  // column c of the MMAs is query row row0 + (SPLIT ? c & 3 : c); rows that do not exist are zeros
  for (int i = threadIdx.x; i < Shape::COLS * 16; i += QA_WARPS * 32) {
    const int c = i >> 4, r = SPLIT ? (c & 3) : c;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (r < n_rows) {
      const int rr = row0 + r, t = (int)a.by_g.div((uint32_t)rr), g = rr - t * a.G;
      const int b = s / v.H, h = s - b * v.H;
      w = __ldcg(reinterpret_cast<const uint4*>(a.q + ((((long long)b * a.T + t) * v.H + h) * a.G + g) * D + (i & 15) * 8));
    }
    *reinterpret_cast<uint4*>(Qs + c * D + (i & 15) * 8) = w;
  }
  __syncthreads();
  constexpr bool Q_REGS = NT == 1;
  uint4 qf[Q_REGS ? 4 : 1];      // column g8: the numbers 32 j + 8 t4 .. + 7
  if constexpr (Q_REGS) {
#pragma unroll
    for (int j = 0; j < 4; ++j) qf[j] = *reinterpret_cast<const uint4*>(Qs + g8 * D + 32 * j + 8 * t4);
  }
  float qsum[NT][2][2];          // [half][column 2 t4, 2 t4 + 1]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 w = *reinterpret_cast<const uint4*>(Qs + (nt * 8 + g8) * D + 64 * h + 32 * j + 8 * t4);
        sum += (bf16lo(w.x) + bf16hi(w.x)) + (bf16lo(w.y) + bf16hi(w.y)) + (bf16lo(w.z) + bf16hi(w.z)) + (bf16lo(w.w) + bf16hi(w.w));
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);      // of column g8, in its four lanes
      qsum[nt][h][0] = __shfl_sync(0xffffffffu, sum, 8 * t4);
      qsum[nt][h][1] = __shfl_sync(0xffffffffu, sum, 8 * t4 + 4);
    }
  const float sl2 = a.scale * 1.44269504088896340736f;      // logits in log2 units
  int last_pos[NT][2];                                       // causal: the last position a column sees
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int c = nt * 8 + 2 * t4 + x, rr = row0 + (SPLIT ? (c & 3) : c);
      last_pos[nt][x] = a.causal ? n - a.T + (int)a.by_g.div((uint32_t)min(rr, R - 1)) : 0x7fffffff;
    }

  float acc[NT][8][4];           // [m]: dims d = 64 (m / 4) + 8 g8 + 2 (m % 4) and d + 1, columns 2 t4 and 2 t4 + 1: (d, c), (d, c + 1), (d + 1, c), (d + 1, c + 1)
  float ref[NT][2], l[NT][2], zs[NT][2][2];      // per column: reference; this lane's rows' share of the sum of weights, and of weights times what the codes' offset stands for
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int m = 0; m < 8; ++m)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[nt][m][x] = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) { ref[nt][x] = -INFINITY; l[nt][x] = 0.f; zs[nt][0][x] = zs[nt][1][x] = 0.f; }
  }

  // Logits of 16 rows (log2 units; [row g8: c, c + 1; row g8 + 8: c, c + 1]) to weights in place; raises the reference where it has to
  auto weigh = [&](float (&x)[NT][4]) {
    bool over = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) over |= x[nt][i] > ref[nt][i & 1] + QA_SLACK;
    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float top = fmaxf(x[nt][c], x[nt][2 + c]);
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          const float to = fmaxf(ref[nt][c], top);
          const float f = to == -INFINITY ? 1.f : ex2_fast(ref[nt][c] - to);
          ref[nt][c] = to;
          l[nt][c] *= f; zs[nt][0][c] *= f; zs[nt][1][c] *= f;
#pragma unroll
          for (int m = 0; m < 8; ++m) { acc[nt][m][c] *= f; acc[nt][m][2 + c] *= f; }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float r = ref[nt][i & 1];
        x[nt][i] = ex2_fast(x[nt][i] - (r == -INFINITY ? 0.f : r));      // (only logits of -inf so far: weights 0)
        l[nt][i & 1] += x[nt][i];
      }
  };
  // two weights as bf16: the plane of the SPLIT column, or both planes
  auto planes = [&](float w0, float w1, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16x2(w0, w1);
    lo = pack_bf16x2(w0 - bf16lo(hi), w1 - bf16hi(hi));
    if (SPLIT) hi = t4 >= 2 ? lo : hi;
  };

  for (int i = 0; i < mine; ++i) {
    const int stage = i % STAGES;
    if (!mbar_wait_bounded(&full[stage], (uint32_t)((i / STAGES) & 1))) {
      if (lane == 0) set_status(v.status, ERR_TIMEOUT);
      ring_drain<STAGES>(full, min(i + STAGES, mine));
      break;
    }
    const unsigned char* base = ring + stage * QA_TILE_BYTES;
    const int j = j0 + warp + i * QA_WARPS;
    if (j < e1) {
      // ================= packed rows =================
      const int jj = j < e0 ? j : j - e0, within = jj - (int)a.by_tiles4.div((uint32_t)jj) * per4;
      const int units = min(2, per16 / 2 - within * 2);
      for (int u = 0; u < units; ++u) {
        const unsigned char* kb = base + u * Q4_UNIT_BYTES;
        const unsigned char* vb = kb + QA_V_OFF;
        const uint4 ka = *reinterpret_cast<const uint4*>(kb + lane * 16), kc = *reinterpret_cast<const uint4*>(kb + 512 + lane * 16);
        const uint2 ha = *reinterpret_cast<const uint2*>(kb + Q4_CODE_BYTES + g8 * 8), hc = *reinterpret_cast<const uint2*>(kb + Q4_CODE_BYTES + 64 + g8 * 8);
        float x[NT][4];
        {
          const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wc[4] = {kc.x, kc.y, kc.z, kc.w};
          float d[NT][2][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int y = 0; y < 4; ++y) d[nt][h][y] = 0.f;
#pragma unroll
          for (int jw = 0; jw < 4; ++jw) {
            uint32_t pa[4], pc[4];
            q4_spread(wa[jw], pa);
            q4_spread(wc[jw], pc);
            const uint32_t A0[4] = {pa[0], pc[0], pa[1], pc[1]}, A1[4] = {pa[2], pc[2], pa[3], pc[3]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint4 qw = Q_REGS ? qf[Q_REGS ? jw : 0] : *reinterpret_cast<const uint4*>(Qs + (nt * 8 + g8) * D + 32 * jw + 8 * t4);
              mma_bf16_16816(d[nt][jw >> 1], A0, qw.x, qw.y);
              mma_bf16_16816(d[nt][jw >> 1], A1, qw.z, qw.w);
            }
          }
          // x = low + 16 s ((1 + c / 16) - 1): the sum over a group is 16 s (what the MMAs give) + (low - 16 s) (sum of q)
          const float sa0 = 16.f * bf16lo(ha.x), sa1 = 16.f * bf16lo(ha.y), sc0 = 16.f * bf16lo(hc.x), sc1 = 16.f * bf16lo(hc.y);
          const float za0 = bf16hi(ha.x) - sa0, za1 = bf16hi(ha.y) - sa1, zc0 = bf16hi(hc.x) - sc0, zc1 = bf16hi(hc.y) - sc1;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              x[nt][c] = (fmaf(d[nt][0][c], sa0, za0 * qsum[nt][0][c]) + fmaf(d[nt][1][c], sa1, za1 * qsum[nt][1][c])) * sl2;
              x[nt][2 + c] = (fmaf(d[nt][0][2 + c], sc0, zc0 * qsum[nt][0][c]) + fmaf(d[nt][1][2 + c], sc1, zc1 * qsum[nt][1][c])) * sl2;
            }
        }
        weigh(x);
        const uint2 va = *reinterpret_cast<const uint2*>(vb + Q4_CODE_BYTES + g8 * 8), vc = *reinterpret_cast<const uint2*>(vb + Q4_CODE_BYTES + 64 + g8 * 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // values enter as (c - 8) / 16: x = (low + 8 s) + 16 s (c - 8) / 16
          const uint32_t ga = h ? va.y : va.x, gc = h ? vc.y : vc.x;
          const float s_a = 16.f * bf16lo(ga), s_c = 16.f * bf16lo(gc), z_a = fmaf(0.5f, s_a, bf16hi(ga)), z_c = fmaf(0.5f, s_c, bf16hi(gc));
          uint32_t bh[NT][2], bl[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            planes(x[nt][0] * s_a, x[nt][1] * s_a, bh[nt][0], bl[nt][0]);
            planes(x[nt][2] * s_c, x[nt][3] * s_c, bh[nt][1], bl[nt][1]);
#pragma unroll
            for (int c = 0; c < 2; ++c) zs[nt][h][c] = fmaf(x[nt][c], z_a, fmaf(x[nt][2 + c], z_c, zs[nt][h][c]));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              bh[nt][y] = transpose_8x8(bh[nt][y]);
              if (!SPLIT) bl[nt][y] = transpose_8x8(bl[nt][y]);
            }
          }
          const uint4 vw = *reinterpret_cast<const uint4*>(vb + h * 512 + lane * 16);
          const uint32_t w[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            uint32_t A[4];
            q4_spread(w[m], A);
#pragma unroll
            for (int y = 0; y < 4; ++y) A[y] = sub_bf16x2(A[y], 0x3fc03fc0u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma_bf16_16816(acc[nt][4 * h + m], A, bh[nt][0], bh[nt][1]);
              if (!SPLIT) mma_bf16_16816(acc[nt][4 * h + m], A, bl[nt][0], bl[nt][1]);
            }
          }
        }
      }
    } else {
      // ================= bf16 rows: eight of them =================
      const int jj = j < e2 ? j - e1 : j - e2;
      const int rows = j < e2 ? QA_ROWS16 : min(QA_ROWS16, tail - jj * QA_ROWS16), pos = c_tail * v.C + jj * QA_ROWS16;      // (pos: of tail rows)
      float x[NT][4];
      {
        float d[NT][2][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int y = 0; y < 4; ++y) d[nt][h][y] = 0.f;
        const uint4* kr = reinterpret_cast<const uint4*>(base + qa_k_row(g8)) + t4;
#pragma unroll
        for (int jw = 0; jw < 4; ++jw) {
          const uint4 kw = kr[4 * jw];
          const uint32_t A0[4] = {kw.x, 0u, kw.y, 0u}, A1[4] = {kw.z, 0u, kw.w, 0u};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const uint4 qw = Q_REGS ? qf[Q_REGS ? jw : 0] : *reinterpret_cast<const uint4*>(Qs + (nt * 8 + g8) * D + 32 * jw + 8 * t4);
            mma_bf16_16816(d[nt][jw >> 1], A0, qw.x, qw.y);
            mma_bf16_16816(d[nt][jw >> 1], A1, qw.z, qw.w);
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const bool seen = g8 < rows && (j < e2 || pos + g8 <= last_pos[nt][c]);
            x[nt][c] = seen ? (d[nt][0][c] + d[nt][1][c]) * sl2 : -INFINITY;
            x[nt][2 + c] = -INFINITY;
          }
      }
      weigh(x);
      uint32_t bh[NT], bl[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        planes(x[nt][0], x[nt][1], bh[nt], bl[nt]);
        bh[nt] = transpose_8x8(bh[nt]);
        if (!SPLIT) bl[nt] = transpose_8x8(bl[nt]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 e = *reinterpret_cast<const uint4*>(base + qa_v_row(2 * t4) + h * 128 + g8 * 16), o = *reinterpret_cast<const uint4*>(base + qa_v_row(2 * t4 + 1) + h * 128 + g8 * 16);
        if (2 * t4 >= rows) e = make_uint4(0u, 0u, 0u, 0u);      // what an earlier tile left there may be anything
        if (2 * t4 + 1 >= rows) o = make_uint4(0u, 0u, 0u, 0u);
        const uint32_t ew[4] = {e.x, e.y, e.z, e.w}, ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const uint32_t a0 = __byte_perm(ew[m], ow[m], 0x5410), a1 = __byte_perm(ew[m], ow[m], 0x7632);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_bf16_1688(acc[nt][4 * h + m], a0, a1, bh[nt]);
            if (!SPLIT) mma_bf16_1688(acc[nt][4 * h + m], a0, a1, bl[nt]);
          }
        }
      }
    }
    __syncwarp();
    if (i + STAGES < mine) issue(i + STAGES);
  }

  // ---- the warps' states meet in shared memory ----
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int o = 4; o <= 16; o <<= 1) {
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], o);
        zs[nt][0][c] += __shfl_xor_sync(0xffffffffu, zs[nt][0][c], o);
        zs[nt][1][c] += __shfl_xor_sync(0xffffffffu, zs[nt][1][c], o);
      }
  if constexpr (SPLIT) {      // the two planes
#pragma unroll
    for (int m = 0; m < 8; ++m)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[0][m][x] += __shfl_xor_sync(0xffffffffu, acc[0][m][x], 2);
  }
  __syncthreads();      // every warp's last tile has been read
  float* states = reinterpret_cast<float*>(smem);      // [warp][column][132]
  if (!SPLIT || t4 < 2) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float* st = states + ((warp * Shape::COLS) + nt * 8 + 2 * t4 + c) * ATTN_PARTIAL_FLOATS;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float zv = zs[nt][h][c];
          float* o = st + 64 * h + 8 * g8;
          *reinterpret_cast<float4*>(o) = make_float4(acc[nt][4 * h][c] + zv, acc[nt][4 * h][2 + c] + zv, acc[nt][4 * h + 1][c] + zv, acc[nt][4 * h + 1][2 + c] + zv);
          *reinterpret_cast<float4*>(o + 4) = make_float4(acc[nt][4 * h + 2][c] + zv, acc[nt][4 * h + 2][2 + c] + zv, acc[nt][4 * h + 3][c] + zv, acc[nt][4 * h + 3][2 + c] + zv);
        }
        if (g8 == 0) { st[128] = ref[nt][c]; st[129] = l[nt][c]; }
      }
  }
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
  auto finish = [&](int rr, float4 o, float top, float sum) {      // a warp writes query row rr
    const float inv = sum == 0.f ? 0.f : 1.f / sum;                // (no row, or weights of 0 only: 0; NaN stays)
    const int t = (int)a.by_g.div((uint32_t)rr), g = rr - t * a.G, b = s / v.H, h = s - b * v.H;
    const long long at = (((long long)b * a.T + t) * v.H + h) * a.G + g;
    *reinterpret_cast<uint2*>(a.out + at * D + lane * 4) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994530942f;
  };
  for (int r = warp; r < n_rows; r += QA_WARPS) {
    const float* st = states + r * ATTN_PARTIAL_FLOATS;
    constexpr int STRIDE = Shape::COLS * ATTN_PARTIAL_FLOATS;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < QA_WARPS; ++w) top = fmaxf(top, st[w * STRIDE + 128]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < QA_WARPS; ++w) {
      const float m = st[w * STRIDE + 128], f = m == -INFINITY ? 0.f : exp2f(m - top);
      const float4 x = *reinterpret_cast<const float4*>(st + w * STRIDE + lane * 4);
      sum = fmaf(st[w * STRIDE + 129], f, sum);
      o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
    }
    if (a.splits == 1) {
      finish(row0 + r, o, top, sum);
    } else {
      float* rec = a.partials + (((long long)s * a.splits + part) * R + row0 + r) * ATTN_PARTIAL_FLOATS;
      *reinterpret_cast<float4*>(rec + lane * 4) = o;
      if (lane == 0) { rec[128] = top; rec[129] = sum; }
    }
  }
  if (a.splits == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    int arrived;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(arrived) : "l"(a.counters + (long long)z * v.S + s) : "memory");
    *flag = arrived == a.splits - 1 ? 1 : 0;
  }
  __syncthreads();
  if (*flag == 0) return;
  __threadfence();
  for (int r = warp; r < n_rows; r += QA_WARPS) {
    const float* rec = a.partials + ((long long)s * a.splits * R + row0 + r) * ATTN_PARTIAL_FLOATS;
    const long long stride = (long long)R * ATTN_PARTIAL_FLOATS;
    float top = -INFINITY, sum = 0.f;
    for (int p = lane; p < a.splits; p += 32) top = fmaxf(top, __ldcg(rec + p * stride + 128));
    top = warp_max(top);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int p = 0; p < a.splits; ++p) {
      const float m = __ldcg(rec + p * stride + 128), lp = __ldcg(rec + p * stride + 129);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(rec + p * stride + lane * 4));
      const float f = m == -INFINITY ? 0.f : exp2f(m - top);
      sum = fmaf(lp, f, sum);
      o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
    }
    finish(row0 + r, o, top, sum);
  }
  if (threadIdx.x == 0) a.counters[(long long)z * v.S + s] = 0;      // clean for the next launch
}

int q4_attn_row_groups(int rows) { return rows <= 16 ? 1 : (rows + 31) / 32; }

cudaError_t launch_attn_q4(const LayerView& v, const Q4Pages& p, bool dense, int T, int G, bool causal, int splits, const void* q, void* out, float* lse,
                           float scale, float* partials, int32_t* counters, cudaStream_t st) {
  Q4AttnArgs a;
  a.v = v; a.p = p;
  a.by_g = fast_div((uint32_t)G);
  a.by_tiles4 = fast_div((uint32_t)((v.C + QA_ROWS4 - 1) / QA_ROWS4));
  a.by_tiles16 = fast_div((uint32_t)(v.C / QA_ROWS16));
  a.dense = dense ? 1 : 0; a.T = T; a.G = G; a.causal = causal ? 1 : 0; a.splits = splits;
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse = lse; a.scale = scale;
  a.partials = partials; a.counters = counters;
  const int R = T * G;
  const dim3 grid((unsigned)splits, (unsigned)v.S, (unsigned)q4_attn_row_groups(R));
  auto launch = [&](auto kernel, DeviceFlags& opted, int smem) {
    const cudaError_t e = smem_opt_in(opted, kernel, smem);
    return e != cudaSuccess ? e : launch_pdl(kernel, grid, dim3(QA_WARPS * 32), (size_t)smem, st, a);
  };
  static DeviceFlags f4, f8, f16, f32;
  if (R <= 4) return launch(kve_decode_attn_q4_kernel<1, true>, f4, QaShape<1>::SMEM);
  if (R <= 8) return launch(kve_decode_attn_q4_kernel<1, false>, f8, QaShape<1>::SMEM);
  if (R <= 16) return launch(kve_decode_attn_q4_kernel<2, false>, f16, QaShape<2>::SMEM);
  return launch(kve_decode_attn_q4_kernel<4, false>, f32, QaShape<4>::SMEM);
}

}  // namespace kve
