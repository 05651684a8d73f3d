// Attention of a tree of drafted tokens over the paged, un-rotated context (see mepic_attn_tree in mepic.h).
//
// Mathematics.  An item is (request, kv head, tile of 128 / G drafted rows): its 128 query vectors (rows x the G query
// heads of the kv head) against the request's keys, first the context's slots, then the request's drafted rows under the
// mask.  Keys are taken 128 at a time: S = Q' K'^T, P = 2^(S - reference), O += P V, with Q' = R(row_pos) q * sm_scale *
// log2(e) and K' = R(pos) k, a reference per row that only moves when a score lies more than 2^8 above it, and the sum of
// P in fp32.  Q', K' and P are rounded to bf16 once each, because the MMA takes both operands in one 16-bit type and the pages'
// V is bf16: fp16 would keep three bits more of them, but it ends at 65504, which bf16 pages may pass.  Everything else is fp32,
// the sum of P too, which takes the weights as they are before their rounding.
//
// What bounds it.  One key tile is 512 D bytes of K and V and 4 * 128 * 128 * D operations: with up to 128 query vectors an
// item is bound by HBM (a tile's bytes take an SM's share of the bandwidth 1.5 us, its MMAs 0.6), beyond that items share
// their tiles through L2 and the softmax (16 exponentials a clock) and the MMAs come level.  So one kernel shape serves all
// sizes: a persistent CTA per SM that never lets the loads stop, and one 128-row MMA tile however few rows are live.
//
// Split.  The key tiles of all items lie on a line per LEVEL (level m = the m-th row tile of every request that has one);
// the CTAs are dealt to the levels in proportion to their lines and each level's line is cut into equal pieces, one per CTA.
// A request whose rows fill several tiles is thus read by CTAs that walk its keys side by side, which is what lets L2 serve
// the second reader; a batch with one wide tree in it does not leave the other CTAs idle.  An item that a cut divides leaves
// partials (reference, sum, unnormalised O), at most two per CTA, and a second kernel merges them.  Every CTA derives the
// cut from row_offsets and kv_len, so no plan is built or uploaded and a captured call may be replayed with other lengths.
//
// Roles (640 threads, one CTA per SM):
//   softmax warps : a thread per row, two warpgroups (even and odd key tiles).  Loads, rotates and stages the row's q; then per key tile the
//                   row's 128 scores come to registers: maximum, 2^(S - reference), and back as bf16 over the scores' columns,
//                   where the PV MMA takes P from.
//   rotator warps : rotate the K tile in place in shared memory, fp32 arithmetic, one rounding.  They also bring the drafted
//                   K rows (plain loads: one tile per item, at positions of their own).
//   loader warps  : one for K, one for V; TMA boxes of 16 rows x 64 dims (128-byte swizzle) per 16-slot group, the next
//                   tile's page ids fetched while the ring is full.  The V loader also clears V rows past kv_len,
//                   brings the drafted V rows and takes non-finite elements out of them: 0 x inf would reach rows that the
//                   mask hides them from.  The rows that do see such an element get it added in the epilogue.
//                   Over 8-bit pages the loaders bring the codes into rings of their own (untiled bulk copies); the rotators
//                   widen K on the way through the rotation, the softmax warps V; the K scales go into (cos, sin), the V scales
//                   into P.
//   MMA warps     : one issues S = Q' K'^T (three score buffers, each of which becomes its tile's P), one O += P V.
// Every wait is bounded; a lost wait raises a flag that ends every role.  However a role ends, the loaders and the issuers first
// wait (bounded) for what they have started.
//
// Measured (G = 4, D = 128, 8 kv heads, pages of 16).  32 requests x 16 rows over 8,256 slots: 209 us in a burst of calls, 230
// to 243 in a run of them (the GPU is at its power limit then, and its clock at 1.66 to 1.76 GHz), of it 6 the merge; 986 MB of
// DRAM traffic, 55 % of the bandwidth; the tensor pipe is active 30 % of the time, the exponential unit 14, issue slots 40.
// 8 x 96 rows over 16,640: 295 us in a burst, 314 to 324 in a run (146 GFLOP, 450 TFLOP/s).  8 x 32 rows over 65,536 slots of
// 8-bit pages: 432 and 448 to 464 us.  One request of 8 rows over 203 slots: 12.3 us, two launches.  A pass (row tile x key
// tile) takes 2.3 to 2.4 us in all three large ones, whatever its rows, bytes and type: what bounds them is none of the units but
// the hand-over of a tile from role to role (load, rotate, QK^T, softmax, PV: each waits for latency, and for instructions, which
// twenty warps with five programs fetch through one cache).  Warp instructions per pass: 5,400, with full row tiles 6,400, over
// 8-bit pages 9,000 (issue slots 57 %).
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "mepic.h"
#include "mepic_internal.h"
#include "mepic_ptx.cuh"
#include "mepic_rows.cuh"
#include "mepic_tcgen05.cuh"

namespace {

using namespace mepic_dev;

constexpr int kTileN = 128;                 // keys per tile
constexpr int kBlockBytes = 128 * 128;      // one [128 rows x 64 bf16] swizzled block
constexpr int kSoftmaxWarps = 8;             // two warpgroups: one takes the even key tiles, one the odd ones
constexpr int kRotatorWarp0 = 8, kRotatorWarps = 8;                  // two groups of four, again even and odd tiles
constexpr int kRotGroupWarps = 4, kRotators = kRotGroupWarps * 32;   // ... threads that share a tile
constexpr int kKLoaderWarp = 16, kVLoaderWarp = 17, kQkWarp = 18, kPvWarp = 19;
constexpr int kThreads = 640;
constexpr int kTmemCols = 512;              // the scores of three tiles at 0, 128, 256 (each becomes its P), O at 384
constexpr int kSD = 3;                      // score buffers
constexpr uint32_t kColO = 384;
constexpr float kRescaleThreshold = 8.f;    // move a row's reference only when a score lies more than 2^8 above it
constexpr int kMaxLevels = MEPIC_TREE_MAX_ROWS / 16;      // 128 / G >= 16 rows per tile
constexpr int kSlots = 2;                   // partials a CTA may leave: of the item its piece starts in the middle of, and of the one it ends in

struct TreeParams {
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  const int32_t* row_offsets;
  const int32_t* row_pos;
  const int32_t* tree_mask;
  const void* k_pool;
  const void* v_pool;
  const float* k_scales;       // 8-bit pools only
  const float* v_scales;
  const int32_t* page_ids;
  const int32_t* pos_base;
  const int32_t* kv_len;
  const float* rope;
  uint16_t* out;
  int32_t* status;
  int4* desc;                  // [CTAs] what the merge of the item this CTA begins is (row, rows, kv head, parts; 0 parts: nothing)
  float2* part_ml;             // [CTAs][kSlots][128] (reference, sum)
  float* part_o;               // [CTAs][kSlots][128][D]
  int table_stride, batch, total_rows, max_rows, mask_words, q_stride, kv_stride;
  int n_kv_heads, group, page_size, page_shift, num_pages, max_position;
  int rows_per_tile, max_levels;
  float scale_log2;
  int spin_limit, skip_tile;   // test hooks
};

#define TMEM_LD16(taddr, r)                                                                                          \
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" \
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),      \
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) \
               : "r"(taddr) : "memory")

#define TMEM_ST8(taddr, r)                                                                                           \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"                               \
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory")

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// ---------------------------------------------------------------- the cut
// What a request contributes: its rows, its key tiles, the row tiles (levels) it has.
struct Request { int row0, n, kvl, n_ctx, n_all, levels; bool bad_rows, bad_len; };
__device__ __forceinline__ Request request_of(const TreeParams& p, int b) {
  Request r;
  const RowRange rr = rows_of(p.row_offsets, b, p.total_rows, p.max_rows);
  r.row0 = rr.lo; r.n = rr.n; r.bad_rows = rr.bad;
  const int len = __ldg(p.kv_len + b);
  const long long room = static_cast<long long>(p.table_stride) << p.page_shift;
  r.kvl = len < 0 ? 0 : (len > room ? static_cast<int>(room) : len);
  r.bad_len = r.kvl != len;
  r.n_ctx = static_cast<int>((static_cast<long long>(r.kvl) + kTileN - 1) / kTileN);
  r.n_all = r.n_ctx + (r.n + kTileN - 1) / kTileN;
  r.levels = (r.n + p.rows_per_tile - 1) / p.rows_per_tile;
  return r;
}

// One CTA's piece: tiles [lo, hi) of its level's line, which has `line` tiles in `pieces` pieces; it starts at key tile t of
// (request b, kv head h).
struct Piece { int level, piece, pieces, b, h, t; long long lo, hi, line; Request r; };
struct PlanScratch {
  unsigned long long hist[kMaxLevels];
  long long warp_sum[kThreads / 32];
};
__device__ __forceinline__ long long mul_div(long long a, int b, long long c) {      // a b / c, b <= 2^11
  if (a < (1 << 20) && c < (1ll << 31)) return static_cast<uint32_t>(a) * static_cast<uint32_t>(b) / static_cast<uint32_t>(c);
  return a / c * b + a % c * b / c;
}
__device__ __forceinline__ long long cut_at(long long line, int pieces, int k) { return mul_div(line, k, pieces); }
// Executed by the whole CTA.
__device__ __noinline__ void plan_piece(const TreeParams& p, PlanScratch* sh, Piece* out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < kMaxLevels; i += kThreads) sh->hist[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int b = tid; b < p.batch; b += kThreads) {
    const Request r = request_of(p, b);
    if (blockIdx.x == 0) {
      if (r.bad_rows) atomicOr(p.status, MEPIC_DEV_BAD_TREE);
      if (r.bad_len) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
    }
    if (r.levels > 0) atomicAdd(&sh->hist[r.levels - 1], static_cast<unsigned long long>(r.n_all) * p.n_kv_heads);
  }
  __syncthreads();
  if (tid == 0) {
    long long all = 0, line = 0;
    int used = 0;
#pragma unroll 1
    for (int m = p.max_levels - 1; m >= 0; --m) {
      line += static_cast<long long>(sh->hist[m]);
      sh->hist[m] = static_cast<unsigned long long>(line);       // now the length of level m's line
      all += line;
      used += line > 0;
    }
    Piece c{-1, 0, 0, 0, 0, 0, 0, 0, 0, {}};
    int cta = blockIdx.x;
    const long long spare = static_cast<long long>(gridDim.x) - used;      // every level has one CTA, the rest go by length
#pragma unroll 1
    for (int m = 0; m < used; ++m) {
      const long long len = static_cast<long long>(sh->hist[m]);
      long long n = 1 + mul_div(len, static_cast<int>(spare), all);
      n = n < len ? n : len;                                     // no empty pieces
      if (cta < n) {
        c.level = m; c.piece = cta; c.pieces = static_cast<int>(n); c.line = len;
        c.lo = cut_at(len, c.pieces, c.piece); c.hi = cut_at(len, c.pieces, c.piece + 1);
        break;
      }
      cta -= static_cast<int>(n);
    }
    *out = c;
  }
  __syncthreads();
  const int level = (*out).level;
  const long long lo = (*out).lo;
  if (level < 0) return;
  long long before = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    const int b = b0 + tid;
    long long w = 0;
    int n_all = 1;
    if (b < p.batch) {
      const Request r = request_of(p, b);
      n_all = r.n_all;
      if (r.levels > level) w = static_cast<long long>(r.n_all) * p.n_kv_heads;
    }
    long long incl = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long up = __shfl_up_sync(kFull, incl, d);
      if (lane >= d) incl += up;
    }
    if (lane == 31) sh->warp_sum[warp] = incl;
    __syncthreads();
    long long at = before + incl - w, chunk = 0;
#pragma unroll
    for (int k = 0; k < kThreads / 32; ++k) {
      if (k < warp) at += sh->warp_sum[k];
      chunk += sh->warp_sum[k];
    }
    if (at <= lo && lo < at + w) {
      const long long off = lo - at;
      const Request r = request_of(p, b);
      out->r = r;
      out->b = b;
      out->h = off < (1ll << 31) ? static_cast<uint32_t>(off) / static_cast<uint32_t>(n_all) : static_cast<int>(off / n_all);
      out->t = static_cast<int>(off - static_cast<long long>(out->h) * n_all);
    }
    before += chunk;
    __syncthreads();
    if (before > lo) break;
  }
  __syncthreads();
}

// The same by one warp, a request per lane, for up to 32 requests: no barrier of the CTA on the way.
__device__ __forceinline__ long long warp_sum64(long long v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
  return v;
}
__device__ __forceinline__ void plan_by_warp(const TreeParams& p, Piece* out, int lane) {
  Request r{0, 0, 0, 0, 0, 0, false, false};
  if (lane < p.batch) {
    r = request_of(p, lane);
    if (blockIdx.x == 0) {
      if (r.bad_rows) atomicOr(p.status, MEPIC_DEV_BAD_TREE);
      if (r.bad_len) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
    }
  }
  const long long w = r.levels > 0 ? static_cast<long long>(r.n_all) * p.n_kv_heads : 0;
  const long long all = warp_sum64(w * r.levels);
  const int used = __reduce_max_sync(kFull, r.levels), spare = static_cast<int>(gridDim.x) - used;
  int cta = blockIdx.x, level = -1, n = 0;
  long long len = 0;
#pragma unroll 1
  for (int m = 0; m < used; ++m) {
    len = warp_sum64(r.levels > m ? w : 0);
    const long long share = 1 + mul_div(len, spare, all);
    n = static_cast<int>(share < len ? share : len);
    if (cta < n) { level = m; break; }
    cta -= n;
  }
  if (lane == 0) out->level = level;
  if (level < 0) return;
  const long long lo = cut_at(len, n, cta), mine = r.levels > level ? w : 0;
  long long at = mine;                           // inclusive sum, then this request's first place on the line
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long up = __shfl_up_sync(kFull, at, d);
    if (lane >= d) at += up;
  }
  at -= mine;
  if (at <= lo && lo < at + mine) {              // one lane
    out->piece = cta; out->pieces = n; out->line = len; out->lo = lo; out->hi = cut_at(len, n, cta + 1);
    const long long off = lo - at;
    out->b = lane; out->r = r;
    out->h = off < (1ll << 31) ? static_cast<uint32_t>(off) / static_cast<uint32_t>(r.n_all) : static_cast<int>(off / r.n_all);
    out->t = static_cast<int>(off - static_cast<long long>(out->h) * r.n_all);
  }
}

// The segments of a piece, one per item it touches, in order.  The K loader walks them and publishes each to the other roles.
struct Walk {
  Request r;
  long long left;
  int b, h, t, level;
};
// Key tiles t0 .. t1 - 1 of item (request b, kv head h); the request's first row, rows, length, context tiles, all tiles.
// t1 = 0: there are no more.
struct Segment { int t0, t1, b, h, row0, n, kvl, n_ctx, n_all; };
__device__ __forceinline__ Walk walk_of(const Piece& c) {
  Walk w;
  w.level = c.level; w.left = c.hi - c.lo; w.b = c.b; w.h = c.h; w.t = c.t; w.r = c.r;
  return w;
}
__device__ __forceinline__ Segment next_segment(const TreeParams& p, Walk& w) {
  Segment s{0, 0, 0, 0, 0, 0, 0, 0, 0};
  if (w.left <= 0) return s;
  if (w.t >= w.r.n_all) {
    w.t = 0;
    if (++w.h >= p.n_kv_heads) {
      w.h = 0;
#pragma unroll 1
      do {
        if (++w.b >= p.batch) { w.left = 0; return s; }          // not reached: `left` ends first
        w.r = request_of(p, w.b);
      } while (w.r.levels <= w.level);
    }
  }
  const int n = static_cast<int>(w.left < w.r.n_all - w.t ? w.left : w.r.n_all - w.t);
  s.t0 = w.t; s.t1 = w.t + n;
  s.b = w.b; s.h = w.h; s.row0 = w.r.row0; s.n = w.r.n; s.kvl = w.r.kvl; s.n_ctx = w.r.n_ctx; s.n_all = w.r.n_all;
  w.t += n; w.left -= n;
  return s;
}

// ---------------------------------------------------------------- attention
// 8-bit pages: the K loader publishes the scales of a tile's blocks beside its K codes.  When it gets to tile i the rotators
// are through with the K codes of i - 2; that tile's K stage was free, so QK^T of i - 4 was complete, so PV of i - 7 was, so
// the softmax was through with tile i - 8.
constexpr int kScaleRing = 8;
constexpr int kSegRing = 3;            // segments published and not yet read by everybody
template <bool FP8>
struct Small {
  float ks[FP8 ? 2 : 1][8], vs[FP8 ? kScaleRing : 1][8];
  union {
    PlanScratch plan;                  // before the roles begin
    float ref[2][128];                 // [warpgroup][row] the row's reference after that warpgroup's latest tile
  };
  float sum[2][128];                   // [warpgroup][row] its sum at an item's end
  Piece piece;
  Segment seg[kSegRing];
  uint32_t tmem;
  int abort_flag;
  int odd_v;                           // a drafted V row of this CTA's holds a non-finite element
};
template <int D, bool FP8>
struct TreeSmem {
  static constexpr int NB = D / 64;
  static constexpr int kStage = NB * kBlockBytes;
  static constexpr int KD = FP8 ? 2 : 3, VD = FP8 ? 2 : 3;       // stages of bf16 K and V tiles
  static constexpr int CD = 2;                                   // 8-bit pages: stages of K and of V codes
  static constexpr int kCodes = kTileN * D;
  static constexpr int kQ = 0;                                   // Q' of the item, as the QK^T MMA reads it
  static constexpr int kK = kQ + kStage;
  static constexpr int kV = kK + KD * kStage;
  static constexpr int kC = kV + VD * kStage;
  static constexpr int kBars = kC + (FP8 ? 2 * CD * kCodes : 0);
  static constexpr int kSmall = kBars + 472;                     // Small
  static constexpr int kBytes = kSmall + sizeof(Small<FP8>);
};
static_assert(TreeSmem<128, false>::kBytes <= 232448 && TreeSmem<128, true>::kBytes <= 232448, "shared memory of an SM");

// barriers
// A wait names a phase by its parity only, so a waiter must have seen the phase before complete.  Roles that take every second
// tile have not, where the phase before belongs to the other group: those barriers come one per tile modulo 6, an even number.
constexpr int kBarKLanded = 0, kBarSFull = 6;                          // [tile % 6]
constexpr int kBarKReady = 12, kBarKFree = 15;                         // [stage]
constexpr int kBarVLanded = 18, kBarVReady = 21, kBarVFree = 24;
constexpr int kBarCFree = 27;                                          // 8-bit pages: [K codes 0, 1, V codes 0, 1]
constexpr int kBarPFull = 31, kBarPvDone = 34;                         // [score buffer]
constexpr int kBarQReady = 37, kBarOFree = 38;
constexpr int kBarRef = 39, kBarItem = 47;                             // [warpgroup * 4 + warp], [warp]
constexpr int kBarDrain = 51;                                          // [QK, PV] at the role's end: its MMAs are done
constexpr int kBarSegFull = 53, kBarSegFree = 56;                      // [segment % 3]
constexpr int kNumBars = 59;
static_assert(kNumBars * 8 <= 472, "barrier block");

// Rotates, scales and rounds the q rows of an item's tile into the staged tile: a thread takes a 16-byte piece and its partner
// in the other half of a row at a time, neighbours in one row (a thread per row left 32 cache lines per load: 5,000 cycles).
// Rows without a drafted row are zeros up to the next multiple of 32 and stay as they are beyond: only their own scores
// come of it.
template <int D>
__device__ __noinline__ void stage_q(const TreeParams& p, unsigned char* Qs, int first, int n_rows, int head0, int tid) {
  constexpr int CH = D / 16;
  const int G = p.group, live = n_rows * G;
#pragma unroll 2
  for (int idx = tid; idx < ((live + 31) & ~31) * CH; idx += kSoftmaxWarps * 32) {
    const int r = idx / CH, c = idx % CH, lc = c, hc = CH + c;
    uint32_t lo_w[4] = {0, 0, 0, 0}, hi_w[4] = {0, 0, 0, 0};
    if (r < live) {
      const int row = first + r / G;
      int pos = __ldg(p.row_pos + row);
      if (pos < 0 || pos > p.max_position) { atomicOr(p.status, MEPIC_DEV_BAD_POSITION); pos = pos < 0 ? 0 : p.max_position; }
      const uint16_t* src = p.q + static_cast<size_t>(row) * p.q_stride + static_cast<size_t>(head0 + r % G) * D + 8 * c;
      const float4* cs = reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(pos) * D + 16 * c);
      const uint4 lo = *reinterpret_cast<const uint4*>(src), hi = *reinterpret_cast<const uint4*>(src + D / 2);
      const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 t = __ldg(cs + j);                      // (cos, sin) of pairs 8c + 2j and 8c + 2j + 1
        const float2 x = bf16x2_to_float2(lw[j]), y = bf16x2_to_float2(hw[j]);
        lo_w[j] = pack_bf16x2((x.x * t.x - y.x * t.y) * p.scale_log2, (x.y * t.z - y.y * t.w) * p.scale_log2);
        hi_w[j] = pack_bf16x2((x.x * t.y + y.x * t.x) * p.scale_log2, (x.y * t.w + y.y * t.z) * p.scale_log2);
      }
    }
    *reinterpret_cast<uint4*>(Qs + (lc / 8) * kBlockBytes + sw128(r, lc % 8)) = make_uint4(lo_w[0], lo_w[1], lo_w[2], lo_w[3]);
    *reinterpret_cast<uint4*>(Qs + (hc / 8) * kBlockBytes + sw128(r, hc % 8)) = make_uint4(hi_w[0], hi_w[1], hi_w[2], hi_w[3]);
  }
}

// V of a tile that does not end with its last key, and of drafted rows (whose stage no copy fills): zeros up to the next
// multiple of 16 keys, which is how far the PV product goes (P is 0 there, but 0 x NaN is NaN), and the drafted rows without
// their non-finite elements.  Eight 16-byte pieces per thread, `step` apart.
template <int D>
__device__ __noinline__ void mend_rows(const TreeParams& p, unsigned char* Vb, int* odd_v, bool draft, int left, int row, int h, int at, int step) {
  constexpr int CH = D / 16, B = 8;
  const int end = (left + 15) & ~15;
  uint4 v[B];
#pragma unroll
  for (int u = 0; u < B; ++u) {
    const int idx = at + u * step, kk = idx / (2 * CH), ch = idx % (2 * CH);
    v[u] = make_uint4(0, 0, 0, 0);
    if (draft && kk < left) v[u] = *reinterpret_cast<const uint4*>(p.v_new + static_cast<size_t>(row + kk) * p.kv_stride + static_cast<size_t>(h) * D + 8 * ch);
  }
#pragma unroll
  for (int u = 0; u < B; ++u) {
    const int idx = at + u * step, kk = idx / (2 * CH), ch = idx % (2 * CH);
    if (kk >= end) break;
    uint32_t vw[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if ((vw[j] & 0x7f80u) == 0x7f80u) { vw[j] &= 0xffff0000u; odd = true; }
      if ((vw[j] & 0x7f800000u) == 0x7f800000u) { vw[j] &= 0x0000ffffu; odd = true; }
    }
    if (odd) *reinterpret_cast<volatile int*>(odd_v) = 1;
    *reinterpret_cast<uint4*>(Vb + (ch / 8) * kBlockBytes + sw128(kk, ch % 8)) = make_uint4(vw[0], vw[1], vw[2], vw[3]);
  }
}

template <int D, bool FP8, bool HOOKS>
__global__ void __launch_bounds__(kThreads, 1)
mepic_tree_attn(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using L = TreeSmem<D, FP8>;
  constexpr int NB = L::NB, KD = L::KD, VD = L::VD, CD = L::CD;
  constexpr int CH = D / 16;                      // (lo, hi) chunk pairs per row: chunk c pairs dims [8c, 8c+8) with [D/2+8c, ...)
  constexpr int KPT = kTileN * CH / kRotators;    // consecutive keys a rotator thread takes
  constexpr uint32_t kIdescQK = instr_desc(128, kTileN, 0, 0);
  constexpr uint32_t kIdescPV = instr_desc(128, D, 0, 1);
  constexpr uint32_t kGroupBytes = 16u * D * (FP8 ? 1u : 2u);

  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* Qs = smem + L::kQ;
  unsigned char* Ks = smem + L::kK;
  unsigned char* Vs = smem + L::kV;
  unsigned char* Kc = smem + L::kC;
  unsigned char* Vc = Kc + CD * L::kCodes;
  const uint32_t bar0 = smem_u32(smem + L::kBars);
  auto BAR = [&](int which, int slot = 0) { return bar0 + static_cast<uint32_t>((which + slot) * 8); };
  Small<FP8>* sm = reinterpret_cast<Small<FP8>*>(smem + L::kSmall);
  volatile int* abort_flag = &sm->abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int spin = HOOKS ? p.spin_limit : kSpinLimit;

  if ((smem_u32(smem) & 1023u) != 0) {            // cannot happen with the alignment requested above; never run misaligned
    if (tid == 0) atomicOr(p.status, MEPIC_DEV_WAIT_EXPIRED);
    return;
  }
  if (tid == 0) {
    for (int s = 0; s < 3; ++s) {
      mbar_init(BAR(kBarKReady, s), kRotGroupWarps); mbar_init(BAR(kBarKFree, s), 1);
      mbar_init(BAR(kBarVLanded, s), 1); mbar_init(BAR(kBarVReady, s), FP8 ? 4 : 1); mbar_init(BAR(kBarVFree, s), 1);
      mbar_init(BAR(kBarPFull, s), 4); mbar_init(BAR(kBarPvDone, s), 1);
    }
    for (int s = 0; s < 4; ++s) mbar_init(BAR(kBarCFree, s), kRotGroupWarps);
    for (int s = 0; s < 6; ++s) { mbar_init(BAR(kBarKLanded, s), 1); mbar_init(BAR(kBarSFull, s), 1); }
    for (int s = 0; s < 8; ++s) mbar_init(BAR(kBarRef, s), 1);
    for (int s = 0; s < 4; ++s) mbar_init(BAR(kBarItem, s), 2);
    for (int s = 0; s < kSegRing; ++s) { mbar_init(BAR(kBarSegFull, s), 1); mbar_init(BAR(kBarSegFree, s), kThreads / 32 - 1); }
    mbar_init(BAR(kBarQReady), kSoftmaxWarps); mbar_init(BAR(kBarOFree), kSoftmaxWarps); mbar_init(BAR(kBarDrain, 0), 1); mbar_init(BAR(kBarDrain, 1), 1);
    sm->abort_flag = 0;
    sm->odd_v = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == kPvWarp) tmem_alloc(smem_u32(&sm->tmem), kTmemCols);
  if (p.batch > 32) plan_piece(p, &sm->plan, &sm->piece);
  else if (warp == kKLoaderWarp) plan_by_warp(p, &sm->piece, lane);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the merge may become resident; it waits for this grid's end
  tc_fence_before();
  __syncthreads();                                // barriers initialised, tensor memory allocated, the piece known
  tc_fence_after();
  const uint32_t tmem = sm->tmem;
  const Piece& piece = sm->piece;
  const int G = p.group, n_q_heads = p.n_kv_heads * G;
  const bool has_work = piece.level >= 0;
  if (!has_work && tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);

  // A wait of a whole warp; false ends the role.
  auto wait_warp = [&](uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (int i = 0; i < spin; ++i) {
      if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
      if ((i & 255) == 255 && *abort_flag) return false;
    }
    *abort_flag = 1;
    atomicOr(p.status, MEPIC_DEV_WAIT_EXPIRED);
    return false;
  };

  // The k-th segment, for a role other than the K loader; false ends the role (no more segments, or a lost wait).
  auto take_segment = [&](int k, Segment& s) {
    const int at = k % kSegRing;
    if (!wait_warp(BAR(kBarSegFull, at), static_cast<uint32_t>(k / kSegRing) & 1u)) { s.t1 = -1; return false; }
    const volatile Segment* v = &sm->seg[at];
    s.t0 = v->t0; s.t1 = v->t1; s.b = v->b; s.h = v->h; s.row0 = v->row0; s.n = v->n; s.kvl = v->kvl; s.n_ctx = v->n_ctx; s.n_all = v->n_all;
    __syncwarp();
    if (lane == 0) mbar_arrive(BAR(kBarSegFree, at));
    return s.t1 > 0;
  };
  const int level = piece.level;

  if (has_work && warp < kSoftmaxWarps) {
    // =============================================================== softmax warps: thread = row (lane of tensor memory)
    // Warpgroup wg takes the key tiles of parity wg, so that one's exponentials run while the other waits for scores or
    // barriers.  Both accumulate into one O and so must agree on a row's reference: it is handed from tile to tile (from the
    // thread of a row to its twin in the other warpgroup), as soon as a tile's maximum is known.
    const int wg = warp >> 2, wq = warp & 3, r = tid & 127;      // row of the tile: drafted row r / G, query head r % G of the kv head
    const uint32_t t_row = tmem + (static_cast<uint32_t>(wq * 32) << 16);
    const int row_in_tile = r / G, g = r % G;
    Segment seg;
    int n_seg = 0;
    bool more = take_segment(n_seg++, seg);
    auto put_q = [&](const Segment& a) {
      const int at = level * p.rows_per_tile;
      stage_q<D>(p, Qs, a.row0 + at, min(p.rows_per_tile, a.n - at), a.h * G, tid);
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(kBarQReady));
    };
    // 8-bit pages: key tile t of segment a, this CTA's tile i, from V codes to the bf16 stage the PV product reads (their scale
    // goes into P).  A warpgroup widens the V of the tile after its own, which the other warpgroup is at: the V stage is free
    // by then, and the rotators, who have K, are the busier role.  (K and V by the rotators: 520 us on 8 x 65,536 slots.)
    auto widen_v = [&](int i, int t, const Segment& a) {
      const int rt = tid & 127, st = i % VD;
      unsigned char* Vb = Vs + st * L::kStage;
      if (!wait_warp(BAR(kBarVLanded, i % CD), static_cast<uint32_t>(i / CD) & 1u)) return false;
      if (i >= VD && !wait_warp(BAR(kBarVFree, st), static_cast<uint32_t>(i / VD - 1) & 1u)) return false;
      const bool draft = t >= a.n_ctx;
      const int left = min(draft ? a.n - (t - a.n_ctx) * kTileN : a.kvl - t * kTileN, kTileN);
      const int end = (left + 15) & ~15;           // the PV product goes over whole groups of 16 keys
      if (draft) {
#pragma unroll 1
        for (int i0 = rt & ~31; i0 < end * 2 * CH; i0 += 128 * 8)
          mend_rows<D>(p, Vb, &sm->odd_v, true, left, a.row0 + (t - a.n_ctx) * kTileN, a.h, i0 + lane, 128);
      } else {
        const unsigned char* codes = Vc + (i % CD) * L::kCodes;
#pragma unroll 1
        for (int idx = rt; idx < end * 8; idx += 128) {
          const int kk = idx >> 3, ch = 2 * (idx & 7);
          uint32_t w8[8] = {0, 0, 0, 0, 0, 0, 0, 0};
          if (kk < left) {
            const uint4 cd = *reinterpret_cast<const uint4*>(codes + kk * 128 + 8 * ch);
            const uint32_t cw[4] = {cd.x, cd.y, cd.z, cd.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t f0, f1;
              e4m3x4_to_f16x2x2(cw[j], f0, f1);
              const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&f0)), y = __half22float2(*reinterpret_cast<const __half2*>(&f1));
              w8[2 * j] = pack_bf16x2(x.x, x.y);
              w8[2 * j + 1] = pack_bf16x2(y.x, y.y);
            }
          }
          *reinterpret_cast<uint4*>(Vb + (ch / 8) * kBlockBytes + sw128(kk, ch % 8)) = make_uint4(w8[0], w8[1], w8[2], w8[3]);
          *reinterpret_cast<uint4*>(Vb + (ch / 8) * kBlockBytes + sw128(kk, ch % 8 + 1)) = make_uint4(w8[4], w8[5], w8[6], w8[7]);
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(BAR(kBarVReady, st));
        mbar_arrive(BAR(kBarCFree, 2 + i % CD));
      }
      return true;
    };
    if (more) put_q(seg);
    int gi = 0, item = 0;                         // key tiles and items of this CTA so far
    bool ok = true, begun = false;
    if (FP8 && more && wg == 1) ok = widen_v(0, seg.t0, seg);
    while (more && ok) {
      const int n = seg.n, n_ctx = seg.n_ctx, n_all = seg.n_all, kvl = seg.kvl, h = seg.h, row0 = seg.row0;
      const int at = level * p.rows_per_tile + row_in_tile;            // this thread's drafted row within the request
      const bool live = row_in_tile < p.rows_per_tile && at < n;
      const bool warp_live = level * p.rows_per_tile + (wq * 32) / G < n;
      const int t0 = seg.t0, t1 = seg.t1;
      float m_ref = -INFINITY, l_run = 0.f;       // reference at this warpgroup's latest tile, and its sum under it
#pragma unroll 1
      for (int t = t0; t < t1; ++t, ++gi) {
        if ((gi & 1) != wg) continue;
        const int sb = gi % kSD;
        const uint32_t t_S = t_row + static_cast<uint32_t>(sb * 128);
        // which of the tile's keys this row sees, where that is not all of them: bit c of word q = key 32 q + c
        const int left = t < n_ctx ? kvl - t * kTileN : n - (t - n_ctx) * kTileN;        // keys that exist
        const bool masked = t >= n_ctx || left < kTileN;
        uint32_t vis[4] = {~0u, ~0u, ~0u, ~0u};
        if (masked && warp_live) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t m = left >= 32 * (q + 1) ? ~0u : (left <= 32 * q ? 0u : (1u << (left - 32 * q)) - 1u);
            if (t >= n_ctx) {
              const int wd = (t - n_ctx) * 4 + q;
              m &= live && wd < p.mask_words ? static_cast<uint32_t>(__ldg(p.tree_mask + static_cast<size_t>(row0 + at) * p.mask_words + wd)) : 0u;
            }
            vis[q] = m;
          }
        }
        if (!wait_warp(BAR(kBarSFull, gi % 6), static_cast<uint32_t>(gi / 6) & 1u)) { ok = false; break; }
        tc_fence_after();
        if (warp_live) {
          // (Short loop bodies, here and in the other roles: the roles that share a scheduler run different code, and what they
          // wait for first is instructions.  A row's scores held in registers, chunks fetched ahead of their use, unrolled
          // rotations: each saved latency on paper and lost time.)
          if (masked) {
            // hidden scores become -inf where they are, so that the passes below need not know
#pragma unroll 1
            for (int q = 0; q < 8; ++q) {
              uint32_t sv[16];
              TMEM_LD16(t_S + 16 * q, sv);
              const uint32_t m = (q < 4 ? (q < 2 ? vis[0] : vis[1]) : (q < 6 ? vis[2] : vis[3])) >> (16 * (q & 1));
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 16; ++c) sv[c] = (m >> c) & 1u ? sv[c] : 0xff800000u;
              TMEM_ST16(t_S + 16 * q, sv);
            }
            tmem_wait_st();
          }
          // ---- pass 1: the maximum of the row's 128 scores
          float mx = -INFINITY;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            uint32_t sv[32];
            TMEM_LD32(t_S + 32 * q, sv, 0);
            tmem_wait_ld();
            float m4[4] = {mx, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) m4[k] = max3(m4[k], __uint_as_float(sv[c + 2 * k]), __uint_as_float(sv[c + 2 * k + 1]));
            }
            mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          }
          // ---- the reference: the one the tile before left, raised to this tile's maximum if that lies more than 2^8 above
          float m_in = -INFINITY;
          if (t > t0) {
            if (!wait_warp(BAR(kBarRef, (wg ^ 1) * 4 + wq), static_cast<uint32_t>((gi - 1) >> 1) & 1u)) { ok = false; break; }
            m_in = *reinterpret_cast<volatile float*>(&sm->ref[wg ^ 1][r]);
          }
          const float m_now = mx > m_in + kRescaleThreshold ? mx : m_in;      // always mx on the first tile that shows the row a key
          *reinterpret_cast<volatile float*>(&sm->ref[wg][r]) = m_now;
          __syncwarp();
          if (lane == 0) mbar_arrive(BAR(kBarRef, wg * 4 + wq));
          if (t > t0 && __any_sync(kFull, m_now != m_in)) {
            // O holds the earlier tiles' PV: wait for the last of them, then scale the row.  (A barrier per score buffer: that
            // this tile's scores are here means that PV of three tiles ago has completed, so the parity names one phase.)
            if (!wait_warp(BAR(kBarPvDone, (gi - 1) % kSD), static_cast<uint32_t>((gi - 1) / kSD) & 1u)) { ok = false; break; }
            tc_fence_after();
            const float alpha = m_now != m_in ? ex2(m_in - m_now) : 1.f;      // 2^-inf = 0: nothing has been summed yet
#pragma unroll 1
            for (int cb = 0; cb < D; cb += 16) {
              uint32_t o[16];
              TMEM_LD16(t_row + kColO + cb, o);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
              TMEM_ST16(t_row + kColO + cb, o);
            }
          }
          if (m_now != m_ref) {                                    // this warpgroup's sum is still under its own latest reference
            l_run *= ex2(m_ref - m_now);                           // (0 x 0 before its first tile)
            m_ref = m_now;
          }
          // ---- pass 2: P = 2^(S - reference), bf16, over columns whose scores are consumed
          const float m_use = m_now == -INFINITY ? 0.f : m_now;    // a row that has seen nothing: every score is -inf, P = 0
          const float2 ref2 = make_float2(m_use, m_use);
          float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
          for (int q = 0; q < 8; ++q) {                            // keys 16 q .. 16 q + 15
            uint32_t sv[16], pw[8];
            TMEM_LD16(t_S + 16 * q, sv);
            const float s = FP8 ? sm->vs[gi % kScaleRing][q] : 1.f;              // the scale of the group's V block (1 for drafted rows)
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 16; c += 4) {
              const float2 d0 = sub2(make_float2(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), ref2);
              const float2 d1 = sub2(make_float2(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), ref2);
              float2 p0 = make_float2(ex2(d0.x), ex2(d0.y)), p1 = make_float2(ex2(d1.x), ex2(d1.y));
              sum2[0] = add2(sum2[0], p0);
              sum2[1] = add2(sum2[1], p1);
              if constexpr (FP8) { p0 = mul2(p0, make_float2(s, s)); p1 = mul2(p1, make_float2(s, s)); }
              pw[c / 2] = pack_bf16x2(p0.x, p0.y);
              pw[c / 2 + 1] = pack_bf16x2(p1.x, p1.y);
            }
            TMEM_ST8(t_S + 8 * q, pw);
          }
          l_run += (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          tmem_wait_st();
        } else if (lane == 0) {
          mbar_arrive(BAR(kBarRef, wg * 4 + wq));                  // no live row: only the phases are kept
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(kBarPFull, sb));
        if (FP8 && t + 1 < t1 && !widen_v(gi + 1, t + 1, seg)) { ok = false; break; }
      }
      if (!ok) break;
      // ---- the item's end: the twins exchange their sums
      const int last = gi - 1;                    // the item's last tile
      *reinterpret_cast<volatile float*>(&sm->ref[wg][r]) = m_ref;      // (what it holds, or -inf where this warpgroup had no tile)
      sm->sum[wg][r] = l_run;
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(kBarItem, wq));
      if (!wait_warp(BAR(kBarItem, wq), static_cast<uint32_t>(item) & 1u)) { ok = false; break; }
      const float m_twin = *reinterpret_cast<volatile float*>(&sm->ref[wg ^ 1][r]), l_twin = *reinterpret_cast<volatile float*>(&sm->sum[wg ^ 1][r]);
      // the next item's q is staged while this one's last PV runs; the staged q is free once the last QK^T has completed
      if (!wait_warp(BAR(kBarSFull, last % 6), static_cast<uint32_t>(last / 6) & 1u)) { ok = false; break; }
      more = take_segment(n_seg++, seg);
      if (seg.t1 < 0) { ok = false; break; }
      if (more) put_q(seg);
      if (FP8 && more && (last & 1) == wg && !widen_v(gi, seg.t0, seg)) { ok = false; break; }
      // (a reference only ever rises, so the larger of the two is the one O is under)
      const float m_end = fmaxf(m_ref, m_twin);
      const float l_end = (m_ref == m_end ? l_run : l_run * ex2(m_ref - m_end)) + (m_twin == m_end ? l_twin : l_twin * ex2(m_twin - m_end));
      if (!wait_warp(BAR(kBarPvDone, last % kSD), static_cast<uint32_t>(last / kSD) & 1u)) { ok = false; break; }
      tc_fence_after();
      const bool whole = t0 == 0 && t1 == n_all;
      if (warp_live) {
        // each of the twins writes half of the row's head dims
        const size_t part = (static_cast<size_t>(blockIdx.x) * kSlots + (t0 > 0 ? 0 : 1)) * 128 + r;
        if (!whole && live && wg == 0) p.part_ml[part] = make_float2(m_end, l_end);
        const float inv = l_end == 0.f ? 0.f : 1.f / l_end;        // nothing seen: zeros
        uint16_t* dst = p.out + (static_cast<size_t>(row0 + at) * n_q_heads + static_cast<size_t>(h) * G + g) * D;
        const bool odd = *reinterpret_cast<volatile int*>(&sm->odd_v) != 0 && t1 > n_ctx;
#pragma unroll 1
        for (int cb = wg * (D / 2); cb < (wg + 1) * (D / 2); cb += 32) {
          uint32_t o[32];
          TMEM_LD32(t_row + kColO + cb, o, 0);
          tmem_wait_ld();
          if (odd && live) {
            // non-finite elements of the drafted V rows this row sees (they were left out of the product): weight > 0
#pragma unroll 1
            for (int j = (max(t0, n_ctx) - n_ctx) * kTileN; j < min(n, (t1 - n_ctx) * kTileN); ++j) {
              if ((j >> 5) >= p.mask_words || !((__ldg(p.tree_mask + static_cast<size_t>(row0 + at) * p.mask_words + (j >> 5)) >> (j & 31)) & 1)) continue;
              const uint16_t* v = p.v_new + static_cast<size_t>(row0 + j) * p.kv_stride + static_cast<size_t>(h) * D + cb;
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                const uint32_t bits = static_cast<uint32_t>(v[c]) << 16;
                if ((bits & 0x7f800000u) == 0x7f800000u) o[c] = __float_as_uint(__uint_as_float(o[c]) + __uint_as_float(bits));
              }
            }
          }
          if (live) {
            if (whole) {
#pragma unroll
              for (int c = 0; c < 32; c += 8) {
                uint4 x;
                x.x = pack_bf16x2(__uint_as_float(o[c + 0]) * inv, __uint_as_float(o[c + 1]) * inv);
                x.y = pack_bf16x2(__uint_as_float(o[c + 2]) * inv, __uint_as_float(o[c + 3]) * inv);
                x.z = pack_bf16x2(__uint_as_float(o[c + 4]) * inv, __uint_as_float(o[c + 5]) * inv);
                x.w = pack_bf16x2(__uint_as_float(o[c + 6]) * inv, __uint_as_float(o[c + 7]) * inv);
                *reinterpret_cast<uint4*>(dst + cb + c) = x;
              }
            } else {
#pragma unroll
              for (int c = 0; c < 32; c += 4) *reinterpret_cast<uint4*>(p.part_o + part * D + cb + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
            }
          }
        }
      }
      if (tid == 0 && t0 == 0 && t1 < n_all) {
        // this CTA holds the first part of an item that goes on in the next pieces: leave the merge its description
        const long long end = piece.hi + (n_all - t1);
        int parts = 1;
#pragma unroll 1
        while (cut_at(piece.line, piece.pieces, piece.piece + parts) < end) ++parts;
        p.desc[blockIdx.x] = make_int4(row0 + level * p.rows_per_tile, min(p.rows_per_tile, n - level * p.rows_per_tile), h, parts);
        begun = true;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(BAR(kBarOFree));
      ++item;
    }
    if (tid == 0 && !begun) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  } else if (has_work && warp < kRotatorWarp0 + kRotatorWarps) {
    // =============================================================== rotator warps
    // A group of four warps takes every second tile, so that one group's fixed latencies (barriers, the table row) run behind
    // the other's arithmetic; the table row of a group's next tile is fetched while it rotates this one.
    const int group = (warp - kRotatorWarp0) / kRotGroupWarps;
    const int rt = (tid - kRotatorWarp0 * 32) & (kRotators - 1);
    const int c = rt % CH;                        // chunk pair
    const int k0 = (rt / CH) * KPT;               // first of this thread's KPT consecutive keys (within one 16-slot group)
    const int lc = c, hc = CH + c;
    // constants: the rotation by the thread's offset in its group, and by one position
    float2 oc[4], os[4], c1[4], s1[4], ns1[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(k0 & 15) * D + 16 * c) + j);
      const float4 b1 = __ldg(reinterpret_cast<const float4*>(p.rope + D + 16 * c) + j);
      oc[j] = make_float2(a.x, a.z); os[j] = make_float2(a.y, a.w);
      c1[j] = make_float2(b1.x, b1.z); s1[j] = make_float2(b1.y, b1.w); ns1[j] = make_float2(-b1.y, -b1.w);
    }
    Segment seg;
    int gi = 0, n_seg = 0;
    bool ok = true;
    while (ok && take_segment(n_seg++, seg)) {
      const int n = seg.n, n_ctx = seg.n_ctx, kvl = seg.kvl, row0 = seg.row0, h = seg.h;
      const int32_t* bases = p.pos_base + static_cast<size_t>(seg.b) * p.table_stride;
      // position of the first slot of this thread's 16-slot group of tile t (0 where it has no slots), and its table row
      auto position = [&](int t) {
        const long long slot = static_cast<long long>(t) * kTileN + (k0 & ~15);
        return t < n_ctx && slot < kvl ? __ldg(bases + (slot >> p.page_shift)) + (static_cast<int>(slot) & (p.page_size - 1)) : 0;
      };
      float4 base[4];
      auto fetch_row = [&](int pos) {
        if (pos < 0 || pos > p.max_position) { atomicOr(p.status, MEPIC_DEV_BAD_POSITION); pos = 0; }
        const float4* row = reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(pos) * D + 16 * c);
#pragma unroll
        for (int j = 0; j < 4; ++j) base[j] = __ldg(row + j);
      };
      int ahead = position(seg.t0 + ((gi & 1) ^ group));           // this group's first tile of the segment, then two tiles ahead
      fetch_row(ahead);
      ahead = position(seg.t0 + ((gi & 1) ^ group) + 2);
#pragma unroll 1
      for (int t = seg.t0; t < seg.t1; ++t, ++gi) {
        if ((gi & 1) != group) continue;
        const int ks = gi % KD;
        unsigned char* Kb = Ks + ks * L::kStage;
        const bool draft = t >= n_ctx;
        const int left = min(draft ? n - (t - n_ctx) * kTileN : kvl - t * kTileN, kTileN);       // keys that exist
        const bool have = !draft && (k0 & ~15) < left;
        float2 cc[4], ss[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 bc = make_float2(base[j].x, base[j].z), bs = make_float2(base[j].y, base[j].w);
          cc[j] = sub2(mul2(oc[j], bc), mul2(os[j], bs));
          ss[j] = fma2(os[j], bc, mul2(oc[j], bs));
        }
        if (t + 2 < seg.t1) {
          fetch_row(ahead);
          ahead = position(t + 4);
        }
        if (!wait_warp(BAR(kBarKLanded, gi % 6), static_cast<uint32_t>(gi / 6) & 1u)) { ok = false; break; }
        if constexpr (FP8) {
          // (this role fills the bf16 stage itself: every QK^T that read its previous tenant has completed.  With two stages a
          // group always has the same one.)
          if (gi >= KD && !wait_warp(BAR(kBarKFree, ks), static_cast<uint32_t>(gi / KD - 1) & 1u)) { ok = false; break; }
          if (have) {
            // codes widened exactly, the block's scale folded into (cos, sin): the one-position step is a pure rotation
            const float sc = *reinterpret_cast<volatile float*>(&sm->ks[gi & 1][k0 >> 4]);
#pragma unroll
            for (int j = 0; j < 4; ++j) { cc[j] = mul2(cc[j], make_float2(sc, sc)); ss[j] = mul2(ss[j], make_float2(sc, sc)); }
            const unsigned char* codes = Kc + (gi % CD) * L::kCodes + k0 * 128 + 8 * c;
#pragma unroll 1
            for (int i = 0; i < KPT; ++i) {
              const uint2 lo = *reinterpret_cast<const uint2*>(codes + i * 128), hi = *reinterpret_cast<const uint2*>(codes + i * 128 + 64);
              uint32_t lh[4], hh[4], lo_w[4], hi_w[4];
              e4m3x4_to_f16x2x2(lo.x, lh[0], lh[1]); e4m3x4_to_f16x2x2(lo.y, lh[2], lh[3]);
              e4m3x4_to_f16x2x2(hi.x, hh[0], hh[1]); e4m3x4_to_f16x2x2(hi.y, hh[2], hh[3]);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lh[j])), y = __half22float2(*reinterpret_cast<const __half2*>(&hh[j]));
                const float2 a = sub2(mul2(x, cc[j]), mul2(y, ss[j]));
                const float2 b = fma2(x, ss[j], mul2(y, cc[j]));
                lo_w[j] = pack_bf16x2(a.x, a.y);
                hi_w[j] = pack_bf16x2(b.x, b.y);
              }
              *reinterpret_cast<uint4*>(Kb + (lc / 8) * kBlockBytes + sw128(k0 + i, lc % 8)) = make_uint4(lo_w[0], lo_w[1], lo_w[2], lo_w[3]);
              *reinterpret_cast<uint4*>(Kb + (hc / 8) * kBlockBytes + sw128(k0 + i, hc % 8)) = make_uint4(hi_w[0], hi_w[1], hi_w[2], hi_w[3]);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float2 cn = fma2(ss[j], ns1[j], mul2(cc[j], c1[j]));
                ss[j] = fma2(ss[j], c1[j], mul2(cc[j], s1[j]));
                cc[j] = cn;
              }
            }
          }
        } else if (have) {
#pragma unroll 1
          for (int i = 0; i < KPT; ++i) {
            uint4* plo = reinterpret_cast<uint4*>(Kb + (lc / 8) * kBlockBytes + sw128(k0 + i, lc % 8));
            uint4* phi = reinterpret_cast<uint4*>(Kb + (hc / 8) * kBlockBytes + sw128(k0 + i, hc % 8));
            const uint4 lo = *plo, hi = *phi;
            const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
            uint32_t lo_w[4], hi_w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 x = bf16x2_to_float2(lw[j]), y = bf16x2_to_float2(hw[j]);
              const float2 a = sub2(mul2(x, cc[j]), mul2(y, ss[j]));                          // lo cos - hi sin
              const float2 b = fma2(x, ss[j], mul2(y, cc[j]));                                // lo sin + hi cos
              lo_w[j] = pack_bf16x2(a.x, a.y);
              hi_w[j] = pack_bf16x2(b.x, b.y);
            }
            *plo = make_uint4(lo_w[0], lo_w[1], lo_w[2], lo_w[3]);
            *phi = make_uint4(hi_w[0], hi_w[1], hi_w[2], hi_w[3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {          // (cos, sin)(pos + 1) = (cos, sin)(pos) x (cos, sin)(1)
              const float2 cn = fma2(ss[j], ns1[j], mul2(cc[j], c1[j]));
              ss[j] = fma2(ss[j], c1[j], mul2(cc[j], s1[j]));
              cc[j] = cn;
            }
          }
        }
        if (draft) {
          // ---- drafted rows: brought by plain loads, each at its own position, dealt to the threads one by one.  (Rows past
          // the last keep whatever the stage holds: their scores are masked.)
          const int first = row0 + (t - n_ctx) * kTileN;
#pragma unroll 2
          for (int kk = rt / CH; kk < left; kk += kRotators / CH) {
            int at = __ldg(p.row_pos + first + kk);
            if (at < 0 || at > p.max_position) { atomicOr(p.status, MEPIC_DEV_BAD_POSITION); at = at < 0 ? 0 : p.max_position; }
            const uint16_t* src = p.k_new + static_cast<size_t>(first + kk) * p.kv_stride + static_cast<size_t>(h) * D + 8 * c;
            const uint4 lo = *reinterpret_cast<const uint4*>(src), hi = *reinterpret_cast<const uint4*>(src + D / 2);
            const float4* cs = reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(at) * D + 16 * c);
            const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
            uint32_t lo_w[4], hi_w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 b = __ldg(cs + j);
              const float2 x = bf16x2_to_float2(lw[j]), y = bf16x2_to_float2(hw[j]);
              lo_w[j] = pack_bf16x2(x.x * b.x - y.x * b.y, x.y * b.z - y.y * b.w);
              hi_w[j] = pack_bf16x2(x.x * b.y + y.x * b.x, x.y * b.w + y.y * b.z);
            }
            *reinterpret_cast<uint4*>(Kb + (lc / 8) * kBlockBytes + sw128(kk, lc % 8)) = make_uint4(lo_w[0], lo_w[1], lo_w[2], lo_w[3]);
            *reinterpret_cast<uint4*>(Kb + (hc / 8) * kBlockBytes + sw128(kk, hc % 8)) = make_uint4(hi_w[0], hi_w[1], hi_w[2], hi_w[3]);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(kBarKReady, ks));
        if (FP8 && lane == 0) mbar_arrive(BAR(kBarCFree, gi % CD));             // the K codes have been read
      }
    }
  } else if (has_work) {
    if (warp == kKLoaderWarp || warp == kVLoaderWarp) {
    // =============================================================== loader warps: lane g < 8 loads 16-slot group g
    const bool is_k = warp == kKLoaderWarp;
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    unsigned char* ring = FP8 ? (is_k ? Kc : Vc) : (is_k ? Ks : Vs);
    constexpr int kRingStage = FP8 ? L::kCodes : L::kStage;
    const int depth = FP8 ? CD : (is_k ? KD : VD);
    Walk w;
    if (is_k) w = walk_of(sm->piece);
    Segment seg;
    int n_seg = 0;
    // the K loader finds the segments and publishes them; the V loader is one of those who read them
    auto advance = [&]() {
      if (!is_k) return take_segment(n_seg++, seg);
      seg = next_segment(p, w);
      const int at = n_seg % kSegRing;
      if (n_seg >= kSegRing && !wait_warp(BAR(kBarSegFree, at), static_cast<uint32_t>(n_seg / kSegRing - 1) & 1u)) return false;
      if (lane == 0) {
        sm->seg[at] = seg;
        mbar_arrive(BAR(kBarSegFull, at));
      }
      ++n_seg;
      __syncwarp();
      return seg.t1 > 0;
    };
    struct Next { int page, slot0, h, left, row; bool live, draft, special; float ks, vs; };      // left: keys that exist; row: first drafted row
    auto look_up = [&](int t) {
      const bool draft = t >= seg.n_ctx;
      const int left = min(draft ? seg.n - (t - seg.n_ctx) * kTileN : seg.kvl - t * kTileN, kTileN);
      Next x{0, 0, seg.h, left, seg.row0 + (t - seg.n_ctx) * kTileN, false, draft, draft || left < kTileN, 1.f, 1.f};
      const long long slot = static_cast<long long>(t) * kTileN + lane * 16;
      x.live = !x.draft && lane < 8 && slot < seg.kvl;
      if (x.live) {
        const size_t e = static_cast<size_t>(seg.b) * p.table_stride + static_cast<size_t>(slot >> p.page_shift);
        x.slot0 = static_cast<int>(slot) & (p.page_size - 1);
        x.page = __ldg(p.page_ids + e);
        if (static_cast<unsigned>(x.page) >= static_cast<unsigned>(p.num_pages)) { atomicOr(p.status, MEPIC_DEV_BAD_PAGE); x.page = 0; }
        if (FP8 && is_k) {
          const size_t block = static_cast<size_t>(x.page) * p.n_kv_heads + seg.h;
          x.ks = __ldg(p.k_scales + block);
          x.vs = __ldg(p.v_scales + block);
        }
      }
      return x;
    };
    bool more = advance();
    int t = seg.t0;
    Next nx = look_up(t);
    int gi = 0, issued = 0;                       // tiles so far; tiles whose copies were started
#pragma unroll 1
    while (more) {
      const Next x = nx;
      const int st = gi % depth;
      if (gi >= depth && !wait_warp(FP8 ? BAR(kBarCFree, is_k ? st : 2 + st) : BAR(is_k ? kBarKFree : kBarVFree, st), static_cast<uint32_t>(gi / depth - 1) & 1u)) break;
      const uint32_t landed = is_k ? BAR(kBarKLanded, gi % 6) : BAR(kBarVLanded, st);
      if (FP8 && is_k && lane < 8) { sm->ks[gi & 1][lane] = x.ks; sm->vs[gi % kScaleRing][lane] = x.vs; }
      const unsigned live = __ballot_sync(kFull, x.live);
      const bool skip = HOOKS && is_k && blockIdx.x == 0 && gi == p.skip_tile;      // (test hook: a K tile that never comes)
      __syncwarp();                               // the scales are written before lane 0's arrival, which publishes them
      if (lane == 0 && !skip) {
        if (live) mbar_expect_tx(landed, static_cast<uint32_t>(__popc(live)) * kGroupBytes);
        else mbar_arrive(landed);                 // drafted rows: the rotators and the V loader bring them into the stage
      }
      __syncwarp();
      if (x.live && !skip) {
        const uint32_t dst = smem_u32(ring + st * kRingStage) + static_cast<uint32_t>(lane * 16 * 128);
        if constexpr (FP8) {
          const size_t row = (static_cast<size_t>(x.page) * p.n_kv_heads + x.h) * p.page_size + x.slot0;      // of the pool viewed as [rows][128 bytes]
          bulk_g2s(dst, static_cast<const unsigned char*>(is_k ? p.k_pool : p.v_pool) + row * 128, kGroupBytes, landed);
        } else {
          const int y = (x.page * p.n_kv_heads + x.h) * p.page_size + x.slot0;       // row of the pool viewed as [rows][D]
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) tma_load_2d(dst + nb * kBlockBytes, map, nb * 64, y, landed);
        }
      }
      issued = gi + 1;
      if (!FP8 && !is_k && x.special) {
        if (live && !wait_warp(landed, static_cast<uint32_t>(gi / depth) & 1u)) break;
        const int end = ((x.left + 15) & ~15) * 2 * CH;
#pragma unroll 1
        for (int i0 = x.draft ? 0 : x.left * 2 * CH; i0 < end; i0 += 8 * 32) mend_rows<D>(p, Vs + st * L::kStage, &sm->odd_v, x.draft, x.left, x.row, x.h, i0 + lane, 32);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(BAR(kBarVReady, st));
      }
      // the page ids of the next tile are on their way while this role waits for room for it
      if (++t >= seg.t1) { more = advance(); t = seg.t0; }
      if (more) nx = look_up(t);
      ++gi;
    }
    // The copies started last have landed before shared memory is given up.  Always looked after, not only when this role
    // itself lost a wait: another may lose one when this role is through.
    for (int j = max(0, issued - depth); j < issued; ++j)
      for (int i = 0; i < spin && !mbar_try_wait(is_k ? BAR(kBarKLanded, j % 6) : BAR(kBarVLanded, j % depth), static_cast<uint32_t>(is_k ? j / 6 : j / depth) & 1u); ++i) {}
    } else if (warp == kQkWarp) {
      // =============================================================== QK^T issuer
      // S of tile j goes to the buffer that held tile j - 3, once that tile's PV is through with it: the softmax finds the
      // scores of its next tiles ready.  QK^T and PV are issued by a warp each: one thread's waits, issues and commits for both
      // took 3,300 cycles a tile and held everything else up.
      const uint64_t q_desc = smem_desc(smem_u32(Qs), 16, 1024);
      const uint64_t k_desc0 = smem_desc(smem_u32(Ks), 16, 1024);
      Segment seg;
      bool ok = true;
      int j = 0, items = 0, n_seg = 0;
      while (ok && take_segment(n_seg++, seg)) {
        if (!wait_warp(BAR(kBarQReady), static_cast<uint32_t>(items++) & 1u)) { ok = false; break; }
#pragma unroll 1
        for (int t = seg.t0; t < seg.t1; ++t, ++j) {
          const int ks = j % KD, sb = j % kSD;
          if (j >= kSD && !wait_warp(BAR(kBarPvDone, sb), static_cast<uint32_t>(j / kSD - 1) & 1u)) { ok = false; break; }
          if (!wait_warp(BAR(kBarKReady, ks), static_cast<uint32_t>(j / KD) & 1u)) { ok = false; break; }
          tc_fence_after();
          if (lane == 0) {
            const uint64_t kd = k_desc0 + static_cast<uint64_t>(ks) * (L::kStage >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint64_t off = static_cast<uint64_t>(((k / 4) * kBlockBytes + (k % 4) * 32) >> 4);
              tc_mma(tmem + static_cast<uint32_t>(sb * 128), q_desc + off, kd + off, kIdescQK, k > 0);
            }
            tc_commit(BAR(kBarSFull, j % 6));
            tc_commit(BAR(kBarKFree, ks));
          }
          __syncwarp();
        }
      }
      if (lane == 0) {
        // tensor memory may only be released once the MMAs issued so far are done: the softmax sees the last of them when all
        // goes well, nobody does after a lost wait (anybody's)
        tc_commit(BAR(kBarDrain, 0));
        for (int i = 0; i < spin && !mbar_try_wait(BAR(kBarDrain, 0), 0); ++i) {}
      }
    } else {
      // =============================================================== PV issuer
      const uint64_t v_desc0 = smem_desc(smem_u32(Vs), kBlockBytes, 1024);
      Segment seg;
      bool ok = true;
      int i = 0, items = 0, n_seg = 0;
      uint32_t v_parity = 0;                      // bit s: parity of the loader's own work on stage s
      while (ok && take_segment(n_seg++, seg)) {
#pragma unroll 1
        for (int t = seg.t0; t < seg.t1; ++t, ++i) {
          const int st = i % VD, sb = i % kSD;
          const int left = min(t < seg.n_ctx ? seg.kvl - t * kTileN : seg.n - (t - seg.n_ctx) * kTileN, kTileN);
          if (FP8) {
            if (!wait_warp(BAR(kBarVReady, st), static_cast<uint32_t>(i / VD) & 1u)) { ok = false; break; }      // the softmax warps fill every V stage
          } else if (!wait_warp(BAR(kBarVLanded, st), static_cast<uint32_t>(i / VD) & 1u)) {
            ok = false; break;
          }
          if (!FP8 && (t >= seg.n_ctx || left < kTileN)) {
            if (!wait_warp(BAR(kBarVReady, st), (v_parity >> st) & 1u)) { ok = false; break; }
            v_parity ^= 1u << st;
          }
          if (t == seg.t0 && items++ > 0 && !wait_warp(BAR(kBarOFree), static_cast<uint32_t>(items - 2) & 1u)) { ok = false; break; }      // the item before has left O
          if (!wait_warp(BAR(kBarPFull, sb), static_cast<uint32_t>(i / kSD) & 1u)) { ok = false; break; }
          tc_fence_after();
          if (lane == 0) {
            const uint64_t vd = v_desc0 + static_cast<uint64_t>(st) * (L::kStage >> 4);
            const int n_groups = (left + 15) >> 4;
#pragma unroll
            for (int k = 0; k < kTileN / 16; ++k)
              if (k < n_groups)
                tc_mma_ts(tmem + kColO, tmem + static_cast<uint32_t>(sb * 128 + k * 8), vd + static_cast<uint64_t>((k * 2048) >> 4), kIdescPV,
                          t > seg.t0 || k > 0 ? 1u : 0u);
            tc_commit(BAR(kBarVFree, st));
            tc_commit(BAR(kBarPvDone, sb));
          }
          __syncwarp();
        }
      }
      if (lane == 0) {
        tc_commit(BAR(kBarDrain, 1));
        for (int k = 0; k < spin && !mbar_try_wait(BAR(kBarDrain, 1), 0); ++k) {}
      }
    }
  }

  // ---- common exit: nothing of this CTA may still be in flight when tensor memory is released
  tc_fence_before();
  __syncthreads();
  if (warp == kPvWarp) tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------- merge of the parts of a divided item
// Block (c, y) combines four rows of the item that CTA c began, a warp each: m* = max m, l* = sum l 2^(m - m*),
// out = sum o 2^(m - m*) / l*.  The parts' (m, l) are read side by side by the lanes, then the outputs eight parts at a time.
// (Four rows to a warp, one after the other, took 11 us: a chain of a dozen trips to L2.)
constexpr int kMergeRows = 4;
template <int D>
__global__ void __launch_bounds__(kMergeRows * 32) mepic_tree_merge(const __grid_constant__ TreeParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");               // launched as a programmatic dependent of the attention kernel
  const int4 d = p.desc[blockIdx.x];
  const int parts = d.w, G = p.group, lane = threadIdx.x & 31, r = blockIdx.y * kMergeRows + (threadIdx.x >> 5);
  if (parts == 0 || r >= d.y * G) return;
  auto at = [&](int k) { return ((static_cast<size_t>(blockIdx.x) + k) * kSlots + (k == 0 ? 1 : 0)) * 128 + r; };
  float m_star = -INFINITY;
  for (int k = lane; k < parts; k += 32) m_star = fmaxf(m_star, p.part_ml[at(k)].x);
#pragma unroll
  for (int s = 16; s; s >>= 1) m_star = fmaxf(m_star, __shfl_xor_sync(kFull, m_star, s));
  float l_star = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int k0 = 0; k0 < parts; k0 += 8) {
    float wgt = 0.f;
    if (lane < 8 && k0 + lane < parts) {
      const float2 ml = p.part_ml[at(k0 + lane)];
      wgt = ml.x == -INFINITY ? 0.f : ex2(ml.x - m_star);          // a part that held nothing this row sees
      l_star += ml.x == -INFINITY ? ml.y : ml.y * wgt;             // (its sum is 0, or NaN, which must show)
    }
    float4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k0 + k < parts && lane < D / 4) x[k] = *reinterpret_cast<const float4*>(p.part_o + at(k0 + k) * D + 4 * lane);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float wk = __shfl_sync(kFull, wgt, k);
      // (a weight that underflows leaves nothing of what is finite, and NaN of what is not, as 0 x inf does inside a part)
      if (wk != 0.f) { o.x += x[k].x * wk; o.y += x[k].y * wk; o.z += x[k].z * wk; o.w += x[k].w * wk; }
      else if (k0 + k < parts) { o.x += x[k].x - x[k].x; o.y += x[k].y - x[k].y; o.z += x[k].z - x[k].z; o.w += x[k].w - x[k].w; }
    }
  }
#pragma unroll
  for (int s = 4; s; s >>= 1) l_star += __shfl_xor_sync(kFull, l_star, s);
  l_star = __shfl_sync(kFull, l_star, 0);
  const float inv = l_star == 0.f ? 0.f : 1.f / l_star;
  if (lane < D / 4) {
    const size_t to = (static_cast<size_t>(d.x + r / G) * (p.n_kv_heads * G) + static_cast<size_t>(d.z) * G + r % G) * D + 4 * lane;
    *reinterpret_cast<uint2*>(p.out + to) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  }
}

template <int D, bool FP8, bool HOOKS>
int32_t launch_tree(const TreeParams& p, int ctas, int device, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t st) {
  constexpr int smem = TreeSmem<D, FP8>::kBytes;
  static std::atomic<uint64_t> prepared{0};      // bit d: the kernel's shared-memory limit is set on device d
  cudaError_t e = cudaSuccess;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (!(prepared.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(mepic_tree_attn<D, FP8, HOOKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) { mepic_set_error("attn_tree: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
    prepared.fetch_or(bit, std::memory_order_relaxed);
  }
  mepic_tree_attn<D, FP8, HOOKS><<<ctas, kThreads, smem, st>>>(p, map_k, map_v);
  e = cudaGetLastError();
  if (e == cudaSuccess) {
    const int live = std::min(p.max_rows, p.rows_per_tile) * p.group;
    e = launch_dependent(mepic_tree_merge<D>, dim3(ctas, (live + kMergeRows - 1) / kMergeRows), dim3(kMergeRows * 32), st, p);
  }
  if (e != cudaSuccess) { mepic_set_error("attn_tree: launch: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(2);
  return MEPIC_OK;
}

// SM count of the current device (0 without one); *device: its index.
int sm_count(int* device) {
  static std::atomic<int> known[64];             // a device's count does not change: asked once
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  *device = dev;
  if (dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
  return sms;
}
int rows_per_tile(const mepic_config_t* cfg) { return 128 / (cfg->n_q_heads / cfg->n_kv_heads); }
// One CTA per SM, or one per level where there are more levels (row tiles of a request) than SMs.
int cta_count(const mepic_config_t* cfg, int max_rows, int sms) {
  const int q = rows_per_tile(cfg);
  return std::max(sms, (max_rows + q - 1) / q);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

size_t workspace_bytes(const mepic_config_t* cfg, int max_rows, int* device, int* sms_out) {
  const int sms = sm_count(device);
  if (sms <= 0) { mepic_set_error("attn_tree: no CUDA device"); return 0; }
  *sms_out = sms;
  const size_t n = static_cast<size_t>(cta_count(cfg, max_rows, sms));
  return n * (sizeof(int4) + kSlots * 128 * (sizeof(float2) + static_cast<size_t>(cfg->head_dim) * sizeof(float)));
}

int32_t tree_call(const mepic_config_t* cfg, const mepic_attn_tree_args_t* a, const float* k_scales, const float* v_scales, bool fp8, void* cuda_stream) {
  const char* what = fp8 ? "attn_tree_fp8" : "attn_tree";
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("%s: NULL argument", what); return MEPIC_E_INVAL; }
  if (fp8 && cfg->head_dim != 128) { mepic_set_error("%s: head_dim %d: 8-bit pages are built for head_dim 128", what, cfg->head_dim); return MEPIC_E_INVAL; }
  if (a->batch < 1 || a->table_stride < 1 || a->total_rows < 0) { mepic_set_error("%s: batch and table_stride must be positive, total_rows not negative", what); return MEPIC_E_INVAL; }
  if (a->max_rows < 0 || a->max_rows > MEPIC_TREE_MAX_ROWS) { mepic_set_error("%s: max_rows %d not in 0..%d", what, a->max_rows, MEPIC_TREE_MAX_ROWS); return MEPIC_E_INVAL; }
  if (a->total_rows == 0 || a->max_rows == 0) return MEPIC_OK;
  if (a->mask_words < 1 || a->max_rows > 32LL * a->mask_words) { mepic_set_error("%s: %d mask words for %d rows", what, a->mask_words, a->max_rows); return MEPIC_E_INVAL; }
  if (!a->q || !a->k_new || !a->v_new || !a->row_offsets || !a->row_pos || !a->tree_mask || !a->k_pool || !a->v_pool || !a->page_ids ||
      !a->pos_base || !a->kv_len || !a->rope_table || !a->out || !a->workspace || !a->status) {
    mepic_set_error("%s: NULL pointer argument", what); return MEPIC_E_INVAL;
  }
  if (fp8 && (!k_scales || !v_scales)) { mepic_set_error("%s: NULL scale pointer", what); return MEPIC_E_INVAL; }
  if (!aligned16(a->q) || !aligned16(a->k_new) || !aligned16(a->v_new) || !aligned16(a->k_pool) || !aligned16(a->v_pool) ||
      !aligned16(a->rope_table) || !aligned16(a->out) || !aligned16(a->workspace)) {
    mepic_set_error("%s: pointers must be 16-byte aligned", what); return MEPIC_E_INVAL;
  }
  const long long q_packed = static_cast<long long>(cfg->n_q_heads) * cfg->head_dim, kv_packed = static_cast<long long>(cfg->n_kv_heads) * cfg->head_dim;
  const long long q_stride = a->q_stride ? a->q_stride : q_packed, kv_stride = a->kv_stride ? a->kv_stride : kv_packed;
  if (q_packed > 0x7fffffffLL || q_stride < q_packed || kv_stride < kv_packed || q_stride % 8 || kv_stride % 8) {
    mepic_set_error("%s: row strides must be 0 or multiples of 8 of at least a packed row", what); return MEPIC_E_INVAL;
  }
  int device = 0, sms = 0;
  const size_t need = workspace_bytes(cfg, a->max_rows, &device, &sms);
  if (need == 0) return MEPIC_E_CUDA;
  if (a->workspace_bytes < need) { mepic_set_error("%s: workspace of %zu bytes, %zu needed", what, a->workspace_bytes, need); return MEPIC_E_INVAL; }
  TreeParams p;
  p.q = static_cast<const uint16_t*>(a->q); p.k_new = static_cast<const uint16_t*>(a->k_new); p.v_new = static_cast<const uint16_t*>(a->v_new);
  p.row_offsets = a->row_offsets; p.row_pos = a->row_pos; p.tree_mask = a->tree_mask;
  p.k_pool = a->k_pool; p.v_pool = a->v_pool; p.k_scales = k_scales; p.v_scales = v_scales;
  p.page_ids = a->page_ids; p.pos_base = a->pos_base; p.kv_len = a->kv_len; p.rope = a->rope_table;
  p.out = static_cast<uint16_t*>(a->out); p.status = a->status;
  p.table_stride = a->table_stride; p.batch = a->batch; p.total_rows = a->total_rows; p.max_rows = a->max_rows; p.mask_words = a->mask_words;
  p.q_stride = static_cast<int>(q_stride); p.kv_stride = static_cast<int>(kv_stride);
  p.n_kv_heads = cfg->n_kv_heads; p.page_size = cfg->page_size; p.num_pages = cfg->num_pages; p.max_position = cfg->max_position;
  p.page_shift = 0;
  while ((1 << p.page_shift) < cfg->page_size) ++p.page_shift;
  p.scale_log2 = a->sm_scale * 1.4426950408889634f;
  p.group = cfg->n_q_heads / cfg->n_kv_heads;
  p.rows_per_tile = rows_per_tile(cfg);
  p.max_levels = (a->max_rows + p.rows_per_tile - 1) / p.rows_per_tile;
  const int ctas = cta_count(cfg, a->max_rows, sms);
  unsigned char* ws = static_cast<unsigned char*>(a->workspace);
  p.desc = reinterpret_cast<int4*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + sizeof(int4) * ctas);
  p.part_o = reinterpret_cast<float*>(p.part_ml + static_cast<size_t>(ctas) * kSlots * 128);
  p.spin_limit = mepic_test_spin_limit(kSpinLimit); p.skip_tile = mepic_test_skip_tile();
  alignas(64) CUtensorMap map_k, map_v;
  if (fp8) {
    memset(&map_k, 0, sizeof(map_k)); memset(&map_v, 0, sizeof(map_v));      // codes come by untiled bulk copies
  } else {
    int32_t rc = mepic_make_pool_map(cfg, a->k_pool, &map_k);
    if (rc == MEPIC_OK) rc = mepic_make_pool_map(cfg, a->v_pool, &map_v);
    if (rc != MEPIC_OK) return rc;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool hooks = p.spin_limit != kSpinLimit || p.skip_tile >= 0;
  if (cfg->head_dim == 64) return hooks ? launch_tree<64, false, true>(p, ctas, device, map_k, map_v, st) : launch_tree<64, false, false>(p, ctas, device, map_k, map_v, st);
  if (fp8) return hooks ? launch_tree<128, true, true>(p, ctas, device, map_k, map_v, st) : launch_tree<128, true, false>(p, ctas, device, map_k, map_v, st);
  return hooks ? launch_tree<128, false, true>(p, ctas, device, map_k, map_v, st) : launch_tree<128, false, false>(p, ctas, device, map_k, map_v, st);
}

}  // namespace

extern "C" size_t mepic_attn_tree_workspace(const mepic_config_t* cfg, int32_t max_rows) {
  if (!mepic_config_ok(cfg)) return 0;
  if (max_rows < 0 || max_rows > MEPIC_TREE_MAX_ROWS) { mepic_set_error("attn_tree_workspace: max_rows %d not in 0..%d", max_rows, MEPIC_TREE_MAX_ROWS); return 0; }
  int device = 0, sms = 0;
  return workspace_bytes(cfg, max_rows, &device, &sms);
}
extern "C" int32_t mepic_attn_tree(const mepic_config_t* cfg, const mepic_attn_tree_args_t* a, void* cuda_stream) {
  return tree_call(cfg, a, nullptr, nullptr, false, cuda_stream);
}
extern "C" int32_t mepic_attn_tree_fp8(const mepic_config_t* cfg, const mepic_attn_tree_args_t* a, const float* k_scales,
                                       const float* v_scales, void* cuda_stream) {
  return tree_call(cfg, a, k_scales, v_scales, true, cuda_stream);
}
