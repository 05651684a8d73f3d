// Attention of the newest token of every beam over the paged, un-rotated context, each page that beams of a request share read
// once (see mepic_beam_plan and mepic_attn_beam in mepic.h).
//
// Bound: HBM, for bf16 pages.  A request's W beams of G query heads are columns of one matrix product per kv head, so a page's K and
// V serve them all for one read.  As in the per-request decode the keys are the M rows of both products (S^T = K' Q^T, O^T = V^T P^T
// on mma.sync) and the columns are the N side: 8 columns a tile of the instruction, one or two such tiles (NT), which is what fits in
// registers with 32 bits an element of Q and of O.  More columns are more blocks, and a page is read once for each: of 8 x 8 beams of
// 4 heads, two blocks, 0.92 GB come from HBM where 0.50 would do.  (Blocks that walk a page together halved that: 151
// us against 155, the bound being the latency of a tile's instructions by then, but 5 x 5 heads took 39 us against 37 and 8-bit pages,
// out of registers, 123 against 107; 32-column blocks spill.)  The (column block, kv
// head, 16-key tile) triples of the batch form one line, cut into equal pieces, one per warp of a persistent grid, each with a ring
// of TMA stages of its own; pieces that end inside a column block leave partials (reference, sum, unnormalised output) that a second
// kernel joins in a fixed order.
//
// Measured, without the plan: 32 x 4 beams of 4 heads, 8 kv heads, over 8,300 slots 164 us (6 TB/s of what has to be read); 8 x 8 beams over 17,300 slots,
// 700 of them their own, 154 us; 8 x 4 beams over 33,000 slots of 8-bit pages 106 us (4.2 TB/s; bound by instructions and their
// latency); one request of 4 beams over 224 slots 11 us: launch, then the chain plan -> line -> page -> partials -> merge.
//
// Rotation.  <R(qpos) q, R(pos) k> = <R(qpos - a) q, R(pos - a) k> for any anchor a.  A warp keeps its queries rotated for an anchor
// and turns each key by pos - a from a table of angles in shared memory, 192 positions of it (8-bit pages: 512); the anchor moves once
// in as many consecutive positions.  So the keys are rotated once for all columns, and the work that grows with the columns is done
// for one tile in twelve.  Queries held in fp32 move on with the anchor where they are; others are rotated anew from the caller's.
//
// Precision.  bf16 pages: rotated q and K stay fp32 and enter tf32 products (ten bits of mantissa, cut off), which costs no time that
// rounding them to bf16 would save (twice the products, but no packing) and halves the error; the softmax weights are rounded to bf16,
// the type of V.  8-bit pages: codes are exact in fp16; angles, rotated q and K and the weights are rounded to it.  All sums are
// fp32.
//
// Who sees what.  A record of the plan is one page of one column block: page, position, the beams that hold it, its filled slots.
// Where every beam of the block holds it, nothing is masked.  Where only some do, the other columns' scores are -infinity and
// their outputs are left as they are (not "plus 0 x V": V may hold anything that is not finite).
#include <cuda.h>
#include <cuda_runtime.h>
#include <float.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "mepic.h"
#include "mepic_internal.h"
#include "mepic_ptx.cuh"
#include "mepic_tcgen05.cuh"      // arithmetic on pairs of floats

namespace {

using namespace mepic_dev;

constexpr int kTile = 16;            // keys per staged tile
constexpr int kMaxColumns = 16;      // columns of a column block
// Cutting a number off after ten bits of mantissa makes it smaller, by 2^-11 of its power of two in the mean and by 2^-11 / (2 ln 2) of
// itself where mantissas are spread as those of products are; the scores are made larger by as much for either factor.  (Scores of 30,
// 320 of them: off by 3e-5 of themselves in the mean.  Where nothing is cut it is too much: by half of it, 3.5e-4 of the score, for a key
// at its anchor, whose angle is 0.)
constexpr float kTf32Cut = 1.f + 2.f * 0x1p-11f * 0.7213475f;
constexpr float kLag = 8.f;                      // weights may reach 2^8
// 8-bit pages: O is kept in units of a power of two, which starts as the first one and follows the V scales of pages that all columns
// hold, down to 2^-60 of the largest scale met (so that what a page with a large one left does not overflow).
constexpr float kFirstUnit = 0x1p-7f, kLeastUnit = 0x1p-60f, kMostUnit = 0x1p126f, kBelowTop = 0x1p-60f;
constexpr float kWeight = 0x1p5f;             // weights (2^8 at most) are carried as 2^5 of them, times at most 4: below 65504, and normal in fp16 from 2^-17 on
constexpr int kSeg = 256;            // table entries a CTA of the plan looks at
constexpr int kNowhere = INT_MIN;    // position of a query that sees nothing

// ---------------------------------------------------------------- the plan's layout
// ints: [0, kHead) header, then the running sums of records per (column block, segment), then the rows' lengths, then (16-byte
// aligned) the records {page, pos_base, beams, filled slots}, kSeg * beams of a block for each (column block, segment).
constexpr int kHead = 16;
constexpr int kPlanMagic = 0x4d424d31;
enum { kHMagic, kHGroups, kHWidth, kHStride, kHPage, kHGroupSize, kHKvHeads, kHBeams, kHSegments, kHPages };

struct PlanShape {
  int groups, width, blocks, beams, segments;      // column blocks of a group, beams of a block, segments of a row
  size_t off_len, off_rec, bytes;                  // in ints, in ints, in bytes
};
// A group's beams are dealt evenly to as few column blocks of at most kMaxColumns columns as hold them.
bool plan_shape(const mepic_config_t* cfg, int groups, int width, int stride, const char* what, PlanShape* s) {
  if (groups < 1 || width < 1 || width > MEPIC_BEAM_MAX_WIDTH) { mepic_set_error("%s: groups must be positive, width in 1..%d", what, MEPIC_BEAM_MAX_WIDTH); return false; }
  if (stride < 1 || static_cast<long long>(groups) * width * stride > 0x40000000LL || static_cast<long long>(groups) * width > 0xffffLL * 16) {
    mepic_set_error("%s: table_stride must be positive and the tables below 2^30 entries", what); return false;
  }
  const int most = kMaxColumns / (cfg->n_q_heads / cfg->n_kv_heads);
  s->groups = groups; s->width = width;
  s->blocks = (width + most - 1) / most;
  s->beams = (width + s->blocks - 1) / s->blocks;
  s->segments = (stride + kSeg - 1) / kSeg;
  const size_t n = static_cast<size_t>(groups) * s->blocks * s->segments;
  if (n * kSeg * s->beams > 0x7fffffffULL) { mepic_set_error("%s: the plan would have more than 2^31 records", what); return false; }
  s->off_len = kHead + n + 1;
  s->off_rec = (s->off_len + static_cast<size_t>(groups) * width + 3) & ~static_cast<size_t>(3);
  s->bytes = s->off_rec * 4 + n * kSeg * s->beams * 16;
  return true;
}

struct PlanParams {
  const int32_t* page_ids;
  const int32_t* pos_base;
  const int32_t* kv_len;
  int32_t* sums;         // running sums; the first launch leaves the counts here
  int32_t* lens;
  int4* records;
  int32_t* head;
  int32_t* status;
  int stride, groups, width, blocks, beams, segments, page_shift, num_pages, group_size, n_kv_heads;
};

__device__ __forceinline__ void write_header(const PlanParams& p) {
  p.head[kHMagic] = kPlanMagic; p.head[kHGroups] = p.groups; p.head[kHWidth] = p.width; p.head[kHStride] = p.stride;
  p.head[kHPage] = 1 << p.page_shift; p.head[kHGroupSize] = p.group_size; p.head[kHKvHeads] = p.n_kv_heads;
  p.head[kHBeams] = p.beams; p.head[kHSegments] = p.segments; p.head[kHPages] = p.num_pages;
}

// ---------------------------------------------------------------- plan
// A CTA per (column block, segment of 256 table entries), a thread per entry: the block's beams fall into classes that hold the
// same page at the same position with the same number of slots.  Counted, summed up over the CTA, written.
__global__ void __launch_bounds__(kSeg) mepic_beam_plan_classes(const __grid_constant__ PlanParams p) {
  __shared__ int len[MEPIC_BEAM_MAX_WIDTH];
  __shared__ int warp_n[kSeg / 32];
  __shared__ int mixed[kSeg], n_mixed;         // entries that not all of their beams hold alike
  __shared__ unsigned mixed_held[kSeg];
  extern __shared__ int held_pages[];          // [page ids, position bases, beams that hold the same][beams of the block][kSeg]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int block = blockIdx.x, seg = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = block / p.blocks, first = (block - group * p.blocks) * p.beams, nb = min(p.beams, p.width - first);
  const int P = 1 << p.page_shift;
  const size_t row0 = static_cast<size_t>(group) * p.width + first;
  if (tid < nb) {
    const long long room = min(static_cast<long long>(p.stride) << p.page_shift, 0x7fffffffll);
    int n = __ldg(p.kv_len + row0 + tid);
    if (n < 0 || n > room) { if (seg == 0) atomicOr(p.status, MEPIC_DEV_BAD_SLOT); n = n < 0 ? 0 : static_cast<int>(room); }
    len[tid] = n;
    if (seg == 0) p.lens[row0 + tid] = n;
  }
  if (tid == 0) n_mixed = 0;
  __syncthreads();
  const int e = seg * kSeg + tid;
  const long long from = static_cast<long long>(e) << p.page_shift;
  unsigned held = 0;
  if (e < p.stride)
    for (int i = 0; i < nb; ++i) if (len[i] > from) held |= 1u << i;
  const int32_t* ids = p.page_ids + row0 * p.stride + e;
  const int32_t* base = p.pos_base + row0 * p.stride + e;
  auto fill = [&](int i) { return static_cast<int>(min(static_cast<long long>(P), len[i] - from)); };
  // everything the entry's beams hold, asked for side by side and kept in shared memory, a column per thread
  int* my_ids = held_pages + tid;
  int* my_base = held_pages + nb * kSeg + tid;
  const int lead = held ? __ffs(held) - 1 : 0;
  bool one = true;                              // all beams that hold anything here hold the same, as over a shared context
  for (int i0 = 0; i0 < nb; i0 += 8) {
    int a[8], b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k < nb && (held >> (i0 + k) & 1)) { a[k] = __ldg(ids + static_cast<size_t>(i0 + k) * p.stride); b[k] = __ldg(base + static_cast<size_t>(i0 + k) * p.stride); }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k < nb && (held >> (i0 + k) & 1)) { my_ids[(i0 + k) * kSeg] = a[k]; my_base[(i0 + k) * kSeg] = b[k]; }
  }
  for (unsigned m = held; m; m &= m - 1) {
    const int i = __ffs(m) - 1;
    one = one && my_ids[i * kSeg] == my_ids[lead * kSeg] && my_base[i * kSeg] == my_base[lead * kSeg] && fill(i) == fill(lead);
  }
  // where they do not, every (entry, beam) pair of the CTA finds the beams that hold the same, a pair a thread
  int* my_same = held_pages + 2 * nb * kSeg + tid;
  mixed_held[tid] = one ? 0 : held;
  if (!one) mixed[atomicAdd(&n_mixed, 1)] = tid;         // (in any order: what is found for an entry is kept at the entry)
  __syncthreads();
  for (int q = tid; q < n_mixed * nb; q += kSeg) {
    const int at = mixed[q / nb], i = q % nb;
    const unsigned those = mixed_held[at];
    if (!(those >> i & 1)) continue;
    const int* col_ids = held_pages + at;
    const int* col_base = held_pages + nb * kSeg + at;
    const long long start = static_cast<long long>(seg * kSeg + at) << p.page_shift;
    auto slots = [&](int b) { return min(static_cast<long long>(P), len[b] - start); };
    unsigned same = 0;
    for (unsigned m = those; m; m &= m - 1) {
      const int b = __ffs(m) - 1;
      if (col_ids[b * kSeg] == col_ids[i * kSeg] && col_base[b * kSeg] == col_base[i * kSeg] && slots(b) == slots(i)) same |= 1u << b;
    }
    held_pages[(2 * nb + i) * kSeg + at] = static_cast<int>(same);
  }
  __syncthreads();
  auto each_class = [&](auto use) {
    if (one) { if (held) use(my_ids[lead * kSeg], my_base[lead * kSeg], held, fill(lead)); return; }
    for (unsigned left = held; left;) {
      const int i = __ffs(left) - 1;
      const unsigned same = static_cast<unsigned>(my_same[i * kSeg]);
      left &= ~same;
      use(my_ids[i * kSeg], my_base[i * kSeg], same, fill(i));
    }
  };
  int n = 0;
  each_class([&](int, int, unsigned, int) { ++n; });
  int incl = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(kFull, incl, d); if (lane >= d) incl += y; }
  if (lane == 31) warp_n[warp] = incl;
  __syncthreads();
  int at = incl - n, total = 0;
  for (int w = 0; w < kSeg / 32; ++w) {
    if (w < warp) at += warp_n[w];
    total += warp_n[w];
  }
  const size_t part = static_cast<size_t>(block) * p.segments + seg;
  if (tid == 0) {
    if (gridDim.x * gridDim.y > 1) p.sums[part] = total;
    else { p.sums[0] = 0; p.sums[1] = total; write_header(p); }      // the only part: its sums are known
  }
  int4* out = p.records + part * kSeg * p.beams;
  each_class([&](int page, int pos, unsigned same, int slots) {
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) { atomicOr(p.status, MEPIC_DEV_BAD_PAGE); page = 0; }
    out[at++] = make_int4(page, pos, static_cast<int>(same), slots);
  });
}

// One CTA: counts -> running sums, and the header.
constexpr int kScanThreads = 1024;
__global__ void __launch_bounds__(kScanThreads) mepic_beam_plan_sums(const __grid_constant__ PlanParams p) {
  __shared__ int warp_n[kScanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = p.groups * p.blocks * p.segments;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int before = 0;
  for (int i0 = 0; i0 < n; i0 += kScanThreads) {
    const int c = i0 + tid < n ? p.sums[i0 + tid] : 0;
    int incl = c;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(kFull, incl, d); if (lane >= d) incl += y; }
    if (lane == 31) warp_n[warp] = incl;
    __syncthreads();
    int w = warp_n[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(kFull, w, d); if (lane >= d) w += y; }
    const int mine = __shfl_sync(kFull, w, max(warp - 1, 0)), all = __shfl_sync(kFull, w, 31);
    if (i0 + tid < n) p.sums[i0 + tid] = before + (warp ? mine : 0) + incl - c;
    before += all;
    __syncthreads();
  }
  if (tid == 0) {
    p.sums[n] = before;
    write_header(p);
  }
}

// ---------------------------------------------------------------- attention
struct BeamParams {
  const uint16_t* q;
  const int32_t* q_pos;
  const int32_t* head;
  const int32_t* sums;
  const int32_t* lens;
  const int4* records;
  const float* rope;
  const float* k_scales;   // 8-bit pools only: [num_pages][n_kv_heads]
  const float* v_scales;
  float* part_o;           // [slots][columns][D]
  float2* part_ml;         // [slots][columns] (reference in log2 units, sum)
  uint16_t* out;
  int32_t* status;
  int groups, width, stride, blocks, beams, segments, group_size, columns;
  int n_kv_heads, page_size, log2_tpp, num_pages, max_position, q_stride, workers;
  int spin_limit, skip_tile;
  float scale_log2;
};

template <typename T> __device__ __forceinline__ T plain(const T* at) { return *at; }
// The plan is one of this call's shape, and its sums are ones that its shape allows.
__device__ __forceinline__ bool plan_fits(const BeamParams& p) {
  const int32_t* h = p.head;
  const long long n = static_cast<long long>(p.groups) * p.blocks * p.segments, total = plain(p.sums + n);
  return plain(h + kHMagic) == kPlanMagic && plain(h + kHGroups) == p.groups && plain(h + kHWidth) == p.width && plain(h + kHStride) == p.stride &&
         plain(h + kHPage) == p.page_size && plain(h + kHGroupSize) == p.group_size && plain(h + kHKvHeads) == p.n_kv_heads &&
         plain(h + kHBeams) == p.beams && plain(h + kHSegments) == p.segments && plain(h + kHPages) == p.num_pages &&
         total >= 0 && total <= n * kSeg * p.beams;
}
// a / b where both are positive, in 32 bits where they fit (a tenth of the instructions).
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}
struct Cut { long long total, piece; };
__device__ __forceinline__ Cut cut_of_line(const BeamParams& p) {
  Cut c;
  c.total = (static_cast<long long>(plain(p.sums + static_cast<size_t>(p.groups) * p.blocks * p.segments)) << p.log2_tpp) * p.n_kv_heads;
  c.piece = max(quotient(c.total + p.workers - 1, p.workers), 1ll);
  return c;
}
// A unit of the line: a column block under one kv head, records r0 .. r1-1 of the plan.
struct Unit { int block, head, r0, r1; };
__device__ __forceinline__ int begin_of(const BeamParams& p, int block) { return plain(p.sums + static_cast<size_t>(block) * p.segments); }
// The unit after (block, head); false: there is none.
__device__ __forceinline__ bool next_unit(const BeamParams& p, int& block, int& head) {
  if (++head < p.n_kv_heads) return true;
  head = 0;
  do {
    if (++block >= p.groups * p.blocks) return false;
  } while (begin_of(p, block) >= begin_of(p, block + 1));
  return true;
}
// The column block that place x of the line falls into, 32 candidates at a time (by a whole warp).  candidate_of: a lane's first one,
// which does not depend on x.
__device__ __forceinline__ int candidate_of(const BeamParams& p, int lane) {
  const int n = p.groups * p.blocks;
  return begin_of(p, min(lane * ((n + 31) / 32), n));
}
__device__ __forceinline__ Unit unit_at(const BeamParams& p, long long x, int lane, int candidate) {
  const int all = p.groups * p.blocks;
  int lo = 0, n = all, begin = candidate;               // in [lo, lo + n): the last block whose begin is <= x
  for (;;) {
    const int step = (n + 31) / 32;
    const bool below = lane * step < n && (static_cast<long long>(begin) << p.log2_tpp) * p.n_kv_heads <= x;
    const int k = 31 - __clz(__ballot_sync(kFull, below) | 1u);
    if (step == 1) {
      Unit u{lo + k, 0, __shfl_sync(kFull, begin, k), __shfl_sync(kFull, begin, min(k + 1, 31))};
      if (k == 31) u.r1 = begin_of(p, u.block + 1);
      return u;
    }
    n = min(step, n - k * step);
    lo += k * step;
    begin = begin_of(p, min(lo + lane * ((n + 31) / 32), all));
  }
}

template <int D, bool FP8> constexpr int stage_bytes = 2 * kTile * D * (FP8 ? 1 : 2);
// Per position of the table, for every two pairs of dims: (c, c', s, s') in fp32 or fp16.
template <int D, bool FP8> constexpr int angle_bytes = D / 2 * (FP8 ? 4 : 8);
// Stages of a warp's ring; positions of the table, as many as fit beside the rings (an anchor lasts as long).
constexpr int kStages = 2;
template <bool FP8> constexpr int angles_of = FP8 ? 512 : 192;
constexpr int kWarpWords = 128;      // bytes a warp has beside its ring: per stage 16 of tile data, 8 of scales and a barrier of 8
template <int D, bool FP8, int W> constexpr size_t smem_bytes = static_cast<size_t>(W) * (kStages * stage_bytes<D, FP8> + kWarpWords) + (angles_of<FP8> + 1) * angle_bytes<D, FP8> + 1024;

// NT: tiles of 8 columns; W: warps of a CTA.
__device__ __forceinline__ float4 lds128(uint32_t addr) {
  float4 v;
  asm("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{ .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p; }" : "=r"(is));
  return is != 0;
}

template <int D, int NT, bool FP8, int W>
__global__ void __launch_bounds__(W * 32, 1)
mepic_beam_attn(const __grid_constant__ BeamParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr int NB = D / 64;                 // 64-dim blocks (128-byte swizzled rows) per K or V row
  constexpr int KS = D / 16, KH = KS / 2;    // k-steps of the QK^T product; step j pairs with step j + KH
  constexpr int NV = D / 16;                 // 16-dim blocks of the output
  constexpr int KB = FP8 ? 1 : NB;
  constexpr int kBlockBytes = kTile * 128;
  constexpr int kStageBytes = stage_bytes<D, FP8>;
  static_assert(kStages * 32 <= kWarpWords, "tile data, scales and barriers of the ring");
  constexpr int kAngleBytes = angle_bytes<D, FP8>, kAngles = angles_of<FP8>;

  extern __shared__ unsigned char smem_dyn[];
  // 1024-byte alignment: the swizzle pattern is a function of the address bits
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~static_cast<uintptr_t>(1023));
  const int lane = threadIdx.x & 31, wic = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0);      // (known to be the same in a warp)
  unsigned char* stage0 = smem + static_cast<size_t>(wic) * kStages * kStageBytes;
  unsigned char* angles = smem + static_cast<size_t>(W) * kStages * kStageBytes;
  unsigned char* words = angles + (kAngles + 1) * kAngleBytes + wic * kWarpWords;
  const uint32_t meta = smem_u32(words);                 // per stage: position, beams, valid slots of the tile
  const uint32_t scl = meta + kStages * 16;              // per stage: K and V scale of the page
  uint64_t* bars = reinterpret_cast<uint64_t*>(words + kStages * 24);

  const int g = lane >> 2, t = lane & 3;     // fragment row (key, dim, or column of Q) and column group
  // 8-bit pages: ldmatrix on bytes hands a lane four consecutive dims of a key, its transposing form four consecutive keys of a
  // dim; which dim or key stands at which place of the contraction is free as long as both operands agree.
  auto pair_of = [&](int j, int r) { return FP8 ? 16 * j + 4 * t + 2 * r : 16 * j + 2 * t + 8 * r; };
  // what ldmatrix wants of this lane: the row (key) that it names of a tile, and its first 16-byte chunk under the swizzle
  uint32_t k_lane, v_lane;
  {
    const int mi = lane >> 3, rr = lane & 7;
    const int kk = FP8 ? 4 * (rr >> 1) + (rr & 1) + 2 * (mi & 1) : ((mi & 1) << 3) + rr, kc = FP8 ? KH * (mi >> 1) : mi >> 1;
    const int vk = FP8 ? lane & 15 : ((mi >> 1) << 3) + rr, vc = FP8 ? lane >> 4 : mi & 1;
    k_lane = kk * 128 + ((kc ^ (kk & 7)) << 4);
    v_lane = vk * 128 + ((vc ^ (vk & 7)) << 4);
  }
  const int keyA = FP8 ? 4 * (g >> 1) + (g & 1) : g, keyB = FP8 ? keyA + 2 : g + 8;      // keys of the lane's two rows

  // What the launches before this one wrote (the plan, the queries, pages) is complete and visible from here on; the CTAs may have been
  // in place before, so their loads are plain ones, not of the read-only path.  (One request, plan and attention launched one by one:
  // 16.4 us before, 14.9 so; replayed from a graph the same.)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("fence.proxy.async.global;" ::: "memory");            // ... for the copies of pages, too
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the merge kernel may move in as CTAs of this one retire
  const int candidate = candidate_of(p, lane);
  if (!plan_fits(p)) return;                                         // (reported by the merge kernel)
  const Cut cut = cut_of_line(p);
  // Pieces of one tile each (fewer tiles than warps) are dealt round to the SMs, longer ones to the warps of a CTA in a row: they
  // mostly share a unit, and its queries in the first-level cache.
  const bool spread = cut.piece == 1;
  if ((spread ? static_cast<long long>(blockIdx.x) : static_cast<long long>(blockIdx.x) * W * cut.piece) >= cut.total) return;

  // The table of angles is made of products, R(16 k + f) = R(16 k) R(f): only these 16 + kAngles / 16 rows of the caller's table are read
  // (all 192 or 512 of them, by every SM at once, took 4.7 and 6.9 us; this takes 1.6 and 2).  A warp has the rows k = warp, warp + W
  // ..., a lane two pairs of dims; asked for here, used once the first tiles are under way.
  constexpr int kCoarse = (kAngles / kTile + W) / W;            // rows 16 k of a warp, that of kAngles among them
  auto row_of = [&](int at) { return lane < D / 4 ? plain(reinterpret_cast<const float4*>(p.rope + static_cast<size_t>(min(at, p.max_position)) * D + 4 * lane)) : make_float4(0.f, 0.f, 0.f, 0.f); };
  float4 coarse[kCoarse], fine[kTile / 2];                      // c, s, c', s'
  if (!spread) {
#pragma unroll
    for (int k = 0; k < kCoarse; ++k) coarse[k] = row_of(kTile * (wic + W * k));
#pragma unroll
    for (int f = 0; f < kTile / 2; ++f) fine[f] = row_of(f);
  }

  if (lane == 0) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) mbar_init(smem_u32(&bars[s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();

  const long long w = spread ? static_cast<long long>(wic) * gridDim.x + blockIdx.x : static_cast<long long>(blockIdx.x) * W + wic;
  const int n_tiles = static_cast<int>(max(min(cut.piece, cut.total - w * cut.piece), 0ll));      // 0: the line ends before this warp
  const long long x0 = min(w * cut.piece, cut.total - 1);
  const int G = p.group_size, tpp_mask = (1 << p.log2_tpp) - 1;

  // ---- producer: the next tile to stage
  int p_block, p_head, pr, pr_end, pt;                                 // column block, kv head, record, the block's last one, tile of the page
  int c_block, c_head, c_left;                                         // consumer: its unit, and the unit's tiles still to come
  {
    const Unit u = unit_at(p, x0, lane, candidate);
    const long long in = x0 - (static_cast<long long>(u.r0) << p.log2_tpp) * p.n_kv_heads, per = static_cast<long long>(u.r1 - u.r0) << p.log2_tpp;
    const int head = static_cast<int>(quotient(in, per));
    const long long in_head = in - head * per;
    p_block = c_block = u.block; p_head = c_head = head;
    pr = u.r0 + static_cast<int>(in_head >> p.log2_tpp);
    pr_end = u.r1;
    pt = static_cast<int>(in_head) & tpp_mask;
    c_left = static_cast<int>(min(per - in_head, static_cast<long long>(INT_MAX)));
  }
  int pseg = p_block * p.segments;                                    // segment of the producer's record
  int win0 = 0, win_n = 0;                                             // records win0 .. win0 + win_n - 1, one per lane
  int4 win = make_int4(0, 0, 0, 0);
  float win_ks = 0.f, win_vs = 0.f;
  int issued = 0;                                                      // tiles handed to the ring
  // A tile behind its page's filled slots goes by the position of the page's last tile that has any: its keys are masked, but an anchor
  // has to be where a key is, within reach of the rope table.  How far that one is from a tile with n_valid filled slots (0 or fewer: none).
  // (bf16 pages: where the tile is issued, 8-bit pages: where it moves the anchor; the other way takes 8-bit pages 2 % and bf16 pages 1 %.)
  auto last_filled = [](int n_valid) { return (n_valid - 1) & -kTile; };
  auto issue = [&](int stage) {
    if (pr < win0 || pr >= win0 + win_n) {
      for (unsigned past = kFull; past == kFull; pseg += __popc(past))      // the segment that record pr lies in
        past = __ballot_sync(kFull, pseg + 1 + lane < p.groups * p.blocks * p.segments && plain(p.sums + pseg + 1 + lane) <= pr);
      const int s0 = plain(p.sums + pseg);
      const int at = pr - s0 + lane;
      win0 = pr;
      win_n = min(32, plain(p.sums + pseg + 1) - pr);
      const bool in = lane < win_n && at >= 0 && at < kSeg * p.beams;
      win = in ? plain(p.records + static_cast<size_t>(pseg) * kSeg * p.beams + at) : make_int4(0, 0, 0, 0);
      if (static_cast<unsigned>(win.x) >= static_cast<unsigned>(p.num_pages)) win.x = 0;
      if constexpr (FP8) {
        win_ks = plain(p.k_scales + static_cast<size_t>(win.x) * p.n_kv_heads + p_head);
        win_vs = plain(p.v_scales + static_cast<size_t>(win.x) * p.n_kv_heads + p_head);
      }
    }
    auto copy = [&](int page) {
      if (w == 0 && issued == p.skip_tile) return;          // (test hook: one copy that never comes)
      const uint32_t bar = smem_u32(&bars[stage]), dst = smem_u32(stage0 + stage * kStageBytes);
      const int y = (page * p.n_kv_heads + p_head) * p.page_size + pt * kTile;      // row of the pool viewed as [rows][D]
      mbar_expect_tx(bar, kStageBytes);
      if constexpr (FP8) {
        tma_load_2d(dst, &map_k, 0, y, bar);
        tma_load_2d(dst + kBlockBytes, &map_v, 0, y, bar);
      } else {
        tma_load_3d(dst, &map_k, 0, y, 0, bar);
        tma_load_3d(dst + NB * kBlockBytes, &map_v, 0, y, 0, bar);
      }
    };
    // The lane that holds the record leaves what the tile's consumer needs.  bf16 pages: it also issues the copies (no registers for
    // another way: 8 x 8 beams 157 us against 164); 8-bit pages: an elected one does, which takes fewer instructions (108 us against 111).
    const int holds = pr - win0;
    if (lane == holds) {
      const int n_valid = min(win.w - pt * kTile, kTile);
      const int pos = win.y + pt * kTile + (FP8 ? 0 : last_filled(n_valid));
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%3};" ::"r"(meta + stage * 16), "r"(pos), "r"(win.z), "r"(n_valid) : "memory");
      if constexpr (FP8) asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(scl + stage * 8), "f"(win_ks), "f"(win_vs) : "memory");
      else copy(win.x);
    }
    if constexpr (FP8) {
      const int page = __shfl_sync(kFull, win.x, holds);
      if (elect_one()) copy(page);
    }
    ++issued;
    if (pt < tpp_mask) { ++pt; return; }
    pt = 0;
    if (++pr < pr_end) return;
    if (!next_unit(p, p_block, p_head)) return;            // (the line's end: nothing is issued any more)
    pr = begin_of(p, p_block);
    pr_end = begin_of(p, p_block + 1);
    pseg = p_block * p.segments;
    win_n = 0;                                              // another head: its scales, another block: its records
  };
  for (int s = 0; s < kStages && issued < n_tiles; ++s) issue(s);

  // positions the table has to reach: those of a piece, where it is short; no more than the caller's table has
  const int span = static_cast<int>(min(static_cast<long long>(min(kAngles, max((p.max_position + 1) / kTile, 1) * kTile)), max(cut.piece, 1ll) * kTile));
  // ---- the table of angles: for position a and pairs 2u, 2u+1 the quadruple (c, c', s, s'), rows swizzled so that the eight lanes
  // that load together (two keys, four column groups) meet all banks
  // (the last row is that of `span` positions, by which an anchor moves)
  auto put_row = [&](int at, const float4& cs) {      // c, s, c', s'
    const int a = at < span ? at : kAngles;
    if (at > span || lane >= D / 4) return;
    if constexpr (FP8) {
      *reinterpret_cast<uint2*>(angles + a * kAngleBytes + ((lane * 8) ^ ((a & 1) << 6))) = make_uint2(pack_f16x2(cs.x, cs.z), pack_f16x2(cs.y, cs.w));
    } else {
      *reinterpret_cast<float4*>(angles + a * kAngleBytes + ((lane * 16) ^ ((a & 1) << 6))) = make_float4(cs.x, cs.z, cs.y, cs.w);
    }
  };
  if (spread) {                                        // pieces of a tile: no more than 17 rows
    for (int at = wic; at <= span; at += W) put_row(at, row_of(at));
  } else {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int k = 0; k < kCoarse; ++k) {
        const float4 b = coarse[k];
#pragma unroll
        for (int f = 0; f < kTile / 2; ++f) {
          const float4 x = fine[f];
          put_row(kTile * (wic + W * k) + half * (kTile / 2) + f,
                  make_float4(fmaf(b.x, x.x, -(b.y * x.y)), fmaf(b.x, x.y, b.y * x.x), fmaf(b.z, x.z, -(b.w * x.w)), fmaf(b.z, x.w, b.w * x.z)));
        }
      }
      if (half == 0)
#pragma unroll
        for (int f = 0; f < kTile / 2; ++f) fine[f] = row_of(kTile / 2 + f);
    }
  }
  __syncthreads();
  const uint32_t angles_addr = smem_u32(angles);

  // ---- state of the unit
  int u_block = -1, u_head = -1;
  unsigned all_beams = 0;
  int anchor = INT_MIN;
  unsigned see[NT][2];                       // beam bit of the columns 8 nt + 2 t, + 1 of this lane (0: no such column)
  int q_at[NT];                              // position of column 8 nt + g
  // B fragments of Q'^T, column 8 nt + g: bf16 pages in fp32 (the product takes them as tf32), 8-bit pages in fp16
  float qt[FP8 ? 1 : NT][KS][4];             // dims of the k-step's two column halves, pairs
  uint32_t qf[FP8 ? NT : 1][KS][2];
  float2 m_neg[NT], l_run[NT];               // the negative of the reference, and this lane's share of the sum, of columns 2 t, 2 t + 1
  float acc[NT][NV][4];                      // O^T: [dim g: column 2t, 2t+1 | dim g + 8: the same]
  float v_unit = kFirstUnit, v_least = kLeastUnit;      // 8-bit pages: acc is in units of v_unit / kWeight; the least that it may be

  auto flush = [&]() {
    if (u_block < 0) return;
    const long long slot = static_cast<long long>(u_block) * p.n_kv_heads + u_head + w;
    const float unit = FP8 ? v_unit * (1.f / kWeight) : 1.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float l = c ? l_run[nt].y : l_run[nt].x;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(kFull, l, o);
        const int col = 8 * nt + 2 * t + c;
        if (col < p.columns) {
          float* dst = p.part_o + (slot * p.columns + col) * D;
#pragma unroll
          for (int db = 0; db < NV; ++db) { dst[16 * db + g] = acc[nt][db][c] * unit; dst[16 * db + 8 + g] = acc[nt][db][2 + c] * unit; }
          if (g == 0) p.part_ml[slot * p.columns + col] = make_float2(-(c ? m_neg[nt].y : m_neg[nt].x), l);
        }
      }
  };
  // The queries of the unit, rotated by their position less the anchor.  One table row does for all columns where their positions are
  // the same, as they are but for beams that have ended.
  auto rotate_queries = [&]() {
    const int first = (u_block % p.blocks) * p.beams, nb = min(p.beams, p.width - first), row0 = u_block / p.blocks * p.width + first;
    const uint16_t* q_src[NT];
    const float* turn[NT];
    float sign[NT];
    const int q0 = __shfl_sync(kFull, q_at[0], 0);
    bool same = true;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int col = 8 * nt + g < nb * G ? 8 * nt + g : 0;
      q_src[nt] = p.q + static_cast<size_t>(row0 + col / G) * p.q_stride + (static_cast<size_t>(u_head) * G + col % G) * D;
      const int rel = q_at[nt] == kNowhere ? 0 : q_at[nt] - anchor;
      int arel = rel < 0 ? -rel : rel;
      if (static_cast<unsigned>(arel) > static_cast<unsigned>(p.max_position)) { atomicOr(p.status, MEPIC_DEV_BAD_POSITION); arel = p.max_position; }
      turn[nt] = p.rope + static_cast<size_t>(arel) * D;
      sign[nt] = rel < 0 ? -1.f : 1.f;
      same = same && q_at[nt] == q0;
    }
    // (8-bit pages: the two pairs of a k-step are neighbours, one load: 8 x 4 beams over 33,000 slots 115 -> 113 us)
    auto rotate = [&](int nt, int j, int r, const uint2& raw, const float4& cs, float sn) {
      const float2 lo = bf16x2_to_float2(raw.x), hi = bf16x2_to_float2(raw.y);
      const float2 c = make_float2(cs.x, cs.z), sp = make_float2(cs.y * sn, cs.w * sn), sm = make_float2(-sp.x, -sp.y);
      const float2 a = fma2(lo, c, mul2(hi, sm)), b = fma2(lo, sp, mul2(hi, c));
      if constexpr (!FP8) {
        qt[nt][j][2 * r] = a.x; qt[nt][j][2 * r + 1] = a.y;
        qt[nt][j + KH][2 * r] = b.x; qt[nt][j + KH][2 * r + 1] = b.y;
      } else {
        qf[nt][j][r] = pack_f16x2(a.x, a.y);
        qf[nt][j + KH][r] = pack_f16x2(b.x, b.y);
      }
    };
    auto rotate_step = [&](int nt, int j, const float4 (&cs)[2], float sn) {
      uint2 raw[2];
      if constexpr (FP8) {
        const uint2* src = reinterpret_cast<const uint2*>(q_src[nt] + pair_of(j, 0));
        const uint2 lo = plain(src), hi = plain(src + D / 8);
        raw[0] = make_uint2(lo.x, hi.x); raw[1] = make_uint2(lo.y, hi.y);
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t* src = reinterpret_cast<const uint32_t*>(q_src[nt] + pair_of(j, r));
          raw[r] = make_uint2(plain(src), plain(src + D / 4));
        }
      }
      rotate(nt, j, 0, raw[0], cs[0], sn);
      rotate(nt, j, 1, raw[1], cs[1], sn);
    };
    auto angles_of_step = [&](int nt, int j, float4 (&cs)[2]) {
#pragma unroll
      for (int r = 0; r < 2; ++r) cs[r] = plain(reinterpret_cast<const float4*>(turn[nt] + 2 * pair_of(j, r)));
    };
    const bool one_turn = __all_sync(kFull, same);
#pragma unroll
    for (int j = 0; j < KH; ++j) {
      float4 cs[2];
      angles_of_step(0, j, cs);
      rotate_step(0, j, cs, sign[0]);
#pragma unroll
      for (int nt = 1; nt < NT; ++nt) {
        if (!one_turn) angles_of_step(nt, j, cs);
        rotate_step(nt, j, cs, sign[nt]);
      }
    }
  };

  // The anchor moves on by `span`: queries held in fp32 are turned back by as much where they are.
  auto advance_queries = [&]() {
#pragma unroll
    for (int j = 0; j < KH; ++j)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float4 cs = lds128(angles_addr + kAngles * kAngleBytes + (16 * j + 2 * t + 8 * r) * 8);      // c, c', s, s'  (an even row)
#pragma unroll
        for (int nt = 0; nt < (FP8 ? 0 : NT); ++nt) {
          float &l0 = qt[nt][j][2 * r], &l1 = qt[nt][j][2 * r + 1], &h0 = qt[nt][j + KH][2 * r], &h1 = qt[nt][j + KH][2 * r + 1];
          const float a0 = fmaf(l0, cs.x, h0 * cs.z), b0 = fmaf(h0, cs.x, -(l0 * cs.z)), a1 = fmaf(l1, cs.y, h1 * cs.w), b1 = fmaf(h1, cs.y, -(l1 * cs.w));
          l0 = a0; h0 = b0; l1 = a1; h1 = b1;
        }
      }
  };

  int stage = 0;
  uint32_t parity = 0;
  for (int it = 0; it < n_tiles; ++it) {
    if (c_block != u_block || c_head != u_head) {
      flush();
      u_block = c_block; u_head = c_head;
      anchor = INT_MIN; v_unit = kFirstUnit; v_least = kLeastUnit;
      const int first = (u_block % p.blocks) * p.beams, nb = min(p.beams, p.width - first);
      all_beams = nb == 32 ? ~0u : (1u << nb) - 1;
      const int row0 = u_block / p.blocks * p.width + first;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {                       // a column that is none repeats the first: nobody looks at it
        const int col = 8 * nt + g < nb * G ? 8 * nt + g : 0, row = row0 + col / G;
        const int at = max(plain(p.q_pos + row), kNowhere + 1);
        q_at[nt] = plain(p.lens + row) > 0 ? at : kNowhere;     // a row without slots: nobody's position
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int beam = (8 * nt + 2 * t + c) / G;
          see[nt][c] = beam < nb ? 1u << beam : 0u;
        }
        m_neg[nt] = make_float2(FLT_MAX, FLT_MAX); l_run[nt] = make_float2(0.f, 0.f);
#pragma unroll
        for (int db = 0; db < NV; ++db) { acc[nt][db][0] = 0.f; acc[nt][db][1] = 0.f; acc[nt][db][2] = 0.f; acc[nt][db][3] = 0.f; }
      }
    }
    int pos, n_valid, unused;
    unsigned beams;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(pos), "=r"(beams), "=r"(n_valid), "=r"(unused) : "r"(meta + stage * 16) : "memory");
    auto beyond = [&]() { return anchor == INT_MIN || static_cast<unsigned>(pos - anchor) > static_cast<unsigned>(span - kTile); };
    bool moves = beyond();
    if constexpr (FP8) {
      if (moves) { pos += last_filled(n_valid); moves = beyond(); }
    }
    if (moves) {
      const bool on = !FP8 && anchor != INT_MIN && pos - anchor == span && span <= p.max_position;
      anchor = pos;
      if (on) advance_queries();
      else rotate_queries();
    }
    if (!mbar_wait_bounded(smem_u32(&bars[stage]), parity, p.spin_limit)) {
      // Give the copies still in flight a last bounded chance to land, then leave cleanly.
      if (lane == 0) atomicOr(p.status, MEPIC_DEV_WAIT_EXPIRED);
      for (int s = 0; s < kStages; ++s) mbar_wait_bounded(smem_u32(&bars[s]), s == stage ? parity : (s < stage ? parity ^ 1u : parity), p.spin_limit);
      return;
    }
    const uint32_t ks_addr = smem_u32(stage0 + stage * kStageBytes), vs_addr = ks_addr + KB * kBlockBytes;
    // slots past the filled ones may hold anything: their P is 0, but 0 x NaN is NaN, so V must be finite there
    if (n_valid < kTile) {
      for (int idx = max(n_valid, 0) * 8 * KB + lane; idx < kTile * 8 * KB; idx += 32) {
        const int key = idx / (8 * KB), chk = idx % (8 * KB);
        const uint32_t a = vs_addr + (chk / 8) * kBlockBytes + key * 128 + (((chk % 8) ^ (key & 7)) << 4);
        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(a), "r"(0) : "memory");
      }
      // these generic-proxy stores must be ordered before the TMA (async proxy) write that refills this stage
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    }
    // ---- S^T = K' Q'^T
    float sc[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) { sc[nt][0] = 0.f; sc[nt][1] = 0.f; sc[nt][2] = 0.f; sc[nt][3] = 0.f; }
    // Addresses: stages and rows of angles begin at multiples of 128 bytes, so that a chunk's place under the swizzle is the first
    // chunk's with its number XORed in, and the second key's row of angles a fixed distance from the first's.
    const int at = pos - anchor + keyA;
    const uint32_t cs0 = angles_addr + at * kAngleBytes + ((16 * t) ^ ((at & 1) << 6)), cs1 = cs0 ^ 64;
    constexpr int kRowB = (FP8 ? 2 : 8) * kAngleBytes;
    const uint32_t k0 = ks_addr + k_lane, v0 = vs_addr + v_lane;
#pragma unroll
    for (int j = 0; j < KH; ++j) {
      uint32_t lo[4], hi[4];      // A fragments of k-steps j, j + KH: [key A, key B | key A, key B (second column half)]
      if constexpr (FP8) {
        uint32_t raw[4];          // [key A, key B of chunk j | of chunk j + KH], four dims each
        ldmatrix_x4(raw, k0 ^ (j << 4));
        e4m3x4_to_f16x2x2(raw[0], lo[0], lo[2]);
        e4m3x4_to_f16x2x2(raw[1], lo[1], lo[3]);
        e4m3x4_to_f16x2x2(raw[2], hi[0], hi[2]);
        e4m3x4_to_f16x2x2(raw[3], hi[1], hi[3]);
        const uint32_t cs_at = (j & 1 ? cs1 : cs0) + 128 * (j >> 1);
        const float4 ca = lds128(cs_at), cb = lds128(cs_at + kRowB);
        const uint32_t cc[4] = {__float_as_uint(ca.x), __float_as_uint(cb.x), __float_as_uint(ca.z), __float_as_uint(cb.z)};
        const uint32_t ss[4] = {__float_as_uint(ca.y), __float_as_uint(cb.y), __float_as_uint(ca.w), __float_as_uint(cb.w)};
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const uint32_t a = lo[f], b = hi[f];
          lo[f] = f16x2_fma(a, cc[f], f16x2_neg(f16x2_mul(b, ss[f])));
          hi[f] = f16x2_fma(a, ss[f], f16x2_mul(b, cc[f]));
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_f16(sc[nt], lo[0], lo[1], lo[2], lo[3], qf[nt][j][0], qf[nt][j][1]);
          mma_f16(sc[nt], hi[0], hi[1], hi[2], hi[3], qf[nt][j + KH][0], qf[nt][j + KH][1]);
        }
      } else {
        float2 kx[4], ky[4];      // the same four places of either k-step, rotated, in fp32
        ldmatrix_x4(lo, k0 ^ (j % 4 << 5));      // chunks 2 j and 2 j + 1 of the lower half of the dims, and of the upper
        ldmatrix_x4(hi, D == 128 ? (k0 ^ (j << 5)) + kBlockBytes : k0 ^ ((j + KH) << 5));
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const int r = f >> 1;
          const float4 cs = lds128((r ? cs1 : cs0) + 128 * j + (f & 1) * kRowB);      // c, c', s, s'
          const float2 a = bf16x2_to_float2(lo[f]), b = bf16x2_to_float2(hi[f]);
          const float2 x = make_float2(fmaf(a.x, cs.x, -(b.x * cs.z)), fmaf(a.y, cs.y, -(b.y * cs.w)));
          const float2 y = make_float2(fmaf(a.x, cs.z, b.x * cs.x), fmaf(a.y, cs.w, b.y * cs.y));
          kx[f] = x; ky[f] = y;
        }
        // one k-step of 16 dims is two of eight: a lane's two neighbouring dims stand at places t and t + 4
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            mma_tf32(sc[nt], kx[2 * r].x, kx[2 * r + 1].x, kx[2 * r].y, kx[2 * r + 1].y, qt[nt][j][2 * r], qt[nt][j][2 * r + 1]);
            mma_tf32(sc[nt], ky[2 * r].x, ky[2 * r + 1].x, ky[2 * r].y, ky[2 * r + 1].y, qt[nt][j + KH][2 * r], qt[nt][j + KH][2 * r + 1]);
          }
      }
    }
    // ---- online softmax (log2 domain): keys A (0, 1) and B (2, 3) of columns 2t (0, 2) and 2t + 1 (1, 3)
    // (`some`: not all columns hold the page, or their weights cannot carry its V scale.  The same in every lane: the vote says so to the
    // compiler)
    bool some = (beams & all_beams) != all_beams;
    float v_rel = 1.f, s_scale = FP8 ? p.scale_log2 : p.scale_log2 * kTf32Cut;
    if constexpr (FP8) {
      float ks, vs;
      asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(scl + stage * 8) : "memory");
      s_scale *= ks;
      // A page that all columns hold, with a V scale near the unit: the weights carry it into the product.  Any other: the product is made
      // with the weights alone and multiplied by the scale in fp32, where it is added.  So no page has a say in the precision of
      // columns that do not hold it, nor one of little weight in that of the others: it moves the unit at most, by a power of two.
      // (One reference for all weights, the largest scale met, left of a weight of 0.01 nothing behind a page with a scale 1e10 times
      // the others'.)
      auto over = [](float unit) { return __int_as_float(0x7f000000 - __float_as_int(unit)); };      // 1 / a power of two
      const float size = fabsf(vs);
      v_rel = vs * over(v_unit);
      if (!(size < 4.f * v_unit && size >= 0.25f * v_unit)) {
        const float order = fminf(__int_as_float(__float_as_int(size) & 0x7f800000), kMostUnit);      // (infinity, NaN: no unit follows them)
        if (size <= FLT_MAX) v_least = fmaxf(v_least, order * kBelowTop);
        const float unit = fmaxf(some || !(size <= FLT_MAX) ? v_unit : order, v_least);
        if (unit != v_unit) {
          const float f = v_unit * over(unit);
          v_unit = unit;
          v_rel = vs * over(unit);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int db = 0; db < NV; ++db) { acc[nt][db][0] *= f; acc[nt][db][1] *= f; acc[nt][db][2] *= f; acc[nt][db][3] *= f; }
        }
        some = some || !(size < 4.f * v_unit && size >= 0.25f * v_unit);
      }
    }
    some = __any_sync(kFull, some);
    // d: the scores less the reference, of keys A (0) and B (1)
    float2 d[NT][2];
    const float2 s_scale2 = make_float2(s_scale, s_scale);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      d[nt][0] = fma2(make_float2(sc[nt][0], sc[nt][1]), s_scale2, m_neg[nt]);
      d[nt][1] = fma2(make_float2(sc[nt][2], sc[nt][3]), s_scale2, m_neg[nt]);
    }
    if (n_valid < kTile) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (keyA >= n_valid) d[nt][0] = make_float2(-INFINITY, -INFINITY);
        if (keyB >= n_valid) d[nt][1] = make_float2(-INFINITY, -INFINITY);
      }
    }
    if (some) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (!(see[nt][0] & beams)) { d[nt][0].x = -INFINITY; d[nt][1].x = -INFINITY; }
        if (!(see[nt][1] & beams)) { d[nt][0].y = -INFINITY; d[nt][1].y = -INFINITY; }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) top = fmaxf(fmaxf(fmaxf(top, d[nt][0].x), fmaxf(d[nt][0].y, d[nt][1].x)), d[nt][1].y);
    // the references move only if some lane saw a score well above: any reference gives the same softmax as long as no weight
    // overflows (with 16 columns some column's largest score moves in two tiles of five, by little)
    if (__any_sync(kFull, top > kLag)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        // (once more from the scores: less a reference of -FLT_MAX nothing is left of them)
        auto score = [&](float less, float x) { return less == -INFINITY ? less : x * s_scale; };
        float mx0 = fmaxf(score(d[nt][0].x, sc[nt][0]), score(d[nt][1].x, sc[nt][2])), mx1 = fmaxf(score(d[nt][0].y, sc[nt][1]), score(d[nt][1].y, sc[nt][3]));
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) { mx0 = fmaxf(mx0, __shfl_xor_sync(kFull, mx0, o)); mx1 = fmaxf(mx1, __shfl_xor_sync(kFull, mx1, o)); }
        const float2 n = make_float2(fminf(m_neg[nt].x, -mx0), fminf(m_neg[nt].y, -mx1));
        const float a0 = ex2(n.x - m_neg[nt].x), a1 = ex2(n.y - m_neg[nt].y);
        m_neg[nt] = n;
        l_run[nt] = mul2(l_run[nt], make_float2(a0, a1));
#pragma unroll
        for (int db = 0; db < NV; ++db) { acc[nt][db][0] *= a0; acc[nt][db][1] *= a1; acc[nt][db][2] *= a0; acc[nt][db][3] *= a1; }
        auto less = [&](float was, float x, float m) { return was == -INFINITY ? was : fmaf(x, s_scale, m); };
        d[nt][0] = make_float2(less(d[nt][0].x, sc[nt][0], n.x), less(d[nt][0].y, sc[nt][1], n.y));
        d[nt][1] = make_float2(less(d[nt][1].x, sc[nt][2], n.x), less(d[nt][1].y, sc[nt][3], n.y));
      }
    }
    uint32_t pb[NT][2];                    // B fragments of P^T: the transposes of the two 8 x 8 blocks (key row, columns)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float2 pa = make_float2(ex2(d[nt][0].x), ex2(d[nt][0].y)), pc = make_float2(ex2(d[nt][1].x), ex2(d[nt][1].y));
      l_run[nt] = add2(l_run[nt], add2(pa, pc));
      if constexpr (FP8) {
        const float v = some ? kWeight : v_rel * kWeight;
        const float2 v2 = make_float2(v, v);
        pa = mul2(pa, v2); pc = mul2(pc, v2);
        pb[nt][0] = movmatrix_trans(pack_f16x2(pa.x, pa.y));
        pb[nt][1] = movmatrix_trans(pack_f16x2(pc.x, pc.y));
      } else {
        pb[nt][0] = movmatrix_trans(pack_bf16x2(pa.x, pa.y));
        pb[nt][1] = movmatrix_trans(pack_bf16x2(pc.x, pc.y));
      }
    }
    // ---- O^T += V^T P^T
    auto v_block = [&](int db, uint32_t (&va)[4]) {      // a0 dims g x keys 0-7, a1 dims g+8 x keys 0-7, a2 dims g x keys 8-15, a3 dims g+8 x keys 8-15
      ldmatrix_x4_trans(va, (v0 ^ (db % 4 << 5)) + db / 4 * kBlockBytes);
    };
    auto v_blocks = [&](int c, uint32_t (&va)[2][4]) {      // 8-bit pages: dim blocks c and c + 1, keys 4t .. 4t+3 a lane
      uint32_t raw[4];          // [block c: dim g, dim g + 8 | block c + 1: the same]
      ldmatrix_b8_trans_x2(raw, v0 ^ (c << 4));
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        e4m3x4_to_f16x2x2(raw[2 * m], va[m][0], va[m][2]);
        e4m3x4_to_f16x2x2(raw[2 * m + 1], va[m][1], va[m][3]);
      }
    };
    auto mma = [&](float (&d)[4], const uint32_t (&va)[4], const uint32_t (&b)[2]) {
      if constexpr (FP8) mma_f16(d, va[0], va[1], va[2], va[3], b[0], b[1]);
      else mma_bf16(d, va[0], va[1], va[2], va[3], b[0], b[1]);
    };
    auto each_block = [&](auto use) {
#pragma unroll
      for (int db = 0; db < NV; db += 2) {
        uint32_t va[2][4];
        if constexpr (FP8) v_blocks(db, va);
        else { v_block(db, va[0]); v_block(db + 1, va[1]); }
        use(db, va[0]);
        use(db + 1, va[1]);
      }
    };
    if (!some) {
      each_block([&](int db, const uint32_t (&va)[4]) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma(acc[nt][db], va, pb[nt]);
      });
    } else {
      each_block([&](int db, const uint32_t (&va)[4]) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[4] = {0.f, 0.f, 0.f, 0.f};
          mma(x, va, pb[nt]);
          if constexpr (FP8) {
            if (see[nt][0] & beams) { acc[nt][db][0] = fmaf(x[0], v_rel, acc[nt][db][0]); acc[nt][db][2] = fmaf(x[2], v_rel, acc[nt][db][2]); }
            if (see[nt][1] & beams) { acc[nt][db][1] = fmaf(x[1], v_rel, acc[nt][db][1]); acc[nt][db][3] = fmaf(x[3], v_rel, acc[nt][db][3]); }
          } else {
            if (see[nt][0] & beams) { acc[nt][db][0] += x[0]; acc[nt][db][2] += x[2]; }
            if (see[nt][1] & beams) { acc[nt][db][1] += x[1]; acc[nt][db][3] += x[3]; }
          }
        }
      });
    }
    __syncwarp();   // every lane is done with this stage
    if (issued < n_tiles) issue(stage);
    __syncwarp();
    if (--c_left == 0) {
      if (next_unit(p, c_block, c_head))
        c_left = static_cast<int>(min(static_cast<long long>(begin_of(p, c_block + 1) - begin_of(p, c_block)) << p.log2_tpp, static_cast<long long>(INT_MAX)));
    }
    if (++stage == kStages) { stage = 0; parity ^= 1u; }
  }
  flush();
}

// ---------------------------------------------------------------- merge
// PER warps a (unit, column): the column's partials are dealt round to them, a lane owns D / 32 output dims.  Each warp joins its
// own partials against the largest reference among them, and the PER results are joined in order.  Few partials a unit (a batch):
// one warp (32 x 4 beams, attention and merge: 165 us against 167 with four); many (one long request): four.
constexpr int kMergeWarps = 8;
template <int D, int PER>
__global__ void __launch_bounds__(kMergeWarps * 32) mepic_beam_merge(const __grid_constant__ BeamParams p) {
  constexpr int E = D / 32;
  const int unit = blockIdx.x, wv = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = wv % PER;
  const int col = blockIdx.y * (kMergeWarps / PER) + wv / PER;
  __shared__ float sh_m[kMergeWarps], sh_l[kMergeWarps];
  __shared__ float sh_o[kMergeWarps][D];
  const int block = unit / p.n_kv_heads, head = unit - block * p.n_kv_heads, group = block / p.blocks;
  const int beam = (block - group * p.blocks) * p.beams + col / p.group_size;
  const bool live = col < p.columns && beam < p.width;
  const size_t row = static_cast<size_t>(group) * p.width + (live ? beam : 0);
  const bool fits = plan_fits(p);
  if (!fits && unit == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.status, MEPIC_DEV_BAD_PLAN);
  long long w0 = 0, w1 = -1;
  bool shows = false;
  if (fits && live) {
    const Cut cut = cut_of_line(p);
    const int r0 = begin_of(p, block);
    const long long per = static_cast<long long>(begin_of(p, block + 1) - r0) << p.log2_tpp, begin = (static_cast<long long>(r0) << p.log2_tpp) * p.n_kv_heads + head * per;
    if (per > 0) { w0 = quotient(begin, cut.piece); w1 = quotient(begin + per - 1, cut.piece); }
    shows = __ldg(p.lens + row) > 0;
  }
  // launched as a programmatic dependent of the attention kernel: its partials are complete and visible after this
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float m = -FLT_MAX, l = 0.f, o[E];
#pragma unroll
  for (int i = 0; i < E; ++i) o[i] = 0.f;
  // 32 partials at a time, a lane each for their references and sums
  for (long long k0 = w0 + sub; k0 <= w1; k0 += 32 * PER) {
    const long long mine = k0 + static_cast<long long>(lane) * PER;
    const float2 ml = mine <= w1 ? p.part_ml[(unit + mine) * p.columns + col] : make_float2(-FLT_MAX, 0.f);
    float top = fmaxf(ml.x, m);
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
    const float wgt = mine <= w1 ? ex2(ml.x - top) : 0.f, was = ex2(m - top);
    float add = mine <= w1 ? ml.y * wgt : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(kFull, add, d);
    l = l * was + add;
    m = top;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= was;
    const int n = static_cast<int>(min((w1 - k0) / PER + 1, 32ll));
    for (int q = 0; q < n; q += 4) {      // four of them side by side; eight take registers that keep CTAs out: 32 x 4 beams 167 us against 165
      float x[4][E] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (q + k < n) {
          const float* src = p.part_o + ((unit + k0 + static_cast<long long>(q + k) * PER) * p.columns + col) * D + E * lane;
          if constexpr (E == 4) *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(src);
          else *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(src);
        }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = __shfl_sync(kFull, wgt, (q + k) & 31);      // (0 past the last)
        if (q + k < n) {
#pragma unroll
          for (int i = 0; i < E; ++i) o[i] += x[k][i] * w;
        }
      }
    }
  }
  if constexpr (PER > 1) {
    if (lane == 0) { sh_m[wv] = m; sh_l[wv] = l; }
#pragma unroll
    for (int i = 0; i < E; ++i) sh_o[wv][E * lane + i] = o[i];
    __syncthreads();
    if (sub != 0) return;
    float top = m;
#pragma unroll
    for (int q = 1; q < PER; ++q) top = fmaxf(top, sh_m[wv + q]);
    float f = ex2(m - top);
    l *= f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= f;
#pragma unroll
    for (int q = 1; q < PER; ++q) {
      f = ex2(sh_m[wv + q] - top);
      l += sh_l[wv + q] * f;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] += sh_o[wv + q][E * lane + i] * f;
    }
  }
  if (!live) return;
  // l = 0 where the row has slots: every score is -infinity, 0 / 0
  uint32_t bits[E / 2];
#pragma unroll
  for (int i = 0; i < E; i += 2)
    bits[i / 2] = static_cast<uint32_t>(f32_to_bf16_bits(shows ? o[i] / l : 0.f)) | static_cast<uint32_t>(f32_to_bf16_bits(shows ? o[i + 1] / l : 0.f)) << 16;
  uint16_t* dst = p.out + (row * p.n_kv_heads * p.group_size + static_cast<size_t>(head) * p.group_size + col % p.group_size) * D + E * lane;
  if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(bits[0], bits[1]);
  else *reinterpret_cast<uint32_t*>(dst) = bits[0];
}

// ---------------------------------------------------------------- host side
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
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
// Warps of a CTA.  bf16 pages: HBM is the bound, and more tiles under way than those of eight warps make it slower (12 warps, which
// spill besides: 226 us against 181 on 32 x 4 beams over 8,300 slots).  8-bit pages are bound by instructions and their latency: twelve
// (122 us against 130 on 8 x 4 beams over 33,000 slots).
constexpr int kMaxWarps = 12;
template <bool FP8> constexpr int warps_of = FP8 ? kMaxWarps : 8;
size_t slots_of(const PlanShape& s, int n_kv_heads, int sms) { return static_cast<size_t>(s.groups) * s.blocks * n_kv_heads + static_cast<size_t>(sms) * kMaxWarps; }
size_t workspace_bytes(const mepic_config_t* cfg, const PlanShape& s, int sms) {
  const size_t columns = static_cast<size_t>(s.beams) * (cfg->n_q_heads / cfg->n_kv_heads);
  return slots_of(s, cfg->n_kv_heads, sms) * columns * (cfg->head_dim + 2) * sizeof(float);
}

template <int D, int NT, bool FP8>
int32_t launch_beam(BeamParams& p, int sms, int device, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t st) {
  constexpr int W = warps_of<FP8>;
  constexpr size_t smem = smem_bytes<D, FP8, W>;
  static_assert(smem <= 232448, "shared memory of a CTA");
  static std::atomic<unsigned long long> prepared{0};      // devices on which the limit is raised
  const unsigned long long bit = device < 64 ? 1ull << device : 0;
  cudaError_t e = cudaSuccess;
  if (!(prepared.load(std::memory_order_relaxed) & bit) || !bit) {
    e = cudaFuncSetAttribute(mepic_beam_attn<D, NT, FP8, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) { mepic_set_error("attn_beam: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
    prepared.fetch_or(bit, std::memory_order_relaxed);
  }
  p.workers = sms * W;
  e = launch_dependent(mepic_beam_attn<D, NT, FP8, W>, dim3(sms), dim3(W * 32), smem, st, p, map_k, map_v);
  if (e == cudaSuccess) e = cudaGetLastError();
  const int units = p.groups * p.blocks * p.n_kv_heads;
  if (e == cudaSuccess) {
    if (p.workers <= 16LL * units) e = launch_dependent(mepic_beam_merge<D, 1>, dim3(units, (p.columns + kMergeWarps - 1) / kMergeWarps), dim3(kMergeWarps * 32), st, p);
    else e = launch_dependent(mepic_beam_merge<D, 4>, dim3(units, (p.columns + kMergeWarps / 4 - 1) / (kMergeWarps / 4)), dim3(kMergeWarps * 32), st, p);
  }
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) { mepic_set_error("attn_beam: launch: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(2);
  return MEPIC_OK;
}

int32_t beam_call(const mepic_config_t* cfg, const mepic_attn_beam_args_t* a, const float* k_scales, const float* v_scales, bool fp8, void* cuda_stream) {
  const char* what = fp8 ? "attn_beam_fp8" : "attn_beam";
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("%s: NULL argument", what); return MEPIC_E_INVAL; }
  if (fp8 && cfg->head_dim != 128) { mepic_set_error("%s: head_dim %d: 8-bit pages are built for head_dim 128", what, cfg->head_dim); return MEPIC_E_INVAL; }
  PlanShape s;
  if (!plan_shape(cfg, a->groups, a->width, a->table_stride, what, &s)) return MEPIC_E_INVAL;
  if (!a->q || !a->q_pos || !a->plan || !a->k_pool || !a->v_pool || !a->rope_table || !a->out || !a->workspace || !a->status) {
    mepic_set_error("%s: NULL pointer argument", what); return MEPIC_E_INVAL;
  }
  if (fp8 && (!k_scales || !v_scales)) { mepic_set_error("%s: NULL scale pointer", what); return MEPIC_E_INVAL; }
  if (!aligned16(a->q) || !aligned16(a->plan) || !aligned16(a->k_pool) || !aligned16(a->v_pool) || !aligned16(a->rope_table) || !aligned16(a->out) || !aligned16(a->workspace)) {
    mepic_set_error("%s: pointers must be 16-byte aligned", what); return MEPIC_E_INVAL;
  }
  const long long packed = static_cast<long long>(cfg->n_q_heads) * cfg->head_dim, q_stride = a->q_stride ? a->q_stride : packed;
  if (packed > 0x7fffffffLL || q_stride < packed || q_stride % 8) { mepic_set_error("%s: q_stride %d must be 0 or a multiple of 8 of at least a packed row", what, a->q_stride); return MEPIC_E_INVAL; }
  if (static_cast<long long>(s.groups) * s.blocks * cfg->n_kv_heads > 0x7fffffffLL) { mepic_set_error("%s: too many beams and heads", what); return MEPIC_E_INVAL; }
  int device = 0;
  const int sms = sm_count(&device);
  if (sms <= 0) { mepic_set_error("%s: no CUDA device", what); return MEPIC_E_CUDA; }
  const size_t need = workspace_bytes(cfg, s, sms);
  if (a->workspace_bytes < need) { mepic_set_error("%s: workspace of %zu bytes, %zu needed", what, a->workspace_bytes, need); return MEPIC_E_INVAL; }
  BeamParams p;
  p.q = static_cast<const uint16_t*>(a->q); p.q_pos = a->q_pos;
  p.head = static_cast<const int32_t*>(a->plan);
  p.sums = p.head + kHead; p.lens = p.head + s.off_len;
  p.records = reinterpret_cast<const int4*>(p.head + s.off_rec);
  p.rope = a->rope_table; p.k_scales = k_scales; p.v_scales = v_scales;
  p.out = static_cast<uint16_t*>(a->out); p.status = a->status;
  p.groups = s.groups; p.width = s.width; p.stride = a->table_stride; p.blocks = s.blocks; p.beams = s.beams; p.segments = s.segments;
  p.group_size = cfg->n_q_heads / cfg->n_kv_heads; p.columns = s.beams * p.group_size;
  p.n_kv_heads = cfg->n_kv_heads; p.page_size = cfg->page_size; p.num_pages = cfg->num_pages; p.max_position = cfg->max_position;
  p.log2_tpp = 0;
  while ((kTile << p.log2_tpp) < cfg->page_size) ++p.log2_tpp;
  p.q_stride = static_cast<int>(q_stride);
  p.scale_log2 = a->sm_scale * 1.4426950408889634f;
  p.spin_limit = mepic_test_spin_limit(kSpinLimit); p.skip_tile = mepic_test_skip_tile();
  p.part_o = static_cast<float*>(a->workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + slots_of(s, cfg->n_kv_heads, sms) * p.columns * cfg->head_dim);
  alignas(64) CUtensorMap map_k, map_v;
  int32_t rc = fp8 ? mepic_make_pool_map_u8(cfg, a->k_pool, &map_k) : mepic_make_pool_map_halves(cfg, a->k_pool, &map_k);
  if (rc == MEPIC_OK) rc = fp8 ? mepic_make_pool_map_u8(cfg, a->v_pool, &map_v) : mepic_make_pool_map_halves(cfg, a->v_pool, &map_v);
  if (rc != MEPIC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool two = p.columns > 8;      // tiles of eight columns
  if (fp8) return two ? launch_beam<128, 2, true>(p, sms, device, map_k, map_v, st) : launch_beam<128, 1, true>(p, sms, device, map_k, map_v, st);
  if (cfg->head_dim == 128) return two ? launch_beam<128, 2, false>(p, sms, device, map_k, map_v, st) : launch_beam<128, 1, false>(p, sms, device, map_k, map_v, st);
  return two ? launch_beam<64, 2, false>(p, sms, device, map_k, map_v, st) : launch_beam<64, 1, false>(p, sms, device, map_k, map_v, st);
}

}  // namespace

extern "C" size_t mepic_beam_plan_bytes(const mepic_config_t* cfg, int32_t groups, int32_t width, int32_t table_stride) {
  PlanShape s;
  return mepic_config_ok(cfg) && plan_shape(cfg, groups, width, table_stride, "beam_plan", &s) ? s.bytes : 0;
}

extern "C" int32_t mepic_beam_plan(const mepic_config_t* cfg, const mepic_beam_plan_args_t* a, void* cuda_stream) {
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("beam_plan: NULL argument"); return MEPIC_E_INVAL; }
  PlanShape s;
  if (!plan_shape(cfg, a->groups, a->width, a->table_stride, "beam_plan", &s)) return MEPIC_E_INVAL;
  if (!a->page_ids || !a->pos_base || !a->kv_len || !a->plan || !a->status) { mepic_set_error("beam_plan: NULL pointer argument"); return MEPIC_E_INVAL; }
  if (!aligned16(a->plan)) { mepic_set_error("beam_plan: the plan must be 16-byte aligned"); return MEPIC_E_INVAL; }
  if (a->plan_bytes < s.bytes) { mepic_set_error("beam_plan: a plan of %zu bytes, %zu needed", a->plan_bytes, s.bytes); return MEPIC_E_INVAL; }
  if (s.segments > 65535) { mepic_set_error("beam_plan: table_stride %d is too large", a->table_stride); return MEPIC_E_INVAL; }
  PlanParams p;
  p.page_ids = a->page_ids; p.pos_base = a->pos_base; p.kv_len = a->kv_len; p.status = a->status;
  p.head = static_cast<int32_t*>(a->plan);
  p.sums = p.head + kHead; p.lens = p.head + s.off_len;
  p.records = reinterpret_cast<int4*>(p.head + s.off_rec);
  p.stride = a->table_stride; p.groups = s.groups; p.width = s.width; p.blocks = s.blocks; p.beams = s.beams; p.segments = s.segments;
  p.page_shift = 0;
  while ((1 << p.page_shift) < cfg->page_size) ++p.page_shift;
  p.num_pages = cfg->num_pages; p.group_size = cfg->n_q_heads / cfg->n_kv_heads; p.n_kv_heads = cfg->n_kv_heads;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const size_t smem = static_cast<size_t>(s.beams) * kSeg * 3 * sizeof(int);
  cudaError_t e = cudaSuccess;
  // always the largest: another thread's call may need more than this one
  if (smem > 40 * 1024) e = cudaFuncSetAttribute(mepic_beam_plan_classes, cudaFuncAttributeMaxDynamicSharedMemorySize, MEPIC_BEAM_MAX_WIDTH * kSeg * 3 * static_cast<int>(sizeof(int)));
  if (e != cudaSuccess) { mepic_set_error("beam_plan: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_beam_plan_classes<<<dim3(static_cast<unsigned>(s.groups) * s.blocks, s.segments), kSeg, smem, st>>>(p);
  e = cudaGetLastError();
  const bool sums = static_cast<long long>(s.groups) * s.blocks * s.segments > 1;
  if (e == cudaSuccess && sums) e = launch_dependent(mepic_beam_plan_sums, dim3(1), dim3(kScanThreads), st, p);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) { mepic_set_error("beam_plan: launch: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(sums ? 2 : 1);
  return MEPIC_OK;
}

extern "C" size_t mepic_attn_beam_workspace(const mepic_config_t* cfg, int32_t groups, int32_t width) {
  PlanShape s;
  if (!mepic_config_ok(cfg) || !plan_shape(cfg, groups, width, 1, "attn_beam_workspace", &s)) return 0;
  int device = 0;
  const int sms = sm_count(&device);
  if (sms <= 0) { mepic_set_error("attn_beam_workspace: no CUDA device"); return 0; }
  return workspace_bytes(cfg, s, sms);
}
extern "C" int32_t mepic_attn_beam(const mepic_config_t* cfg, const mepic_attn_beam_args_t* args, void* cuda_stream) {
  return beam_call(cfg, args, nullptr, nullptr, false, cuda_stream);
}
extern "C" int32_t mepic_attn_beam_fp8(const mepic_config_t* cfg, const mepic_attn_beam_args_t* args, const float* k_scales, const float* v_scales,
                                       void* cuda_stream) {
  return beam_call(cfg, args, k_scales, v_scales, true, cuda_stream);
}
