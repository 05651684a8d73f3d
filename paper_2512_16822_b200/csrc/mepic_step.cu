// The integer side of a step with drafted tokens, and the commit of its rows: layout of the trees, acceptance, block tables
// and slot maps from lengths, K/V rows into their physical slots (see "drafted tokens" in mepic.h).
//
// The first three move kilobytes: what they cost is launch latency plus one chain of dependent loads, so each is ONE launch,
// reads its inputs once, side by side, and does everything that depends on them in shared memory.  The commit is a copy.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "mepic.h"
#include "mepic_internal.h"
#include "mepic_ptx.cuh"
#include "mepic_rows.cuh"
#include "mepic_tcgen05.cuh"      // arithmetic on pairs of floats

namespace {

using namespace mepic_dev;

// ---------------------------------------------------------------- tree layout
// One CTA per request.  Ancestors by doubling: every row starts with its own bit and a pointer to its parent; in a round it
// takes over the bits of the row it points to and then points where that row pointed, so after k rounds it holds its 2^k
// nearest ancestors and log2(depth) rounds do.  (A thread per row walking up its chain took 8 us on trees of 200 rows and
// depth 45.)  A row may read another's words while those grow: they only ever hold true ancestors, so whatever it reads is
// right, and the pointers, of which that is not so, are kept twice.  The depth is the number of bits.
// Bound by latency: 2.3 us for one tree of 8 rows, 5.4 us for 128 trees of 200 rows (device time, calls replayed in a graph).
constexpr int kLayoutThreads = 512;
__global__ void __launch_bounds__(kLayoutThreads) mepic_tree_layout_kernel(const mepic_tree_layout_args_t a, int page_shift) {
  __shared__ int16_t up[2][MEPIC_TREE_MAX_ROWS];
  extern __shared__ uint32_t bits[];             // [32 mask_words][mask_words]
  const int b = blockIdx.x, tid = threadIdx.x, W = a.mask_words;
  const RowRange rr = rows_of(a.row_offsets, b, a.total_rows, 0x7fffffff);
  int kvl = __ldg(a.kv_len + b);
  const int n = min(rr.n, 32 * W);
  bool bad = rr.bad || rr.n > n;
  const float inv_w = 1.f / static_cast<float>(W);      // k / W = int((k + 1/2) inv_w) for every k below 2^15 here
  for (int i = tid; i < n; i += kLayoutThreads) {
    int p = __ldg(a.parent + rr.lo + i);
    if (p < -1 || p >= i) { bad = true; p = -1; }
    up[0][i] = static_cast<int16_t>(p);
  }
  for (int k = tid; k < n * W; k += kLayoutThreads) {
    const int r = static_cast<int>((static_cast<float>(k) + 0.5f) * inv_w);
    bits[k] = (r >> 5) == k - r * W ? 1u << (r & 31) : 0u;
  }
  if (bad) atomicOr(a.status, MEPIC_DEV_BAD_TREE);
  const long long room = static_cast<long long>(a.table_stride) << page_shift;
  if (kvl < 0 || kvl > room) {
    if (tid == 0) atomicOr(a.status, MEPIC_DEV_BAD_SLOT);
    kvl = kvl < 0 ? 0 : static_cast<int>(room);
  }
  int next = 0;
  if (kvl > 0) next = __ldg(a.pos_base + static_cast<size_t>(b) * a.table_stride + ((kvl - 1) >> page_shift)) + ((kvl - 1) & ((1 << page_shift) - 1)) + 1;
  __syncthreads();
  for (int from = 0, more = n > 0; more; from ^= 1) {
    for (int k = tid; k < n * W; k += kLayoutThreads) {
      const int r = static_cast<int>((static_cast<float>(k) + 0.5f) * inv_w), w = k - r * W;
      const int u = up[from][r];
      if (u >= 0 && w <= (u >> 5)) bits[k] |= *reinterpret_cast<volatile uint32_t*>(bits + u * W + w);      // ancestors of u lie in words up to u's
    }
    bool left = false;
    for (int i = tid; i < n; i += kLayoutThreads) {
      const int u = up[from][i], to = u >= 0 ? up[from][u] : -1;
      up[from ^ 1][i] = static_cast<int16_t>(to);
      left = left || to >= 0;
    }
    more = __syncthreads_or(left);
  }
  int32_t* out = a.tree_mask + static_cast<size_t>(rr.lo) * W;
  for (int k = tid; k < n * W; k += kLayoutThreads) out[k] = static_cast<int32_t>(bits[k]);
  for (int i = tid; i < n; i += kLayoutThreads) {
    int depth = -1;
    for (int w = 0; w <= (i >> 5); ++w) depth += __popc(bits[i * W + w]);
    a.row_pos[rr.lo + i] = next + depth;
  }
  for (long long i = n + tid; i < rr.n; i += kLayoutThreads) {      // rows the mask has no room for (reported)
    for (int w = 0; w < W; ++w) out[static_cast<size_t>(i) * W + w] = 0;
    a.row_pos[rr.lo + i] = next;
  }
}

// ---------------------------------------------------------------- acceptance
// One CTA per request.  Whether a row fits (its draft is the choice made at its parent) does not depend on the path, so all
// rows are tested at once and each parent keeps its first fitting child (a minimum: no order of the atomics changes it);
// the path is then a walk down those children in shared memory.  Bound by latency: 2.5 us for one tree of 8 rows, 2.7 us for
// 256 trees of 64 rows; the walk is a shared-memory load per accepted row.
constexpr int kAcceptThreads = 128;
__global__ void __launch_bounds__(kAcceptThreads) mepic_tree_accept_kernel(const mepic_tree_accept_args_t a) {
  __shared__ int child[MEPIC_TREE_MAX_ROWS + 1];       // [0]: of the context, [i + 1]: of row i
  __shared__ int target[MEPIC_TREE_MAX_ROWS];
  __shared__ int path[MEPIC_TREE_MAX_ROWS];
  __shared__ int path_n;
  const int b = blockIdx.x, tid = threadIdx.x;
  const RowRange rr = rows_of(a.row_offsets, b, a.total_rows, MEPIC_TREE_MAX_ROWS);
  bool bad = rr.bad;
  const int root = __ldg(a.root + b);
  for (int i = tid; i <= rr.n; i += kAcceptThreads) {
    child[i] = 0x7fffffff;
    if (i < rr.n) target[i] = __ldg(a.target + rr.lo + i);
  }
  __syncthreads();
  for (int i = tid; i < rr.n; i += kAcceptThreads) {
    const int p = __ldg(a.parent + rr.lo + i), d = __ldg(a.draft + rr.lo + i);
    if (p < -1 || p >= i) { bad = true; continue; }
    if (d == (p < 0 ? root : target[p])) atomicMin(&child[p + 1], i);
  }
  if (bad) atomicOr(a.status, MEPIC_DEV_BAD_TREE);
  __syncthreads();
  if (tid == 0) {
    int n = 0, at = child[0];
    while (at != 0x7fffffff && n < a.max_accept) { path[n++] = at; at = child[at + 1]; }      // children follow their parents: at most rr.n steps
    path_n = n;
    a.n_accept[b] = n;
    a.next_token[b] = n > 0 ? target[path[n - 1]] : root;
  }
  __syncthreads();
  const int n = path_n;
  for (long long k = tid; k < a.max_accept; k += kAcceptThreads)       // (any int32 length: counters that step past it are 64 bits wide)
    a.accept_rows[static_cast<size_t>(b) * a.max_accept + k] = k < n ? rr.lo + path[k] : -1;
}

// ---------------------------------------------------------------- step tables
// Every CTA scans all requests' lengths (a few kilobytes out of L2) and keeps the running sums of rows and new pages in
// shared memory; it then writes its share of the outputs, which all follow from those sums, by binary search.  No CTA reads
// what another writes: an appended row's page comes from the table only where the entry existed before the call.  (One CTA
// for the sums and a second launch for the rest would cost a launch, 2 us, to save a scan of a few hundred loads.)  Bound by
// latency: 4.0 us for 32 requests that gain 4 slots each, 4.7 us for 64 prompts of up to 2,048 rows.
constexpr int kTablesThreads = 512;
__device__ __forceinline__ int find_request(const int* off, int batch, int r) {       // the b with off[b] <= r < off[b + 1]
  int lo = 0, hi = batch;                       // off[lo] <= r < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}
__global__ void __launch_bounds__(kTablesThreads) mepic_step_tables_kernel(const mepic_step_tables_args_t a, int page_shift, int num_pages) {
  extern __shared__ int sh[];
  int* row_off = sh;                            // [batch + 1]
  int* page_off = sh + a.batch + 1;             // [batch + 1]
  __shared__ long long warp_rows[kTablesThreads / 32], warp_pages[kTablesThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int P = 1 << page_shift;
  const long long room = min(static_cast<long long>(a.table_stride) << page_shift, 0x7fffffffll);       // lengths are int32
  auto entries = [&](long long len) { return static_cast<int>((len + P - 1) >> page_shift); };        // table entries of `len` slots
  const int used = __ldg(a.reserve_used);
  // ---- sums: a thread owns `per` consecutive requests
  const int per = (a.batch + kTablesThreads - 1) / kTablesThreads, b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
  long long rows = 0, pages = 0;
  bool bad = used < 0;
  for (int b = b0; b < b1; ++b) {
    const long long kv = __ldg(a.kv_len + b), nn = __ldg(a.n_new + b);
    if (kv < 0 || nn < 0 || kv + nn > room) { bad = true; continue; }
    rows += nn;
    pages += entries(kv + nn) - entries(kv);
  }
  long long r_in = rows, p_in = pages;          // inclusive over the warp
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long r = __shfl_up_sync(kFull, r_in, d), p = __shfl_up_sync(kFull, p_in, d);
    if (lane >= d) { r_in += r; p_in += p; }
  }
  if (lane == 31) { warp_rows[warp] = r_in; warp_pages[warp] = p_in; }
  bad = __syncthreads_or(bad) != 0;
  long long r_at = r_in - rows, p_at = p_in - pages, r_all = 0, p_all = 0;
#pragma unroll
  for (int w = 0; w < kTablesThreads / 32; ++w) {
    if (w < warp) { r_at += warp_rows[w]; p_at += warp_pages[w]; }
    r_all += warp_rows[w]; p_all += warp_pages[w];
  }
  bad = bad || r_all > a.max_rows || used + p_all > a.n_reserve;        // the same answer in every thread of every CTA
  for (int b = b0; b < b1; ++b) {
    row_off[b] = bad ? 0 : static_cast<int>(r_at);
    page_off[b] = bad ? 0 : static_cast<int>(p_at);
    if (bad) continue;
    const long long kv = __ldg(a.kv_len + b), nn = __ldg(a.n_new + b);
    r_at += nn;
    p_at += entries(kv + nn) - entries(kv);
  }
  if (tid == 0) { row_off[a.batch] = bad ? 0 : static_cast<int>(r_all); page_off[a.batch] = bad ? 0 : static_cast<int>(p_all); }
  __syncthreads();
  const int n_rows = row_off[a.batch], n_pages = page_off[a.batch];
  const int gid = blockIdx.x * kTablesThreads + tid, step = gridDim.x * kTablesThreads;
  if (gid == 0) {
    if (bad) atomicOr(a.status, MEPIC_DEV_NO_PAGES);
    *a.reserve_used_out = used + n_pages;
    a.row_offsets[a.batch] = n_rows;
  }
  // ---- per request
  for (int b = gid; b < a.batch; b += step) {
    const int kv = __ldg(a.kv_len + b), end = kv + (row_off[b + 1] - row_off[b]);
    a.row_offsets[b] = row_off[b];
    a.kv_len_out[b] = end;
    if (a.q_pos) {
      int pos = -1;
      if (end > 0 && end <= room) {
        const int held = entries(kv), e = (end - 1) >> page_shift;
        const int32_t* base = a.pos_base + static_cast<size_t>(b) * a.table_stride;
        pos = (e < held ? base[e] : (held > 0 ? base[held - 1] + (e - held + 1) * P : e * P)) + ((end - 1) & (P - 1));
      }
      a.q_pos[b] = pos;
    }
  }
  // ---- per new table entry
  for (long long at = gid; at < n_pages; at += step) {
    const int t = static_cast<int>(at);
    const int b = find_request(page_off, a.batch, t);
    const int held = entries(__ldg(a.kv_len + b)), k = t - page_off[b];
    const int page = __ldg(a.reserve + used + t);
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(num_pages)) atomicOr(a.status, MEPIC_DEV_BAD_PAGE);
    const size_t row = static_cast<size_t>(b) * a.table_stride;
    a.page_ids[row + held + k] = page;
    a.pos_base[row + held + k] = held > 0 ? a.pos_base[row + held - 1] + (k + 1) * P : k * P;
  }
  // ---- per appended row
  if (!a.row_slot && !a.slot_map) return;
  for (long long at = gid; at < a.max_rows; at += step) {
    const int r = static_cast<int>(at);
    int slot = -1;
    long long phys = -1;
    if (r < n_rows) {
      const int b = find_request(row_off, a.batch, r);
      const int kv = __ldg(a.kv_len + b), held = entries(kv);
      slot = kv + r - row_off[b];
      const int e = slot >> page_shift;
      const int page = e < held ? a.page_ids[static_cast<size_t>(b) * a.table_stride + e] : __ldg(a.reserve + used + page_off[b] + e - held);
      if (static_cast<unsigned>(page) < static_cast<unsigned>(num_pages)) phys = (static_cast<long long>(page) << page_shift) + (slot & (P - 1));
      else atomicOr(a.status, MEPIC_DEV_BAD_PAGE);
    }
    if (a.row_slot) a.row_slot[r] = slot;
    if (a.slot_map) a.slot_map[r] = phys;
  }
}

// ---------------------------------------------------------------- commit of rows
struct CommitParams {
  const uint16_t* src[2];      // K, V
  void* pool[2];
  float* scales[2];
  const int32_t* row_offsets;
  const int64_t* slot_map;
  const int32_t* src_rows;
  int32_t* status;
  int src_stride, batch, max_rows, n_sources, kv_stride, n_kv_heads, page_size, page_shift;
  long long n_slots;           // num_pages * page_size
};

// Where appended row r comes from: the row itself, or the entry of src_rows that belongs to it.  -1: nowhere (reported).
// Called by a whole warp for one row.  The request is found 32 candidates at a time (the offsets ascend).
__device__ __forceinline__ int source_of(const CommitParams& p, int r, int lane) {
  int src = r;
  if (p.src_rows) {
    int lo = 0, n = p.batch;                    // the request is in [lo, lo + n)
    while (n > 1) {
      const int step = (n + 31) / 32, at = lo + lane * step;
      const bool below = lane * step < n && __ldg(p.row_offsets + at) <= r;
      const int k = 31 - __clz(__ballot_sync(kFull, below) | 1u);
      n = min(step, lo + n - (lo + k * step));
      lo += k * step;
    }
    const int k = r - __ldg(p.row_offsets + lo);
    src = k >= 0 && k < p.src_stride ? __ldg(p.src_rows + static_cast<size_t>(lo) * p.src_stride + k) : -1;
  }
  if (src < 0 || src >= p.n_sources) {
    if (lane == 0) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
    return -1;
  }
  return src;
}

// The same for one lane (a row of its own), and without a word where there is none.
__device__ __forceinline__ int lane_source_or_none(const CommitParams& p, int r) {
  int src = r;
  if (p.src_rows) {
    int lo = 0, hi = p.batch;                    // row_offsets[lo] <= r < row_offsets[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(p.row_offsets + mid) <= r) lo = mid; else hi = mid;
    }
    const int k = r - __ldg(p.row_offsets + lo);
    src = k >= 0 && k < p.src_stride ? __ldg(p.src_rows + static_cast<size_t>(lo) * p.src_stride + k) : -1;
  }
  return src < 0 || src >= p.n_sources ? -1 : src;
}

// bf16 pages: a warp per row, 16 bytes a lane, K and V together.  Bound by latency where it is used most: 128 accepted rows of
// 8 kv heads (0.8 MB) take 3.7 us, a launch and five dependent loads (row count, offsets search, offset, source, row); 12,900
// prompt rows (106 MB) 25 us, 4.3 TB/s.
constexpr int kCopyRows = 8;         // rows per CTA, one warp each
template <int D>
__global__ void __launch_bounds__(kCopyRows * 32) mepic_rows_commit_kernel(const __grid_constant__ CommitParams p) {
  constexpr int C = D / 8;           // 16-byte chunks per head row
  const int lane = threadIdx.x & 31;
  const unsigned at = blockIdx.x * kCopyRows + (threadIdx.x >> 5);
  const int owned = __ldg(p.row_offsets), n_rows = __ldg(p.row_offsets + p.batch);      // rows before the first request's are nobody's
  if (n_rows > p.max_rows && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
  if (at < static_cast<unsigned>(max(owned, 0)) || at >= static_cast<unsigned>(max(min(n_rows, p.max_rows), 0))) return;
  const int r = static_cast<int>(at);
  const long long slot = __ldg(reinterpret_cast<const long long*>(p.slot_map) + r);
  const int src = source_of(p, r, lane);
  if (src < 0) return;
  if (slot < 0 || slot >= p.n_slots) { if (lane == 0) atomicOr(p.status, MEPIC_DEV_BAD_PAGE); return; }
  const int page = static_cast<int>(slot >> p.page_shift), in_page = static_cast<int>(slot) & (p.page_size - 1);
  const size_t from = static_cast<size_t>(src) * p.kv_stride;
  for (int c = lane; c < p.n_kv_heads * C; c += 32) {
    const int h = c / C, cc = c % C;
    const size_t to = ((static_cast<size_t>(page) * p.n_kv_heads + h) * p.page_size + in_page) * D + 8 * cc;
#pragma unroll
    for (int w = 0; w < 2; ++w)
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.pool[w]) + to) = *reinterpret_cast<const uint4*>(p.src[w] + from + static_cast<size_t>(c) * 8);
  }
}

// 8-bit pages.  A CTA looks at kRunRows consecutive rows and does the runs (rows that go to one page) that START among
// them, whole; each of its warps takes one (pool, kv head) of a run at a time, so a block's maximum, scale and codes stay
// in one warp.  (A CTA per row left 15 of 16 CTAs of a prompt with nothing to do.)  12,900 prompt rows of 8 kv heads (79 MB
// read and written): 39 us (2.0 TB/s), 31 with the inputs in L2; about 1,250 instructions per block of 16 rows and a chain of
// dependent look-ups (slots, sources, rows, maximum, codes), which the CTAs of an SM hide from one another only in part: issue
// slots 50 %, DRAM 16.  A few rows per request make many short runs, which a CTA does one after the other: 32 x 4 rows 25 us,
// 256 x 4 28, 256 x 1 47.  (Prompts, inputs in L2, with CTAs of 8 warps 31; of 2 46; each warp two blocks of a run 34; rolled
// loops over a lane's eight pieces 35.)
constexpr int kRunRows = 16;
constexpr int kRunWarps = 4;
// Eight elements -> E4M3(x / sc), the quotient rounded to fp32 first, as the format is defined.  With y = RN(1 / sc) and no
// overflow or underflow on the way, q <- q - y (q sc - x) in fused arithmetic, begun at q = x y and done twice, ends at the
// rounded quotient (Markstein's correction; this order of signs keeps a zero's): two and a half instructions an element, two
// elements at a time, where a division takes a dozen.  For a scale outside [2^-80, 2^80] the division is used.
__device__ __noinline__ uint2 e4m3x8_by_division(uint4 v, float sc) {
  const float2 a = bf16x2_to_float2(v.x), b = bf16x2_to_float2(v.y), c = bf16x2_to_float2(v.z), d = bf16x2_to_float2(v.w);
  return make_uint2(e4m3x4_of(__fdiv_rn(a.x, sc), __fdiv_rn(a.y, sc), __fdiv_rn(b.x, sc), __fdiv_rn(b.y, sc)),
                    e4m3x4_of(__fdiv_rn(c.x, sc), __fdiv_rn(c.y, sc), __fdiv_rn(d.x, sc), __fdiv_rn(d.y, sc)));
}
// most: what saturates anyway must not overflow on the way, so |x| is cut to it first; 0: no element is above the block's maximum
// and none is cut.  NaN stays.
__device__ __forceinline__ uint2 e4m3x8_of(const uint4& v, float sc, float inv, float most) {
  const uint32_t w[4] = {v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u};      // -x
  const float2 sc2 = make_float2(sc, sc), ninv2 = make_float2(-inv, -inv);
  float2 q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float2 nx = bf16x2_to_float2(w[j]);
    if (most != 0.f) {
      nx.x = nx.x > most ? most : (nx.x < -most ? -most : nx.x);
      nx.y = nx.y > most ? most : (nx.y < -most ? -most : nx.y);
    }
    q[j] = mul2(nx, ninv2);
    q[j] = fma2(fma2(q[j], sc2, nx), ninv2, q[j]);
    q[j] = fma2(fma2(q[j], sc2, nx), ninv2, q[j]);
  }
  return make_uint2(e4m3x4_of(q[0].x, q[0].y, q[1].x, q[1].y), e4m3x4_of(q[2].x, q[2].y, q[3].x, q[3].y));
}
// Two running maxima of absolute values; a NaN operand is dropped.
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t m, uint32_t x) {
  asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(x & 0x7fff7fffu));
  return m;
}
// Rows r0 .. r0 + min(n, 16) - 1 of pool w, kv head h: a lane's 16-byte pieces of eight rows (half a warp takes a row), and in
// lane k < 16 the in-page slot of row k (-1: nothing to write).  known: in lane k, the source of row cta_r0 + k.
__device__ __forceinline__ void load_block(const CommitParams& p, int w, int r0, int n, int h, int lane, int cta_r0, int known, uint4 (&v)[8], int& slot) {
  const int found = p.src_rows ? __shfl_sync(kFull, known, (r0 + lane - cta_r0) & 31) : -1;
  int src = -1;
  slot = -1;
  if (lane < 16 && lane < n) {
    src = p.src_rows && r0 + lane - cta_r0 < kRunRows ? found : lane_source_or_none(p, r0 + lane);
    if (src < 0) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
    slot = src < 0 ? -1 : static_cast<int>(__ldg(reinterpret_cast<const long long*>(p.slot_map) + r0 + lane)) & (p.page_size - 1);
  }
  const uint16_t* base = p.src[w] + h * 128 + 8 * (lane & 15);
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int s = __shfl_sync(kFull, src, 2 * u + (lane >> 4));
    v[u] = s < 0 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(base + static_cast<size_t>(s) * p.kv_stride);
  }
}
__global__ void __launch_bounds__(kRunWarps * 32, 6) mepic_rows_commit_fp8_kernel(const __grid_constant__ CommitParams p) {
  constexpr int D = 128;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r0 = blockIdx.x * kRunRows;
  const int owned = max(__ldg(p.row_offsets), 0);      // the first row that is anybody's
  const int all = __ldg(p.row_offsets + p.batch), n_rows = min(all, p.max_rows);
  if (all > p.max_rows && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.status, MEPIC_DEV_BAD_SLOT);
  if (r0 >= n_rows) return;
  const long long* slots = reinterpret_cast<const long long*>(p.slot_map);
  auto page_of = [&](int r) -> int {
    const long long s = __ldg(slots + r);
    return s < 0 || s >= p.n_slots ? -1 : static_cast<int>(s >> p.page_shift);
  };
  // the sources of this CTA's rows, looked up once, beside their slots (again for each run and block: 2 us more on 32 requests
  // of 4 rows), and which of the rows start a run
  const int known = lane < kRunRows && r0 + lane < n_rows ? lane_source_or_none(p, r0 + lane) : -1;
  const unsigned sourced = __ballot_sync(kFull, known >= 0);
  bool starts = false;
  if (lane < kRunRows && r0 + lane >= owned && r0 + lane < n_rows) {
    const int mine = page_of(r0 + lane);
    if (mine < 0) { if (warp == 0) atomicOr(p.status, MEPIC_DEV_BAD_PAGE); }
    else starts = r0 + lane == owned || page_of(r0 + lane - 1) != mine;
  }
  for (unsigned todo = __ballot_sync(kFull, starts); todo; todo &= todo - 1) {
    const int first = r0 + __ffs(todo) - 1;
    const int page = page_of(first);
    // length of the run and whether it writes in-page slot 0, 32 rows at a time; lane k keeps rows first + k + 32 j
    int n = 0;
    bool fresh = false;
    for (bool more = true; more;) {
      const int r = first + n + lane;
      const bool in = n + lane < min(p.page_size, n_rows - first) && page_of(r) == page;
      const unsigned m = __ballot_sync(kFull, in);
      const int got = m == kFull ? 32 : __ffs(~m) - 1;
      const bool begins = lane < got && (__ldg(slots + r) & (p.page_size - 1)) == 0;      // a skipped row writes nothing, slot 0 neither
      fresh = fresh || __any_sync(kFull, begins && (r - r0 < kRunRows ? ((sourced >> (r - r0)) & 1) != 0 : lane_source_or_none(p, r) >= 0));
      n += got;
      more = got == 32;
    }
    // half a warp takes a row: cc is the 16-byte piece of 8 elements.  A block of 16 rows is 8 pieces per lane, all in flight
    // at once; a run of one block keeps them in registers between its two passes (maximum, codes).
    const int half = lane >> 4, cc = lane & 15;
    for (int unit = blockIdx.y * kRunWarps + warp; unit < 2 * p.n_kv_heads; unit += gridDim.y * kRunWarps) {
      const int w = unit & 1, h = unit >> 1;
      const size_t block = static_cast<size_t>(page) * p.n_kv_heads + h;
      uint4 v[8];
      int slot = 0;                                // lane k < 16: in-page slot of row k of the block, -1 where there is nothing to write
      float sc;
      if (fresh) {
        uint32_t m2[2] = {0, 0};                   // bf16 maxima are exact
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += 16) {
          load_block(p, w, first + k0, n - k0, h, lane, r0, known, v, slot);
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            m2[0] = max_abs_bf16x2(max_abs_bf16x2(m2[0], v[u].x), v[u].y);
            m2[1] = max_abs_bf16x2(max_abs_bf16x2(m2[1], v[u].z), v[u].w);
          }
        }
        const float2 m = bf16x2_to_float2(max_abs_bf16x2(m2[0], m2[1]));
        float amax = fmaxf(m.x, m.y);              // a NaN element does not set the scale
#pragma unroll
        for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, d));
        sc = amax > 0.f ? __fdiv_rn(amax, 448.f) : 1.f;
        if (lane == 0) p.scales[w][block] = sc;
      } else {
        sc = p.scales[w][block];
      }
      const float inv = __frcp_rn(sc), most = fresh ? 0.f : 600.f * sc;
      const bool plain = sc >= 8.2718061e-25f && sc <= 1.2089258e24f;       // 2^-80 .. 2^80
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 16) {
        if (!fresh || n > 16) load_block(p, w, first + k0, n - k0, h, lane, r0, known, v, slot);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int in_page = __shfl_sync(kFull, slot, 2 * u + half);
          const uint2 out = plain ? e4m3x8_of(v[u], sc, inv, most) : e4m3x8_by_division(v[u], sc);
          if (in_page >= 0) *reinterpret_cast<uint2*>(static_cast<unsigned char*>(p.pool[w]) + (block * p.page_size + in_page) * D + 8 * cc) = out;
        }
      }
    }
  }
}

int shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}
long long ceil_div(long long a, int b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int32_t launched(const char* what, int n = 1) {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { mepic_set_error("%s: launch: %s", what, cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(n);
  return MEPIC_OK;
}

int32_t commit_call(const mepic_config_t* cfg, const mepic_rows_commit_args_t* a, float* k_scales, float* v_scales, bool fp8, void* cuda_stream) {
  const char* what = fp8 ? "rows_commit_fp8" : "rows_commit";
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("%s: NULL argument", what); return MEPIC_E_INVAL; }
  if (fp8 && cfg->head_dim != 128) { mepic_set_error("%s: head_dim %d: 8-bit pages are built for head_dim 128", what, cfg->head_dim); return MEPIC_E_INVAL; }
  if (a->batch < 1 || a->max_rows < 0 || a->n_sources < 0) { mepic_set_error("%s: batch must be positive, max_rows and n_sources not negative", what); return MEPIC_E_INVAL; }
  const long long packed = static_cast<long long>(cfg->n_kv_heads) * cfg->head_dim;
  const long long stride = a->kv_stride ? a->kv_stride : packed;
  if (packed > 0x7fffffffLL || stride < packed || stride % 8) {
    mepic_set_error("%s: kv_stride %d must be 0 or a multiple of 8 of at least n_kv_heads * head_dim", what, a->kv_stride); return MEPIC_E_INVAL;
  }
  if (a->max_rows == 0) return MEPIC_OK;
  if ((a->n_sources > 0 && (!a->k_new || !a->v_new)) || !a->row_offsets || !a->slot_map || !a->k_pool || !a->v_pool || !a->status) {
    mepic_set_error("%s: NULL pointer argument", what); return MEPIC_E_INVAL;
  }
  if (a->src_rows && a->src_stride < 1) { mepic_set_error("%s: src_stride must be positive", what); return MEPIC_E_INVAL; }
  if (fp8 && (!k_scales || !v_scales)) { mepic_set_error("%s: NULL scale pointer", what); return MEPIC_E_INVAL; }
  if (!aligned(a->k_new, 16) || !aligned(a->v_new, 16) || !aligned(a->k_pool, 16) || !aligned(a->v_pool, 16) || !aligned(a->slot_map, 8)) {
    mepic_set_error("%s: rows and pools must be 16-byte aligned, slot_map 8-byte aligned", what); return MEPIC_E_INVAL;
  }
  CommitParams p;
  p.src[0] = static_cast<const uint16_t*>(a->k_new); p.src[1] = static_cast<const uint16_t*>(a->v_new);
  p.pool[0] = a->k_pool; p.pool[1] = a->v_pool;
  p.scales[0] = k_scales; p.scales[1] = v_scales;
  p.row_offsets = a->row_offsets; p.slot_map = a->slot_map; p.src_rows = a->src_rows; p.status = a->status;
  p.src_stride = a->src_stride; p.batch = a->batch; p.max_rows = a->max_rows; p.n_sources = a->n_sources;
  p.kv_stride = static_cast<int>(stride); p.n_kv_heads = cfg->n_kv_heads; p.page_size = cfg->page_size;
  p.page_shift = shift_of(cfg->page_size);
  p.n_slots = static_cast<long long>(cfg->num_pages) * cfg->page_size;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // a CTA takes up to four of a run's (pool, kv head) blocks, one per warp: several CTAs fit an SM and hide one another's look-ups
  const unsigned run_ctas = static_cast<unsigned>(ceil_div(a->max_rows, kRunRows)), copy_ctas = static_cast<unsigned>(ceil_div(a->max_rows, kCopyRows));
  if (fp8) mepic_rows_commit_fp8_kernel<<<dim3(run_ctas, std::min((2 * cfg->n_kv_heads + kRunWarps - 1) / kRunWarps, 64)), kRunWarps * 32, 0, st>>>(p);
  else if (cfg->head_dim == 128) mepic_rows_commit_kernel<128><<<copy_ctas, kCopyRows * 32, 0, st>>>(p);
  else mepic_rows_commit_kernel<64><<<copy_ctas, kCopyRows * 32, 0, st>>>(p);
  return launched(what);
}

}  // namespace

extern "C" int32_t mepic_tree_layout(const mepic_config_t* cfg, const mepic_tree_layout_args_t* a, void* cuda_stream) {
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("tree_layout: NULL argument"); return MEPIC_E_INVAL; }
  if (a->batch < 1 || a->table_stride < 1 || a->total_rows < 0) { mepic_set_error("tree_layout: batch and table_stride must be positive, total_rows not negative"); return MEPIC_E_INVAL; }
  if (a->mask_words < 1 || a->mask_words > MEPIC_TREE_MAX_ROWS / 32) {
    mepic_set_error("tree_layout: mask_words %d not in 1..%d", a->mask_words, MEPIC_TREE_MAX_ROWS / 32); return MEPIC_E_INVAL;
  }
  if (a->total_rows == 0) return MEPIC_OK;
  if (!a->parent || !a->row_offsets || !a->kv_len || !a->pos_base || !a->row_pos || !a->tree_mask || !a->status) {
    mepic_set_error("tree_layout: NULL pointer argument"); return MEPIC_E_INVAL;
  }
  const size_t smem = static_cast<size_t>(32 * a->mask_words) * a->mask_words * sizeof(uint32_t);
  if (smem > 40 * 1024) {                        // beside the static 4 KB.  Always the largest: another thread's call may need more than this one
    const cudaError_t e = cudaFuncSetAttribute(mepic_tree_layout_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MEPIC_TREE_MAX_ROWS * MEPIC_TREE_MAX_ROWS / 8);
    if (e != cudaSuccess) { mepic_set_error("tree_layout: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  }
  mepic_tree_layout_kernel<<<a->batch, kLayoutThreads, smem, static_cast<cudaStream_t>(cuda_stream)>>>(*a, shift_of(cfg->page_size));
  return launched("tree_layout");
}

extern "C" int32_t mepic_tree_accept(const mepic_tree_accept_args_t* a, void* cuda_stream) {
  if (!a) { mepic_set_error("tree_accept: NULL argument"); return MEPIC_E_INVAL; }
  if (a->batch < 1 || a->total_rows < 0 || a->max_accept < 1) { mepic_set_error("tree_accept: batch and max_accept must be positive, total_rows not negative"); return MEPIC_E_INVAL; }
  if (!a->row_offsets || !a->root || !a->n_accept || !a->accept_rows || !a->next_token || !a->status ||
      (a->total_rows > 0 && (!a->parent || !a->draft || !a->target))) {
    mepic_set_error("tree_accept: NULL pointer argument"); return MEPIC_E_INVAL;
  }
  mepic_tree_accept_kernel<<<a->batch, kAcceptThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(*a);
  return launched("tree_accept");
}

extern "C" int32_t mepic_step_tables(const mepic_config_t* cfg, const mepic_step_tables_args_t* a, void* cuda_stream) {
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("step_tables: NULL argument"); return MEPIC_E_INVAL; }
  if (a->batch < 1 || a->batch > MEPIC_STEP_MAX_BATCH) { mepic_set_error("step_tables: batch %d not in 1..%d", a->batch, MEPIC_STEP_MAX_BATCH); return MEPIC_E_INVAL; }
  if (a->table_stride < 1 || a->max_rows < 0 || a->n_reserve < 0) { mepic_set_error("step_tables: table_stride must be positive, max_rows and n_reserve not negative"); return MEPIC_E_INVAL; }
  if (!a->kv_len || !a->n_new || !a->page_ids || !a->pos_base || (a->n_reserve > 0 && !a->reserve) || !a->reserve_used || !a->row_offsets ||
      !a->kv_len_out || !a->reserve_used_out || !a->status) {
    mepic_set_error("step_tables: NULL pointer argument"); return MEPIC_E_INVAL;
  }
  if (a->kv_len_out == a->kv_len || a->kv_len_out == a->n_new || a->reserve_used_out == a->reserve_used) {
    mepic_set_error("step_tables: outputs must not overlap inputs"); return MEPIC_E_INVAL;
  }
  if (a->slot_map && !aligned(a->slot_map, 8)) { mepic_set_error("step_tables: slot_map must be 8-byte aligned"); return MEPIC_E_INVAL; }
  const size_t smem = 2 * (static_cast<size_t>(a->batch) + 1) * sizeof(int);
  if (smem > 40 * 1024) {                        // beside the static sums.  Always the largest, as above
    const cudaError_t e = cudaFuncSetAttribute(mepic_step_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               2 * (MEPIC_STEP_MAX_BATCH + 1) * static_cast<int>(sizeof(int)));
    if (e != cudaSuccess) { mepic_set_error("step_tables: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  }
  const int work = std::max(a->row_slot || a->slot_map ? a->max_rows : 0, a->batch);
  const int ctas = static_cast<int>(std::min<long long>(ceil_div(work, 2 * kTablesThreads), 296));
  mepic_step_tables_kernel<<<ctas, kTablesThreads, smem, static_cast<cudaStream_t>(cuda_stream)>>>(*a, shift_of(cfg->page_size), cfg->num_pages);
  return launched("step_tables");
}

extern "C" int32_t mepic_rows_commit(const mepic_config_t* cfg, const mepic_rows_commit_args_t* a, void* cuda_stream) {
  return commit_call(cfg, a, nullptr, nullptr, false, cuda_stream);
}
extern "C" int32_t mepic_rows_commit_fp8(const mepic_config_t* cfg, const mepic_rows_commit_args_t* a, float* k_scales, float* v_scales,
                                         void* cuda_stream) {
  return commit_call(cfg, a, k_scales, v_scales, true, cuda_stream);
}
