// A decode with beams, apart from its attention: selection over beams and vocabulary, block tables of the new beams, page copies
// (see "beams" in mepic.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include <algorithm>

#include "mepic.h"
#include "mepic_internal.h"
#include "mepic_ptx.cuh"
#include "mepic_tcgen05.cuh"      // arithmetic on pairs of floats

namespace {

using namespace mepic_dev;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWidth = MEPIC_BEAM_MAX_WIDTH;

// ---------------------------------------------------------------- selection
// Two launches.  The first is a pass over the logits, bound by HBM: every warp leaves the sum of its tokens' exponentials and every
// four threads (a SET: 128 fp32 or 256 16-bit tokens) their largest logit, nothing else.  The second has a CTA per group: the n_select best
// tokens are not below the n_select-th largest of the sets' maxima, so only the few sets that reach it are read again, and of those
// only the tokens that reach it are ranked.  (Every segment keeping its own n_select best, in the first pass, took a dozen
// instructions a token more: 64 x 8 beams over 100,003 fp32 tokens in 65 us against 41.)  The pass alone
// takes 33 of them (6.2 TB/s); the join is a chain of five dependent round trips.
constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr float kFusedRef = 65536.f;           // largest magnitude of a maximum that the fused form of its exponentials is for
constexpr int kSelPieces = 8;                  // 16-byte pieces a thread reads
constexpr int kSelSets = kSelThreads / 4;      // sets of a segment (the tokens of a CTA of the first pass)
static_assert(kSelSets >= MEPIC_BEAM_MAX_SELECT, "as many maxima as tokens to select");

template <typename T> constexpr int kVec = 16 / sizeof(T);
template <typename T> __device__ __forceinline__ void widen(const uint4& c, float (&x)[kVec<T>]);
template <> __device__ __forceinline__ void widen<float>(const uint4& c, float (&x)[4]) {
  x[0] = __uint_as_float(c.x); x[1] = __uint_as_float(c.y); x[2] = __uint_as_float(c.z); x[3] = __uint_as_float(c.w);
}
template <> __device__ __forceinline__ void widen<__nv_bfloat16>(const uint4& c, float (&x)[8]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = bf16x2_to_float2(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}
template <> __device__ __forceinline__ void widen<__half>(const uint4& c, float (&x)[8]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}
// The largest element of a piece; a NaN is dropped.
template <typename T> __device__ __forceinline__ float largest(const uint4& c);
template <> __device__ __forceinline__ float largest<float>(const uint4& c) {
  return fmaxf(fmaxf(__uint_as_float(c.x), __uint_as_float(c.y)), fmaxf(__uint_as_float(c.z), __uint_as_float(c.w)));
}
template <> __device__ __forceinline__ float largest<__nv_bfloat16>(const uint4& c) {
  uint32_t a, b;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(c.x), "r"(c.y));
  asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(c.z), "r"(c.w));
  asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  const float2 f = bf16x2_to_float2(a);
  return fmaxf(f.x, f.y);
}
template <> __device__ __forceinline__ float largest<__half>(const uint4& c) {
  uint32_t a, b;
  asm("max.f16x2 %0, %1, %2;" : "=r"(a) : "r"(c.x), "r"(c.y));
  asm("max.f16x2 %0, %1, %2;" : "=r"(b) : "r"(c.z), "r"(c.w));
  asm("max.f16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a));
  return fmaxf(f.x, f.y);
}
template <typename T> __device__ __forceinline__ T minus_infinity();
template <> __device__ __forceinline__ float minus_infinity<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __nv_bfloat16 minus_infinity<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half minus_infinity<__half>() { return __ushort_as_half(0xfc00); }

struct WarpSum { double sum; float top; float pad; };      // sum of exp(x - top) over a warp's tokens; NaN: the row is to be given up

struct SelectParams {
  mepic_beam_select_args_t a;
  WarpSum* sums;         // [rows][segments][kSelWarps]
  float* tops;           // [rows][segments][kSelSets]; -infinity where a set has no candidate
  int segments;
  long long stride;
};

// Pieces are 16 bytes by address, so that a row may begin and end inside one: the elements of a row that its first piece lacks.
template <typename T> __device__ __forceinline__ int lead_of(const T* row) { return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)); }
// Token of the first element of piece k of a thread (negative before the row).
template <typename T> __device__ __forceinline__ int token_of(int lead, int seg, int k, int thread) {
  return ((seg * kSelPieces + k) * kSelThreads + thread) * kVec<T> - lead;
}

// (five CTAs an SM: 51 million bf16 logits in 23 us, with three 28; fp32 33 either way, where HBM is the bound)
template <typename T>
__global__ void __launch_bounds__(kSelThreads, 5) mepic_beam_pass(const __grid_constant__ SelectParams p) {
  constexpr int N = kVec<T>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = blockIdx.y, seg = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float score = __ldg(p.a.score + row);
  if (score == -INFINITY || (p.a.done && __ldg(p.a.done + row) != 0)) return;        // nobody reads what such a row leaves
  const T* x = static_cast<const T*>(p.a.logits) + row * p.stride;
  const int lead = lead_of(x), V = p.a.vocab;
  uint4 c[kSelPieces];
#pragma unroll
  for (int k = 0; k < kSelPieces; ++k) {
    const int at = token_of<T>(lead, seg, k, tid);
    if (at >= 0 && at + N <= V) c[k] = __ldcs(reinterpret_cast<const uint4*>(x + at));
    else {
      alignas(16) T e[N];
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = at + i >= 0 && at + i < V ? x[at + i] : minus_infinity<T>();
      c[k] = *reinterpret_cast<const uint4*>(e);
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < kSelPieces; ++k) top = fmaxf(top, largest<T>(c[k]));
  const float ref = top == -INFINITY ? 0.f : top;
  float2 sum2 = make_float2(0.f, 0.f);
  auto add_all = [&](auto exponents) {
#pragma unroll
    for (int k = 0; k < kSelPieces; ++k) {
      float v[N];
      widen<T>(c[k], v);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float2 d = exponents(make_float2(v[i], v[i + 1]));
        sum2 = add2(sum2, make_float2(ex2(d.x), ex2(d.y)));      // +infinity - +infinity and NaN - anything: NaN
      }
    }
  };
  const float2 l2 = make_float2(kLog2e, kLog2e);
  float sum;
  if (fabsf(ref) <= kFusedRef) {
    // 2^(x log2e - c) with c = ref log2e as rounded, in one fused step an element; what the rounding of c took (2^-8 at most: 2^16 log2e
    // is below 2^17) is divided by, so that the maximum itself counts exactly 1.  (1 / y is 2 - y but for (1 - y)^2 < 2^-17; one Newton step on
    // the quotient leaves 2^-34.  A division: 1 to 3 % of a 16-bit batch.)
    const float c0 = ref * kLog2e;
    add_all([&](float2 v) { return fma2(v, l2, make_float2(-c0, -c0)); });
    const float y = ex2(fmaf(ref, kLog2e, -c0)), all = sum2.x + sum2.y, q = all * (2.f - y);
    sum = fmaf(fmaf(-q, y, all), 2.f - y, q);
  } else {                                        // ref log2e would be rounded by more than a factor can give back (or ref is infinite)
    add_all([&](float2 v) { return mul2(add2(v, make_float2(-ref, -ref)), l2); });
    sum = sum2.x + sum2.y;
  }
  const size_t part = static_cast<size_t>(row) * p.segments + seg;
  float wtop = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
  wtop = fmaxf(wtop, __shfl_xor_sync(kFull, wtop, 2));
  if ((lane & 3) == 0) p.tops[part * kSelSets + (tid >> 2)] = wtop;
#pragma unroll
  for (int d = 4; d < 32; d <<= 1) wtop = fmaxf(wtop, __shfl_xor_sync(kFull, wtop, d));
  double s = static_cast<double>(sum) * (top == -INFINITY ? 1.0 : static_cast<double>(ex2((top - wtop) * kLog2e)));
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(kFull, s, d);
  if (lane == 0) p.sums[part * kSelWarps + warp] = WarpSum{s, wtop, 0.f};
}

// A candidate: its score in 64 bits, ordered as an unsigned number (0: none), and where it stands, beam * vocab + token.
struct Candidate { uint64_t order; long long flat; };
__device__ __forceinline__ bool better(const Candidate& x, const Candidate& y) { return x.order > y.order || (x.order == y.order && x.order && x.flat < y.flat); }
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return u ^ ((u >> 63) ? ~0ull : 0x8000000000000000ull);
}
__device__ __forceinline__ double score_of(uint64_t order) {
  return __longlong_as_double(static_cast<long long>(order ^ ((order >> 63) ? 0x8000000000000000ull : ~0ull)));
}

// The same order for floats.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t order) { return __uint_as_float(order ^ ((order >> 31) ? 0x80000000u : 0xffffffffu)); }

// Two sums of the same terms, relative to one another: each term is off by 2^-22 (ex2) and 2^-23 (its argument), the 31 additions of a
// thread's terms by 2^-25 each; both sums at most by 1.3e-6 therefore.  (A logarithm taken for another's is off by this much at most.)
constexpr double kSame = 0x1p-18;
constexpr int kJoinSets = 512;           // sets that are read again
constexpr int kJoinList = 1536;          // tokens that are ranked
constexpr int kJoinBatch = 8;            // pieces of four maxima a thread has under way
// (three CTAs an SM: the compiler keeps to 64 registers otherwise and spills, 64 x 8 beams over 100,003 bf16 tokens 35 us against 33)
template <typename T>
__global__ void __launch_bounds__(kSelThreads, 3) mepic_beam_join(const __grid_constant__ SelectParams p) {
  __shared__ double lse[kWidth], base[kWidth];
  __shared__ float off[kWidth];                   // base - lse in fp32; -infinity where a beam offers no tokens
  __shared__ int kind[kWidth];                    // 0: offers nothing, 1: live, 2: finished
  __shared__ int like[kWidth];                    // the first beam with the same logarithm
  __shared__ alignas(16) uint32_t quad_top[kSelSets];
  __shared__ uint64_t set_order[kJoinSets];
  __shared__ int sets[kJoinSets];
  __shared__ Candidate list[kJoinList];
  __shared__ uint64_t threshold;
  __shared__ uint32_t threshold0;
  __shared__ int n_sets, n_listed;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int W = p.a.width, S = p.segments, K = p.a.n_select, V = p.a.vocab;
  const float* tops = p.tops + static_cast<size_t>(g) * W * S * kSelSets;
  const int n = W * S * kSelSets, per = S * kSelSets;
  const float inv_per = 1.f / static_cast<float>(per);
  if (tid == 0) { n_sets = 0; n_listed = 0; threshold = 0; }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // the maxima of a batch, side by side; the first batch is on its way while the sums are taken together
  float4 top[kJoinBatch];
  auto place = [&](int i0, int k) { return i0 + 4 * (k * kSelThreads + tid); };
  auto load_batch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k)
      top[k] = place(i0, k) < n ? *reinterpret_cast<const float4*>(tops + place(i0, k)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
  };
  load_batch(0);
  // ---- log-sum-exp of the rows
  for (int w = warp; w < W; w += kSelWarps) {
    const int row = g * W + w, parts = S * kSelWarps;
    const WarpSum* part = p.sums + static_cast<size_t>(row) * parts;
    auto part_at = [&](int i) { return i < parts ? part[i] : WarpSum{0.0, -INFINITY, 0.f}; };
    // (asked for before it is known whether the row counts: one that does not left nothing, and nothing is made of it)
    WarpSum first[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) first[k] = part_at(lane + 32 * k);
    const float score = __ldg(p.a.score + row);
    int what = 1;
    bool bad = !(score < INFINITY);
    double l = 0.0;
    if (p.a.done && __ldg(p.a.done + row) != 0) what = 2;
    else if (score > -INFINITY) {
      float most = fmaxf(fmaxf(first[0].top, first[1].top), fmaxf(first[2].top, first[3].top));
      for (int i = lane + 128; i < parts; i += 32) most = fmaxf(most, part[i].top);
#pragma unroll
      for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, d));
      double sum = 0.0;
      auto add = [&](const WarpSum& v) { sum += v.top == -INFINITY ? v.sum : v.sum * static_cast<double>(ex2((v.top - most) * kLog2e)); };
#pragma unroll
      for (int k = 0; k < 4; ++k) add(first[k]);
      for (int i = lane + 128; i < parts; i += 32) add(part[i]);
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
      bad = bad || !(sum < INFINITY);              // NaN
      if (!(sum > 0.0)) what = 0;                  // every token is masked
      else l = static_cast<double>(most) + log(sum);
      bad = bad || !(fabs(static_cast<double>(score) - l) <= FLT_MAX);      // what is added to every logit
    }
    if (score == -INFINITY) what = 0;
    if (bad) what = 0;
    if (lane == 0) {
      lse[w] = l; base[w] = score; kind[w] = what;
      off[w] = what == 1 ? static_cast<float>(static_cast<double>(score) - l) : -INFINITY;
      if (bad) atomicOr(p.a.status, MEPIC_DEV_BAD_LOGITS);
    }
  }
  __syncthreads();
  auto order_at = [&](int w, float x) -> uint64_t {
    const double d = base[w] + (static_cast<double>(x) - lse[w]);
    return d >= -FLT_MAX ? order_of(d) : 0;          // (x = -infinity, or a score that fp32 does not hold: no candidate)
  };
  auto beam_of = [&](int i) {                      // i / per
    int w = static_cast<int>(static_cast<float>(i) * inv_per);
    return w + (i - w * per >= per ? 1 : i < w * per ? -1 : 0);
  };
  const uint64_t ended = tid < W && kind[tid] == 2 ? order_of(base[tid]) : 0;      // a finished beam's one candidate
  // Scores in fp32 do to leave out what cannot be among the best: x + off is off by 2^-24 of off and of itself at most.
  float most_off = 0.f;
  for (int w = 0; w < W; ++w) if (off[w] > -INFINITY) most_off = fmaxf(most_off, fabsf(off[w]));
  auto lowered = [&](float x) { return x - 0x1p-21f * (most_off + fabsf(x)) - static_cast<float>(kSame); };      // (off is that of the sums as they are)
  // Beams with the same logits have the same logarithm.  The sums of two such rows are rounded differently where the rows begin
  // at different places of their 16 bytes, by less than kSame: one that near to an earlier beam's is taken to be the same.  (Found here, put
  // in place behind the next barrier and used behind the one after it: nothing is compared in 64 bits before.)
  for (int w = warp; w < W; w += kSelWarps) {
    const bool same = lane < w && kind[w] == 1 && kind[lane] == 1 && fabs(lse[w] - lse[lane]) <= kSame + fabs(lse[w]) * 0x1p-52;
    const unsigned those = __ballot_sync(kFull, same);
    if (lane == 0) like[w] = those ? __ffs(those) - 1 : w;
  }
  // ---- a first threshold, from the best of every four threads (no two equal: a number of their own in the last bits)
  float mine = ended ? static_cast<float>(base[tid]) : -INFINITY;
  for (int i0 = 0; i0 < n; i0 += 4 * kJoinBatch * kSelThreads) {
    if (i0) load_batch(i0);
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k)
      if (place(i0, k) < n) mine = fmaxf(mine, fmaxf(fmaxf(top[k].x, top[k].y), fmaxf(top[k].z, top[k].w)) + off[beam_of(place(i0, k))]);
  }
  float quad = fmaxf(mine, __shfl_xor_sync(kFull, mine, 1));
  quad = fmaxf(quad, __shfl_xor_sync(kFull, quad, 2));
  if ((lane & 3) == 0) quad_top[tid >> 2] = (order_of(quad) & ~(kSelSets - 1u)) | (tid >> 2);
  __syncthreads();
  if (warp == 0) {                                 // a lane a beam: all are read before any is written
    const double l = lane < W ? lse[like[lane]] : 0.0;
    __syncwarp();
    if (lane < W) lse[lane] = l;
  }
  {
    const int i = tid >> 2, q0 = (tid & 3) * (kSelSets / 4);
    const uint32_t me = quad_top[i];
    int above = 0;
#pragma unroll
    for (int q = q0; q < q0 + kSelSets / 4; q += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(quad_top + q);
      above += (o.x > me) + (o.y > me) + (o.z > me) + (o.w > me);
    }
    above += __shfl_xor_sync(kFull, above, 1);
    above += __shfl_xor_sync(kFull, above, 2);
    if ((tid & 3) == 0 && above == K - 1) threshold0 = me & ~(kSelSets - 1u);
  }
  __syncthreads();
  // ---- the sets that may reach it; the threshold proper is the n_select-th largest among them, in 64 bits
  const float least0 = threshold0 > order_of(-INFINITY) ? lowered(float_of(threshold0)) : -INFINITY;
  if (mine >= least0) {
    for (int i0 = 0; i0 < n; i0 += 4 * kJoinBatch * kSelThreads) {
      if (n > 4 * kJoinBatch * kSelThreads) load_batch(i0);
#pragma unroll
      for (int k = 0; k < kJoinBatch; ++k) {
        if (place(i0, k) >= n) continue;
        const int w = beam_of(place(i0, k));
        if (!(fmaxf(fmaxf(top[k].x, top[k].y), fmaxf(top[k].z, top[k].w)) + off[w] >= least0)) continue;
        const float x[4] = {top[k].x, top[k].y, top[k].z, top[k].w};
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (x[c] + off[w] >= least0 && x[c] + off[w] > -INFINITY) {
            const int at = atomicAdd(&n_sets, 1);
            if (at < kJoinSets) { sets[at] = place(i0, k) + c; set_order[at] = order_at(w, x[c]); }
          }
      }
    }
  }
  __syncthreads();
  const int m = min(n_sets, kJoinSets);
  const bool all_sets = n_sets <= kJoinSets;
  for (int i = tid; i < m; i += kSelThreads) {
    const uint64_t me = set_order[i];
    int above = 0;
    for (int q = 0; q < m; ++q) above += set_order[q] > me || (set_order[q] == me && q < i);
    if (above == K - 1) threshold = me;            // (never below what it was)
  }
  __syncthreads();
  // (fewer sets than that: the others that reached the first threshold are finished beams, and it holds)
  uint64_t least = max(threshold, least0 > -INFINITY ? order_of(static_cast<double>(least0)) : static_cast<uint64_t>(1));
  // ---- the tokens that reach it: a set a warp, the warp's loads side by side
  const T* logits = static_cast<const T*>(p.a.logits) + static_cast<long long>(g) * W * p.stride;
  constexpr int kRun = 4 * kVec<T>, kLoads = kSelPieces * kRun / 32;      // consecutive tokens of a set's piece; tokens of a set a lane has
  auto each_token = [&](int set, uint64_t from, auto use) {               // those whose order is `from` or more
    // (below the lowest score's order there is no number to compare with: 1 and 2 would be read as NaN)
    const float from_f = from >= order_of(static_cast<double>(-FLT_MAX)) ? lowered(static_cast<float>(score_of(from))) : -INFINITY;
    const int w = beam_of(set);
    const T* x = logits + w * p.stride;
    const int first = token_of<T>(lead_of(x), (set - w * per) / kSelSets, lane / kRun, (set % kSelSets) * 4) + lane % kRun;
    float y[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int v = first + k * (32 / kRun) * kSelThreads * kVec<T>;      // (a warp covers 32 / kRun pieces at a time)
      y[k] = v >= 0 && v < V ? static_cast<float>(x[v]) : -INFINITY;
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (y[k] + off[w] >= from_f && y[k] > -INFINITY) {
        const Candidate c{order_at(w, y[k]), static_cast<long long>(w) * V + first + k * (32 / kRun) * kSelThreads * kVec<T>};
        if (c.order >= from) use(c);
      }
  };
  auto append = [&](const Candidate& c) {
    const int at = atomicAdd(&n_listed, 1);
    if (at < kJoinList) list[at] = c;
  };
  if (all_sets) {
    if (ended >= least) append(Candidate{ended, static_cast<long long>(tid) * V + p.a.pad_token});
    for (int q = warp; q < m; q += kSelWarps)
      if (set_order[q] >= least) each_token(sets[q], least, append);
  }
  __syncthreads();
  auto write = [&](int k, const Candidate& c) {
    const size_t at = static_cast<size_t>(g) * K + k;
    const bool any = c.order != 0;
    const int w = any ? static_cast<int>(c.flat / V) : -1, v = any ? static_cast<int>(c.flat - static_cast<long long>(w) * V) : -1;
    const bool stops = any && (kind[w] == 2 || v == p.a.eos_token);
    p.a.parent[at] = w; p.a.token[at] = v;
    p.a.score_out[at] = any ? static_cast<float>(score_of(c.order)) : -INFINITY;
    p.a.done_out[at] = stops; p.a.n_new[at] = any && !stops;
  };
  auto write_list = [&](int n_of) {                // the list's best, by their ranks
    for (int i = tid; i < n_of; i += kSelThreads) {
      const Candidate me = list[i];
      int above = 0;
      for (int q = 0; q < n_of; ++q) above += better(list[q], me);
      if (above < K) write(above, me);
    }
  };
  if (all_sets && n_listed <= kJoinList) {
    write_list(n_listed);
    for (int k = n_listed + tid; k < K; k += kSelThreads) write(k, Candidate{0, 0});
    return;
  }
  // ---- More of them than the lists hold: thousands of equal logits, or of neighbours above the threshold.  What lies above the
  // threshold is listed without what equals it; where that is too much, the threshold rises to the n_select-th largest of what the
  // list got hold of.  (So does every round; two or three are the most that was seen.)
  for (;;) {
    __syncthreads();
    if (tid == 0) n_sets = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {
      const int w = beam_of(i);
      const uint64_t o = kind[w] == 1 ? order_at(w, tops[i]) : 0;
      if (o > least) {
        const int at = atomicAdd(&n_sets, 1);
        if (at < kJoinSets) { sets[at] = i; set_order[at] = o; }
      }
    }
    __syncthreads();
    if (n_sets <= kJoinSets) break;
    for (int i = tid; i < kJoinSets; i += kSelThreads) {
      int above = 0;
      for (int q = 0; q < kJoinSets; ++q) above += set_order[q] > set_order[i] || (set_order[q] == set_order[i] && q < i);
      if (above == K - 1) threshold = set_order[i];
    }
    __syncthreads();
    least = threshold;
  }
  const int m2 = n_sets;
  for (;;) {
    __syncthreads();
    if (tid == 0) n_listed = 0;
    __syncthreads();
    if (ended > least) append(Candidate{ended, static_cast<long long>(tid) * V + p.a.pad_token});
    for (int q = warp; q < m2; q += kSelWarps)
      if (set_order[q] > least) each_token(sets[q], least + 1, append);
    __syncthreads();
    if (n_listed <= kJoinList) break;
    for (int i = tid; i < kJoinList; i += kSelThreads) {
      int above = 0;
      for (int q = 0; q < kJoinList; ++q) above += list[q].order > list[i].order || (list[q].order == list[i].order && q < i);
      if (above == K - 1) threshold = list[i].order;
    }
    __syncthreads();
    least = threshold;
  }
  write_list(n_listed);
  // ... and what equals it in order of beam and token, until there is enough
  int found = n_listed;
  for (int w = 0; w < W && found < K && least > 1; ++w) {
    if (kind[w] == 2) {
      if (order_of(base[w]) == least) { if (tid == 0) write(found, Candidate{least, static_cast<long long>(w) * V + p.a.pad_token}); ++found; }
      continue;
    }
    if (kind[w] == 0) continue;
    for (int v0 = 0; v0 < V && found < K; v0 += 8 * kSelThreads) {
      const T* x = logits + w * p.stride + v0 + 8 * tid;       // eight consecutive tokens a thread
      unsigned hit = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) if (v0 + 8 * tid + i < V && order_at(w, static_cast<float>(x[i])) == least) hit |= 1u << i;
      if (!__syncthreads_or(hit != 0)) continue;
      int incl = __popc(hit);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(kFull, incl, d); if (lane >= d) incl += y; }
      if (lane == 31) sets[warp] = incl;
      __syncthreads();
      int at = found + incl - __popc(hit);
      for (int q = 0; q < kSelWarps; ++q) {
        if (q < warp) at += sets[q];
        found += sets[q];
      }
      for (; hit && at < K; hit &= hit - 1, ++at) write(at, Candidate{least, static_cast<long long>(w) * V + v0 + 8 * tid + __ffs(hit) - 1});
      __syncthreads();
    }
  }
  for (int k = found + tid; k < K; k += kSelThreads) write(k, Candidate{0, 0});
}

// ---------------------------------------------------------------- fork
// Two launches: the first finds, a CTA per group and stretch of entries, which pages nobody holds any more and how many copies a
// group needs.  The second copies the tables meanwhile (it is a programmatic dependent), and then every CTA sums the counts up for
// itself and writes its share of the reserve and the copy list.
constexpr int kForkThreads = 256;
struct ForkParams {
  mepic_beam_fork_args_t a;
  int* n_freed;          // [groups][stretches]
  int* n_copies;         // [groups]
  int* freed;            // [groups][stretches][width_in * stretch]
  int page_shift, num_pages, stretches, stretch;
};

// What a group's CTA knows of it: parents, lengths, and which new beams need a copy of their last page.
struct Group {
  int parent[kWidth], len[kWidth];       // new beam -> beam (-1: none); beam -> slots
  unsigned copies;                       // new beams that copy
};
__device__ void load_lengths(const ForkParams& p, int g, Group& s, bool report) {
  const int tid = threadIdx.x, Wi = p.a.width_in, Wo = p.a.width_out;
  const long long room = min(static_cast<long long>(p.a.table_stride) << p.page_shift, 0x7fffffffll);
  if (tid == 0) s.copies = 0;
  if (tid < Wi) {
    int n = __ldg(p.a.kv_len + static_cast<size_t>(g) * Wi + tid);
    if (n < 0 || n > room) { if (report) atomicOr(p.a.status, MEPIC_DEV_BAD_SLOT); n = n < 0 ? 0 : static_cast<int>(room); }
    s.len[tid] = n;
  }
  if (tid >= 32 && tid - 32 < Wo) {
    int q = __ldg(p.a.parent + static_cast<size_t>(g) * Wo + tid - 32);
    if (q < -1 || q >= Wi) { if (report) atomicOr(p.a.status, MEPIC_DEV_BAD_BEAM); q = -1; }
    s.parent[tid - 32] = q;
  }
  __syncthreads();
}
// Every pair (k, j) of new beams side by side: does j keep k from keeping its partly filled last page?
struct Pair { int page, other; bool asks; };      // k's last page, what j holds there, whether there is such a page
__device__ __forceinline__ Pair load_pair(const ForkParams& p, int g, const Group& s, int i) {
  const int Wo = p.a.width_out, k = i / Wo, j = i - k * Wo, stride = p.a.table_stride;
  Pair r{-1, -1, false};
  if (i >= Wo * Wo || s.parent[k] < 0 || s.parent[j] < 0) return r;
  const int n = s.len[s.parent[k]], e = n >> p.page_shift;
  r.asks = (n & ((1 << p.page_shift) - 1)) != 0;
  if (!r.asks) return r;
  const int32_t* ids = p.a.page_ids + static_cast<size_t>(g) * p.a.width_in * stride + e;
  r.page = __ldg(ids + static_cast<size_t>(s.parent[k]) * stride);
  if (s.len[s.parent[j]] > (static_cast<long long>(e) << p.page_shift)) r.other = __ldg(ids + static_cast<size_t>(s.parent[j]) * stride);
  return r;
}
__device__ __forceinline__ void settle_pair(const ForkParams& p, Group& s, int i, const Pair& r) {
  if (!r.asks) return;
  const int Wo = p.a.width_out, k = i / Wo, j = i - k * Wo;
  const long long from = static_cast<long long>(s.len[s.parent[k]] >> p.page_shift) << p.page_shift, m = s.len[s.parent[j]];
  bool lost;
  if (j == k) lost = static_cast<unsigned>(r.page) >= static_cast<unsigned>(p.num_pages) || __ldg(p.a.owned + r.page) == 0;
  else lost = m > from && (j < k || m >= from + (1 << p.page_shift)) && r.other == r.page;
  if (lost) atomicOr(&s.copies, 1u << k);
}
__device__ void find_copies(const ForkParams& p, int g, Group& s, Pair first) {      // first: the thread's first pair
  const int pairs = p.a.width_out * p.a.width_out;
  for (int i = threadIdx.x; i < pairs; i += kForkThreads) {
    settle_pair(p, s, i, first);
    first = load_pair(p, g, s, i + kForkThreads);
  }
  __syncthreads();
}

__global__ void __launch_bounds__(kForkThreads) mepic_beam_fork_count(const __grid_constant__ ForkParams p) {
  __shared__ Group s;
  __shared__ int warp_n[kForkThreads / 32];
  extern __shared__ int at_entry[];              // [width_in][kForkThreads]: what the beams hold at a thread's entry
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int g = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int Wi = p.a.width_in, Wo = p.a.width_out, stride = p.a.table_stride;
  load_lengths(p, g, s, part == 0);
  const Pair first = load_pair(p, g, s, tid);
  unsigned kept = 0;
  for (int k = 0; k < Wo; ++k) if (s.parent[k] >= 0) kept |= 1u << s.parent[k];
  const unsigned dropped = ~kept & (Wi == 32 ? ~0u : (1u << Wi) - 1);
  const int32_t* ids = p.a.page_ids + static_cast<size_t>(g) * Wi * stride;
  int* out = p.freed + (static_cast<size_t>(g) * p.stretches + part) * p.stretch * Wi;
  int longest = 0;
  for (unsigned m = dropped; m; m &= m - 1) longest = max(longest, s.len[__ffs(m) - 1]);
  const int e_end = min(min(stride, (part + 1) * p.stretch), static_cast<int>((longest + (1ll << p.page_shift) - 1) >> p.page_shift));
  // what all beams hold at entry e, asked for side by side
  auto fetch = [&](int e) {
    if (e >= e_end) return;
    const long long from = static_cast<long long>(e) << p.page_shift;
    for (int q0 = 0; q0 < Wi; q0 += 8) {
      int page[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) page[q] = q0 + q < Wi && s.len[q0 + q] > from ? __ldg(ids + static_cast<size_t>(q0 + q) * stride + e) : -1;
#pragma unroll
      for (int q = 0; q < 8; ++q) if (q0 + q < Wi) at_entry[(q0 + q) * kForkThreads + tid] = page[q];
    }
  };
  fetch(part * p.stretch + tid);                   // (beside the pairs' pages)
  if (part == 0) {
    find_copies(p, g, s, first);
    if (tid == 0) p.n_copies[g] = __popc(s.copies);
  }
  int total = 0;
  for (int e0 = part * p.stretch; e0 < e_end; e0 += kForkThreads) {
    const int e = e0 + tid;
    unsigned back = 0;
    if (e0 > part * p.stretch) fetch(e);
    if (e < e_end) {
      const long long from = static_cast<long long>(e) << p.page_shift;
      for (unsigned m = dropped; m; m &= m - 1) {
        const int r = __ffs(m) - 1;
        if (s.len[r] <= from) continue;
        const int page = at_entry[r * kForkThreads + tid];
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) { atomicOr(p.a.status, MEPIC_DEV_BAD_PAGE); continue; }
        bool held = false;                          // by a beam that goes on, or by an earlier one that does not
        for (unsigned o = kept | (dropped & ((1u << r) - 1)); o; o &= o - 1) {
          const int q = __ffs(o) - 1;
          held = held || (s.len[q] > from && at_entry[q * kForkThreads + tid] == page);
        }
        if (!held && __ldg(p.a.owned + page) != 0) back |= 1u << r;
      }
    }
    const int n = __popc(back);
    int incl = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int y = __shfl_up_sync(kFull, incl, d); if (lane >= d) incl += y; }
    if (lane == 31) warp_n[warp] = incl;
    __syncthreads();
    int at = total + incl - n;
    for (int w = 0; w < kForkThreads / 32; ++w) {
      if (w < warp) at += warp_n[w];
      total += warp_n[w];
    }
    for (; back; back &= back - 1) out[at++] = at_entry[(__ffs(back) - 1) * kForkThreads + tid];
    __syncthreads();
  }
  if (tid == 0) p.n_freed[g * p.stretches + part] = total;
}

// Exclusive running sums of na counts into sa[0 .. na] and of nb into sb[0 .. nb] (shared memory), both in one scan.
__device__ void running_sums(const int* ca, int na, int* sa, const int* cb, int nb, int* sb) {
  __shared__ long long warp_n[kForkThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int pa = (na + kForkThreads - 1) / kForkThreads, a0 = min(tid * pa, na), a1 = min(a0 + pa, na);
  const int pb = (nb + kForkThreads - 1) / kForkThreads, b0 = min(tid * pb, nb), b1 = min(b0 + pb, nb);
  int in_a = 0, in_b = 0;
  for (int i = a0; i < a1; ++i) in_a += ca[i];
  for (int i = b0; i < b1; ++i) in_b += cb[i];
  const long long mine = static_cast<long long>(in_b) << 32 | static_cast<unsigned>(in_a);      // (counts: neither half reaches 2^31)
  long long incl = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) { const long long y = __shfl_up_sync(kFull, incl, d); if (lane >= d) incl += y; }
  if (lane == 31) warp_n[warp] = incl;
  __syncthreads();
  long long before = incl - mine;
  for (int w = 0; w < warp; ++w) before += warp_n[w];
  int at_a = static_cast<int>(before), at_b = static_cast<int>(before >> 32);
  for (int i = a0; i < a1; ++i) { sa[i] = at_a; at_a += ca[i]; }
  for (int i = b0; i < b1; ++i) { sb[i] = at_b; at_b += cb[i]; }
  if (a1 == na && a0 < na) sa[na] = at_a;
  if (b1 == nb && b0 < nb) sb[nb] = at_b;
  __syncthreads();
}

__global__ void __launch_bounds__(kForkThreads) mepic_beam_fork_write(const __grid_constant__ ForkParams p) {
  __shared__ Group s;
  __shared__ int fresh[kWidth];
  extern __shared__ int sums[];
  const int g = blockIdx.x, tid = threadIdx.x;
  const int Wi = p.a.width_in, Wo = p.a.width_out, stride = p.a.table_stride, groups = p.a.groups, S = p.stretches;
  int* freed_at = sums;                              // [groups * stretches + 1]
  int* copies_at = sums + groups * S + 1;            // [groups + 1]
  const int part = blockIdx.y, parts = gridDim.y;
  load_lengths(p, g, s, false);
  find_copies(p, g, s, load_pair(p, g, s, tid));
  // ---- tables: they do not depend on the counts, but for the pages of the copies; four rows side by side
  bool none = false;                                 // a page outside the pool, in a beam that goes on (others: by the first launch)
  for (int k0 = 0; k0 < Wo; k0 += 4) {
    int ents[4], most = 0;
    size_t from[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int parent = k0 + k < Wo ? s.parent[k0 + k] : -1;
      ents[k] = parent >= 0 ? static_cast<int>((static_cast<long long>(s.len[parent]) + (1 << p.page_shift) - 1) >> p.page_shift) : 0;
      from[k] = (static_cast<size_t>(g) * Wi + max(parent, 0)) * stride;
      most = max(most, ents[k]);
    }
    for (int e = part * kForkThreads + tid; e < most; e += parts * kForkThreads) {
      int page[4], pos[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) if (e < ents[k]) { page[k] = __ldg(p.a.page_ids + from[k] + e); pos[k] = __ldg(p.a.pos_base + from[k] + e); }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (e < ents[k]) {
          const size_t to = (static_cast<size_t>(g) * Wo + k0 + k) * stride + e;
          p.a.page_ids_out[to] = page[k]; p.a.pos_base_out[to] = pos[k];
          none = none || static_cast<unsigned>(page[k]) >= static_cast<unsigned>(p.num_pages);
        }
    }
  }
  if (none) atomicOr(p.a.status, MEPIC_DEV_BAD_PAGE);
  const long long used = __ldg(p.a.reserve_used);
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  running_sums(p.n_freed, groups * S, freed_at, p.n_copies, groups, copies_at);
  const long long n_freed = freed_at[groups * S], n_copies = copies_at[groups];
  const bool bad = used < 0 || used > p.a.n_reserve || n_freed > used, full = !bad && used - n_freed + n_copies > p.a.n_reserve;
  const bool ok = !bad && !full;
  // ---- the counts, and the unused end of the copy list
  if (g == 0 && part == 0 && tid == 0) {
    if (bad) atomicOr(p.a.status, MEPIC_DEV_BAD_BEAM);
    if (full) atomicOr(p.a.status, MEPIC_DEV_NO_PAGES);
    *p.a.n_copies = ok ? static_cast<int>(n_copies) : 0;
    *p.a.reserve_used_out = static_cast<int>(ok ? used - n_freed + n_copies : used);
  }
  const long long rows = static_cast<long long>(groups) * Wo;
  for (long long i = (ok ? n_copies : 0) + (static_cast<long long>(g) * parts + part) * kForkThreads + tid; i < rows; i += static_cast<long long>(groups) * parts * kForkThreads) {
    p.a.copy_src[i] = -1; p.a.copy_dst[i] = -1; p.a.copy_slots[i] = -1;
  }
  if (part == 0 && tid < Wo) p.a.kv_len_out[static_cast<size_t>(g) * Wo + tid] = ok && s.parent[tid] >= 0 ? s.len[s.parent[tid]] : 0;
  if (!ok) return;
  // ---- pages that go back
  for (int q = part; q < S; q += parts) {
    const int* list = p.freed + (static_cast<size_t>(g) * S + q) * p.stretch * Wi;
    const int n = freed_at[g * S + q + 1] - freed_at[g * S + q];
    for (int i = tid; i < n; i += kForkThreads) p.a.reserve[used - n_freed + freed_at[g * S + q] + i] = list[i];
  }
  // ---- copies of this group: their pages come from the top of the reserve as it is with the returned ones on it
  if (tid < Wo) {
    fresh[tid] = -1;
    if (s.copies >> tid & 1) {
      const int rank = copies_at[g] + __popc(s.copies & ((1u << tid) - 1));
      int page;
      if (rank < n_freed) {
        int lo = 0, hi = groups * S;                 // freed_at[lo] <= rank < freed_at[hi]
        while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (freed_at[mid] <= rank) lo = mid; else hi = mid; }
        page = p.freed[static_cast<size_t>(lo) * p.stretch * Wi + rank - freed_at[lo]];
      } else {
        page = p.a.reserve[used + rank - n_freed];
      }
      fresh[tid] = page;
      if (part == 0) {
        const int n = s.len[s.parent[tid]];
        const int src = __ldg(p.a.page_ids + (static_cast<size_t>(g) * Wi + s.parent[tid]) * stride + (n >> p.page_shift));
        if (static_cast<unsigned>(src) >= static_cast<unsigned>(p.num_pages) || static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages))
          atomicOr(p.a.status, MEPIC_DEV_BAD_PAGE);
        p.a.copy_src[rank] = src; p.a.copy_dst[rank] = page; p.a.copy_slots[rank] = n & ((1 << p.page_shift) - 1);
      }
    }
  }
  __syncthreads();
  // ---- the copies' places in the tables (this CTA wrote them above with the parents' pages)
  if (tid < Wo && (s.copies >> tid & 1)) {
    const int last = s.len[s.parent[tid]] >> p.page_shift;
    if (last / kForkThreads % parts == part) p.a.page_ids_out[(static_cast<size_t>(g) * Wo + tid) * stride + last] = fresh[tid];
  }
}

// ---------------------------------------------------------------- page copies
// A warp per (copy, pool, kv head): its filled slots are one contiguous stretch on both sides.
constexpr int kCopyWarps = 8;
struct CopyParams {
  mepic_pages_copy_args_t a;
  float* scales[2];
  int n_kv_heads, page_size, num_pages, row_bytes;
};
__global__ void __launch_bounds__(kCopyWarps * 32) mepic_pages_copy_kernel(const __grid_constant__ CopyParams p) {
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * kCopyWarps + (threadIdx.x >> 5);
  int n = p.a.n_copies ? __ldg(p.a.n_copies) : p.a.max_copies;
  if (n < 0 || n > p.a.max_copies) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.a.status, MEPIC_DEV_BAD_SLOT);
    n = n < 0 ? 0 : p.a.max_copies;
  }
  const int units = 2 * p.n_kv_heads;
  const long long i = unit / units;
  if (i >= n) return;
  const int u = static_cast<int>(unit - i * units), w = u / p.n_kv_heads, h = u - w * p.n_kv_heads;
  const int src = __ldg(p.a.src + i), dst = __ldg(p.a.dst + i);
  const int slots = p.a.slots ? min(max(__ldg(p.a.slots + i), 0), p.page_size) : p.page_size;
  if (static_cast<unsigned>(src) >= static_cast<unsigned>(p.num_pages) || static_cast<unsigned>(dst) >= static_cast<unsigned>(p.num_pages)) {
    if (lane == 0) atomicOr(p.a.status, MEPIC_DEV_BAD_PAGE);
    return;
  }
  unsigned char* pool = static_cast<unsigned char*>(w ? p.a.v_pool : p.a.k_pool);
  const size_t block = static_cast<size_t>(p.page_size) * p.row_bytes;
  const uint4* from = reinterpret_cast<const uint4*>(pool + (static_cast<size_t>(src) * p.n_kv_heads + h) * block);
  uint4* to = reinterpret_cast<uint4*>(pool + (static_cast<size_t>(dst) * p.n_kv_heads + h) * block);
  const int chunks = slots * (p.row_bytes / 16);
  for (int c0 = lane; c0 < chunks; c0 += 8 * 32) {
    uint4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) if (c0 + 32 * k < chunks) v[k] = from[c0 + 32 * k];
#pragma unroll
    for (int k = 0; k < 8; ++k) if (c0 + 32 * k < chunks) to[c0 + 32 * k] = v[k];
  }
  if (p.scales[w] && lane == 0) p.scales[w][static_cast<size_t>(dst) * p.n_kv_heads + h] = p.scales[w][static_cast<size_t>(src) * p.n_kv_heads + h];
}

// ---------------------------------------------------------------- host side
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}
int32_t launched(const char* what, cudaError_t e, int n) {
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) { mepic_set_error("%s: launch: %s", what, cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(n);
  return MEPIC_OK;
}
size_t up16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

// a row that begins inside a 16-byte piece may need one segment more
int segments_of(long long vocab, int type) {
  const int n = kSelThreads * kSelPieces * (type == MEPIC_LOGITS_FP32 ? 4 : 8);
  return static_cast<int>((vocab + 7 + n - 1) / n);
}
bool select_shape_ok(int32_t groups, int32_t width, int32_t n_select, int32_t vocab) {
  if (groups < 1 || width < 1 || width > MEPIC_BEAM_MAX_WIDTH) { mepic_set_error("beam_select: groups must be positive, width in 1..%d", MEPIC_BEAM_MAX_WIDTH); return false; }
  if (n_select < 1 || n_select > MEPIC_BEAM_MAX_SELECT) { mepic_set_error("beam_select: n_select %d not in 1..%d", n_select, MEPIC_BEAM_MAX_SELECT); return false; }
  if (vocab < 1 || vocab > (1 << 24)) { mepic_set_error("beam_select: vocab %d not in 1..2^24", vocab); return false; }
  if (static_cast<long long>(groups) * width > 65535) { mepic_set_error("beam_select: more than 65535 beams"); return false; }
  return true;
}
size_t select_bytes(int32_t groups, int32_t width, int segments) {
  return static_cast<size_t>(groups) * width * segments * (kSelWarps * sizeof(WarpSum) + kSelSets * sizeof(float));
}

// how the entries of a group are cut for the first launch of a fork: enough CTAs to fill the GPU, few enough counts to sum up
void fork_cut(int groups, int table_stride, int* stretches, int* stretch) {
  int n = std::max(1, std::min((table_stride + kForkThreads - 1) / kForkThreads, 1024 / std::max(1, groups)));
  int len = (table_stride + n - 1) / n;
  len = (len + kForkThreads - 1) / kForkThreads * kForkThreads;
  *stretch = len;
  *stretches = (table_stride + len - 1) / len;
}
bool fork_shape_ok(int32_t groups, int32_t width_in, int32_t width_out, int32_t table_stride) {
  if (groups < 1 || groups > MEPIC_STEP_MAX_BATCH) { mepic_set_error("beam_fork: groups %d not in 1..%d", groups, MEPIC_STEP_MAX_BATCH); return false; }
  if (width_in < 1 || width_in > MEPIC_BEAM_MAX_WIDTH || width_out < 1 || width_out > MEPIC_BEAM_MAX_WIDTH) {
    mepic_set_error("beam_fork: widths must be in 1..%d", MEPIC_BEAM_MAX_WIDTH); return false;
  }
  if (table_stride < 1 || table_stride > (1 << 24) || static_cast<long long>(groups) * std::max(width_in, width_out) * table_stride > 0x7fffffffLL) {
    mepic_set_error("beam_fork: table_stride must be in 1..2^24 and the tables below 2^31 entries"); return false;
  }
  return true;
}
size_t fork_bytes(int32_t groups, int32_t width_in, int32_t table_stride) {
  int n, len;
  fork_cut(groups, table_stride, &n, &len);
  return up16(static_cast<size_t>(groups) * n * 4) + up16(static_cast<size_t>(groups) * 4) + static_cast<size_t>(groups) * n * len * width_in * 4;
}

int32_t copy_call(const mepic_config_t* cfg, const mepic_pages_copy_args_t* a, float* k_scales, float* v_scales, bool fp8, void* cuda_stream) {
  const char* what = fp8 ? "pages_copy_fp8" : "pages_copy";
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("%s: NULL argument", what); return MEPIC_E_INVAL; }
  if (fp8 && cfg->head_dim != 128) { mepic_set_error("%s: head_dim %d: 8-bit pages are built for head_dim 128", what, cfg->head_dim); return MEPIC_E_INVAL; }
  if (a->max_copies < 0) { mepic_set_error("%s: max_copies must not be negative", what); return MEPIC_E_INVAL; }
  if (a->max_copies == 0) return MEPIC_OK;
  if (!a->src || !a->dst || !a->k_pool || !a->v_pool || !a->status) { mepic_set_error("%s: NULL pointer argument", what); return MEPIC_E_INVAL; }
  if (fp8 && (!k_scales || !v_scales)) { mepic_set_error("%s: NULL scale pointer", what); return MEPIC_E_INVAL; }
  if (!aligned(a->k_pool, 16) || !aligned(a->v_pool, 16)) { mepic_set_error("%s: pools must be 16-byte aligned", what); return MEPIC_E_INVAL; }
  CopyParams p;
  p.a = *a;
  p.scales[0] = k_scales; p.scales[1] = v_scales;
  p.n_kv_heads = cfg->n_kv_heads; p.page_size = cfg->page_size; p.num_pages = cfg->num_pages;
  p.row_bytes = cfg->head_dim * (fp8 ? 1 : 2);
  const long long warps = 2LL * cfg->n_kv_heads * a->max_copies, ctas = (warps + kCopyWarps - 1) / kCopyWarps;
  if (ctas > 0x7fffffffLL) { mepic_set_error("%s: max_copies %d is too large", what, a->max_copies); return MEPIC_E_INVAL; }
  mepic_pages_copy_kernel<<<static_cast<unsigned>(ctas), kCopyWarps * 32, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p);
  return launched(what, cudaSuccess, 1);
}

}  // namespace

extern "C" size_t mepic_beam_select_workspace(int32_t groups, int32_t width, int32_t n_select, int32_t vocab) {
  if (!select_shape_ok(groups, width, n_select, vocab)) return 0;
  return select_bytes(groups, width, segments_of(vocab, MEPIC_LOGITS_FP32));       // enough for every type
}

extern "C" int32_t mepic_beam_select(const mepic_beam_select_args_t* a, void* cuda_stream) {
  if (!a) { mepic_set_error("beam_select: NULL argument"); return MEPIC_E_INVAL; }
  if (!select_shape_ok(a->groups, a->width, a->n_select, a->vocab)) return MEPIC_E_INVAL;
  if (a->logits_type < MEPIC_LOGITS_BF16 || a->logits_type > MEPIC_LOGITS_FP32) { mepic_set_error("beam_select: logits_type %d is none of MEPIC_LOGITS_*", a->logits_type); return MEPIC_E_INVAL; }
  if (!a->logits || !a->score || !a->parent || !a->token || !a->score_out || !a->done_out || !a->n_new || !a->workspace || !a->status) {
    mepic_set_error("beam_select: NULL pointer argument"); return MEPIC_E_INVAL;
  }
  const long long stride = a->logits_stride ? a->logits_stride : a->vocab;
  if (stride < a->vocab || stride > (1LL << 40)) { mepic_set_error("beam_select: logits_stride %lld must be 0 or at least vocab", static_cast<long long>(a->logits_stride)); return MEPIC_E_INVAL; }
  if (a->eos_token < -1 || a->eos_token >= a->vocab || a->pad_token < 0 || a->pad_token >= a->vocab) {
    mepic_set_error("beam_select: eos_token must be -1 or a token, pad_token a token of the vocabulary"); return MEPIC_E_INVAL;
  }
  if (!aligned(a->logits, a->logits_type == MEPIC_LOGITS_FP32 ? 4 : 2) || !aligned(a->workspace, 16)) {
    mepic_set_error("beam_select: logits must be aligned to their type, the workspace to 16 bytes"); return MEPIC_E_INVAL;
  }
  if (a->score_out == a->score || (a->done && a->done_out == a->done)) { mepic_set_error("beam_select: outputs must not overlap inputs"); return MEPIC_E_INVAL; }
  SelectParams p;
  p.a = *a;
  p.segments = segments_of(a->vocab, a->logits_type);
  p.stride = stride;
  const size_t need = select_bytes(a->groups, a->width, p.segments), rows = static_cast<size_t>(a->groups) * a->width;
  if (a->workspace_bytes < need) { mepic_set_error("beam_select: workspace of %zu bytes, %zu needed", a->workspace_bytes, need); return MEPIC_E_INVAL; }
  p.sums = static_cast<WarpSum*>(a->workspace);
  p.tops = reinterpret_cast<float*>(p.sums + rows * p.segments * kSelWarps);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const dim3 grid(p.segments, static_cast<unsigned>(rows)), groups(a->groups);
  cudaError_t e;
  if (a->logits_type == MEPIC_LOGITS_BF16) {
    mepic_beam_pass<__nv_bfloat16><<<grid, kSelThreads, 0, st>>>(p);
    if ((e = cudaGetLastError()) == cudaSuccess) e = launch_dependent(mepic_beam_join<__nv_bfloat16>, groups, dim3(kSelThreads), st, p);
  } else if (a->logits_type == MEPIC_LOGITS_FP16) {
    mepic_beam_pass<__half><<<grid, kSelThreads, 0, st>>>(p);
    if ((e = cudaGetLastError()) == cudaSuccess) e = launch_dependent(mepic_beam_join<__half>, groups, dim3(kSelThreads), st, p);
  } else {
    mepic_beam_pass<float><<<grid, kSelThreads, 0, st>>>(p);
    if ((e = cudaGetLastError()) == cudaSuccess) e = launch_dependent(mepic_beam_join<float>, groups, dim3(kSelThreads), st, p);
  }
  return launched("beam_select", e, 2);
}

extern "C" size_t mepic_beam_fork_workspace(int32_t groups, int32_t width_in, int32_t width_out, int32_t table_stride) {
  if (!fork_shape_ok(groups, width_in, width_out, table_stride)) return 0;
  return fork_bytes(groups, width_in, table_stride);
}

extern "C" int32_t mepic_beam_fork(const mepic_config_t* cfg, const mepic_beam_fork_args_t* a, void* cuda_stream) {
  if (!mepic_config_ok(cfg)) return MEPIC_E_INVAL;
  if (!a) { mepic_set_error("beam_fork: NULL argument"); return MEPIC_E_INVAL; }
  if (!fork_shape_ok(a->groups, a->width_in, a->width_out, a->table_stride)) return MEPIC_E_INVAL;
  if (a->n_reserve < 0) { mepic_set_error("beam_fork: n_reserve must not be negative"); return MEPIC_E_INVAL; }
  if (!a->parent || !a->kv_len || !a->page_ids || !a->pos_base || !a->owned || (a->n_reserve > 0 && !a->reserve) || !a->reserve_used || !a->page_ids_out ||
      !a->pos_base_out || !a->kv_len_out || !a->copy_src || !a->copy_dst || !a->copy_slots || !a->n_copies || !a->reserve_used_out || !a->workspace || !a->status) {
    mepic_set_error("beam_fork: NULL pointer argument"); return MEPIC_E_INVAL;
  }
  if (a->page_ids_out == a->page_ids || a->pos_base_out == a->pos_base || a->kv_len_out == a->kv_len || a->reserve_used_out == a->reserve_used) {
    mepic_set_error("beam_fork: outputs must not overlap inputs"); return MEPIC_E_INVAL;
  }
  if (!aligned(a->workspace, 16)) { mepic_set_error("beam_fork: the workspace must be 16-byte aligned"); return MEPIC_E_INVAL; }
  const size_t need = fork_bytes(a->groups, a->width_in, a->table_stride);
  if (a->workspace_bytes < need) { mepic_set_error("beam_fork: workspace of %zu bytes, %zu needed", a->workspace_bytes, need); return MEPIC_E_INVAL; }
  ForkParams p;
  p.a = *a;
  p.page_shift = shift_of(cfg->page_size); p.num_pages = cfg->num_pages;
  fork_cut(a->groups, a->table_stride, &p.stretches, &p.stretch);
  unsigned char* ws = static_cast<unsigned char*>(a->workspace);
  p.n_freed = reinterpret_cast<int*>(ws);
  ws += up16(static_cast<size_t>(a->groups) * p.stretches * 4);
  p.n_copies = reinterpret_cast<int*>(ws);
  ws += up16(static_cast<size_t>(a->groups) * 4);
  p.freed = reinterpret_cast<int*>(ws);
  const size_t smem = (static_cast<size_t>(a->groups) * (p.stretches + 1) + 2) * sizeof(int);
  cudaError_t e = cudaSuccess;
  if (smem > 40 * 1024) e = cudaFuncSetAttribute(mepic_beam_fork_write, cudaFuncAttributeMaxDynamicSharedMemorySize, (2 * MEPIC_STEP_MAX_BATCH + 2) * static_cast<int>(sizeof(int)));
  if (e != cudaSuccess) { mepic_set_error("beam_fork: cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  mepic_beam_fork_count<<<dim3(a->groups, p.stretches), kForkThreads, static_cast<size_t>(a->width_in) * kForkThreads * sizeof(int), st>>>(p);
  e = cudaGetLastError();
  // entries of a group's tables: one a thread, but no more CTAs than give each of 148 SMs four; every CTA sums the counts up for itself
  constexpr int kCtas = 4 * 148;
  const int parts = std::max(1, std::min((a->table_stride + kForkThreads - 1) / kForkThreads, std::max(1, kCtas / a->groups)));
  if (e == cudaSuccess) e = launch_dependent(mepic_beam_fork_write, dim3(a->groups, parts), dim3(kForkThreads), smem, st, p);
  return launched("beam_fork", e, 2);
}

extern "C" int32_t mepic_pages_copy(const mepic_config_t* cfg, const mepic_pages_copy_args_t* a, void* cuda_stream) {
  return copy_call(cfg, a, nullptr, nullptr, false, cuda_stream);
}
extern "C" int32_t mepic_pages_copy_fp8(const mepic_config_t* cfg, const mepic_pages_copy_args_t* a, float* k_scales, float* v_scales,
                                        void* cuda_stream) {
  return copy_call(cfg, a, k_scales, v_scales, true, cuda_stream);
}
