// Attention of a tree of drafted tokens over the paged, un-rotated context (see mepic_attn_tree in mepic.h).
//
// One warp per (drafted row, query head): a lane holds D / 32 dims of the head as rotation pairs (i, i + D/2), every key
// is rotated by its row of the table as it is read, and the softmax runs online in fp32.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mepic.h"
#include "mepic_internal.h"
#include "mepic_ptx.cuh"
#include "mepic_rows.cuh"

namespace {

using namespace mepic_dev;

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
  int table_stride, batch, total_rows, max_rows, mask_words, q_stride, kv_stride;
  int n_kv_heads, page_size, page_shift, num_pages, max_position;
  float scale_log2;
};

template <int D, bool FP8>
__global__ void __launch_bounds__(128) mepic_tree_attn(const TreeParams p, int n_q_heads) {
  constexpr int N = D / 64;                       // rotation pairs per lane: lane + 32 j
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int row = static_cast<int>(unit / n_q_heads), hq = static_cast<int>(unit % n_q_heads);
  if (row >= p.total_rows) return;
  int b = -1;
  RowRange rr{0, 0, false};
  for (int i = 0; i < p.batch; ++i) {
    const RowRange ri = rows_of(p.row_offsets, i, p.total_rows, p.max_rows);
    if (ri.bad) atomicOr(p.status, MEPIC_DEV_BAD_TREE);
    if (b < 0 && row >= ri.lo && row < ri.lo + ri.n) { b = i; rr = ri; }
  }
  if (b < 0) return;
  const int row0 = rr.lo, n_rows = rr.n, h = hq / (n_q_heads / p.n_kv_heads);
  int kvl = p.kv_len[b];
  const long long room = static_cast<long long>(p.table_stride) << p.page_shift;
  if (kvl < 0 || kvl > room) { atomicOr(p.status, MEPIC_DEV_BAD_SLOT); kvl = kvl < 0 ? 0 : static_cast<int>(room); }
  auto bounded = [&](int pos) {
    if (pos < 0 || pos > p.max_position) { atomicOr(p.status, MEPIC_DEV_BAD_POSITION); pos = pos < 0 ? 0 : p.max_position; }
    return pos;
  };
  auto bf = [](uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); };
  float ql[N], qh[N], ol[N], oh[N], m = -INFINITY, l = 0.f;
  const float2* cq = reinterpret_cast<const float2*>(p.rope) + static_cast<size_t>(bounded(p.row_pos[row])) * (D / 2);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = lane + 32 * j;
    const uint16_t* q = p.q + static_cast<size_t>(row) * p.q_stride + hq * D;
    const float lo = bf(q[i]), hi = bf(q[i + D / 2]);
    const float2 t = cq[i];
    ql[j] = (lo * t.x - hi * t.y) * p.scale_log2; qh[j] = (lo * t.y + hi * t.x) * p.scale_log2;
    ol[j] = oh[j] = 0.f;
  }
  auto value = [&](const void* base, size_t at, float sc) {
    if (FP8) {
      uint32_t two;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"(static_cast<uint16_t>(static_cast<const unsigned char*>(base)[at])));
      return __half2float(__low2half(*reinterpret_cast<const __half2*>(&two))) * sc;
    }
    return bf(static_cast<const uint16_t*>(base)[at]);
  };
  auto key = [&](const float* kl, const float* kh, const float* vl, const float* vh, int pos) {
    const float2* ck = reinterpret_cast<const float2*>(p.rope) + static_cast<size_t>(bounded(pos)) * (D / 2);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float2 t = ck[lane + 32 * j];
      s += ql[j] * (kl[j] * t.x - kh[j] * t.y) + qh[j] * (kl[j] * t.y + kh[j] * t.x);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(kFull, s, d);
    const float mn = fmaxf(m, s), a = ex2(m - mn), w = ex2(s - mn);
    l = l * a + w;
#pragma unroll
    for (int j = 0; j < N; ++j) { ol[j] = ol[j] * a + w * vl[j]; oh[j] = oh[j] * a + w * vh[j]; }
    m = mn;
  };
  float kl[N], kh[N], vl[N], vh[N];
  for (int t = 0; t < kvl; ++t) {
    const int e = t >> p.page_shift, in_page = t & (p.page_size - 1);
    int page = p.page_ids[static_cast<size_t>(b) * p.table_stride + e];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) { atomicOr(p.status, MEPIC_DEV_BAD_PAGE); page = 0; }
    const size_t block = static_cast<size_t>(page) * p.n_kv_heads + h, at = (block * p.page_size + in_page) * D;
    const float ks = FP8 ? p.k_scales[block] : 1.f, vs = FP8 ? p.v_scales[block] : 1.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = lane + 32 * j;
      kl[j] = value(p.k_pool, at + i, ks); kh[j] = value(p.k_pool, at + i + D / 2, ks);
      vl[j] = value(p.v_pool, at + i, vs); vh[j] = value(p.v_pool, at + i + D / 2, vs);
    }
    key(kl, kh, vl, vh, p.pos_base[static_cast<size_t>(b) * p.table_stride + e] + in_page);
  }
  for (int t = 0; t < n_rows; ++t) {
    if (!((p.tree_mask[static_cast<size_t>(row) * p.mask_words + (t >> 5)] >> (t & 31)) & 1)) continue;
    const size_t at = static_cast<size_t>(row0 + t) * p.kv_stride + h * D;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = lane + 32 * j;
      kl[j] = bf(p.k_new[at + i]); kh[j] = bf(p.k_new[at + i + D / 2]);
      vl[j] = bf(p.v_new[at + i]); vh[j] = bf(p.v_new[at + i + D / 2]);
    }
    key(kl, kh, vl, vh, p.row_pos[row0 + t]);
  }
  uint16_t* o = p.out + (static_cast<size_t>(row) * n_q_heads + hq) * D;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = lane + 32 * j;
    o[i] = l > 0.f || l != l ? f32_to_bf16_bits(ol[j] / l) : 0;
    o[i + D / 2] = l > 0.f || l != l ? f32_to_bf16_bits(oh[j] / l) : 0;
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

size_t workspace_bytes(const mepic_config_t* cfg, int max_rows) { (void)cfg; (void)max_rows; return 16; }

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
  const size_t need = workspace_bytes(cfg, a->max_rows);
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
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const long long units = static_cast<long long>(a->total_rows) * cfg->n_q_heads;
  const unsigned grid = static_cast<unsigned>((units + 3) / 4);
  if (fp8) mepic_tree_attn<128, true><<<grid, 128, 0, st>>>(p, cfg->n_q_heads);
  else if (cfg->head_dim == 128) mepic_tree_attn<128, false><<<grid, 128, 0, st>>>(p, cfg->n_q_heads);
  else mepic_tree_attn<64, false><<<grid, 128, 0, st>>>(p, cfg->n_q_heads);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { mepic_set_error("%s: launch: %s", what, cudaGetErrorString(e)); return MEPIC_E_CUDA; }
  mepic_count_launches(1);
  return MEPIC_OK;
}

}  // namespace

extern "C" size_t mepic_attn_tree_workspace(const mepic_config_t* cfg, int32_t max_rows) {
  if (!mepic_config_ok(cfg)) return 0;
  if (max_rows < 0 || max_rows > MEPIC_TREE_MAX_ROWS) { mepic_set_error("attn_tree_workspace: max_rows %d not in 0..%d", max_rows, MEPIC_TREE_MAX_ROWS); return 0; }
  return workspace_bytes(cfg, max_rows);
}
extern "C" int32_t mepic_attn_tree(const mepic_config_t* cfg, const mepic_attn_tree_args_t* a, void* cuda_stream) {
  return tree_call(cfg, a, nullptr, nullptr, false, cuda_stream);
}
extern "C" int32_t mepic_attn_tree_fp8(const mepic_config_t* cfg, const mepic_attn_tree_args_t* a, const float* k_scales,
                                       const float* v_scales, void* cuda_stream) {
  return tree_call(cfg, a, k_scales, v_scales, true, cuda_stream);
}
