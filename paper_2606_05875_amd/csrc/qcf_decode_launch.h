// Internal launchers of the decoding calls (host side).  Arguments were validated by the C ABI
// layer; each launcher enqueues its kernels on `stream` and returns the HIP launch status.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace qcf {

// A launch takes fewer than 2^32 threads along x: longer grids go on along y.
constexpr int kGridLog2 = 23;
inline dim3 grid_of(int64_t blocks) {
  const int64_t x = (int64_t)1 << kGridLog2;
  return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)((blocks + x - 1) >> kGridLog2));
}

struct PagePlan {
  int32_t* block_table;
  int64_t table_stride;
  int max_pages, batch;
  const int32_t *kv_len, *new_len, *pages_held, *free_pages;
  int64_t n_free;
  const int32_t* free_head;
  int64_t n_pages;
  int page_log2;
  const int32_t* parents;
  uint32_t* tree_mask;
  int mask_words;
  int32_t *slots, *positions;
  int64_t n_rows;
  int32_t *cu_new, *kv_end, *pages_held_out, *free_head_out;
};
hipError_t launch_page_plan(const PagePlan& p, hipStream_t stream);

struct RopeStore {
  void *k_cache, *v_cache;
  int64_t n_slots, cache_stride;
  void* q_out;
  const void *k_new, *v_new;
  int64_t new_stride;
  const void* q_new;
  int64_t q_stride, n_src_rows;
  const int32_t* src_idx;
  int64_t n_rows;
  const int32_t *slots, *positions;
  const double* freq;
  int rotary_dim;
  float magnitude;
  int hq, hkv;
};
hipError_t launch_rope_store(const RopeStore& p, bool bf16, int head_dim, bool interleaved,
                             hipStream_t stream);

struct TreeAttn {
  void* out;
  float* lse;
  const void* q;
  int64_t n_rows;
  const int32_t* cu_q;
  const void *k_cache, *v_cache;
  int64_t n_pages, kv_stride;
  const int32_t* block_table;
  int64_t table_stride;
  int max_pages, page_log2;
  const int32_t* kv_len;
  const uint32_t* tree_mask;
  int mask_words;
  int batch, max_q, max_kv, hq, hkv;
  float scale;
};
// Whether a call whose units are taken whole, a block each, is one grid (cut ones always are).
bool tree_attn_fits(int batch, int max_q, int max_kv, int hq, int hkv, bool bf16);
size_t tree_attn_workspace(int batch, int max_q, int max_kv, int hq, int hkv, int head_dim, bool bf16);
hipError_t launch_tree_attn_f32(const TreeAttn& p, int head_dim, void* ws, hipStream_t stream);
hipError_t launch_tree_attn(const TreeAttn& p, bool bf16, int head_dim, void* ws, hipStream_t stream);

struct VerifyDrafts {
  int32_t *n_out, *path, *out_tokens;
  const void *target, *draft;
  int64_t row_stride, n_rows;
  int vocab;
  const int32_t *tokens, *parents;
  int batch;
  const int32_t* cu_rows;
  int max_rows;
  const float *u_accept, *u_next;
  const int32_t* slots;
  int32_t *move_src, *move_dst;
};
constexpr int kVerifyMaxBatch = (1 << 22) - 1;       // blocks of 1024 threads along x
constexpr int kVerifyMaxVocab = (1 << 28) - 8192;    // pieces of 4096 tokens along y
size_t verify_drafts_workspace(int batch, int vocab);
hipError_t launch_verify_drafts(const VerifyDrafts& p, bool bf16, void* ws, hipStream_t stream);

}  // namespace qcf
