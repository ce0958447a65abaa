// Internal launchers of the calls of qcf_turns.h (host side).  Arguments were validated by the C ABI
// layer; each launcher enqueues its kernels on `stream` and returns the HIP launch status.
#pragma once
#include "qcf_decode_launch.h"

namespace qcf {

struct NormRopeStore : RopeStore {
  const void *q_weight, *k_weight;
  int64_t q_weight_stride, k_weight_stride;
  float eps;
};
hipError_t launch_norm_rope_store(const NormRopeStore& p, bool bf16, int head_dim, bool interleaved,
                                  hipStream_t stream);

struct ChunkAttn : TreeAttn {
  int window;
};
bool chunk_attn_fits(int batch, int max_q, int hq, int hkv, bool bf16);
size_t chunk_attn_workspace(int max_q, int hq, int hkv, int head_dim, bool bf16);
hipError_t launch_chunk_attn_f32(const ChunkAttn& p, int head_dim, void* ws, hipStream_t stream);
hipError_t launch_chunk_attn(const ChunkAttn& p, bool bf16, int head_dim, void* ws, hipStream_t stream);

struct ShapeLogits {
  void* out;
  int64_t out_stride;
  const void* logits;
  int64_t logits_stride, n_rows;
  int vocab, batch;
  const int32_t *cu_rows, *history;
  int64_t history_stride;
  int max_history;
  const int32_t *prompt_len, *hist_len, *tokens;
  const uint32_t* tree_mask;
  int mask_words;
  const float *repetition, *presence, *frequency;
  const int32_t *bias_start, *bias_token;
  const float* bias_value;
  int64_t n_bias;
  const uint32_t* allowed;
  int64_t allowed_words;
  const float* temperature;
};
constexpr int kShapeMaxVocab = 1 << 28;
size_t shape_logits_workspace(int64_t n_rows, int vocab);
hipError_t launch_shape_logits(const ShapeLogits& p, bool in_bf16, bool out_bf16, bool probabilities, void* ws,
                               hipStream_t stream);

struct PageFork {
  int32_t* table_out;
  int64_t table_out_stride;
  int32_t *kv_out, *held_out;
  const int32_t* block_table;
  int64_t table_stride;
  int max_pages, batch;
  const int32_t *kv_len, *source, *keep_len, *free_pages;
  int64_t n_free;
  const int32_t* free_head;
  int64_t n_pages;
  int page_log2;
  int32_t *free_head_out, *copy_src, *copy_dst, *copy_rows;
};
hipError_t launch_page_fork(const PageFork& p, hipStream_t stream);

struct CopyPages {
  void* const* pools;
  int n_pools;
  int64_t n_pages, row_bytes, row_stride;
  int page_log2;
  const int32_t *src_page, *dst_page, *rows;
  int64_t n_pairs;
};
int64_t copy_pages_blocks(const CopyPages& p);
hipError_t launch_copy_pages(const CopyPages& p, hipStream_t stream);

struct PageRelease {
  const int32_t* before;
  int64_t before_stride;
  const int32_t *held_before, *after;
  int64_t after_stride;
  const int32_t* held_after;
  int max_pages, batch;
  int32_t* free_pages;
  int64_t n_free;
  const int32_t* free_head;
  int32_t* free_head_out;
  int64_t n_pages;
};
size_t page_release_workspace(int batch, int max_pages, int64_t n_pages);
hipError_t launch_page_release(const PageRelease& p, void* ws, hipStream_t stream);

}  // namespace qcf
