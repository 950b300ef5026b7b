// Shared declarations of the cache entry points (vq_kv_*): geometry, host-side checks, launchers.
#pragma once

#include "vq_common.cuh"

namespace vq {

// A cache's format with derived quantities, passed by value to kernels.
struct KvGeometry {
  int n_pages, page_tokens, page_shift, heads, dim;
  int int8;             // 1: signed 8-bit keys and values with a binary32 scale per token and head
  int row_bytes;        // one token's keys of one head
};

struct KvPool {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
};

struct KvBooks {
  int* table;
  int* len;
  int n_seqs, table_stride;
  int max_len;          // table_stride * page_tokens
};

// Kernel arguments of the pools of all layers (by value: 32 bytes a layer).
struct KvPools {
  KvPool p[VQ_KV_MAX_LAYERS];
  int n_layers;
};

struct KvRotary {
  const float2* cs;      // [n_positions][rot_dim / 2], or null: nothing is rotated
  int rot_dim, interleaved, n_q_heads;
  const __half* q;
  __half* q_out;
  long long q_stride, q_out_stride;
};

vq_status launch_kv_attention(const KvGeometry& g, const KvPool& pool, const KvBooks& books, int n_q_heads, const __half* q,
                              long long q_stride, __half* out, long long out_stride, float* lse, float scale, int window, void* ws,
                              cudaStream_t s);
size_t kv_attention_workspace_bytes(int head_dim);
bool kv_attention_covers(const KvGeometry& g);

vq_status launch_kv_append(const KvGeometry& g, const KvPool& pool, const KvBooks& books, const int* starts, int n_tokens,
                           const __half* k, long long k_stride, const __half* v, long long v_stride, const KvRotary& rot, cudaStream_t s);

size_t kv_pages_workspace_bytes(const KvGeometry& g, int n_seqs);
vq_status launch_kv_reserve(const KvGeometry& g, const KvBooks& books, int* refs, const int* grow, int* status, void* ws, cudaStream_t s);
vq_status launch_kv_fork(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, const int* pairs, int n_pairs,
                         int* status, void* ws, cudaStream_t s);
vq_status launch_kv_free(const KvGeometry& g, const KvBooks& books, int* refs, const int* slots, int n_slots, cudaStream_t s);
vq_status launch_kv_compact(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, int* status, void* ws,
                            cudaStream_t s);
vq_status launch_kv_copy_pages(const KvGeometry& g, const KvPools& pools, const int* pairs, int n_pairs, cudaStream_t s);

#ifdef __CUDACC__
// Launch with programmatic stream serialisation: the kernel's first statement is pdl_wait(), so only its start overlaps
// the end of the kernel in front of it.
template <class... P, class... A>
inline vq_status launch_dependent(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
    (void)cudaGetLastError();
    return VQ_ERR_CUDA;
  }
  return check_launch();
}
#endif

}  // namespace vq
