// The paged key / value cache as the kernels see it, and their launches (kv_cache.cu,
// kv_attention.cu).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace dcl {

constexpr int KV_EXP_MIN = -64;  // smallest exponent of a stored vector (DCL_KV_EXP_MIN)

struct KvPool {
  void *k, *v;             // [pages][G][page_len][hd] bf16 or E4M3 codes
  int8_t *k_exp, *v_exp;   // [pages][G][page_len], FP8 only
  int pages, page_shift, G, hd, fp8;
  __host__ __device__ int page_len() const { return 1 << page_shift; }
  __host__ __device__ int n_slots() const { return pages << page_shift; }
  // index of the vector of slot (page * page_len + position) and kv head g
  __device__ __forceinline__ int64_t vector_of(int slot, int g) const {
    return (((int64_t)(slot >> page_shift) * G + g) << page_shift) + (slot & (page_len() - 1));
  }
};

// 2^e for e in [-126, 127] (a slot that was never written may hold any exponent: below that, 2^-126)
__device__ __forceinline__ float kv_pow2(int e) { return __int_as_float((max(e, -126) + 127) << 23); }

cudaError_t kv_write_launch(const KvPool& kv, const __nv_bfloat16* k, const __nv_bfloat16* v, int64_t stride,
                            const int* slots, int n, int* err, cudaStream_t stream);
cudaError_t kv_read_launch(const KvPool& kv, const int* slots, int n, __nv_bfloat16* k, __nv_bfloat16* v, int64_t stride,
                           int* err, cudaStream_t stream);

// Attention of the new positions of each sequence over its cached ones.
struct KvAttn {
  const __nv_bfloat16* q;   // [rows][H][hd], row stride q_stride
  int64_t q_stride;
  const int *q_start, *table, *lens;  // [batch + 1], [batch][max_pages], [batch]
  int batch, max_pages, rows, max_new, H, causal;
  float scale;
  __nv_bfloat16* out;       // [rows][H][hd]
  float* lse;               // [rows][H] or NULL
};
// Two kernels: for up to 32 rows (new positions x query heads of a kv head) that share a kv head's keys,
// and for more (not causal).  Scratch of a launch on `sms` SMs: counters, zero before the first launch
// and left zero by each, then the parts of rows whose keys several CTAs share.  The launches of a
// context run one after another on its stream, so that both kernels use the same.
constexpr size_t KV_ATTN_COUNTERS = 4096;                                      // bytes (an int per CTA)
constexpr size_t KV_ATTN_PART_BYTES = 2 * 32 * (128 + 4) * sizeof(float);      // per CTA
constexpr size_t KV_ATTN_TC_PART_BYTES = 2 * 256 * (128 + 4) * sizeof(float);
bool kv_attention_many_rows(const KvPool& kv, const KvAttn& a);
size_t kv_attention_scratch(int sms);
size_t kv_attention_tc_scratch(int sms);
cudaError_t kv_attention_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream);
cudaError_t kv_attention_tc_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream);

// Drawing tokens (sample.cu).
struct SampleArgs {
  const __nv_bfloat16* z;   // [rows][V], row stride z_stride
  const float* noise;       // [rows][V], row stride noise_stride, or NULL
  int64_t z_stride, noise_stride;
  int rows, V;
  const float* temperature; // per row; NULL: 1
  const int* top_k;         // NULL: off
  const float *top_p, *min_p;
  int* token;
  float *prob, *conf;       // may be NULL
};
cudaError_t sample_launch(const SampleArgs& a, cudaStream_t stream);

}  // namespace dcl
