// The paged key / value cache and what stands around it as the kernels see them, and their launches.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace dcl {

constexpr int KV_EXP_MIN = -64;  // smallest exponent of a stored vector (DCL_KV_EXP_MIN)

// How a pool holds its vectors (DCL_KV_*).
enum KvFormat : int { KV_BF16 = 0, KV_FP8 = 1, KV_Q4 = 4 };

struct KvPool {
  void *k, *v;             // [pages][G][page_len][hd] bf16 or E4M3 codes, or [hd / 2] bytes of 4-bit codes
  int8_t *k_exp, *v_exp;   // [pages][G][page_len] exponents (FP8), or [hd / 32] scale bytes each (Q4)
  int pages, page_shift, G, hd, format;
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
// Three kernels: for up to 8 rows (new positions x query heads of a kv head) that share a kv head's keys in 4
// bits, for up to 32 rows, and for more (not causal, or 4 bits).  Scratch of a launch on `sms` SMs: counters, zero before
// the first launch and left zero by each, then the parts of rows whose keys several CTAs share.  The launches of a
// context run one after another on its stream, so that all use the same.
constexpr size_t KV_ATTN_COUNTERS = 4096;                                      // bytes (up to three ints a CTA)
constexpr size_t KV_ATTN_PART_BYTES = 2 * 32 * (128 + 4) * sizeof(float);      // per CTA
constexpr size_t KV_ATTN_TC_PART_BYTES = 2 * 256 * (128 + 4) * sizeof(float);
bool kv_attention_q4_few(const KvPool& kv, const KvAttn& a);
cudaError_t kv_attention_q4_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream);
bool kv_attention_many_rows(const KvPool& kv, const KvAttn& a);
size_t kv_attention_scratch(int sms);
size_t kv_attention_tc_scratch(int sms);
cudaError_t kv_attention_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream);
cudaError_t kv_attention_tc_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream);

// The plan of a step (kv_plan.cu).
struct KvPlan {
  const int *start, *rows_new;  // [batch]: positions that stay, and new ones
  int *table, *held;            // [batch][max_pages], [batch]: pages of each sequence
  int *free, *n_free;           // [n_pages], [1]: a stack of the others
  int *q_start, *seq_len;       // [batch + 1], [batch]
  int *slot, *pos;              // [n_rows]
  int batch, max_pages, page_shift, n_pages, n_rows;
};
cudaError_t kv_plan_launch(const KvPlan& a, int sms, int* err, cudaStream_t stream);

// Norm and rotation of queries and keys (qk_rope.cu).
struct QkRope {
  const __nv_bfloat16 *q, *k;          // [n][H][hd], [n][G][hd]; strides in elements
  __nv_bfloat16 *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  const __nv_bfloat16 *q_gain, *k_gain;  // [hd], or NULL: no norm
  const int* pos;                      // [n]; negative: the row is left out
  int n, H, G, hd, rot;
  float eps;
  uint64_t turns[64];                  // of component i < rot / 2: its frequency, turns a position * 2^64
};
cudaError_t qk_rope_launch(const QkRope& a, int sms, cudaStream_t stream);

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
