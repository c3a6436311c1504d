// Attention of a few new positions of every sequence over its paged keys and values:
// out = softmax(scale q k^T) v over the sequence's cached positions.
#include <cuda_fp8.h>

#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KA_WARPS = 4;

// One block: one (row, query head).  Each warp takes every fourth key, a lane HD / 32 components.
template <int HD, bool FP8>
__global__ void __launch_bounds__(32 * KA_WARPS) kv_attention_kernel(KvPool kv, KvAttn a, int* err) {
  constexpr int E = HD / 32;
  __shared__ float part[KA_WARPS][HD + 2];
  const int row = blockIdx.x / a.H, h = blockIdx.x - row * a.H, g = h / (a.H / kv.G);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int b = 0;  // the sequence whose rows hold this one
  for (; b < a.batch; ++b)
    if (row >= a.q_start[b] && row < a.q_start[b + 1]) break;
  if (b == a.batch) return;
  const int room = a.max_pages << kv.page_shift, len = min(max(a.lens[b], 0), room);
  if (a.lens[b] != len && threadIdx.x == 0) report_error(err, DERR_KV_RANGE);
  const int n = a.causal ? min(len, len - (a.q_start[b + 1] - a.q_start[b]) + (row - a.q_start[b]) + 1) : len;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  for (int i = 0; i < E; ++i) {
    q[i] = __bfloat162float(a.q[row * a.q_stride + (int64_t)h * HD + lane * E + i]) * a.scale;
    o[i] = 0.f;
  }
  auto load = [&](const void* base, const int8_t* exps, int64_t vec, float (&x)[E]) {
    const float s = FP8 ? kv_pow2(exps[vec]) : 1.f;
    for (int i = 0; i < E; ++i) {
      const int64_t at = vec * HD + lane * E + i;
      x[i] = FP8 ? s * __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(base)[at], __NV_E4M3)))
                 : __bfloat162float(static_cast<const __nv_bfloat16*>(base)[at]);
    }
  };
  for (int j = warp; j < n; j += KA_WARPS) {
    const int page = a.table[(int64_t)b * a.max_pages + (j >> kv.page_shift)];
    if (page < 0 || page >= kv.pages) {
      if (lane == 0) report_error(err, DERR_KV_RANGE);
      continue;
    }
    const int64_t vec = kv.vector_of((page << kv.page_shift) + (j & (kv.page_len() - 1)), g);
    float x[E], s = 0.f;
    load(kv.k, kv.k_exp, vec, x);
    for (int i = 0; i < E; ++i) s = fmaf(q[i], x[i], s);
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    const float top = fmaxf(m, s), c = expf(m - top), p = expf(s - top);
    load(kv.v, kv.v_exp, vec, x);
    for (int i = 0; i < E; ++i) o[i] = fmaf(o[i], c, p * x[i]);
    l = fmaf(l, c, p);
    m = top;
  }
  for (int i = 0; i < E; ++i) part[warp][lane * E + i] = o[i];
  if (lane == 0) {
    part[warp][HD] = m;
    part[warp][HD + 1] = l;
  }
  __syncthreads();
  float top = -INFINITY, total = 0.f;
  for (int w = 0; w < KA_WARPS; ++w) top = fmaxf(top, part[w][HD]);
  for (int w = 0; w < KA_WARPS; ++w)
    if (part[w][HD + 1] > 0.f) total += part[w][HD + 1] * expf(part[w][HD] - top);
  for (int i = threadIdx.x; i < HD; i += 32 * KA_WARPS) {
    float s = 0.f;
    for (int w = 0; w < KA_WARPS; ++w)
      if (part[w][HD + 1] > 0.f) s += part[w][i] * expf(part[w][HD] - top);
    a.out[((int64_t)row * a.H + h) * HD + i] = __float2bfloat16_rn(n > 0 ? s / total : 0.f);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)row * a.H + h] = n > 0 ? top + logf(total) : -INFINITY;
}

}  // namespace

cudaError_t kv_attention_launch(const KvPool& kv, const KvAttn& a, int* err, cudaStream_t stream) {
  const unsigned grid = (unsigned)a.rows * (unsigned)a.H;
  if (kv.hd == 128 && kv.fp8) kv_attention_kernel<128, true><<<grid, 32 * KA_WARPS, 0, stream>>>(kv, a, err);
  else if (kv.hd == 128) kv_attention_kernel<128, false><<<grid, 32 * KA_WARPS, 0, stream>>>(kv, a, err);
  else if (kv.fp8) kv_attention_kernel<64, true><<<grid, 32 * KA_WARPS, 0, stream>>>(kv, a, err);
  else kv_attention_kernel<64, false><<<grid, 32 * KA_WARPS, 0, stream>>>(kv, a, err);
  return cudaGetLastError();
}

}  // namespace dcl
