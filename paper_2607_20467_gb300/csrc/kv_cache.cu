// The paged key / value cache: writing the keys and values of new positions into their pages
// (quantising them on the way) and reading positions back.
//
// A page holds page_len positions of every kv head as [kv head][position][hd], so that the keys of
// one head that an attention walks are contiguous.  FP8 storage: one vector of hd components is
// codes (E4M3) and one exponent e, a ~ code * 2^e with e the least integer that fits the largest
// finite component into 448 * 2^e (at least KV_EXP_MIN), so scaling by 2^-e and widening a code to
// bf16 are both exact: the code's rounding is the only one.
#include <cuda_fp8.h>

#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KV_THREADS = 256;

// One thread: 8 components of one vector of k or v (HD / 8 threads a vector).
template <int HD, bool FP8>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvPool kv, const __nv_bfloat16* __restrict__ k,
                                                              const __nv_bfloat16* __restrict__ v, int64_t stride,
                                                              const int* __restrict__ slots, int n, int* err) {
  constexpr int TPV = HD / 8;
  const int64_t item = ((int64_t)blockIdx.x * KV_THREADS + threadIdx.x) / TPV;  // [row][k, v][head]
  const int part = threadIdx.x % TPV;
  const int64_t row = item / (2 * kv.G);
  if (row >= n) return;  // (a vector's threads are of one warp and leave together)
  const int which = (int)(item - row * (2 * kv.G)), is_v = which >= kv.G, g = which - is_v * kv.G;
  const int slot = slots[row];
  if (slot < 0) return;
  if (slot >= kv.n_slots()) {
    report_error(err, DERR_KV_RANGE);
    return;
  }
  const uint4 raw = *reinterpret_cast<const uint4*>((is_v ? v : k) + row * stride + (int64_t)g * HD + 8 * part);
  const int64_t vec = kv.vector_of(slot, g);
  if (!FP8) {
    reinterpret_cast<uint4*>(is_v ? kv.v : kv.k)[vec * TPV + part] = raw;
    return;
  }
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t top = 0;  // largest finite magnitude, as bf16 bits (ordered as the values)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    top = max(top, lo < 0x7f80u ? lo : 0u);
    top = max(top, hi < 0x7f80u ? hi : 0u);
  }
  const uint32_t mask = (TPV == 16 ? 0xffffu : 0xffu) << ((threadIdx.x & 31) & ~(TPV - 1));  // the vector's threads
#pragma unroll
  for (int d = TPV / 2; d; d >>= 1) top = max(top, __shfl_xor_sync(mask, top, d));
  // 448 * 2^e = 1.75 * 2^(e + 8): the exponent field decides, and whether the fraction passes 1.75
  const int e = top ? max(KV_EXP_MIN, (int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u)) : 0;
  const float scale = kv_pow2(-e);
  uint32_t out[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t both = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float lo = bf16_lo(w[2 * i + j]) * scale, hi = bf16_hi(w[2 * i + j]) * scale;
      // (the format has no infinities: they become its NaN, so that they are not taken for 448)
      lo = isinf(lo) ? __int_as_float(0x7fffffff) : lo;
      hi = isinf(hi) ? __int_as_float(0x7fffffff) : hi;
      both |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3) << (16 * j);
    }
    out[i] = both;
  }
  reinterpret_cast<uint2*>(is_v ? kv.v : kv.k)[vec * TPV + part] = make_uint2(out[0], out[1]);
  if (part == 0) (is_v ? kv.v_exp : kv.k_exp)[vec] = (int8_t)e;
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvPool kv, const int* __restrict__ slots, int n,
                                                             __nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ v,
                                                             int64_t stride, int* err) {
  constexpr int TPV = HD / 8;
  const int64_t item = ((int64_t)blockIdx.x * KV_THREADS + threadIdx.x) / TPV;
  const int part = threadIdx.x % TPV;
  const int64_t row = item / (2 * kv.G);
  if (row >= n) return;
  const int which = (int)(item - row * (2 * kv.G)), is_v = which >= kv.G, g = which - is_v * kv.G;
  const int slot = slots[row];
  uint4 raw = make_uint4(0, 0, 0, 0);
  if (slot >= kv.n_slots()) {
    report_error(err, DERR_KV_RANGE);
  } else if (slot >= 0) {
    const int64_t vec = kv.vector_of(slot, g);
    if (!FP8) {
      raw = reinterpret_cast<const uint4*>(is_v ? kv.v : kv.k)[vec * TPV + part];
    } else {
      const uint2 codes = reinterpret_cast<const uint2*>(is_v ? kv.v : kv.k)[vec * TPV + part];
      const float scale = kv_pow2((is_v ? kv.v_exp : kv.k_exp)[vec]);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t pair = ((i < 2 ? codes.x : codes.y) >> (16 * (i & 1))) & 0xffffu;
        const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
        w[i] = pack_bf16x2(f.x * scale, f.y * scale);
      }
      raw = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  *reinterpret_cast<uint4*>((is_v ? v : k) + row * stride + (int64_t)g * HD + 8 * part) = raw;
}

}  // namespace

cudaError_t kv_write_launch(const KvPool& kv, const __nv_bfloat16* k, const __nv_bfloat16* v, int64_t stride,
                            const int* slots, int n, int* err, cudaStream_t stream) {
  const int64_t blocks = ((int64_t)n * 2 * kv.G * (kv.hd / 8) + KV_THREADS - 1) / KV_THREADS;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)blocks;
  if (kv.hd == 128 && kv.fp8) kv_write_kernel<128, true><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, err);
  else if (kv.hd == 128) kv_write_kernel<128, false><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, err);
  else if (kv.fp8) kv_write_kernel<64, true><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, err);
  else kv_write_kernel<64, false><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, err);
  return cudaGetLastError();
}

cudaError_t kv_read_launch(const KvPool& kv, const int* slots, int n, __nv_bfloat16* k, __nv_bfloat16* v, int64_t stride,
                           int* err, cudaStream_t stream) {
  const int64_t blocks = ((int64_t)n * 2 * kv.G * (kv.hd / 8) + KV_THREADS - 1) / KV_THREADS;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)blocks;
  if (kv.hd == 128 && kv.fp8) kv_read_kernel<128, true><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, err);
  else if (kv.hd == 128) kv_read_kernel<128, false><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, err);
  else if (kv.fp8) kv_read_kernel<64, true><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, err);
  else kv_read_kernel<64, false><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, err);
  return cudaGetLastError();
}

}  // namespace dcl
