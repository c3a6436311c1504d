// The paged key / value cache: writing the keys and values of new positions into their pages
// (quantising them on the way) and reading positions back.
//
// A page holds page_len positions of every kv head as [kv head][position][hd], so that the keys of
// one head that an attention walks are contiguous.  FP8 storage: one vector of hd components is
// codes (E4M3) and one exponent e, a ~ code * 2^e with e the least integer that fits the largest
// finite component into 448 * 2^e (at least KV_EXP_MIN), so scaling by 2^-e and widening a code to
// bf16 are both exact: the code's rounding is the only one.
//
// Both kernels are bound by memory.  A thread has 16 components of a vector (two 16-byte loads, one
// 16-byte store of codes) of two vectors at once; hd / 16 threads find a vector's maximum by
// shuffles.  12288 positions of 32 heads x 128 (302 MB): written in 47.2 us, 6.4 TB/s, 0.94 of the
// measured copy rate; read back in 52.9 us, 5.7 TB/s, 0.84 (two thirds of that traffic are
// writes).  32 positions: 2 to 3 us of kernel in a call of 5.1.
#include <cuda_fp8.h>

#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_EACH = 2;   // parts of a vector that a thread has in flight
constexpr int KV_COMP = 16;  // components of a part

// A thread's parts: part `at` of the call's [row][k, v][kv head][HD / 16], in blocks of KV_THREADS *
// KV_EACH.  per_row and its reciprocal (rounded up, exact for the few rows of a block) come from
// the host: a 64-bit division per part took longer than the copy.
struct KvPart {
  int row, is_v, g, part;
};
template <int HD>
struct KvWalk {
  static constexpr int TPV = HD / KV_COMP;  // threads of a vector
  int64_t row0;
  uint32_t rest, per_row, inverse;
  int G;
  __device__ KvWalk(int G_, uint32_t inverse_) : per_row(2 * G_ * TPV), inverse(inverse_), G(G_) {
    const int64_t start = (int64_t)blockIdx.x * (KV_THREADS * KV_EACH);
    row0 = start / per_row;
    rest = (uint32_t)(start - row0 * per_row);
  }
  __device__ __forceinline__ KvPart at(int i) const {
    const uint32_t x = rest + i * KV_THREADS + threadIdx.x, r = __umulhi(x, inverse), in_row = x - r * per_row;
    const int vec = (int)(in_row / TPV), is_v = vec >= G;
    return KvPart{(int)(row0 + r), is_v, vec - is_v * G, (int)(in_row % TPV)};
  }
};

// A part in bf16, its codes, and both ways between them.
struct KvBf16 {
  uint4 x[2];
  __device__ __forceinline__ uint32_t& word(int i) { return (&x[i >> 2].x)[i & 3]; }
};

// Codes of a part and its vector's exponent; all threads of a warp call it.
template <int HD>
__device__ __forceinline__ uint4 quantise(KvBf16& a, int& e) {
  constexpr int TPV = HD / KV_COMP;
  // largest magnitude of the vector, as bf16 bits (ordered as the values)
  auto largest = [&]() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, a.word(i) & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int d = TPV / 2; d; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
  };
  uint32_t top = largest();
  uint32_t strange = 0;  // components that are no numbers: out of the exponent, NaN in the end
  if (__any_sync(0xffffffffu, top >= 0x7f80u)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w = a.word(i), lo = (w & 0x7fffu) >= 0x7f80u, hi = (w & 0x7fff0000u) >= 0x7f800000u;
      strange |= lo << (2 * i) | hi << (2 * i + 1);
      a.word(i) = w & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
    }
    top = largest();
  }
  // 448 * 2^e = 1.75 * 2^(e + 8): the exponent field decides, and whether the fraction passes 1.75
  e = top ? max(KV_EXP_MIN, (int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u)) : 0;
  const float scale = kv_pow2(-e);
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t two[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t w = a.word(2 * i + j);
      two[j] = __nv_cvt_float2_to_fp8x2(make_float2(bf16_lo(w) * scale, bf16_hi(w) * scale), __NV_SATFINITE, __NV_E4M3);
    }
    out[i] = two[0] | two[1] << 16;
  }
  if (strange) {  // (the format has no infinities: they become its NaN, so that they are not taken for 448)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (strange >> i & 1) out[i >> 2] |= 0x7fu << (8 * (i & 3));
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvPool kv, const __nv_bfloat16* __restrict__ k,
                                                              const __nv_bfloat16* __restrict__ v, int64_t stride,
                                                              const int* __restrict__ slots, int n, uint32_t inverse,
                                                              int* err) {
  const KvWalk<HD> walk(kv.G, inverse);
  constexpr int TPV = HD / KV_COMP;
  KvBf16 raw[KV_EACH];
  int slot[KV_EACH];
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    raw[i].x[0] = raw[i].x[1] = make_uint4(0, 0, 0, 0);
    slot[i] = -1;
    if (p.row < n) {
      slot[i] = slots[p.row];
      const uint4* from = reinterpret_cast<const uint4*>((p.is_v ? v : k) + p.row * stride + (p.g * HD + KV_COMP * p.part));
      raw[i].x[0] = from[0];
      raw[i].x[1] = from[1];
    }
  }
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    int e = 0;
    uint4 codes;
    if (FP8) codes = quantise<HD>(raw[i], e);
    if (slot[i] < 0) continue;
    if (slot[i] >= kv.n_slots()) {
      report_error(err, DERR_KV_RANGE);
      continue;
    }
    const int64_t vec = kv.vector_of(slot[i], p.g);
    uint4* to = reinterpret_cast<uint4*>(p.is_v ? kv.v : kv.k) + (vec * TPV + p.part) * (FP8 ? 1 : 2);
    if (!FP8) {
      to[0] = raw[i].x[0];
      to[1] = raw[i].x[1];
    } else {
      to[0] = codes;
      if (p.part == 0) (p.is_v ? kv.v_exp : kv.k_exp)[vec] = (int8_t)e;
    }
  }
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvPool kv, const int* __restrict__ slots, int n,
                                                             __nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ v,
                                                             int64_t stride, uint32_t inverse, int* err) {
  const KvWalk<HD> walk(kv.G, inverse);
  constexpr int TPV = HD / KV_COMP;
  int64_t vec[KV_EACH];  // -1: zeros
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    const int slot = p.row < n ? slots[p.row] : -1;
    vec[i] = -1;
    if (slot >= kv.n_slots()) report_error(err, DERR_KV_RANGE);
    else if (slot >= 0) vec[i] = kv.vector_of(slot, p.g);
  }
  KvBf16 raw[KV_EACH];
  int e[KV_EACH];
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    raw[i].x[0] = raw[i].x[1] = make_uint4(0, 0, 0, 0);
    e[i] = 0;
    if (vec[i] < 0) continue;
    const uint4* from = reinterpret_cast<const uint4*>(p.is_v ? kv.v : kv.k) + (vec[i] * TPV + p.part) * (FP8 ? 1 : 2);
    raw[i].x[0] = from[0];
    if (!FP8) raw[i].x[1] = from[1];
    if (FP8) e[i] = (p.is_v ? kv.v_exp : kv.k_exp)[vec[i]];
  }
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    if (p.row >= n) continue;
    if (FP8) {
      const float scale = kv_pow2(e[i]);
      const uint4 codes = raw[i].x[0];
      const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t pair = (c[j >> 1] >> (16 * (j & 1))) & 0xffffu;
        const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
        raw[i].word(j) = pack_bf16x2(f.x * scale, f.y * scale);
      }
    }
    uint4* to = reinterpret_cast<uint4*>((p.is_v ? v : k) + p.row * stride + (p.g * HD + KV_COMP * p.part));
    to[0] = raw[i].x[0];
    to[1] = raw[i].x[1];
  }
}

// Blocks of a call, and the reciprocal of a row's parts for KvWalk: x / per_row is exact for the
// x < per_row + KV_THREADS * KV_EACH that a block divides while x * per_row < 2^32.
bool kv_grid(const KvPool& kv, int n, unsigned* grid, uint32_t* inverse) {
  const int64_t per_row = 2 * (int64_t)kv.G * (kv.hd / KV_COMP), per_block = KV_THREADS * KV_EACH;
  const int64_t blocks = (n * per_row + per_block - 1) / per_block;
  if (blocks > 0x7fffffff || (per_row + per_block) * per_row >= (1ll << 32)) return false;
  *grid = (unsigned)blocks;
  *inverse = (uint32_t)(((1ll << 32) + per_row - 1) / per_row);
  return true;
}

}  // namespace

cudaError_t kv_write_launch(const KvPool& kv, const __nv_bfloat16* k, const __nv_bfloat16* v, int64_t stride,
                            const int* slots, int n, int* err, cudaStream_t stream) {
  unsigned grid;
  uint32_t inv;
  if (!kv_grid(kv, n, &grid, &inv)) return cudaErrorInvalidValue;
  if (kv.hd == 128 && kv.fp8) kv_write_kernel<128, true><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, inv, err);
  else if (kv.hd == 128) kv_write_kernel<128, false><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, inv, err);
  else if (kv.fp8) kv_write_kernel<64, true><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, inv, err);
  else kv_write_kernel<64, false><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, inv, err);
  return cudaGetLastError();
}

cudaError_t kv_read_launch(const KvPool& kv, const int* slots, int n, __nv_bfloat16* k, __nv_bfloat16* v, int64_t stride,
                           int* err, cudaStream_t stream) {
  unsigned grid;
  uint32_t inv;
  if (!kv_grid(kv, n, &grid, &inv)) return cudaErrorInvalidValue;
  if (kv.hd == 128 && kv.fp8) kv_read_kernel<128, true><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, inv, err);
  else if (kv.hd == 128) kv_read_kernel<128, false><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, inv, err);
  else if (kv.fp8) kv_read_kernel<64, true><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, inv, err);
  else kv_read_kernel<64, false><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, inv, err);
  return cudaGetLastError();
}

}  // namespace dcl
