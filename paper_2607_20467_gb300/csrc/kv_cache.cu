// The paged key / value cache: writing the keys and values of new positions into their pages
// (quantising them on the way) and reading positions back.
//
// A page holds page_len positions of every kv head as [kv head][position][hd], so that the keys of
// one head that an attention walks are contiguous.  FP8 storage: one vector of hd components is
// codes (E4M3) and one exponent e, a ~ code * 2^e with e the least integer that fits the largest
// finite component into 448 * 2^e (at least KV_EXP_MIN), so scaling by 2^-e and widening a code to
// bf16 are both exact: the code's rounding is the only one.
//
// 4 bits: groups of 32 components, 4-bit multiples -7 .. 7 of a scale (q4.cuh), the least one that reaches
// the largest, each code the nearest; a group with an infinity or NaN in it is marked as none.
//
// Both kernels are bound by memory.  A thread has 16 components of a vector (two 16-byte loads, one
// 16-byte or 8-byte store of codes) of two vectors at once; hd / 16 threads find a vector's maximum by
// shuffles, two a group's.  12288 positions of 32 heads x 128, FP8 (302 MB): written in 44.8 us, 6.7 TB/s, 0.99 of
// the measured copy rate; read back in 46.9 us, 0.95 (two thirds of that traffic are writes).  4 bits (255 MB):
// 43.8 us, 0.86 (a component's 3.5 instructions beside it: 0.8 of the issue slots) and 44.4 us, 0.85 (four
// fifths writes).  32 positions: 2 us of kernel in a call of 4.5.  (256 threads a block: 1.5 to 2 us more for each.)
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "kv_cache.cuh"
#include "q4.cuh"

namespace dcl {
namespace {

constexpr int KV_THREADS = 64;
constexpr int KV_EACH = 2;   // parts of a vector that a thread has in flight
constexpr int KV_COMP = 16;  // components of a part

// A thread's parts: part `at` of the call's [row][k, v][kv head][HD / 16], in blocks of KV_THREADS *
// KV_EACH.  per_row and its reciprocals (rounded up: 2^32 of it, exact for the few rows of a block, and 2^64,
// exact for all that a call has) come from the host: 64-bit divisions took longer than the copy.
struct KvPart {
  int row, is_v, g, part;
};
struct KvOver {
  uint64_t row64;
  uint32_t row32;
};
template <int HD>
struct KvWalk {
  static constexpr int TPV = HD / KV_COMP;  // threads of a vector
  int64_t row0;
  uint32_t rest, per_row, inverse;
  int G;
  __device__ KvWalk(int G_, const KvOver& over) : per_row(2 * G_ * TPV), inverse(over.row32), G(G_) {
    const uint64_t start = (uint64_t)blockIdx.x * (KV_THREADS * KV_EACH);
    row0 = (int64_t)__umul64hi(start, over.row64);
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

// Codes (16 of 4 bits) and the scale byte of a part's group, which two neighbouring threads share; all
// threads of a warp call it.
//
// The quotient by d = 4 .. 7 times a power of two comes out in fp32 to 2^-21 of itself (a reciprocal to two units
// of its last place, and a product) and is rounded to fp16, which puts ties right: half a whole number is an fp16
// number and nearer than the next by 2^-12 of itself at least; a quotient of 8 bits by 3 that is not halfway is off
// that by 1/255 of itself or more, eight times fp16's half step.  Adding 1.5 2^10 + 8 rounds it to a whole number, 8 above, in the low bits.  Two at a
// time, components i and i + 4 of a word's eight, as their codes lie in it; pairs are put together by
// multiplying and adding, where what stands above their four bits comes to a constant.  That is 3.5 instructions
// a component: with each code rounded and cut out by itself there were ten, and 12288 positions of 32 heads x
// 128 took 55 us instead of 43.8.
__device__ __forceinline__ uint2 quantise_q4(KvBf16& a, uint32_t& scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, a.word(i) & 0x7fff7fffu);
  m = max(m & 0xffffu, m >> 16);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  // The largest is f 2^x, f = 128 .. 255.  7 (4 + i) 2^k, the largest a scale reaches, passes 128 2^x,
  // 140 2^x, ... in turn: 35, 42, 49 at k = x + 2, then 28 and 35 at x + 3.  Bytes count through them.
  const int x = (int)(m >> 7) - 134, f = (int)(m & 0x7fu) + 128;
  const int fits = 4 * (x + 42) + 1 + (f > 140) + (f > 168) + (f > 196) + (f > 224), b = min(Q4_SCALES - 1, max(0, fits));
  scale = m >= 0x7f80u ? Q4_NONE : (uint32_t)b;
  if (m >= 0x7f80u) return make_uint2(0x88888888u, 0x88888888u);
  const float over = __fdividef(1.f, (float)(4 + (b & 3))) * __int_as_float((127 + 40 - (b >> 2)) << 23);
  const __half2 round = __halves2half2(__ushort_as_half(0x6608), __ushort_as_half(0x6608));  // 1.5 2^10 + 8
  constexpr uint32_t ABOVE = 0x66006600u * 0x1111u;  // (what the sums of four have too much)
  uint32_t out[2];
  auto codes = [&](auto limit) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 3; j >= 0; --j) {  // components j and j + 4
        const uint32_t first = a.word(4 * i + j / 2), second = a.word(4 * i + 2 + j / 2);
        const float v0 = j & 1 ? bf16_hi(first) : bf16_lo(first), v1 = j & 1 ? bf16_hi(second) : bf16_lo(second);
        const __half2 y = __hadd2(__floats2half2_rn(limit(v0 * over), limit(v1 * over)), round);
        w = w * 16u + *reinterpret_cast<const uint32_t*>(&y);
      }
      out[i] = w - ABOVE;
    }
  };
  if (fits <= Q4_SCALES - 1) codes([](float y) { return y; });
  else codes([](float y) { return fminf(7.f, fmaxf(-7.f, y)); });  // (past the largest scale)
  return make_uint2(out[0], out[1]);
}

template <int HD, KvFormat F>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvPool kv, const __nv_bfloat16* __restrict__ k,
                                                              const __nv_bfloat16* __restrict__ v, int64_t stride,
                                                              const int* __restrict__ slots, int n, KvOver over,
                                                              int* err) {
  const KvWalk<HD> walk(kv.G, over);
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
    uint2 codes4;
    uint32_t scales;
    if (F == KV_FP8) codes = quantise<HD>(raw[i], e);
    if (F == KV_Q4) {
      codes4 = quantise_q4(raw[i], scales);
      scales <<= 8 * (p.part >> 1);  // the vector's bytes side by side
      scales |= __shfl_xor_sync(0xffffffffu, scales, 2);
      if (HD == 128) scales |= __shfl_xor_sync(0xffffffffu, scales, 4);
    }
    if (slot[i] < 0) continue;
    if (slot[i] >= kv.n_slots()) {
      report_error(err, DERR_KV_RANGE);
      continue;
    }
    const int64_t vec = kv.vector_of(slot[i], p.g);
    if (F == KV_Q4) {
      (reinterpret_cast<uint2*>(p.is_v ? kv.v : kv.k))[vec * TPV + p.part] = codes4;
      if (p.part == 0) {
        int8_t* to = (p.is_v ? kv.v_exp : kv.k_exp) + vec * (HD / Q4_GROUP);
        if (HD == 128) *reinterpret_cast<uint32_t*>(to) = scales;
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)scales;
      }
      continue;
    }
    uint4* to = reinterpret_cast<uint4*>(p.is_v ? kv.v : kv.k) + (vec * TPV + p.part) * (F == KV_FP8 ? 1 : 2);
    if (F == KV_BF16) {
      to[0] = raw[i].x[0];
      to[1] = raw[i].x[1];
    } else {
      to[0] = codes;
      if (p.part == 0) (p.is_v ? kv.v_exp : kv.k_exp)[vec] = (int8_t)e;
    }
  }
}

// A part (32 bytes) stored by two neighbouring threads together with the neighbour's: each store of a warp then
// covers whole sectors, where threads that store their own cover a half of each twice.
__device__ __forceinline__ void store_pair(uint4* to, const KvBf16& a, bool live) {
  const bool odd = threadIdx.x & 1;
  const uint4 mine = odd ? a.x[0] : a.x[1];
  const uint4 other = make_uint4(__shfl_xor_sync(0xffffffffu, mine.x, 1), __shfl_xor_sync(0xffffffffu, mine.y, 1),
                                 __shfl_xor_sync(0xffffffffu, mine.z, 1), __shfl_xor_sync(0xffffffffu, mine.w, 1));
  if (!live) return;
  // the even thread's part, then the odd one's: their first halves by the even thread
  to[odd ? -1 : 0] = odd ? other : a.x[0];
  to[odd ? 1 : 2] = odd ? a.x[1] : other;
}

template <int HD, KvFormat F>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvPool kv, const int* __restrict__ slots, int n,
                                                             __nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ v,
                                                             int64_t stride, KvOver over, int* err) {
  const KvWalk<HD> walk(kv.G, over);
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
    if (F == KV_Q4) {
      const uint2 codes = (reinterpret_cast<const uint2*>(p.is_v ? kv.v : kv.k))[vec[i] * TPV + p.part];
      raw[i].x[0].x = codes.x;
      raw[i].x[0].y = codes.y;
      e[i] = (uint8_t)(p.is_v ? kv.v_exp : kv.k_exp)[vec[i] * (HD / Q4_GROUP) + (p.part >> 1)];
      continue;
    }
    const uint4* from = reinterpret_cast<const uint4*>(p.is_v ? kv.v : kv.k) + (vec[i] * TPV + p.part) * (F == KV_FP8 ? 1 : 2);
    raw[i].x[0] = from[0];
    if (F == KV_BF16) raw[i].x[1] = from[1];
    if (F == KV_FP8) e[i] = (p.is_v ? kv.v_exp : kv.k_exp)[vec[i]];
  }
#pragma unroll
  for (int i = 0; i < KV_EACH; ++i) {
    const KvPart p = walk.at(i);
    if (F == KV_Q4 && vec[i] >= 0) {
      const Q4Scale f = q4_scale_twice((uint32_t)e[i]);
      const uint32_t codes[2] = {raw[i].x[0].x, raw[i].x[0].y};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t y[4];  // components 0 and 4, 1 and 5, ...
#pragma unroll
        for (int z = 0; z < 4; ++z) y[z] = q4_widen(codes[j], z, f);
        raw[i].x[j] = make_uint4(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410),
                                 __byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
      }
    }
    if (F == KV_FP8) {
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
    store_pair(reinterpret_cast<uint4*>((p.is_v ? v : k) + p.row * stride + (p.g * HD + KV_COMP * p.part)), raw[i], p.row < n);
  }
}

// Blocks of a call, and the reciprocal of a row's parts for KvWalk: x / per_row is exact for the
// x < per_row + KV_THREADS * KV_EACH that a block divides while x * per_row < 2^32.
bool kv_grid(const KvPool& kv, int n, unsigned* grid, KvOver* over) {
  const int64_t per_row = 2 * (int64_t)kv.G * (kv.hd / KV_COMP), per_block = KV_THREADS * KV_EACH;
  const int64_t blocks = (n * per_row + per_block - 1) / per_block;
  if (blocks > 0x7fffffff || (per_row + per_block) * per_row >= (1ll << 32)) return false;
  *grid = (unsigned)blocks;
  over->row32 = (uint32_t)(((1ll << 32) + per_row - 1) / per_row);
  over->row64 = ~0ull / (uint64_t)per_row + 1;  // (x * per_row < 2^64 for the x < 2^38 of a grid)
  return true;
}

// The launch of a cache's head size and format.
template <typename Launch>
cudaError_t for_layout(const KvPool& kv, Launch launch) {
  auto as = [&](auto hd) {
    if (kv.format == KV_Q4) launch(hd, std::integral_constant<KvFormat, KV_Q4>{});
    else if (kv.format == KV_FP8) launch(hd, std::integral_constant<KvFormat, KV_FP8>{});
    else launch(hd, std::integral_constant<KvFormat, KV_BF16>{});
  };
  if (kv.hd == 128) as(std::integral_constant<int, 128>{});
  else as(std::integral_constant<int, 64>{});
  return cudaGetLastError();
}

}  // namespace

cudaError_t kv_write_launch(const KvPool& kv, const __nv_bfloat16* k, const __nv_bfloat16* v, int64_t stride,
                            const int* slots, int n, int* err, cudaStream_t stream) {
  unsigned grid;
  KvOver over;
  if (!kv_grid(kv, n, &grid, &over)) return cudaErrorInvalidValue;
  return for_layout(kv, [&](auto hd, auto format) {
    kv_write_kernel<decltype(hd)::value, decltype(format)::value><<<grid, KV_THREADS, 0, stream>>>(kv, k, v, stride, slots, n, over, err);
  });
}

cudaError_t kv_read_launch(const KvPool& kv, const int* slots, int n, __nv_bfloat16* k, __nv_bfloat16* v, int64_t stride,
                           int* err, cudaStream_t stream) {
  unsigned grid;
  KvOver over;
  if (!kv_grid(kv, n, &grid, &over)) return cudaErrorInvalidValue;
  return for_layout(kv, [&](auto hd, auto format) {
    kv_read_kernel<decltype(hd)::value, decltype(format)::value><<<grid, KV_THREADS, 0, stream>>>(kv, slots, n, k, v, stride, over, err);
  });
}

}  // namespace dcl
