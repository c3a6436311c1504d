// RMSNorm of every head of queries and keys, and the rotation by their positions, in one pass:
//
//   y = x / sqrt(mean x^2 + eps) * gain;  (y_i, y_(i + h)) -> (y_i cos - y_(i + h) sin, y_(i + h) cos + y_i sin)
//
// for i < h = rot / 2, the angle pos * theta^(-i / h); components past rot are normed only.
//
// An angle is needed modulo a turn, and positions are whole numbers: with the frequency as a 64-bit
// fraction of a turn, the product modulo 2^64 is the fraction exactly, however far the position (a
// product in fp32 is off by 2^-24 of up to 10^5 turns).
#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int QR_THREADS = 256;

__device__ __forceinline__ void unpack8(const uint4& x, float* f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo(w[i]);
    f[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// hd / 16 threads have a head, two chunks of 8 components each: i and i + h of those that rotate.
template <int HD>
__global__ void __launch_bounds__(QR_THREADS) qk_rope_kernel(QkRope a) {
  constexpr int LANES = HD / 16, PER_BLOCK = QR_THREADS / LANES;
  const int t = threadIdx.x % LANES, heads = a.H + a.G, turning = a.rot / 16;
  const int64_t vec = (int64_t)blockIdx.x * PER_BLOCK + threadIdx.x / LANES;
  const int64_t row = vec / heads;
  if (row >= a.n) return;
  const int pos = a.pos[row];
  if (pos < 0) return;
  const int h = (int)(vec - row * heads), is_k = h >= a.H, at = is_k ? h - a.H : h;
  const bool turns = t < turning;
  const int c0 = turns ? t : 2 * t, c1 = turns ? t + turning : 2 * t + 1;  // (2 turning + 2 (t - turning))
  const __nv_bfloat16* src = (is_k ? a.k + row * a.k_stride : a.q + row * a.q_stride) + (int64_t)at * HD;
  __nv_bfloat16* dst = (is_k ? a.k_out + row * a.k_out_stride : a.q_out + row * a.q_out_stride) + (int64_t)at * HD;
  float x[16];
  unpack8(*reinterpret_cast<const uint4*>(src + 8 * c0), x);
  unpack8(*reinterpret_cast<const uint4*>(src + 8 * c1), x + 8);
  const __nv_bfloat16* gain = is_k ? a.k_gain : a.q_gain;
  const unsigned peers = ((1u << LANES) - 1u) << (threadIdx.x % 32 / LANES * LANES);
  if (gain) {
    auto mean = [&](float f) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s = fmaf(x[i] * f, x[i] * f, s);
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) s += __shfl_xor_sync(peers, s, d);
      return s * (1.f / HD);
    };
    float m = mean(1.f), up = 1.f;
    if (!(m < 3e38f)) {  // squares past the largest number: of values 2^-70 as large
      up = 0x1p-70f;
      m = mean(up);
    }
    const float f = rsqrtf(m + (up == 1.f ? a.eps : 0.f)) * up;
    float g[16];
    unpack8(*reinterpret_cast<const uint4*>(gain + 8 * c0), g);
    unpack8(*reinterpret_cast<const uint4*>(gain + 8 * c1), g + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * f * g[i];
  }
  if (turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int turn = (int)((uint64_t)(uint32_t)pos * a.turns[8 * t + i] >> 32);  // of 2^32
      const float angle = (float)turn * (float)(6.283185307179586 / 4294967296.0), cs = __cosf(angle), sn = __sinf(angle);
      const float y0 = x[i], y1 = x[8 + i];
      x[i] = y0 * cs - y1 * sn;
      x[8 + i] = y1 * cs + y0 * sn;
    }
  }
  *reinterpret_cast<uint4*>(dst + 8 * c0) = pack8(x);
  *reinterpret_cast<uint4*>(dst + 8 * c1) = pack8(x + 8);
}

}  // namespace

cudaError_t qk_rope_launch(const QkRope& a, int sms, cudaStream_t stream) {
  const int64_t per_block = QR_THREADS / (a.hd / 16), blocks = ((int64_t)a.n * (a.H + a.G) + per_block - 1) / per_block;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  if (a.hd == 128) qk_rope_kernel<128><<<(unsigned)blocks, QR_THREADS, 0, stream>>>(a);
  else qk_rope_kernel<64><<<(unsigned)blocks, QR_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace dcl
