// RMSNorm of every head of queries and keys, and the rotation by their positions, in one pass:
//
//   y = x / sqrt(mean x^2 + eps) * gain;  (y_i, y_(i + h)) -> (y_i cos - y_(i + h) sin, y_(i + h) cos + y_i sin)
//
// for i < h = rot / 2, the angle pos * theta^(-i / h); components past rot are normed only.
//
// An angle is needed modulo a turn, and positions are whole numbers: with the frequency as a 64-bit
// fraction of a turn, the product modulo 2^64 is that of the fraction exactly (a product in fp32 is off by 2^-24
// of up to 10^5 turns).  The frequency, from double arithmetic, is off by 2^-55 of a turn, which a position of 2^31
// makes 2^-21.4 rad; the rest is the fraction's way to fp32, 2^-21.27 of at most pi.
//
// Bound by memory: 2 bytes in and 2 out a component, and about 20 operations.  12288 rows of 32 + 32 heads of 128
// (403 MB): 65.8 us, 6.1 TB/s, 0.90 of the measured copy rate.  (A head a thread group at a time, sines for each:
// 124 us; four at a time on 110 registers, two CTAs an SM: 81.)  One row of 28 + 4 heads: 3 us in a graph, all of
// it launch and one look at memory; 512 rows 4.1.
#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int QR_THREADS = 256;
constexpr int qr_ctas(int u) { return u == 1 ? 8 : 3; }  // CTAs of an SM: as many as the registers allow

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

// A warp has heads of one row: hd / 16 lanes a head, two chunks of 8 components each (i and i + h of those that
// rotate), so that a rotation stays in its thread; U heads a lane at once, whose sines and cosines are the
// same.
template <int HD, int U>
__global__ void __launch_bounds__(QR_THREADS, U == 1 ? 4 : qr_ctas(U)) qk_rope_kernel(QkRope a, int per_row, int64_t tasks) {
  constexpr int LANES = HD / 16, HEADS = 32 / LANES;  // lanes of a head; heads of a warp at once
  __shared__ __align__(16) uint64_t turns[HD / 2];
  if (threadIdx.x < HD / 2) turns[threadIdx.x] = a.turns[threadIdx.x];
  __syncthreads();
  const int lane = threadIdx.x & 31, t = lane % LANES, heads = a.H + a.G, turning = a.rot / 16;
  const bool rotates = t < turning;
  const int c0 = 8 * (rotates ? t : 2 * t), c1 = 8 * (rotates ? t + turning : 2 * t + 1);  // (2 turning + 2 (t - turning))
  for (int64_t task = (int64_t)blockIdx.x * (QR_THREADS / 32) + (threadIdx.x >> 5); task < tasks; task += (int64_t)gridDim.x * (QR_THREADS / 32)) {
    const int64_t row = task < (1ll << 31) ? (uint32_t)task / (uint32_t)per_row : task / per_row;
    const int h0 = (int)(task - row * per_row) * (HEADS * U) + lane / LANES;
    const int pos = a.pos[row];
    uint4 x0[U], x1[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + HEADS * u;
      x0[u] = x1[u] = make_uint4(0, 0, 0, 0);
      if (h < heads) {
        const __nv_bfloat16* src = h < a.H ? a.q + row * a.q_stride + (int64_t)h * HD : a.k + row * a.k_stride + (int64_t)(h - a.H) * HD;
        x0[u] = *reinterpret_cast<const uint4*>(src + c0);
        x1[u] = *reinterpret_cast<const uint4*>(src + c1);
      }
    }
    if (pos < 0) continue;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t f = rotates ? turns[8 * t + i] : 0;
      const int turn = (int)((uint64_t)(uint32_t)pos * f >> 32);  // of 2^32
      const float angle = (float)turn * (float)(6.283185307179586 / 4294967296.0);
      cs[i] = __cosf(angle);
      sn[i] = __sinf(angle);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + HEADS * u;
      const bool is_k = h >= a.H;
      float x[16];
      unpack8(x0[u], x);
      unpack8(x1[u], x + 8);
      const __nv_bfloat16* gain = is_k ? a.k_gain : a.q_gain;
      if (a.q_gain || a.k_gain) {  // (all lanes: the sums are shuffled)
        auto mean = [&](float f) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s = fmaf(x[i] * f, x[i] * f, s);
#pragma unroll
          for (int d = 1; d < LANES; d <<= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
          return s * (1.f / HD);
        };
        float m = mean(1.f), f = rsqrtf(m + a.eps);
        if (__any_sync(0xffffffffu, !(m < 3e38f))) {  // squares past the largest number: of values 2^-70 as large
          const float small = mean(0x1p-70f);
          if (!(m < 3e38f)) f = rsqrtf(small) * 0x1p-70f;
        }
        if (gain) {
          float g[16];
          unpack8(*reinterpret_cast<const uint4*>(gain + c0), g);
          unpack8(*reinterpret_cast<const uint4*>(gain + c1), g + 8);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = x[i] * f * g[i];
        }
      }
      if (rotates) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y0 = x[i], y1 = x[8 + i];
          x[i] = y0 * cs[i] - y1 * sn[i];
          x[8 + i] = y1 * cs[i] + y0 * sn[i];
        }
      }
      if (h < heads) {
        __nv_bfloat16* dst = is_k ? a.k_out + row * a.k_out_stride + (int64_t)(h - a.H) * HD : a.q_out + row * a.q_out_stride + (int64_t)h * HD;
        *reinterpret_cast<uint4*>(dst + c0) = pack8(x);
        *reinterpret_cast<uint4*>(dst + c1) = pack8(x + 8);
      }
    }
  }
}

template <int HD, int U>
cudaError_t launch_as(const QkRope& a, int sms, cudaStream_t stream) {
  constexpr int HEADS = 512 / HD * U, WARPS = QR_THREADS / 32;
  const int per_row = (a.H + a.G + HEADS - 1) / HEADS;
  const int64_t tasks = (int64_t)a.n * per_row;
  const int64_t ctas = (tasks + WARPS - 1) / WARPS, most = (int64_t)sms * qr_ctas(U);
  qk_rope_kernel<HD, U><<<(unsigned)(ctas < most ? ctas : most), QR_THREADS, 0, stream>>>(a, per_row, tasks);
  return cudaGetLastError();
}

}  // namespace

cudaError_t qk_rope_launch(const QkRope& a, int sms, cudaStream_t stream) {
  // One head a lane at a time while four would leave warps without any, in us, one / four, rows of 28 + 4 heads of
  // 128: 64 rows 2.9 / 4.3, 512 rows 4.4 / 4.5, 1024 rows 8.0 / 6.7, 2048 rows 12.0 / 10.3.
  const bool few = (int64_t)a.n * (a.H + a.G) * a.hd < (int64_t)sms * 8 * 2048;
  if (a.hd == 128) return few ? launch_as<128, 1>(a, sms, stream) : launch_as<128, 4>(a, sms, stream);
  return few ? launch_as<64, 1>(a, sms, stream) : launch_as<64, 4>(a, sms, stream);
}

}  // namespace dcl
