// Drawing tokens from logits: temperature, top-k, top-p and min-p, then the largest of
// y + noise over what they keep (with standard Gumbel numbers a draw from the renormalised
// softmax), its probability and its confidence under the whole softmax.
//
// y = (z - max z) / T.  Tokens are ordered by (logit descending, index ascending).  Top-k and top-p
// keep a prefix of that order, described by the logit of its last token and how many tokens of
// that logit it holds; min-p keeps y >= ln(min_p).
#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int SM_THREADS = 1024;

// bf16 bits as a whole number that orders as the values do (-0 as +0, NaN as -inf).
__device__ __forceinline__ uint32_t order_key(uint32_t bits) {
  if ((bits & 0x7fffu) > 0x7f80u) bits = 0xff80u;
  if (bits == 0x8000u) bits = 0;
  return bits & 0x8000u ? 0xffffu - bits : bits | 0x8000u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x8000u ? key & 0x7fffu : 0xffffu - key) << 16);
}
constexpr uint32_t KEY_NEG_INF = 0x007fu;

template <typename T, typename Op>
__device__ T block_reduce(T v, Op op, T* buf) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  __syncthreads();
  if (lane == 0) buf[warp] = v;
  __syncthreads();
  v = buf[lane];
  for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}

__global__ void __launch_bounds__(SM_THREADS) sample_kernel(SampleArgs a) {
  __shared__ double bufd[32];
  __shared__ unsigned long long bufu[32];
  const int row = blockIdx.x, V = a.V;
  const unsigned short* z = reinterpret_cast<const unsigned short*>(a.z) + row * a.z_stride;
  const float* g = a.noise ? a.noise + row * a.noise_stride : nullptr;
  auto maxu = [](unsigned long long x, unsigned long long y) { return x > y ? x : y; };
  auto add = [](auto x, auto y) { return x + y; };
  unsigned long long top = 0;
  for (int i = threadIdx.x; i < V; i += SM_THREADS) top = maxu(top, order_key(z[i]));
  const uint32_t kmax = (uint32_t)block_reduce(top, maxu, bufu);
  if (kmax <= KEY_NEG_INF) {  // nothing to draw from
    if (threadIdx.x == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
      if (a.conf) a.conf[row] = 0.f;
    }
    return;
  }
  const float zmax = key_value(kmax);
  const float T = a.temperature ? a.temperature[row] : 1.f;
  const float inv = __fdiv_rn(1.f, T);
  const bool greedy = !(T > 0.f) || isinf(inv);
  auto rel = [&](uint32_t key) { return key == kmax ? 0.f : __fsub_rn(key_value(key), zmax); };
  auto weight = [&](uint32_t key) { return expf(__fmul_rn(rel(key), inv)); };
  int k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
  if (k <= 0 || k > V) k = V;
  float p = a.top_p && !greedy ? a.top_p[row] : 1.f, mp = a.min_p && !greedy ? a.min_p[row] : 0.f;
  auto count_above = [&](uint32_t t) {  // keys > t
    unsigned long long c = 0;
    for (int i = threadIdx.x; i < V; i += SM_THREADS) c += order_key(z[i]) > t;
    return (int)block_reduce(c, add, bufu);
  };
  auto mass_above = [&](uint32_t t) {
    double s = 0;
    for (int i = threadIdx.x; i < V; i += SM_THREADS) {
      const uint32_t key = order_key(z[i]);
      if (key > t) s += weight(key);
    }
    return block_reduce(s, add, bufd);
  };
  // the prefix: keys above `last` and the first `ties` tokens of key `last`
  uint32_t last = 0;
  int ties = V;
  if (k < V) {  // the least key with fewer than k tokens above it
    uint32_t lo = 0, hi = kmax;
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (count_above(mid) < k) hi = mid; else lo = mid + 1;
    }
    last = lo;
    ties = k - count_above(last);
  }
  if (p < 1.f) {
    const double goal = (double)p * (mass_above(last) + (last ? (double)ties * weight(last) : 0.0));
    uint32_t lo = last, hi = kmax;  // the least key whose tokens begin before the goal
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if (mass_above(mid) < goal) hi = mid; else lo = mid + 1;
    }
    const double before = mass_above(lo), w = weight(lo);
    const double n = w > 0 ? ceil((goal - before) / w) : (double)V;
    const int np = n < 1 ? 1 : n < V ? (int)n : V;
    ties = lo == last ? min(ties, np) : np;
    last = lo;
  }
  // which index the last of the ties has: the least bound below which there are `ties` of them
  int bound = V;
  if (last) {
    int lo = 0, hi = V;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      unsigned long long c = 0;
      for (int i = threadIdx.x; i < mid; i += SM_THREADS) c += order_key(z[i]) == last;
      if ((int)block_reduce(c, add, bufu) >= ties) hi = mid; else lo = mid + 1;
    }
    bound = lo;
  }
  const float floor_y = mp > 0.f ? logf(fminf(mp, 1.f)) : -INFINITY;
  unsigned long long best = 0;  // {ordered key of y + g, ~index}
  double total = 0, full = 0;
  for (int i = threadIdx.x; i < V; i += SM_THREADS) {
    const uint32_t key = order_key(z[i]);
    if (key <= KEY_NEG_INF) continue;
    const float d = rel(key), y = __fmul_rn(d, inv);
    full += expf(d);
    const bool kept = greedy ? key == kmax && i < bound : (key > last || (key == last && i < bound)) && y >= floor_y;
    if (!kept) continue;
    total += greedy ? 1.0 : (double)expf(y);
    float s = greedy ? 0.f : g ? __fadd_rn(y, g[i]) : y;
    if (isnan(s)) s = -INFINITY;
    const uint32_t bits = __float_as_uint(s + 0.f);
    const uint32_t ord = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    best = maxu(best, (unsigned long long)ord << 32 | (0xffffffffu - (uint32_t)i));
  }
  best = block_reduce(best, maxu, bufu);
  total = block_reduce(total, add, bufd);
  full = block_reduce(full, add, bufd);
  if (threadIdx.x) return;
  const int token = (int)(0xffffffffu - (uint32_t)best);
  const float d = rel(order_key(z[token]));
  a.token[row] = token;
  if (a.prob) a.prob[row] = greedy ? 1.f : (float)((double)expf(__fmul_rn(d, inv)) / total);
  if (a.conf) a.conf[row] = (float)((double)expf(d) / full);
}

}  // namespace

cudaError_t sample_launch(const SampleArgs& a, cudaStream_t stream) {
  sample_kernel<<<(unsigned)a.rows, SM_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace dcl
