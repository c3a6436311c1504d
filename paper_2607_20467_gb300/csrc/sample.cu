// Drawing tokens from logits: temperature, top-k, top-p and min-p, then the largest of
// y + noise over what they keep (with standard Gumbel numbers a draw from the renormalised
// softmax), its probability and its confidence under the whole softmax.
//
// y = (z - max z) / T.  Tokens are ordered by (logit descending, index ascending).  Top-k and top-p
// keep a prefix of that order, described by the logit of its last token and how many tokens of
// that logit it holds; min-p keeps y >= ln(min_p).
//
// A row is read once: the CTAs of a cluster keep it in shared memory (a sixteenth to an eighth of a
// large vocabulary each) and exchange what they find through distributed shared memory.  bf16
// logits take few distinct values where it matters (16 octaves below the largest are 2048), so the
// order is found by counting them: a histogram over the values themselves in whole numbers,
// one scan of counts and masses (count times the value's weight, summed in fp64), and both
// boundaries are exact up to the rounding of the weights; nothing is sorted and nothing depends on
// the order in which threads arrive.  A prefix that ends below the histogram's window (flat rows)
// takes a window further down, empty stretches skipped.
#include <cooperative_groups.h>

#include <utility>

#include "common.cuh"
#include "kv_cache.cuh"

namespace cg = cooperative_groups;

namespace dcl {
namespace {

constexpr int SM_THREADS = 256;
constexpr int SM_WARPS = SM_THREADS / 32;
constexpr int SM_BINS = 2048;      // distinct logits of a window
constexpr int SM_CLUSTER = 8;      // most CTAs of a row
constexpr int SM_PER_THREAD = SM_BINS / SM_THREADS;
constexpr uint32_t NEG_INF = 0xff80u;
constexpr uint32_t KEY_NEG_INF = 0x007fu;

// bf16 bits without NaN (-inf in its place) and -0.
__device__ __forceinline__ uint32_t canonical(uint32_t bits) {
  if ((bits & 0x7fffu) > 0x7f80u) bits = NEG_INF;
  return bits == 0x8000u ? 0u : bits;
}
// The same as a whole number that orders as the values do, and back.
__device__ __forceinline__ uint32_t order_key(uint32_t bits) { return bits & 0x8000u ? 0xffffu - bits : bits | 0x8000u; }
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x8000u ? key & 0x7fffu : 0xffffu - key) << 16);
}
__device__ __forceinline__ float exp_fast(float x) {  // e^x, x <= 0: |x| 2^-24 + about 2^-22 of itself
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
  return y;
}

struct Decision {
  int more;         // 1: another window is needed, from bin `start`
  int start;
  int last, ties;   // bin of the last kept logit, tokens of it that are kept
  int count;        // tokens above the window
  double mass;      // their mass
  int k_bin, k_ties;  // the top-k prefix (k_bin < 0: not found yet)
  double goal;      // mass that the top-p prefix has to reach (negative: not known yet)
};

struct SampleShared {
  uint32_t kmax[SM_CLUSTER];            // by rank, in every CTA
  float full[SM_CLUSTER], mass[SM_CLUSTER], total[SM_CLUSTER];  // by rank, in the leader
  uint32_t next[SM_CLUSTER];
  unsigned long long best[SM_CLUSTER];
  Decision dec;
  float red_f[2][SM_WARPS];
  uint32_t red_u[SM_WARPS];
  unsigned long long red_b[SM_WARPS];
  int scan_c[SM_WARPS];
  double scan_m[SM_WARPS];
  int pick;
};

template <typename T, typename Op>
__device__ __forceinline__ T warp_reduce(T v, Op op) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
// Over the block; the result in warp 0's threads (buf: one element a warp, not in use).
template <typename T, typename Op>
__device__ __forceinline__ T block_reduce(T v, Op op, T* buf) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  v = warp_reduce(v, op);
  if (lane == 0) buf[warp] = v;
  __syncthreads();
  if (warp == 0) {
    v = buf[lane & (SM_WARPS - 1)];
#pragma unroll
    for (int d = SM_WARPS / 2; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  }
  return v;
}

struct Best {  // largest s, the lower index of equals
  float s = -INFINITY;
  int at = -1;
  __device__ __forceinline__ void take(float x, int i, bool valid) {
    x = fmaxf(x, -INFINITY);  // (NaN noise: never the largest)
    if (x > s || (at < 0 && valid)) {
      s = x;
      at = i;
    }
  }
  // as one number (0: nothing was taken)
  __device__ __forceinline__ unsigned long long packed() const {
    if (at < 0) return 0;
    const uint32_t bits = __float_as_uint(s + 0.f);
    const uint32_t ord = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return (unsigned long long)ord << 32 | (0xffffffffu - (uint32_t)at);
  }
};

template <bool TRUNC>
__global__ void __launch_bounds__(SM_THREADS) sample_kernel(SampleArgs a, int seg) {
  extern __shared__ __align__(16) uint8_t smem[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem);
  constexpr int HEAD = (sizeof(SampleShared) + 15) / 16 * 16;
  uint32_t* hist = reinterpret_cast<uint32_t*>(smem + HEAD);  // this CTA's counts of the window
  uint32_t* sum = hist + SM_BINS;                             // the leader's: the row's
  uint16_t* zs = reinterpret_cast<uint16_t*>(smem + HEAD + (TRUNC ? 8 * SM_BINS : 0));
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), C = (int)cluster.num_blocks();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / C, V = a.V;
  const uint16_t* z = reinterpret_cast<const uint16_t*>(a.z) + row * a.z_stride;
  const float* g = a.noise ? a.noise + row * a.noise_stride : nullptr;
  SampleShared* leader = cluster.map_shared_rank(&sh, 0);
  auto started = cluster.barrier_arrive();  // (waited for before another CTA's shared memory is touched)
  // element j of this CTA is token base + j: vectors of 8 tokens are aligned in memory
  const int shift = (int)((reinterpret_cast<uintptr_t>(z) >> 1) & 7);
  const int base = rank * seg - shift, lo = max(0, -base), hi = min(seg, V - base), nv = hi > 0 ? (hi + 7) / 8 : 0;

  // ---- the row into shared memory, its largest logit
  uint32_t top = 0;
  for (int v = tid; v < nv; v += SM_THREADS) {
    uint32_t w[4];
    if (8 * v >= lo && 8 * v + 8 <= hi) {
      const uint4 x = *reinterpret_cast<const uint4*>(z + base + 8 * v);
      w[0] = x.x;
      w[1] = x.y;
      w[2] = x.z;
      w[3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 8 * v + 2 * i;
        const uint32_t p = j >= lo && j < hi ? z[base + j] : NEG_INF, q = j + 1 >= lo && j + 1 < hi ? z[base + j + 1] : NEG_INF;
        w[i] = p | q << 16;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p = canonical(w[i] & 0xffffu), q = canonical(w[i] >> 16);
      top = max(top, max(order_key(p), order_key(q)));
      w[i] = p | q << 16;
    }
    reinterpret_cast<uint4*>(zs)[v] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  auto maxu = [](uint32_t x, uint32_t y) { return max(x, y); };
  auto minu = [](uint32_t x, uint32_t y) { return min(x, y); };
  auto addf = [](float x, float y) { return x + y; };
  top = block_reduce(top, maxu, sh.red_u);
  cluster.barrier_wait(std::move(started));
  if (warp == 0 && lane < C) cluster.map_shared_rank(&sh, lane)->kmax[rank] = top;
  if (TRUNC)
    for (int i = tid; i < SM_BINS; i += SM_THREADS) hist[i] = 0;
  cluster.sync();
  uint32_t kmax = 0;
  for (int c = 0; c < C; ++c) kmax = max(kmax, sh.kmax[c]);
  if (kmax <= KEY_NEG_INF) {  // nothing to draw from (every CTA of the row leaves here)
    if (rank == 0 && tid == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
      if (a.conf) a.conf[row] = 0.f;
    }
    return;
  }
  const float zmax = key_value(kmax);
  const float T = a.temperature ? a.temperature[row] : 1.f, inv = __fdiv_rn(1.f, fminf(T, 1e30f));
  const bool greedy = !(T > 0.f) || isinf(inv);
  int k = 0;
  float p = 1.f, mp = 0.f;
  if (TRUNC) {
    if (a.top_k) k = a.top_k[row];
    if (a.top_p) p = a.top_p[row];
    if (a.min_p) mp = a.min_p[row];
  }
  if (k <= 0 || k > V) k = V;
  const bool by_k = k < V, by_p = p < 1.f;  // (NaN: off)
  // (z - max z, 0 at the maximum even where it is infinite)
  auto rel = [&](uint32_t bits) {
    const float x = __uint_as_float(bits << 16);
    return x == zmax ? 0.f : __fsub_rn(x, zmax);
  };
  auto scaled = [&](float d) { return __fmul_rn(d, inv); };
  float full = 0.f, total = 0.f;  // sums of e^(z - max z), and of e^y over the kept tokens
  Best best;

  if (greedy || !TRUNC || !(by_k || by_p)) {
    // ---- no prefix to find: one pass over the row and its noise
    const float floor_y = mp > 0.f ? logf(fminf(mp, 1.f)) : -INFINITY;
    auto element = [&](uint32_t bits, int i, float noise) {
      const float d = rel(bits), e = exp_fast(d);
      full += e;
      if (greedy) {
        if (d == 0.f) best.take(0.f, i, true);
        return;
      }
      const float y = scaled(d);
      if (TRUNC && !(y >= floor_y)) return;
      total += inv == 1.f ? e : exp_fast(y);
      best.take(__fadd_rn(y, noise), i, bits != NEG_INF);
    };
    const bool with_noise = g && !greedy;
    if (with_noise && ((reinterpret_cast<uintptr_t>(g + base) & 15) == 0)) {
      constexpr int U = 2;  // vectors of 8 in flight
      for (int v0 = tid; v0 < nv; v0 += U * SM_THREADS) {
        float4 n[U][2];
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int j = 8 * (v0 + x * SM_THREADS);
          if (j >= lo && j + 8 <= hi) {
            n[x][0] = __ldcs(reinterpret_cast<const float4*>(g + base + j));
            n[x][1] = __ldcs(reinterpret_cast<const float4*>(g + base + j) + 1);
          }
        }
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int v = v0 + x * SM_THREADS, j = 8 * v;
          if (v >= nv) break;
          const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
          const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
          if (j >= lo && j + 8 <= hi) {
            const float* f = &n[x][0].x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              element(w[i] & 0xffffu, base + j + 2 * i, f[2 * i]);
              element(w[i] >> 16, base + j + 2 * i + 1, f[2 * i + 1]);
            }
          } else {
            for (int i = max(j, lo); i < min(j + 8, hi); ++i) element(zs[i], base + i, g[base + i]);
          }
        }
      }
    } else {
      for (int j = lo + tid; j < hi; j += SM_THREADS) element(zs[j], base + j, with_noise ? g[base + j] : 0.f);
    }
  } else if constexpr (TRUNC) {
    // ---- the prefix: windows of SM_BINS distinct logits from the largest down
    float mass = 0.f;
    if (rank == 0 && tid == 0) {
      sh.dec = Decision{};
      sh.dec.k_bin = by_k ? -1 : 1 << 20;  // (past every logit)
      sh.dec.goal = -1.0;
    }
    Decision dec{};
    for (int start = 0, turn = 0;; ++turn) {
      uint32_t next = 0xffffffffu;
      for (int v = tid; v < nv; v += SM_THREADS) {
        const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        const bool inner = 8 * v >= lo && 8 * v + 8 <= hi;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
          if (!inner && (8 * v + i < lo || 8 * v + i >= hi)) continue;
          if (turn == 0) {
            const float d = rel(bits), e = exp_fast(d);
            full += e;
            mass += inv == 1.f ? e : exp_fast(scaled(d));
          }
          const uint32_t bin = kmax - order_key(bits);
          if (bin - (uint32_t)start < SM_BINS) atomicAdd(&hist[bin - start], 1u);
          else if ((int)bin >= start) next = min(next, bin);
        }
      }
      if (turn == 0) {
        full = block_reduce(full, addf, sh.red_f[0]);
        mass = block_reduce(mass, addf, sh.red_f[1]);
      }
      next = block_reduce(next, minu, sh.red_u);
      if (tid == 0) {
        if (turn == 0) {
          leader->full[rank] = full;
          leader->mass[rank] = mass;
        }
        leader->next[rank] = next;
      }
      cluster.sync();
      // the row's counts, a share of the bins each, into the leader
      {
        uint32_t* to = cluster.map_shared_rank(sum, 0);
        const int share = SM_BINS / C;
        for (int i = rank * share + tid; i < (rank + 1) * share; i += SM_THREADS) {
          uint32_t n = 0;
          for (int c = 0; c < C; ++c) n += cluster.map_shared_rank(hist, c)[i];
          to[i] = n;
        }
      }
      cluster.sync();
      if (rank == 0) {
        // scan: thread t holds bins 8 t .. 8 t + 7
        uint32_t n[SM_PER_THREAD];
        double w[SM_PER_THREAD];
        int count = 0;
        double own = 0.0;
#pragma unroll
        for (int i = 0; i < SM_PER_THREAD; ++i) {
          const int bin = start + tid * SM_PER_THREAD + i;
          n[i] = sum[tid * SM_PER_THREAD + i];
          const uint32_t key = kmax - (uint32_t)bin;
          w[i] = 0.0;
          if (n[i]) w[i] = exp_fast(scaled(bin == 0 ? 0.f : __fsub_rn(key_value(key), zmax)));
          count += (int)n[i];
          own += n[i] * w[i];
        }
        int c_up = count;
        double m_up = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int c = __shfl_up_sync(0xffffffffu, c_up, d);
          const double m = __shfl_up_sync(0xffffffffu, m_up, d);
          if (lane >= d) {
            c_up += c;
            m_up += m;
          }
        }
        if (lane == 31) {
          sh.scan_c[warp] = c_up;
          sh.scan_m[warp] = m_up;
        }
        if (tid == 0) sh.pick = -1;
        __syncthreads();
        int c_all = 0, c_before = sh.dec.count + c_up - count;
        double m_all = 0.0, m_before = sh.dec.mass + m_up - own;
        for (int i = 0; i < SM_WARPS; ++i) {
          if (i < warp) {
            c_before += sh.scan_c[i];
            m_before += sh.scan_m[i];
          }
          c_all += sh.scan_c[i];
          m_all += sh.scan_m[i];
        }
        const int c_end = sh.dec.count + c_all;
        const double m_end = sh.dec.mass + m_all, m_start = sh.dec.mass;
        int k_bin = sh.dec.k_bin;
        double goal = sh.dec.goal;
        __syncthreads();  // (dec has been read)
        if (k_bin < 0 && c_end >= k) {  // the top-k prefix ends in this window
          int c = c_before;
          double m = m_before;
#pragma unroll
          for (int i = 0; i < SM_PER_THREAD; ++i) {
            if (c < k && c + (int)n[i] >= k) {
              sh.dec.k_bin = start + tid * SM_PER_THREAD + i;
              sh.dec.k_ties = k - c;
              sh.dec.goal = (double)p * (m + (k - c) * w[i]);
            }
            c += (int)n[i];
            m += n[i] * w[i];
          }
        } else if (!by_k && goal < 0.0 && tid == 0) {
          float all = 0.f;
          for (int c = 0; c < C; ++c) all += sh.mass[c];
          sh.dec.goal = (double)p * all;
        }
        __syncthreads();
        k_bin = sh.dec.k_bin;
        goal = sh.dec.goal;
        uint32_t below = 0xffffffffu;  // where the next window would begin
        for (int c = 0; c < C; ++c) below = min(below, sh.next[c]);
        const bool k_known = k_bin >= 0, rest = below != 0xffffffffu;
        if (k_known && by_p && (m_start < goal || start == 0) && (m_end >= goal || k_bin < start + SM_BINS || !rest)) {
          // the top-p prefix ends in this window: the last logit with less than the goal before it
          int mine = -1, ties = 1;
          double m = m_before;
#pragma unroll
          for (int i = 0; i < SM_PER_THREAD; ++i) {
            const int bin = start + tid * SM_PER_THREAD + i;
            if (n[i] && bin <= k_bin && (m < goal || bin == 0)) {
              mine = bin;
              const double need = w[i] > 0.0 ? ceil((goal - m) / w[i]) : 2e9;
              ties = need < 1.0 ? 1 : need < (double)n[i] ? (int)need : (int)n[i];
            }
            m += n[i] * w[i];
          }
          if (mine >= 0) atomicMax(&sh.pick, mine);
          __syncthreads();
          if (mine >= 0 && mine == sh.pick) {
            sh.dec.last = mine;
            sh.dec.ties = mine == k_bin ? min(ties, sh.dec.k_ties) : ties;
            sh.dec.more = 0;
          }
        } else if (tid == 0) {
          if (k_known && !by_p) {
            sh.dec.last = k_bin;
            sh.dec.ties = sh.dec.k_ties;
            sh.dec.more = 0;
          } else {
            sh.dec.more = 1;
            if (k_known && m_start >= goal) {  // the top-p prefix ended in an earlier window
              sh.dec.start = 0;
              sh.dec.count = 0;
              sh.dec.mass = 0.0;
            } else {
              sh.dec.start = (int)below;
              sh.dec.count = c_end;
              sh.dec.mass = m_end;
            }
          }
        }
      }
      cluster.sync();
      dec = leader->dec;
      if (!dec.more) break;
      start = dec.start;
      for (int i = tid; i < SM_BINS; i += SM_THREADS) hist[i] = 0;
      cluster.sync();  // every CTA has read the decision and the counts
    }
    // ---- which of the tokens of the last logit are this CTA's to keep
    const int last = dec.last;
    int at = 0;
    {
      int start_bin = dec.start;  // (of the window that the histograms hold)
      int before = 0;
      for (int c = 0; c < rank; ++c) before += (int)cluster.map_shared_rank(hist, c)[last - start_bin];
      const int own = (int)hist[last - start_bin], keep = min(max(dec.ties - before, 0), own);
      at = keep == own ? hi : lo;  // tokens of the last logit before element `at`
      if (keep > 0 && keep < own) {  // (uniform over the CTA)
        // a run of elements per thread, in order
        const int run = (hi - lo + SM_THREADS - 1) / SM_THREADS, j0 = min(lo + tid * run, hi), j1 = min(j0 + run, hi);
        int n = 0;
        for (int j = j0; j < j1; ++j) n += kmax - order_key(zs[j]) == (uint32_t)last;
        int up = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, up, d);
          if (lane >= d) up += x;
        }
        if (lane == 31) sh.scan_c[warp] = up;
        __syncthreads();
        int c = up - n;
        for (int i = 0; i < warp; ++i) c += sh.scan_c[i];
        if (c < keep && c + n >= keep) {
          for (int j = j0; j < j1; ++j) {
            if (kmax - order_key(zs[j]) == (uint32_t)last && ++c == keep) {
              sh.pick = j + 1;
              break;
            }
          }
        }
        __syncthreads();
        at = sh.pick;
      }
    }
    // ---- the kept tokens
    const float floor_y = mp > 0.f ? logf(fminf(mp, 1.f)) : -INFINITY;
    for (int v = tid; v < nv; v += SM_THREADS) {
      const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
      const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        const int j = 8 * v + i, bin = (int)(kmax - order_key(bits));
        if (bin > last || (bin == last && j >= at) || bits == NEG_INF || j < lo || j >= hi) continue;
        const float y = scaled(rel(bits));
        if (!(y >= floor_y)) continue;
        total += exp_fast(y);
        best.take(g ? __fadd_rn(y, g[base + j]) : y, base + j, true);
      }
    }
  }

  // ---- the row's token
  auto maxb = [](unsigned long long x, unsigned long long y) { return x > y ? x : y; };
  const unsigned long long b = block_reduce(best.packed(), maxb, sh.red_b);
  __syncthreads();  // (the sums' buffers may still be read)
  total = block_reduce(total, addf, sh.red_f[0]);
  const bool prefix = TRUNC && !greedy && (by_k || by_p);
  if (!prefix) full = block_reduce(full, addf, sh.red_f[1]);
  if (tid == 0) {
    leader->best[rank] = b;
    leader->total[rank] = total;
    if (!prefix) leader->full[rank] = full;
  }
  cluster.sync();
  if (rank == 0 && tid == 0) {
    unsigned long long top_b = 0;
    float all = 0.f, whole = 0.f;
    for (int c = 0; c < C; ++c) {
      top_b = maxb(top_b, sh.best[c]);
      all += sh.total[c];
      whole += sh.full[c];
    }
    const int token = (int)(0xffffffffu - (uint32_t)top_b);
    const float d = rel(canonical(z[token]));
    a.token[row] = token;
    if (a.prob) a.prob[row] = greedy ? 1.f : exp_fast(scaled(d)) / all;
    if (a.conf) a.conf[row] = exp_fast(d) / whole;
  }
}

template <bool TRUNC>
cudaError_t launch_as(const SampleArgs& a, int C, cudaStream_t stream) {
  const int seg = ((a.V + 7 + C - 1) / C + 7) / 8 * 8;  // (7: a row's first vector may hold one token)
  const size_t smem = (sizeof(SampleShared) + 15) / 16 * 16 + (TRUNC ? 8 * SM_BINS : 0) + 2 * (size_t)seg;
  static const cudaError_t set = cudaFuncSetAttribute(sample_kernel<TRUNC>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  if (set != cudaSuccess) return set;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.rows * C);
  cfg.blockDim = dim3(SM_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<TRUNC>, a, seg);
}

}  // namespace

cudaError_t sample_launch(const SampleArgs& a, cudaStream_t stream) {
  int C = 1;
  while (C < SM_CLUSTER && a.V > 4096 * C) C *= 2;
  return a.top_k || a.top_p || a.min_p ? launch_as<true>(a, C, stream) : launch_as<false>(a, C, stream);
}

}  // namespace dcl
