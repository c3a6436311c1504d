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
// one scan of counts and masses (count times the value's weight, in fixed point of 2^-44, which
// 2^19 tokens of weight 1 do not overflow; in fp64 the scan took longer than all else), and both
// boundaries are exact up to the rounding of the weights; nothing is sorted and nothing depends on
// the order in which threads arrive.  A prefix that ends below the histogram's window (flat rows)
// takes a window further down, empty stretches skipped.
//
// Large calls are bound by memory: 512 rows of 152064 with noise for every token (467 MB) take
// 92 us, 5.1 TB/s, 0.74 of the measured copy rate; the noise pass waits for the row's maximum, and
// the CTAs of other rows (three to five an SM) fill that time.  Few rows are bound by latency: a row of 4095
// tokens 10.3 us, 32 rows of 126464 with all three truncations 18.1, in steps of about 1 us (the
// maximum, the histogram, its scan, the boundaries, the draw, each with a barrier of the
// cluster).  A row has up to eight CTAs (C doubles while V > 4096 C): what one CTA loads and counts is
// what such a call waits for.
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
constexpr int SM_FIRST = 256;      // of the first one
constexpr int SM_CLUSTER = 8;      // most CTAs of a row
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

using mass_t = unsigned long long;  // units of 2^-44 of the largest token's weight
constexpr float MASS_ONE = 17592186044416.f;
__device__ __forceinline__ mass_t mass_share(float p, mass_t m) {  // p m, 0 <= p < 1
  return p > 0.f ? (mass_t)((double)p * (double)m) : 0;
}

struct Decision {
  int more;         // 1: another window is needed, from bin `start`
  int start;
  int last, ties;   // bin of the last kept logit, tokens of it that are kept
  int count;        // tokens above the window
  mass_t mass;      // their mass
  int k_bin, k_ties;  // the top-k prefix (k_bin < 0: not found yet)
  int goal_known;
  mass_t goal;      // mass that the top-p prefix has to reach
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
  mass_t scan_m[SM_WARPS];
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

constexpr float LOWEST = -3.402823466e38f;

struct Best {  // largest s, the lower index of equals (a thread meets its tokens in order)
  float s = -INFINITY;
  int at = -1;
  __device__ __forceinline__ void take(float x, int i) {
    if (x > s) {
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
// y + noise.  Noise of -inf or NaN counts as the lowest number, so that a kept token (y finite)
// always beats one that is not (y = -inf).
__device__ __forceinline__ float perturbed(float y, float noise) { return __fadd_rn(y, fmaxf(noise, LOWEST)); }

// What the leader needs to look for the ends of the prefix in a window.
struct PrefixArgs {
  cg::cluster_group& cluster;
  SampleShared& sh;
  uint32_t* hist;
  int C, V;
  uint32_t kmax;
  float zmax, inv;
  int k;
  float p;
  bool by_k, by_p;
  int start, width;
};

// The leader's step: scans the row's counts and masses over the window (PER consecutive bins a
// thread) and writes the decision.  All its threads call it.
template <int PER>
__device__ __forceinline__ void scan_window(const PrefixArgs& q) {
  SampleShared& sh = q.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, start = q.start, k = q.k;
  uint32_t n[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) n[i] = 0;
#pragma unroll
  for (int c = 0; c < SM_CLUSTER; ++c) {
    if (c >= q.C) break;
    const uint32_t* from = q.cluster.map_shared_rank(q.hist, c) + tid * PER;
    if constexpr (PER % 4 == 0) {
#pragma unroll
      for (int i = 0; i < PER / 4; ++i) {
        const uint4 y = reinterpret_cast<const uint4*>(from)[i];
        n[4 * i] += y.x;
        n[4 * i + 1] += y.y;
        n[4 * i + 2] += y.z;
        n[4 * i + 3] += y.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) n[i] += from[i];
    }
  }
  mass_t w[PER];
  int count = 0;
  mass_t own = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int bin = start + tid * PER + i;
    const uint32_t key = q.kmax - (uint32_t)bin;
    w[i] = 0;
    if (n[i]) w[i] = __float2ull_rn(MASS_ONE * exp_fast(__fmul_rn(bin == 0 ? 0.f : __fsub_rn(key_value(key), q.zmax), q.inv)));
    count += (int)n[i];
    own += (mass_t)n[i] * w[i];
  }
  int c_up = count;
  mass_t m_up = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int c = __shfl_up_sync(0xffffffffu, c_up, d);
    const mass_t m = __shfl_up_sync(0xffffffffu, m_up, d);
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
  mass_t m_all = 0, m_before = sh.dec.mass + m_up - own;
  for (int i = 0; i < SM_WARPS; ++i) {
    if (i < warp) {
      c_before += sh.scan_c[i];
      m_before += sh.scan_m[i];
    }
    c_all += sh.scan_c[i];
    m_all += sh.scan_m[i];
  }
  const int c_end = sh.dec.count + c_all;
  const mass_t m_end = sh.dec.mass + m_all, m_start = sh.dec.mass;
  int k_bin = sh.dec.k_bin;
  const bool goal_known = sh.dec.goal_known;
  __syncthreads();  // (dec has been read)
  if (k_bin < 0 && c_end >= k) {  // the top-k prefix ends in this window
    int c = c_before;
    mass_t m = m_before;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (c < k && c + (int)n[i] >= k) {
        sh.dec.k_bin = start + tid * PER + i;
        sh.dec.k_ties = k - c;
        sh.dec.goal = q.by_p ? mass_share(q.p, m + (mass_t)(k - c) * w[i]) : 0;
      }
      c += (int)n[i];
      m += (mass_t)n[i] * w[i];
    }
  } else if (!q.by_k && !goal_known && tid == 0) {
    float all = 0.f;
    for (int c = 0; c < q.C; ++c) all += sh.mass[c];
    sh.dec.goal_known = 1;
    sh.dec.goal = mass_share(q.p, __float2ull_rn(MASS_ONE * all));
  }
  __syncthreads();
  k_bin = sh.dec.k_bin;
  const mass_t goal = sh.dec.goal;
  uint32_t below = 0xffffffffu;  // where the next window would begin, if any token is left
  for (int c = 0; c < q.C; ++c) below = min(below, sh.next[c]);
  const bool k_known = k_bin >= 0, rest = c_end < q.V;
  if (k_known && q.by_p && (m_start < goal || start == 0) && (m_end >= goal || k_bin < start + q.width || !rest)) {
    // the top-p prefix ends in this window: the last logit with less than the goal before it
    int mine = -1, most = 0;
    mass_t m = m_before, room = 0, each = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int bin = start + tid * PER + i;
      if (n[i] && bin <= k_bin && (m < goal || bin == 0)) {
        mine = bin;
        most = (int)n[i];
        each = w[i];
        room = goal > m ? goal - m : 0;
      }
      m += (mass_t)n[i] * w[i];
    }
    if (mine >= 0) atomicMax(&sh.pick, mine);
    __syncthreads();
    if (mine >= 0 && mine == sh.pick) {
      // token i of the logit (from 0) is kept where i of them do not fill the room
      const mass_t need = each ? (room + each - 1) / each : (mass_t)most;
      const int ties = need < 1 ? 1 : need < (mass_t)most ? (int)need : most;
      sh.dec.last = mine;
      sh.dec.ties = mine == k_bin ? min(ties, sh.dec.k_ties) : ties;
      sh.dec.more = 0;
    }
  } else if (tid == 0) {
    if (k_known && !q.by_p) {
      sh.dec.last = k_bin;
      sh.dec.ties = sh.dec.k_ties;
      sh.dec.more = 0;
    } else {
      sh.dec.more = 1;
      if (k_known && m_start >= goal) {  // the top-p prefix ended in an earlier window
        sh.dec.start = 0;
        sh.dec.count = 0;
        sh.dec.mass = 0;
      } else {
        sh.dec.start = (int)below;
        sh.dec.count = c_end;
        sh.dec.mass = m_end;
      }
    }
  }
}

// (a call of its own: inlined it took the registers of the loops over the row)
__device__ __noinline__ void scan_wide(const PrefixArgs& q) { scan_window<SM_BINS / SM_THREADS>(q); }

template <bool TRUNC>
__global__ void __launch_bounds__(SM_THREADS, TRUNC ? 3 : 5) sample_kernel(SampleArgs a, int seg) {
  extern __shared__ __align__(16) uint8_t smem[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem);
  constexpr int HEAD = (sizeof(SampleShared) + 15) / 16 * 16;
  uint32_t* hist = reinterpret_cast<uint32_t*>(smem + HEAD);  // this CTA's counts of the window
  uint16_t* zs = reinterpret_cast<uint16_t*>(smem + HEAD + (TRUNC ? 4 * SM_BINS : 0));
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

  // (asked for before the row, used after it)
  const float T = a.temperature ? a.temperature[row] : 1.f;
  int k = 0;
  float p = 1.f, mp = 0.f;
  if (TRUNC) {
    if (a.top_k) k = a.top_k[row];
    if (a.top_p) p = a.top_p[row];
    if (a.min_p) mp = a.min_p[row];
  }

  // ---- the row into shared memory, its largest logit
  const int v_lo = (lo + 7) / 8, v_hi = max(v_lo, hi / 8);  // vectors that lie inside the row
  // (the others: at most 7 elements at either end)
  const int n_head = min(8 * v_lo, hi) - min(lo, hi), n_edge = n_head + max(0, hi - 8 * v_hi);
  auto edge = [&](int i) { return i < n_head ? lo + i : 8 * v_hi + i - n_head; };
  float top_z = -INFINITY;
  auto keep = [&](int v, uint32_t (&w)[4]) {
    uint32_t odd = 0;  // a sign bit for each NaN (magnitude above 0x7f80) and -0
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = w[i] ^ 0x80008000u;
      odd |= (((w[i] & 0x7fff7fffu) + 0x007f007fu) | ((t - 0x00010001u) & ~t)) & 0x80008000u;
    }
    if (odd) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = canonical(w[i] & 0xffffu) | canonical(w[i] >> 16) << 16;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) top_z = fmaxf(top_z, fmaxf(bf16_lo(w[i]), bf16_hi(w[i])));
    reinterpret_cast<uint4*>(zs)[v] = make_uint4(w[0], w[1], w[2], w[3]);
  };
  constexpr int LD = 4;  // loads in flight
  for (int v0 = v_lo + tid; v0 < v_hi; v0 += LD * SM_THREADS) {
    uint4 x[LD];
#pragma unroll
    for (int i = 0; i < LD; ++i)
      if (v0 + i * SM_THREADS < v_hi) x[i] = __ldcs(reinterpret_cast<const uint4*>(z + base) + v0 + i * SM_THREADS);
#pragma unroll
    for (int i = 0; i < LD; ++i)
      if (v0 + i * SM_THREADS < v_hi) {
        uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        keep(v0 + i * SM_THREADS, w);
      }
  }
  if (tid < 2) {  // the vectors that the row begins and ends in
    const int v = tid ? v_hi : v_lo - 1;
    if (v >= 0 && v < nv && (tid == 0 || v != v_lo - 1)) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 8 * v + 2 * i;
        const uint32_t p = j >= lo && j < hi ? z[base + j] : NEG_INF, q = j + 1 >= lo && j + 1 < hi ? z[base + j + 1] : NEG_INF;
        w[i] = p | q << 16;
      }
      keep(v, w);
    }
  }
  auto maxu = [](uint32_t x, uint32_t y) { return max(x, y); };
  auto minu = [](uint32_t x, uint32_t y) { return min(x, y); };
  auto addf = [](float x, float y) { return x + y; };
  const uint32_t top = block_reduce(order_key(__float_as_uint(top_z) >> 16), maxu, sh.red_u);
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
  const float inv = __fdiv_rn(1.f, fminf(T, 1e30f));
  const bool greedy = !(T > 0.f) || inv > 1e37f;
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
    const bool with_noise = g && !greedy;
    // (infinite maxima take the plain loop: z - max z is 0 or -inf there)
    const bool plain = inv == 1.f, vectors = with_noise && ((reinterpret_cast<uintptr_t>(g + base) & 15) == 0) && !isinf(zmax);
    auto element = [&](int j) {
      const float d = rel(zs[j]), e = exp_fast(d);
      full += e;
      const float y = greedy ? (d == 0.f ? 0.f : -INFINITY) : scaled(d);
      if (TRUNC && !(y >= floor_y)) return;
      total += exp_fast(y);
      best.take(with_noise ? perturbed(y, g[base + j]) : y, base + j);
    };
    if (vectors) {
      if (tid < n_head) element(edge(tid));  // (before the vectors: a thread's tokens in order)
      constexpr int U = 2;  // vectors of 8 in flight
      for (int v0 = v_lo + tid; v0 < v_hi; v0 += U * SM_THREADS) {
        float4 n[U][2];
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int v = v0 + x * SM_THREADS;
          if (v < v_hi) {
            n[x][0] = __ldcs(reinterpret_cast<const float4*>(g + base + 8 * v));
            n[x][1] = __ldcs(reinterpret_cast<const float4*>(g + base + 8 * v) + 1);
          }
        }
#pragma unroll
        for (int x = 0; x < U; ++x) {
          const int v = v0 + x * SM_THREADS;
          if (v >= v_hi) break;
          const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
          const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
          const float* f = &n[x][0].x;
          float s[8], most = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float d = __fsub_rn(i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]), zmax);
            const float y = scaled(d), e = exp_fast(d), ey = plain ? e : exp_fast(y);
            full += e;
            if (TRUNC) {
              const bool in = y >= floor_y;
              total += in ? ey : 0.f;
              s[i] = in ? perturbed(y, f[i]) : -INFINITY;
            } else {
              total += ey;
              s[i] = perturbed(y, f[i]);
            }
            most = fmaxf(most, s[i]);
          }
          if (most > best.s) {
#pragma unroll
            for (int i = 7; i >= 0; --i)
              if (s[i] == most) best.at = base + 8 * v + i;
            best.s = most;
          }
        }
      }
    }
    // what the last vector holds of the row, or without vectors all of it
    if (!vectors) {
      for (int j = lo + tid; j < hi; j += SM_THREADS) element(j);
    } else if (tid >= n_head && tid < n_edge) {
      element(edge(tid));
    }
  } else if constexpr (TRUNC) {
    // ---- the prefix: windows of SM_BINS distinct logits from the largest down
    float mass = 0.f;
    if (rank == 0 && tid == 0) {
      sh.dec = Decision{};
      sh.dec.k_bin = by_k ? -1 : 1 << 20;  // (past every logit)
    }
    Decision dec{};
    const float per_y = inv * kLog2e;  // y in units of log2
    for (int start = 0, turn = 0;; ++turn) {
      // a first window of few logits holds what is usually kept and little of the bulk
      const int width = turn == 0 ? SM_FIRST : SM_BINS;
      // bins start .. start + width - 1 are the logits from `upper` down to `lower`
      const float upper = key_value(kmax - start);
      const int low_key = (int)kmax - start - width + 1;
      const float lower = low_key > (int)KEY_NEG_INF ? key_value((uint32_t)low_key) : -INFINITY;
      float below = -INFINITY;  // the largest logit under the window
      auto sums = [&](float x) {
        const float d = x == zmax ? 0.f : __fsub_rn(x, zmax);
        full += exp_fast(d);
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * per_y));
        mass += e;
      };
      const uint32_t hist_at = static_cast<uint32_t>(__cvta_generic_to_shared(hist)) + 4 * (kmax - start);
      auto count = [&](uint32_t bits) {  // without a branch: lanes differ in what they count
        const float x = __uint_as_float(bits);
        const uint32_t key = (bits ^ ((uint32_t)((int)bits >> 31) | 0x80000000u)) >> 16;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.u32 p, %1, 0;\n\t"
            "@p red.shared.add.u32 [%0], 1;\n\t}" ::"r"(hist_at - 4 * key),
            "r"((uint32_t)(x >= lower && x <= upper))
            : "memory");
        below = fmaxf(below, x >= lower ? -INFINITY : x);
      };
      for (int v = v_lo + tid; v < v_hi; v += SM_THREADS) {
        const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        if (turn == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sums(bf16_lo(w[i]));
            sums(bf16_hi(w[i]));
          }
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(bf16_lo(w[i]), bf16_hi(w[i])));
        if (most < lower) {  // most vectors: all under the window
          below = fmaxf(below, most);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            count(w[i] << 16);
            count(w[i] & 0xffff0000u);
          }
        }
      }
      if (tid < n_edge) {
        const uint32_t bits = (uint32_t)zs[edge(tid)] << 16;
        if (turn == 0) sums(__uint_as_float(bits));
        count(bits);
      }
      uint32_t next = kmax - order_key(__float_as_uint(below) >> 16);
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
      if (rank == 0) {
        const PrefixArgs pa{cluster, sh, hist, C, V, kmax, zmax, inv, k, p, by_k, by_p, start, width};
        if (turn == 0)
          scan_window<1>(pa);
        else
          scan_wide(pa);
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
    const float least = key_value(kmax - last);
    auto element = [&](uint32_t bits, int j) {
      const float x = __uint_as_float(bits);
      if (!(x >= least) || (x == least && j >= at) || x == -INFINITY) return;
      const float y = scaled(x == zmax ? 0.f : __fsub_rn(x, zmax));
      if (!(y >= floor_y)) return;
      total += exp_fast(y);
      best.take(g ? perturbed(y, g[base + j]) : y, base + j);
    };
    if (tid < n_head) element((uint32_t)zs[edge(tid)] << 16, edge(tid));  // (a thread's tokens in order)
    for (int v = v_lo + tid; v < v_hi; v += SM_THREADS) {
      const uint4 w4 = reinterpret_cast<const uint4*>(zs)[v];
      const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
      float most = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(bf16_lo(w[i]), bf16_hi(w[i])));
      if (most >= least)
#pragma unroll 1
        for (int i = 0; i < 8; ++i) element((uint32_t)zs[8 * v + i] << 16, 8 * v + i);
    }
    if (tid >= n_head && tid < n_edge) element((uint32_t)zs[edge(tid)] << 16, edge(tid));
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
    int token = (int)(0xffffffffu - (uint32_t)top_b);
    if (!top_b)  // every kept y + noise overflowed to -inf: the largest logit
      for (token = 0; token < V - 1 && order_key(canonical(z[token])) != kmax;) ++token;
    const float d = rel(canonical(z[token]));
    a.token[row] = token;
    if (a.prob) a.prob[row] = greedy ? 1.f : exp_fast(scaled(d)) / all;
    if (a.conf) a.conf[row] = exp_fast(d) / whole;
  }
}

template <bool TRUNC>
cudaError_t launch_as(const SampleArgs& a, int C, cudaStream_t stream) {
  const int seg = ((a.V + 7 + C - 1) / C + 7) / 8 * 8;  // (7: a row's first vector may hold one token)
  const size_t smem = (sizeof(SampleShared) + 15) / 16 * 16 + (TRUNC ? 4 * SM_BINS : 0) + 2 * (size_t)seg;
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
