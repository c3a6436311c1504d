// Attention of up to 8 rows of a kv head (new positions x the query heads that share it) over pages in 4
// bits: a decode step's.  More rows take the kernels of kv_attention.cu and kv_attention_tc.cu.
//
// Half a byte a component: at the rate at which memory delivers codes an SM has to widen 45 of them a cycle,
// which costs more than their arrival.  So the products stand the other way
// round than those of wider formats: keys and value components are the M side,
//   S^T [16 keys][8 rows] = K q^T,   O^T [16 components][8 rows] += V^T P^T  (m16n8k16, bf16),
// which leaves no half of an operand or of an accumulator empty, so that O takes 32 registers of a lane, not
// 64, and 16 warps share an SM.  A lane's codes are widened where they are operands (q4.cuh): pairs of
// components of a key, which have one scale; pairs of keys of a component, with the two keys' scales.
// The weights go from S^T's layout to P^T's by movmatrix, 8 x 8 at a time.
//
// All operands are bf16, which every stored value is; weights have two parts, and their reference m stands far
// above the largest score and moves seldom, as in kv_attention.cu with bf16 pages.  Work is shared out and
// joined as there (kv_share.cuh).
//
// 28 / 4 heads of 128, one row a sequence: 2 sequences of 131071 positions (143 MB) in 45.8 us, 3.1 TB/s, 0.46 of the
// measured copy rate; 64 ragged sequences to 4096 (74 MB) in 32.8 us; one of 512, 32 heads, 7.7 us.  A warp takes
// 197 instructions for 8 keys and their values, 94 of them on the integer pipe, which has one for two cycles: 56
// bring codes into place (a shift and a mask for two components), and that pipe is 0.6 to 0.8 busy while keys
// are walked.  Over the whole call neither it (0.45, 21 us of the 45.8) nor the issue slots (0.48) are full: the rest are
// waits of fixed latency in a warp's chain (S, maximum, exp2, movmatrix, then the values), with four warps a scheduler
// to cover them.  The rest of a CTA's time: 3900 cycles to find its part of the line, 4700 until its first keys
// are there, 2700 an item's end, 2800 a join of two parts.  (Keys and values on the N side, as for wider
// formats: 57.5 us and 39.7.  Shifts by multiplication, for the other pipe: 53.6.  16 rows a pass this way
// round: 8 sequences of 1536, 32 heads, 32 rows 52 us, 47.5 in kv_attention.cu, both cut.)
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kv_cache.cuh"
#include "kv_share.cuh"
#include "q4.cuh"

namespace dcl {
namespace {

constexpr int K4_START = 2;   // units of keys that beginning an item takes (64 ragged sequences: 3 33.9 us, 2 32.9, 4 34.7)
constexpr int K4_ONE = 48;    // parts of an item that are joined at once
constexpr int K4_KEYS = 32;   // keys that a warp takes at a time
constexpr float K4_ABOVE = 32.f, K4_SLACK = 8.f;  // the reference above the largest score, and how far that may be passed

template <int HD>
struct K4Cfg {
  static constexpr int ROWS = 8;                     // of an item
  static constexpr int WARPS = 8;                    // (as many as the registers allow)
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int ROWB = HD / 2;                // bytes of a key
  static constexpr int SIDE = HD / Q4_GROUP;         // its scales
  static constexpr int TILE = K4_KEYS * ROWB;
  static constexpr int STAGE = 2 * TILE + 2 * K4_KEYS * SIDE;
  static constexpr int LIMIT = 220 * 1024 / KA_CTAS / WARPS / STAGE;
  static constexpr int STAGES = LIMIT > 6 ? 6 : LIMIT;
  static constexpr int RING = STAGES * STAGE;
  static constexpr int O_PITCH = HD + 36;            // a warp's O in the ring's place: [ROWS][O_PITCH] floats, 16 components and 4 on
  static constexpr int O_B = ROWS * O_PITCH * 4;
  static constexpr int RING_B = (std::max(RING, O_B) + 127) & ~127;
  static constexpr int ML = WARPS * RING_B;          // {m, l} [warp][ROWS]
  static constexpr int WT = ML + WARPS * ROWS * 8;  // weights of the warps' parts [ROWS][8], then {m, l} of the rows
  static constexpr int HEAD = WT + ROWS * (8 * 4 + 8);  // the walk's variables
  static constexpr int TODO = HEAD + 48;             // joins left to this CTA: their number, and two at most
  static constexpr size_t SMEM = TODO + 3 * 24;
  static_assert(WARPS <= 8 && STAGES >= 2 && KA_CTAS * (SMEM + 1024) <= 233472, "shared memory of an SM");
  static_assert(sizeof(KaWalk) <= 48 && sizeof(KaJoin) == 24, "their places");
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// (the same without a sum to add to)
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// An 8 x 8 matrix of 16-bit elements, a row's pairs by four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Whether any value group of a step holds no numbers.
template <int BYTES>
__device__ __noinline__ bool any_without_numbers(uint32_t scales, int lane) {
  bool any = false;
  for (int c = lane; c < BYTES; c += 32) any |= lds_u8(scales + c) >= Q4_SCALES;
  return __any_sync(0xffffffffu, any);
}

// Parts of an item, left by every stride-th CTA from c0 on, joined: into the rows' results, or (GROUP) into the
// first of them.  HD / 4 lanes have a row, a lane four of its components, which
// it copies into shared memory a few parts at a time, the next ones on their way (one takes about 1000
// cycles here); the parts' {m, l} and then their weights stand there, too.  (The lanes' weights exchanged by
// shuffles, 25 parts at a time without others on their way: 11000 cycles for 38 parts.)
template <int HD, int ROWS, int THREADS, int ROOM>
__device__ __forceinline__ void join4(const KvAttn& a, const KaJoin& it, int c0, int stride, int n, bool group, int rep, float* parts, uint8_t* smem) {
  using Part = KaPart<HD, ROWS, false>;
  constexpr int LPR = HD / 4, CHUNK = 10;
  static_assert(THREADS / LPR >= ROWS, "a row for every so many threads");
  static_assert(2 * CHUNK * 16 * THREADS + ROWS * KA_MOST * 8 <= ROOM, "shared memory of a join");
  const int l = threadIdx.x % LPR, r = threadIdx.x / LPR;
  if (r / (32 / LPR) * (32 / LPR) >= it.rows) return;  // (whole warps)
  const int rr = min(r, it.rows - 1);
  // (the item's first CTA's part is its second, the others' their first)
  auto part_of = [&](int c) { return parts + (int64_t)(2 * (c0 + c * stride) + (c == 0 && c0 == it.c0)) * Part::FLOATS; };
  const uint32_t mine = smem_addr(smem) + 16 * threadIdx.x;
  float2* weights = reinterpret_cast<float2*>(smem + 2 * CHUNK * 16 * THREADS) + r * KA_MOST;
  auto ask = [&](int at) {
    const uint32_t to = mine + (at / CHUNK & 1) * (CHUNK * 16 * THREADS);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)
      if (at + i < n) copy16(to + 16 * THREADS * i, part_of(at + i) + Part::four(rr, l));
    copy_commit();
  };
  ask(0);
  ask(CHUNK);
  float top = -INFINITY, sum = 0.f;
#pragma unroll 2
  for (int c = l; c < n; c += LPR) {
    const float2 x = __ldcg(reinterpret_cast<const float2*>(part_of(c) + Part::ml(rr)));
    weights[c] = x;
    top = fmaxf(top, x.x);
  }
#pragma unroll
  for (int d = LPR / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  for (int c = l; c < n; c += LPR) {  // (what this lane wrote)
    const float2 x = weights[c];
    const float half = part_half(x.x, top);
    weights[c].x = half * half;
    sum = fmaf(x.y * half, half, sum);
  }
#pragma unroll
  for (int d = LPR / 2; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  __syncwarp();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int at = 0; at < n; at += CHUNK) {
    copy_wait<1>();
    const uint32_t from = mine + (at / CHUNK & 1) * (CHUNK * 16 * THREADS);
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
      if (at + i >= n) break;
      const uint4 y = lds128(from + 16 * THREADS * i);
      add_scaled(acc, make_float4(__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w)), weights[at + i].x);
    }
    ask(at + 2 * CHUNK);
  }
  copy_wait<0>();
  __syncwarp();  // (the weights' places are free again)
  if (r >= it.rows) return;
  if (group) {
    *reinterpret_cast<float4*>(part_of(0) + Part::four(r, l)) = acc;
    if (l == 0) *reinterpret_cast<float2*>(part_of(0) + Part::ml(r)) = make_float2(top, sum);
    return;
  }
  const int tok = (it.first + r) / rep, at = (it.row0 + tok) * a.H + it.head0 + it.first + r - tok * rep;
  if (a.lse && l == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
  finish4<HD>(a, KaRow{sum == 0.f ? 0.f : 1.f / sum, at}, 4 * l, acc);
}

template <int HD, bool GROUPS>
__global__ void __launch_bounds__(K4Cfg<HD>::THREADS, KA_CTAS) kv_attention_q4_kernel(KvPool kv, KvAttn a, KaScratch scratch, int* err) {
  using C = K4Cfg<HD>;
  constexpr int ROWS = C::ROWS, KT = K4_KEYS, SIDE = C::SIDE, ROWB = C::ROWB, CPR = ROWB / 16;
  constexpr int KS = HD / 16;   // k steps of S
  constexpr int MT = HD / 16;   // tiles of 16 components of O
  constexpr int W = HD / 64;    // 8-code words of a value that a lane has
  constexpr uint32_t EIGHT = ROWB == 64 ? 512 : 128;  // 8 keys on, in a tile
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, place = lane & 3;
  const int rep = a.H / kv.G, P = kv.page_len();
  const bool small = kv.page_shift == 4;
  const uint32_t ring = smem_addr(smem) + warp * C::RING_B;
  float2* ml = reinterpret_cast<float2*>(smem + C::ML);
  // where a lane's chunk of a copy lies, its part of key quad, and of values 2 place and 2 place + 1
  const uint32_t copy_at = chunk4_at<ROWB>(lane / CPR, lane % CPR);
  const uint32_t k_at = HD == 128 ? chunk4_at<ROWB>(quad, place) : chunk4_at<ROWB>(quad, place >> 1) + 8 * (place & 1);
  const uint32_t v_at[2] = {chunk4_at<ROWB>(2 * place, quad * (HD / 16) >> 4) + (quad * (HD / 16) & 15),
                            chunk4_at<ROWB>(2 * place + 1, quad * (HD / 16) >> 4) + (quad * (HD / 16) & 15)};
  // a copy's addresses: chunk `lane` of 16 keys; of the scales of a page's keys (16 or 32), then of the values'
  const uint8_t* k_from = static_cast<const uint8_t*>(kv.k) + 16 * lane;
  const uint8_t* v_from = static_cast<const uint8_t*>(kv.v) + 16 * lane;
  const int side_chunks = small ? SIDE : 2 * SIDE, of = lane / side_chunks, side_chunk = 16 * (lane - of * side_chunks);
  const uint8_t* side_from = reinterpret_cast<const uint8_t*>(of ? kv.v_exp : kv.k_exp) + side_chunk;
  const uint32_t side_at = 2 * C::TILE + SIDE * KT * of + side_chunk, page_bytes = (uint32_t)(kv.G * P * ROWB);  // (2^24 at most)
  const int k_group = place * SIDE / 4, v_group = quad * SIDE / 8;
  const float qa = fmaxf(a.scale * kLog2e, 1.2e-38f);  // (not 0: a masked score is -inf)

  const KaLine<ROWS, K4_START, KA_KEEP, KA_FINE> line(kv, a);

  // ---- this CTA's part of the line of all items
  KaWalk& shared_walk = *reinterpret_cast<KaWalk*>(smem + C::HEAD);
  KaJoin* todo = reinterpret_cast<KaJoin*>(smem + C::TODO);
  if (warp == 0) {
    line.begin(&shared_walk, err);
    if (lane == 0) todo[0].rows = 0;
  }
  __syncthreads();
  KaWalk walk = shared_walk;
  KaItem it;
  it.b = -1;

  while (line.next(walk, it)) {
    const int key0 = it.from * KA_UNIT, key1 = min(it.len, it.until * KA_UNIT);
    // the keys that the item's rows see: its first row the fewest, its last the most
    const int lim_min = a.causal ? it.len - it.nq + it.first / rep + 1 : it.len;
    const int lim_max = a.causal ? min(it.len, it.len - it.nq + (it.first + it.rows - 1) / rep + 1) : it.len;

    // ---- q of row quad, this lane's quarter of its components; asked for before the keys, which would be in the way
    uint4 raw[HD / 32];
    {
      const int rr = it.first + quad, tok = rr / rep, h = it.g * rep + rr - tok * rep;
      const __nv_bfloat16* src = a.q + (it.row0 + tok) * a.q_stride + (int64_t)h * HD + place * (HD / 4);
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) raw[c] = quad < it.rows ? *reinterpret_cast<const uint4*>(src + 8 * c) : make_uint4(0, 0, 0, 0);
    }

    const uint32_t head_at = (uint32_t)(it.g * P * ROWB);
    // ---- this warp's steps: keys key0 + KT warp on, then every WARPS-th
    const int stop = max(0, min(key1, lim_max));  // (rows that see nothing may be before key 0)
    const int* table = a.table + (int64_t)it.b * a.max_pages;
    int next = key0 + KT * warp;  // first key of the next step to copy
    uint32_t bad = 0;             // two bits a stage: 16 keys whose page is not the cache's
    uint32_t slot = 0;            // of the ring, in bytes
    int pages[2];                 // of this warp's steps, a step a lane (longer pages than 16 hold a step's keys together)
    int turn = 0;                 // the next step's lane
    auto look_up = [&]() {
      const uint32_t key = (uint32_t)next + KT * C::WARPS * lane;  // (which may pass 2^31)
      pages[0] = key < (uint32_t)stop ? table[key >> kv.page_shift] : 0;
      pages[1] = small && key + 16 < (uint32_t)stop ? table[(key + 16) >> kv.page_shift] : pages[0];
    };
    look_up();
    const uint8_t *k_head = k_from + head_at, *v_head = v_from + head_at, *side_head = side_from + head_at / (ROWB / SIDE);
    auto copy = [&](int page, int in_page, int h, auto rows_) {  // 16 keys or 32 of a page
      constexpr int ROWS = decltype(rows_)::value;
      const uint64_t at = (uint64_t)(unsigned)page * page_bytes + (uint32_t)(in_page * ROWB);
      const uint8_t *k = k_head + at, *v = v_head + at;
      const uint32_t dst = ring + slot + copy_at + 16 * ROWB * h;
#pragma unroll
      for (int i = 0; i < ROWS * ROWB / 512; ++i) {
        copy16(dst + 512 * i, k + 512 * i);
        copy16(dst + C::TILE + 512 * i, v + 512 * i);
      }
      if (lane < 2 * side_chunks) copy16(ring + slot + side_at + 16 * SIDE * h, side_head + at / (ROWB / SIDE));
    };
    auto issue = [&]() {
      uint32_t gone = 0;
      if (next < stop) {
        const int page = __shfl_sync(0xffffffffu, pages[0], turn);
        const bool there = (unsigned)page < (unsigned)kv.pages;
        if (!small) {  // (one page holds all 32, those past the sequence's end too)
          if (there) copy(page, next & (P - 1), 0, std::integral_constant<int, 32>{});
          else gone = 3;
        } else {
          const int page1 = __shfl_sync(0xffffffffu, pages[1], turn);
          if (there) copy(page, 0, 0, std::integral_constant<int, 16>{});
          else gone = 1;
          if (next + 16 < stop) {
            if ((unsigned)page1 < (unsigned)kv.pages) copy(page1, 0, 1, std::integral_constant<int, 16>{});
            else gone |= 2;
          }
        }
        if (gone && lane == 0) report_error(err, DERR_KV_RANGE);
        next += KT * C::WARPS;
        turn = (turn + 1) & 31;
        if (turn == 0) look_up();
      }
      bad = bad << 2 | gone;
      copy_commit();
      slot = slot == C::RING - C::STAGE ? 0 : slot + C::STAGE;
    };
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s) issue();

    // q as the product's operand: of 8 components 0 and 4, 1 and 5, then 2 and 6, 3 and 7, as codes are widened
    uint32_t q[KS][2];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const uint32_t* w = &raw[s >> 1].x + (s & 1);
      q[s][0] = __byte_perm(w[0], w[2], 0x5410);
      q[s][1] = __byte_perm(w[0], w[2], 0x7632);
    }

    // ---- rows 2 place and 2 place + 1 are this lane's in S^T and O^T
    int lim[2];  // keys each sees
    float o[MT][4], m[2], l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 2 * place + i;
      lim[i] = r >= it.rows ? 0 : a.causal ? min(it.len, it.len - it.nq + (it.first + r) / rep + 1) : it.len;
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < MT; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[c][j] = 0.f;

    uint32_t cur = 0;
    for (int key = key0 + KT * warp; key < stop; key += KT * C::WARPS) {
      issue();  // into the stage that the last step left
      copy_wait<C::STAGES - 1>();
      __syncwarp();
      const uint32_t sk = ring + cur, sv = sk + C::TILE, se = sv + C::TILE;
      const uint32_t skip = bad >> (2 * (C::STAGES - 1)) & 3u;  // (this step's was put there so many steps ago)
      cur = cur == C::RING - C::STAGE ? 0 : cur + C::STAGE;
      const bool masked = key + KT > lim_min || skip;
      if (key + KT > lim_max || skip) {  // values that no row sees may be anything; any codes are numbers
        for (int c = lane; c < KT * SIDE; c += 32) {
          const int r = c / SIDE;
          if (key + r >= lim_max || (skip >> (r >> 4) & 1)) sts8(se + KT * SIDE + c, 0);
        }
        __syncwarp();
      }
      // Values that are no numbers and that only some of the rows see (0 * NaN): the rows that do get NaN, and the
      // group a scale that is one.
      if (masked && a.causal && any_without_numbers<KT * SIDE>(se + KT * SIDE, lane)) {
        for (int j = 0; j < KT; ++j) {
          if (lds_u8(se + (KT + j) * SIDE + v_group) < Q4_SCALES) continue;
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (key + j < lim[i])
#pragma unroll
              for (int c = 0; c < MT; ++c) o[c][i] = o[c][2 + i] = NAN;
        }
        __syncwarp();
        for (int c = lane; c < KT * SIDE; c += 32)
          if (lds_u8(se + KT * SIDE + c) >= Q4_SCALES) sts8(se + KT * SIDE + c, 0);
        __syncwarp();
      }
      // ---- S^T = K q^T: tiles of 16 keys, this lane's are quad and quad + 8
      float s[KT / 16][4];
#pragma unroll
      for (int t = 0; t < KT / 16; ++t) {
        uint32_t w[2][2 * W];
        Q4Scale f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t at = sk + k_at + 16 * ROWB * t + EIGHT * i;
          if (HD == 128) {
            const uint4 x = lds128(at);
            w[i][0] = x.x;
            w[i][1] = x.y;
            w[i][2 * W - 2] = x.z;
            w[i][2 * W - 1] = x.w;
          } else {
            const uint2 x = lds64(at);
            w[i][0] = x.x;
            w[i][1] = x.y;
          }
          f[i] = q4_scale_twice(lds_u8(se + (16 * t + 8 * i + quad) * SIDE + k_group));
        }
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          const int i = 2 * (x & 1);
          const uint32_t a0 = q4_widen(w[0][x >> 1], i, f[0]), a1 = q4_widen(w[1][x >> 1], i, f[1]);
          const uint32_t a2 = q4_widen(w[0][x >> 1], i + 1, f[0]), a3 = q4_widen(w[1][x >> 1], i + 1, f[1]);
          if (x == 0) mma_bf16_first(s[t], a0, a1, a2, a3, q[x][0], q[x][1]);
          else mma_bf16(s[t], a0, a1, a2, a3, q[x][0], q[x][1]);
        }
      }
      if (masked) {
#pragma unroll
        for (int t = 0; t < KT / 16; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (key + 16 * t + quad + 8 * (j >> 1) >= lim[j & 1] || (skip >> t & 1)) s[t][j] = -INFINITY;
      }
      // ---- a larger reference where a row's largest score passes it too far, or is its first
      float top[2];
      bool grew = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = fmaxf(s[0][i], s[0][2 + i]);
#pragma unroll
        for (int t = 1; t < KT / 16; ++t) x = fmaxf(x, fmaxf(s[t][i], s[t][2 + i]));
        top[i] = x * qa;
        grew |= top[i] > m[i] - (K4_ABOVE - K4_SLACK);
      }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = top[i];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          const float mn = fmaxf(m[i], x + K4_ABOVE);
          const float alpha = exp2_fast(m[i] - (mn == -INFINITY ? 0.f : mn));
          m[i] = mn;
          l[i] *= alpha;
#pragma unroll
          for (int c = 0; c < MT; ++c) {
            o[c][i] *= alpha;
            o[c][2 + i] *= alpha;
          }
        }
      }
      // ---- P^T in two parts
      uint32_t p[KT / 16][2], p_lo[KT / 16][2];
      const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};  // (nothing seen yet: exp2(-inf) = 0)
#pragma unroll
      for (int t = 0; t < KT / 16; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // keys quad + 8 i
          const float x0 = exp2_fast(fmaf(s[t][2 * i], qa, -ref[0])), x1 = exp2_fast(fmaf(s[t][2 * i + 1], qa, -ref[1]));
          l[0] += x0;
          l[1] += x1;
          p[t][i] = transposed(upper_halves(x0, x1));
          p_lo[t][i] = transposed(pack_bf16x2(fmaf(x0, BF16_LO, minus_upper(x0)), fmaf(x1, BF16_LO, minus_upper(x1))));
        }
      // ---- O^T += V^T P^T, 16 keys at a time; a lane's components are quad * HD / 8 on
#pragma unroll
      for (int t = 0; t < KT / 16; ++t) {
        uint32_t v[4][W], scale[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // keys 2 place, 2 place + 1, and 8 on
          const uint32_t at = sv + v_at[r & 1] + 16 * ROWB * t + EIGHT * (r >> 1);
          if (W == 2) {
            const uint2 x = lds64(at);
            v[r][0] = x.x;
            v[r][W - 1] = x.y;
          } else {
            v[r][0] = lds32(at);
          }
          scale[r] = lds_u8(se + (KT + 16 * t + 2 * place + (r & 1) + 8 * (r >> 1)) * SIDE + v_group);
        }
        const Q4Scale f0 = q4_scale(scale[0] + (scale[1] << 16)), f1 = q4_scale(scale[2] + (scale[3] << 16));
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int up = 0; up < 2; ++up) {  // a word's lower four components, its upper four; two keys side by side
            const uint32_t x0 = __byte_perm(v[0][w], v[1][w], up ? 0x7632 : 0x5410);
            const uint32_t x1 = __byte_perm(v[2][w], v[3][w], up ? 0x7632 : 0x5410);
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              float(&acc)[4] = o[4 * w + 2 * up + j / 2];
              const uint32_t a0 = q4_widen(x0, j, f0), a1 = q4_widen(x0, j + 1, f0), a2 = q4_widen(x1, j, f1), a3 = q4_widen(x1, j + 1, f1);
              mma_bf16(acc, a0, a1, a2, a3, p[t][0], p[t][1]);
              mma_bf16(acc, a0, a1, a2, a3, p_lo[t][0], p_lo[t][1]);
            }
          }
      }
      __syncwarp();
    }
    copy_wait<0>();
    __syncwarp();

    // ---- join the warps
    constexpr int RUN = HD / 8;  // components of a lane
    float* mine = reinterpret_cast<float*>(smem + warp * C::RING_B) + quad * (RUN + 4);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 2 * place + i;
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
      if (quad == 0) ml[warp * ROWS + r] = make_float2(m[i], l[i]);
      if (key0 + KT * warp < stop)
#pragma unroll
        for (int c = 0; c < MT; c += 2)
          *reinterpret_cast<float4*>(mine + r * C::O_PITCH + 2 * c) = make_float4(o[c][i], o[c][2 + i], o[c + 1][i], o[c + 1][2 + i]);
    }
    __syncthreads();
    // a row's weights by a thread, then four components of a row a thread
    float* wt = reinterpret_cast<float*>(smem + C::WT);
    KaRow* row = reinterpret_cast<KaRow*>(smem + C::WT + ROWS * 32);
    float* part = scratch.part + (2 * (int64_t)blockIdx.x + (it.from == 0)) * ROWS * (HD + 4);
    if (threadIdx.x < it.rows) {
      const int r = threadIdx.x;
      float2 x[C::WARPS];
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < C::WARPS; ++w) {
        x[w] = ml[w * ROWS + r];
        top = fmaxf(top, x[w].x);
      }
#pragma unroll
      for (int w = 0; w < C::WARPS; ++w) {
        const float half = part_half(x[w].x, top);
        wt[r * 8 + w] = half * half;
        sum = fmaf(x[w].y * half, half, sum);
      }
      if (it.whole())
        row[r] = finish_row(a, it.row0, it.g * rep, it.first, rep, r, top, sum);
      else
        *reinterpret_cast<float2*>(part + r * (HD + 4) + HD) = make_float2(top, sum);
    }
    __syncthreads();
    constexpr int PART = HD + 4, Q = HD / 4;
    const int active = min(C::WARPS, (stop - key0 + KT - 1) / KT);  // (warps without keys have written no O)
    for (int t = threadIdx.x; t < it.rows * Q; t += C::THREADS) {
      const int r = t / Q, c = 4 * (t % Q);
      const float* o_row = reinterpret_cast<const float*>(smem) + r * C::O_PITCH + c + 4 * (c / RUN);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < C::WARPS; ++w)
        if (w < active) add_scaled(acc, *reinterpret_cast<const float4*>(o_row + w * (C::RING_B / 4)), wt[r * 8 + w]);
      if (it.whole())
        finish4<HD>(a, row[r], c, acc);
      else
        *reinterpret_cast<float4*>(part + r * PART + c) = acc;
    }
    if (!it.whole()) {
      int c0, c1;
      line.sharers(walk, it, c0, c1);
      __syncthreads();
      if (threadIdx.x == 0) {
        // the last to come joins the parts, those of its group first, when it is through with its own
        const KaGroups by(c1 - c0 + 1, GROUPS ? K4_ONE : INT_MAX);
        const int k = by.of(blockIdx.x - c0), at = c0 + k * by.size;
        if (ka_come(by.groups == 1 ? scratch.count + c0 : scratch.count + KA_MOST + 2 * at + (k == 0), by.parts(k)))
          todo[todo[0].rows++ ? 2 : 1] = KaJoin{it.row0, it.g * rep, it.first, it.rows, c0, c1 - c0 + 1};
      }
    } else {
      __syncthreads();  // (the rings are free again)
    }
  }
  __syncthreads();
  for (int i = 0; i < todo[0].rows; ++i) {
    const KaJoin j = todo[1 + i];
    const KaGroups by(j.parts, GROUPS ? K4_ONE : INT_MAX);
    const int k = by.of(blockIdx.x - j.c0);
    bool group = GROUPS && by.groups > 1;
    int c0 = j.c0 + k * by.size, stride = 1, n = by.parts(k);
    while (true) {
      join4<HD, ROWS, C::THREADS, C::ML>(a, j, c0, stride, n, group, rep, scratch.part, smem);
      if (!GROUPS || !group) break;
      __syncthreads();
      if (threadIdx.x == 0) todo[0].parts = ka_come(scratch.count + j.c0, by.groups);
      __syncthreads();
      if (!todo[0].parts) break;
      c0 = j.c0;
      stride = by.size;
      n = by.groups;
      group = false;
    }
  }
}

template <int HD, bool GROUPS>
cudaError_t launch_as(const KvPool& kv, const KvAttn& a, const KaScratch& s, int ctas, int* err, cudaStream_t stream) {
  using C = K4Cfg<HD>;
  static_assert(2 * C::ROWS * (HD + 4) * 4 <= KV_ATTN_PART_BYTES, "scratch");
  auto kern = kv_attention_q4_kernel<HD, GROUPS>;
  static const cudaError_t set = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
  if (set != cudaSuccess) return set;
  kern<<<ctas, C::THREADS, C::SMEM, stream>>>(kv, a, s, err);
  return cudaGetLastError();
}

}  // namespace

bool kv_attention_q4_few(const KvPool& kv, const KvAttn& a) { return kv.format == KV_Q4 && (int64_t)a.max_new * (a.H / kv.G) <= 8; }

cudaError_t kv_attention_q4_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream) {
  const int ctas = KA_CTAS * std::min(sms, KA_MOST / KA_CTAS);
  KaScratch s{reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + KV_ATTN_COUNTERS), static_cast<int*>(scratch)};
  // Joins in two steps, in a kernel of their own (the other's calls took 1 % longer with them), where so few long
  // items may have more parts than K4_ONE.  28 / 4 heads, one row, us in one step / two: 1 x 65536 27.1 / 22.7, 1 x 131072
  // 33.2 / 30.1; 38 parts an item: 2 x 131071 46.3 / 46.0, 32 / 8 heads 1 x 131072 44.6 / 45.0; 24 parts and fewer 1 to 2 us
  // longer in two.
  const bool groups = (int64_t)a.batch * kv.G * K4_ONE < ctas && (int64_t)a.max_pages << kv.page_shift > K4_ONE * KA_FINE * KA_UNIT;
  auto as = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    return groups ? launch_as<HD, true>(kv, a, s, ctas, err, stream) : launch_as<HD, false>(kv, a, s, ctas, err, stream);
  };
  return kv.hd == 128 ? as(std::integral_constant<int, 128>{}) : as(std::integral_constant<int, 64>{});
}

}  // namespace dcl
