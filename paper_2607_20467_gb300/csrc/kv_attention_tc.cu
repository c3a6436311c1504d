// Attention of many new positions of every sequence over its paged keys and values, on the tcgen05
// tensor cores: the rows of an item (up to 256: new positions x the query heads of one kv head)
// fill one or two tiles of 128, and one pass over the keys serves them all.
//
// Per unit of 128 keys: S = Q K^T into TMEM; P = exp2(S scaled - m) in two bf16 parts (2^-16 of itself) takes
// the place of its scores there; O += P V in TMEM.  A thread owns a row, so its statistics need no
// exchange.
//
// All operands are bf16, which holds every value that a cache stores: FP8 codes are widened with their
// exponents, so that nothing is lost whatever the sizes of neighbouring keys and values, and the rows'
// loop knows of no exponents.  Eight warps copy the pages into shared memory (16-byte asynchronous
// copies, one unit ahead), bf16 straight into the operand tiles, FP8 codes into a buffer from which
// they widen them.  (fp16 operands, scaled by the largest exponent of 32 keys, lost those far below it.)
// V's tile is [key][hd], the transposed ("MN-major") form of the B operand, as it comes.
//
// The reference m, 32 above a row's largest score when it is taken, moves only when a unit's passes it
// by more than 8; O is scaled then.  (P stays far below 1, so that no sum of large values overflows.)
//
// 16 sequences of 8192 positions, FP8, 28 / 4 heads of 128, 32 new positions each (224 rows a kv head;
// 143 MB, 60 GFLOP): 109.5 us, 0.28 of the tensor rate.  Neither memory (0.19) nor the tensor pipe
// (0.45 busy, P's second part included) bounds it but the chain S -> maximum -> weights -> O of a
// tile, with two tiles in turn: of 6800 cycles a unit a row's warp takes 2200 to 3000 for the weights, 650
// to 1200 for the maximum, waits 1900 to 2200 for S and has about 900 for an item's q and results.  The
// CTAs' work ends after 88 to 102 us, and the joins come after it.
//
// Roles (544 threads): warps 0-3 and 4-7 have the rows of the two tiles; warps 8-11 copy and widen
// keys, 12-15 values (one group for both was the slowest link: 7800 cycles a unit); warp 16
// allocates TMEM and issues the MMAs.  17 warps leave 96 registers a thread: a row's warp holds 32 scores at
// a time (the next 32 on their way as well spill: 137 us).  Two warps for a tile's 32 rows, half the
// keys each, were no faster (115 us).  Every wait is bounded (DERR_WAIT_TIMEOUT).
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kv_cache.cuh"
#include "kv_share.cuh"
#include "tc_ptx.cuh"

namespace dcl {
namespace {

constexpr int TC_ROWS = 256;      // rows of an item
constexpr int TC_START = 2;       // units of keys that beginning an item takes
constexpr float TC_ABOVE = 32.f;  // of a row's largest score, where its reference is taken
constexpr float TC_SLACK = 8.f;   // by how much a later score may pass that one
constexpr int TC_THREADS = 544;
constexpr int TC_BOX = 128 * 128; // 128 rows of 128 bytes, swizzled
constexpr int TC_JOIN = 8000;     // rows x parts joined at a time

template <int HD, bool FP8>
struct TcCfg {
  static constexpr int KB = HD / 64;                  // boxes along hd
  static constexpr int TILE = KB * TC_BOX;            // 128 rows of q, keys or values, 16 bits each
  static constexpr int NS = 4;                        // operand tiles of keys and values, in turn
  static constexpr int KV = 2 * TILE;                 // (q comes first)
  static constexpr int RAW = KV + NS * TILE;          // FP8: codes of a unit's keys, then of its values
  static constexpr int THERE = RAW + (FP8 ? 2 * 128 * HD : 0);  // [4 units][4 x 32 keys]: a bit for each key that is there
  static constexpr int BAR = THERE + 4 * 4 * 4;                 // (keys may be two units ahead)
  static constexpr int NBARS = 2 * NS + 4 * 2 + 1;
  static constexpr int HOLDER = BAR + 8 * NBARS;      // TMEM address, abort flag
  static constexpr int WALK = HOLDER + 8;
  static constexpr int TODO = WALK + (int)sizeof(KaWalk);
  static constexpr size_t SMEM = TODO + 3 * sizeof(KaJoin);
  static_assert(SMEM <= 232448, "shared memory per CTA");
  static_assert(TC_JOIN * 8 + TC_ROWS * 8 <= THERE, "a join's weights take the place of the operands");
};

// The value of lane 0, which the compiler then knows to be the whole warp's (uniform registers).
__device__ __forceinline__ int warp_uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Descriptor of a [key][hd] tile as the transposed B operand: 128-byte rows of 64 components (the next
// 64 a box on), 8-row swizzle atoms along the keys.
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(TC_BOX >> 4) << 16;  // leading byte offset: the next 64 components
  d |= (uint64_t)(1024 >> 4) << 32;    // stride byte offset: the next 8 keys
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t IDESC_B_MN = 1u << 16;
// D += A B with A (bf16 pairs) in TMEM.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Two E4M3 codes times f (bf16 pairs), exactly: the code by way of fp16 and fp32, which hold it.
__device__ __forceinline__ uint32_t widen(uint32_t w, int half, __nv_bfloat162 f) {
  const uint32_t r = half ? widen_hi(w) : widen_lo(w);
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&r));
  const __nv_bfloat162 y = __hmul2(__floats2bfloat162_rn(x.x, x.y), f);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// The MMAs of an item (the whole warp; one lane issues).  Its operands are made known as the warp's, in
// uniform registers: else an issue takes about 100 cycles, more than most of the products.
template <int HD, bool FP8>
__device__ __forceinline__ bool tc_mma(uint32_t base, uint32_t tmem, int tiles, int n, uint32_t& seq_, uint32_t& items,
                                       uint32_t& units, volatile int* abort_flag) {
  using C = TcCfg<HD, FP8>;
  constexpr uint32_t idesc_s = make_idesc(128, 128);
  constexpr uint32_t idesc_o = make_idesc(128, HD) | IDESC_B_MN;
  base = (uint32_t)warp_uniform((int)base);
  tmem = (uint32_t)warp_uniform((int)tmem);
  tiles = warp_uniform(tiles);
  n = warp_uniform(n);
  uint32_t seq = (uint32_t)warp_uniform((int)seq_);
  const uint32_t full0 = base + C::BAR, empty0 = full0 + 8 * C::NS, s_full0 = empty0 + 8 * C::NS, p_full0 = s_full0 + 16;
  const uint32_t p_empty0 = p_full0 + 16, q_full0 = p_empty0 + 16;
  const bool leader = elect_one();
  auto wait = [&](uint32_t bar, uint32_t parity) {
    return (bool)__all_sync(0xffffffffu, mbar_wait_inline(bar, parity, abort_flag));
  };
  auto full = [&](uint32_t s) { return wait(full0 + 8 * (s % C::NS), (s / C::NS) & 1u); };
  auto issue_s = [&](int t, uint32_t s, bool last) {  // S of the keys at place s
    const uint64_t dq = sw128_desc(base + t * C::TILE), dk = sw128_desc(base + C::KV + (s % C::NS) * C::TILE);
    if (leader) {
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
        umma_bf16(tmem + 128u * t, dq + (k >> 2) * (TC_BOX >> 4) + 2 * (k & 3), dk + (k >> 2) * (TC_BOX >> 4) + 2 * (k & 3),
                  idesc_s, k > 0 ? 1u : 0u);
      umma_commit(s_full0 + 8 * t);
      if (last) umma_commit(empty0 + 8 * (s % C::NS));
    }
    __syncwarp();
  };
  if (!full(seq)) return false;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (t >= tiles) break;
    if (!wait(q_full0 + 8 * t, (items >> (16 * t)) & 1u)) return false;
    items ^= 1u << (16 * t);
    tc_fence_after();
    issue_s(t, seq, t + 1 == tiles);
  }
  for (int u = 0; u < n; ++u, seq += 2) {
    if (!full(seq + 1) || (u + 1 < n && !full(seq + 2))) return false;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (t >= tiles) break;
      if (!wait(p_full0 + 8 * t, (units >> (16 * t)) & 1u)) return false;
      units ^= 1u << (16 * t);
      tc_fence_after();
      const uint64_t dv = sw128_desc_mn(base + C::KV + ((seq + 1) % C::NS) * C::TILE);
      if (leader) {
#pragma unroll
        for (int k = 0; k < 8; ++k)  // (P's parts stand where its scores were: per 32 keys 16 of their columns each)
#pragma unroll
          for (int part = 0; part < 2; ++part)
            umma_bf16_ts(tmem + 256u + (uint32_t)(HD * t), tmem + 128u * t + 32 * (k >> 1) + 16 * part + 8 * (k & 1),
                        dv + k * (2048 >> 4), idesc_o, (u > 0 || k > 0 || part > 0) ? 1u : 0u);
        umma_commit(p_empty0 + 8 * t);
        if (t + 1 == tiles) umma_commit(empty0 + 8 * ((seq + 1) % C::NS));
      }
      __syncwarp();
      if (u + 1 < n) issue_s(t, seq + 2, t + 1 == tiles);
    }
  }
  seq_ = seq;
  return true;
}

template <int HD, bool FP8>
__global__ void __launch_bounds__(TC_THREADS, 1)
    kv_attention_tc_kernel(KvPool kv, KvAttn a, KaScratch scratch, int* err) {
  using C = TcCfg<HD, FP8>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint32_t base = smem_u32(smem);
  asm volatile("" : "+r"(base));
  if (base & 1023u) {  // (the swizzled operands need it; uniform over the grid)
    if (threadIdx.x == 0) report_error(err, DERR_BAD_SHAPE);
    return;
  }
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rep = a.H / kv.G;
  const uint32_t full0 = base + C::BAR, empty0 = full0 + 8 * C::NS, s_full0 = empty0 + 8 * C::NS, p_full0 = s_full0 + 16;
  const uint32_t p_empty0 = p_full0 + 16, q_full0 = p_empty0 + 16, drain = q_full0 + 16;
  volatile uint32_t* holder = reinterpret_cast<volatile uint32_t*>(smem + C::HOLDER);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::HOLDER + 4);
  KaWalk& shared_walk = *reinterpret_cast<KaWalk*>(smem + C::WALK);
  KaJoin* todo = reinterpret_cast<KaJoin*>(smem + C::TODO);
  const KaLine<TC_ROWS, TC_START> line(kv, a);

  if (warp == 0) line.begin(&shared_walk, err);
  if (warp == 16) {
    if (lane == 0) {
      for (int s = 0; s < C::NS; ++s) {
        mbar_init(full0 + 8 * s, 4);   // the copying warps
        mbar_init(empty0 + 8 * s, 1);
      }
      for (int t = 0; t < 2; ++t) {
        mbar_init(s_full0 + 8 * t, 1);
        mbar_init(p_full0 + 8 * t, 4); // the tile's warps
        mbar_init(p_empty0 + 8 * t, 1);
        mbar_init(q_full0 + 8 * t, 4);
      }
      mbar_init(drain, 1);
      fence_mbar_init();
      *abort_flag = 0;
      todo[0].rows = 0;
    }
    __syncwarp();
    tmem_alloc(base + C::HOLDER, 512);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *holder;
  KaWalk walk = shared_walk;
  KaItem it;
  it.b = -1;
  auto wait = [&](uint32_t bar, uint32_t parity) {  // (the whole warp; one outcome for all its lanes)
    return (bool)__all_sync(0xffffffffu, mbar_wait_inline(bar, parity, abort_flag));
  };
  auto gave_up = [&]() {
    *abort_flag = 1;
    if (lane == 0) report_error(err, DERR_WAIT_TIMEOUT);
  };

  if (warp >= 8 && warp < 16) {
    // ================================================================ copies, widening
    // Keys or values of a unit: warp w of the four has keys 32 w .. 32 w + 31, lane l knows of key 32 w + l
    // (its page and exponents); they are copied in chunks of 16 bytes.
    const int values = warp >= 12, w4 = warp & 3;
    constexpr int CH = FP8 ? HD / 16 : HD / 8;       // chunks of a vector
    constexpr int PK = CH / 4;                       // this lane's of a key: key (lane >> 2) + 8 i, chunk (lane & 3) + 4 j
    const int shift = kv.page_shift, P = kv.page_len(), at_key = 32 * w4 + (lane >> 2), at_chunk = lane & 3;
    const void* pool = values ? kv.v : kv.k;
    const int8_t* exps = values ? kv.v_exp : kv.k_exp;
    const uint32_t raw = base + C::RAW + values * (128 * HD);
    uint32_t seq = values;  // operand tiles (keys and values in turn): stage seq % NS
    bool ok = true;
    // (codes: eight lanes read two keys, whose chunks lie in each other's halves of 128 bytes)
    auto raw_at = [&](int k, int c) { return (uint32_t)(k * CH + (CH == 8 ? c ^ (4 * (k & 1)) : c)) * 16; };
    auto tile_at = [&](int k, int c) { return (uint32_t)(c >> 3) * TC_BOX + swz(k, c & 7); };  // 16-bit elements
    auto stage_of = [&](uint32_t s) { return base + C::KV + (s % C::NS) * C::TILE; };
    auto wait_empty = [&](uint32_t s) { return wait(empty0 + 8 * (s % C::NS), ((s / C::NS) & 1u) ^ 1u); };
    while (ok && line.next(walk, it)) {
      const int stop = min(it.len, it.until * KA_UNIT), n = it.until - it.from, first = it.from * KA_UNIT + 32 * w4;
      const int* table = a.table + (int64_t)it.b * a.max_pages;
      auto page_at = [&](int unit) {  // of this lane's key; negative: it is not to be read
        const int key = first + unit * KA_UNIT + lane;
        if (unit >= n || key >= stop) return -1;
        const int page = table[key >> shift];
        if (page >= 0 && page < kv.pages) return page;
        report_error(err, DERR_KV_RANGE);
        return -1;
      };
      auto vec_of = [&](int page, int key) { return kv.vector_of((page << shift) + (key & (P - 1)), it.g); };
      auto issue = [&](int unit, int pages, uint32_t dst) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 16 keys of one page
          const int page = __shfl_sync(0xffffffffu, pages, 16 * h);
          if (page < 0) continue;
          const uint8_t* src = static_cast<const uint8_t*>(pool) + vec_of(page, first + unit * KA_UNIT + 16 * h) * (CH * 16) +
                               ((lane >> 2) * CH + at_chunk) * 16;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < PK; ++j) {
              const int k = at_key + 16 * h + 8 * i, c = at_chunk + 4 * j;
              copy16(dst + (FP8 ? raw_at(k, c) : tile_at(k, c)), src + (8 * i * CH + 4 * j) * 16);
            }
        }
        copy_commit();
      };
      auto exp_at = [&](int unit, int page) {
        return FP8 && page >= 0 ? (int)exps[vec_of(page, first + unit * KA_UNIT + lane)] : 0;
      };
      int pages = page_at(0), pages2 = page_at(1);
      int e = exp_at(0, pages);
      if (!FP8) ok = wait_empty(seq);
      if (ok) issue(0, pages, FP8 ? raw : stage_of(seq));
      for (int u = 0; ok && u < n; ++u) {
        const uint32_t dst = stage_of(seq), here = __ballot_sync(0xffffffffu, pages >= 0);
        copy_wait<0>();
        __syncwarp();
        if (FP8) {
          const float scale = kv_pow2(e);
          const uint32_t mine = pack_bf16x2(scale, scale);  // (exact)
          ok = wait_empty(seq);
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = at_key + 8 * i;
            const uint32_t f2 = __shfl_sync(0xffffffffu, mine, k & 31);
            const __nv_bfloat162 f = *reinterpret_cast<const __nv_bfloat162*>(&f2);
            const bool in = here >> (k & 31) & 1;
            uint4 x[PK];
#pragma unroll
            for (int j = 0; j < PK; ++j) x[j] = lds128(raw + raw_at(k, at_chunk + 4 * j));
#pragma unroll
            for (int j = 0; j < PK; ++j) {
              const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
              uint32_t y[8];
#pragma unroll
              for (int z = 0; z < 8; ++z) y[z] = widen(w[z >> 1], z & 1, f);
              if (here != 0xffffffffu) {
#pragma unroll
                for (int z = 0; z < 8; ++z) y[z] = in ? y[z] : 0u;
              }
              const int c = 2 * (at_chunk + 4 * j);
              st_shared_v4(dst + tile_at(k, c), y[0], y[1], y[2], y[3]);
              st_shared_v4(dst + tile_at(k, c + 1), y[4], y[5], y[6], y[7]);
            }
          }
        } else if (here != 0xffffffffu) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < PK; ++j)
              if (!(here >> ((at_key + 8 * i) & 31) & 1)) st_shared_v4(dst + tile_at(at_key + 8 * i, at_chunk + 4 * j), 0, 0, 0, 0);
        }
        if (!values && lane == 0) *reinterpret_cast<volatile uint32_t*>(smem + C::THERE + (((seq >> 1) & 3) * 4 + w4) * 4) = here;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(full0 + 8 * (seq % C::NS));
        seq += 2;
        if (u + 1 < n) {
          if (!FP8) ok = wait_empty(seq);
          if (!ok) break;
          issue(u + 1, pages2, FP8 ? raw : stage_of(seq));
          e = exp_at(u + 1, pages2);
          pages = pages2;
          pages2 = page_at(u + 2);
        }
      }
      copy_wait<0>();
    }
    copy_wait<0>();
    if (!ok) gave_up();
  } else if (warp == 16) {
    // ================================================================ MMAs
    uint32_t seq = 0, items = 0, units = 0;  // items, units: of tile 0 in the low half, of tile 1 in the high
    bool ok = true;
    const bool leader = elect_one();
    while (warp_uniform(ok && line.next(walk, it)))
      ok = tc_mma<HD, FP8>(base, tmem, it.rows > 128 ? 2 : 1, it.until - it.from, seq, items, units, abort_flag);
    if (!ok) gave_up();
    if (leader) umma_commit(drain);  // every MMA issued here completes before the end
    __syncwarp();
    volatile int no_abort = 0;
    mbar_wait(drain, 0, &no_abort);
  } else {
    // ================================================================ rows
    const int t = warp >> 2, quarter = warp & 3, r = 32 * quarter + lane;  // row r of tile t
    const uint32_t s_at = tmem + 128u * t + ((uint32_t)(32 * quarter) << 16);
    const uint32_t o_at = tmem + 256u + (uint32_t)(HD * t) + ((uint32_t)(32 * quarter) << 16);
    auto rows_bar = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    const float qf = fmaxf(a.scale * kLog2e, 1.2e-38f);  // (not 0: a masked score is -inf)
    uint32_t count = 0, seq = 0;
    // After a wait that ran out a warp goes on through the items without work: the barrier of the rows'
    // warps has one count for all of them.
    bool ok = true;
    auto row_wait = [&](uint32_t bar, uint32_t parity) {
      if (ok && !wait(bar, parity)) {
        ok = false;
        gave_up();
      }
      return ok;
    };
    while (line.next(walk, it)) {
      const int n = it.until - it.from, tiles = it.rows > 128 ? 2 : 1;
      const int row = 128 * t + r;
      const bool live = row < it.rows, band = 128 * t + 32 * quarter < it.rows;
      // ---- q: the band's rows into their tile, 16-byte chunks of a row by neighbouring lanes
      if (ok && t < tiles) {
        constexpr int CPR = HD / 8, RPL = 32 / CPR, LOADS = 32 / RPL;  // chunks of a row, rows of a load, loads
        const int c = lane % CPR;
        uint4 x[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int rb = 32 * quarter + RPL * i + lane / CPR, q = it.first + 128 * t + rb, tk = q / rep;
          x[i] = make_uint4(0, 0, 0, 0);
          if (128 * t + rb < it.rows)
            x[i] = *reinterpret_cast<const uint4*>(a.q + (it.row0 + tk) * a.q_stride + (int64_t)(it.g * rep + q - tk * rep) * HD + 8 * c);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          st_shared_v4(base + t * C::TILE + (uint32_t)(c >> 3) * TC_BOX + swz(32 * quarter + RPL * i + lane / CPR, c & 7),
                       x[i].x, x[i].y, x[i].z, x[i].w);
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full0 + 8 * t);
      } else {
        seq += 2 * n;
      }
      float m = -INFINITY, l = 0.f;
      for (int u = 0; ok && t < tiles && u < n; ++u, seq += 2) {
        const uint32_t blk = seq >> 1;
        if (!row_wait(s_full0 + 8 * t, count & 1u)) break;
        tc_fence_after();
        if (band) {
          const uint32_t there0 = base + C::THERE + (blk & 3) * 16;
          uint32_t s0[32];  // 32 scores
          auto mask = [&](uint32_t (&s)[32], int c) {  // keys that are not there
            const uint32_t there = __float_as_uint(ld_shared_f32(there0 + 4 * c));
            if (there != 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 32; ++i) s[i] = there >> i & 1 ? s[i] : 0xff800000u;
            }
          };
          // ---- the row's largest score
          float top = -INFINITY;
          auto largest = [&](uint32_t (&s)[32], int c) {
            mask(s, c);
            float a0 = -INFINITY, a1 = -INFINITY;
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              a0 = max3f(a0, f32(s[i]), f32(s[i + 1]));
              a1 = max3f(a1, f32(s[i + 2]), f32(s[i + 3]));
            }
            top = fmaxf(top, fmaxf(a0, a1) * qf);
          };
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            tmem_ld32(s_at + 32 * c, s0);
            tmem_ld_wait();
            largest(s0, c);
          }
          // ---- a larger reference where that passes it too far, or is the row's first
          const bool grew = top > m - (TC_ABOVE - TC_SLACK);
          if (__any_sync(0xffffffffu, grew)) {
            const float mn = grew ? top + TC_ABOVE : m, alpha = grew ? ex2_approx(m - mn) : 1.f;
            m = mn;
            l *= alpha;
            if (u > 0) {  // (the product before this unit's scores is done: they came after it)
              tmem_ld_wait();
#pragma unroll 1
              for (int c = 0; c < HD / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(o_at + 32 * c, o);
                tmem_ld_wait();
                float y[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = f32(o[i]) * alpha;
                tmem_st32(o_at + 32 * c, y);
              }
            }
          }
          // ---- P, into the places of its scores: per 32 keys 16 columns of bf16 pairs, and 16 of what they leave
          const float ref = m == -INFINITY ? 0.f : m;
          auto weigh = [&](uint32_t (&s)[32], int c) {
            mask(s, c);
            const unsigned long long qf2 = pk2(qf, qf), add2 = pk2(-ref, -ref), more2 = pk2(BF16_LO, BF16_LO);
            unsigned long long sum2 = pk2(0.f, 0.f);
#pragma unroll
            for (int i0 = 0; i0 < 32; i0 += 16) {
              uint32_t w[8], rest[8];
#pragma unroll
              for (int i = i0; i < i0 + 16; i += 2) {  // (pairs: one instruction for two scores)
                float x0, x1;
                upk2(ffma2(pk2(f32(s[i]), f32(s[i + 1])), qf2, add2), x0, x1);
                const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                sum2 = fadd2(pk2(p0, p1), sum2);
                w[(i - i0) / 2] = upper_halves(p0, p1);
                upk2(ffma2(pk2(p0, p1), more2, pk2(minus_upper(p0), minus_upper(p1))), x0, x1);
                rest[(i - i0) / 2] = pack_bf16x2(x0, x1);
              }
              tmem_st8(s_at + 32 * c + i0 / 2, w);
              tmem_st8(s_at + 32 * c + 16 + i0 / 2, rest);
            }
            float lo, hi;
            upk2(sum2, lo, hi);
            l += lo + hi;
          };
#pragma unroll 1
          for (int c = 3; c >= 0; --c) {  // (the last 32 are here still)
            if (c < 3) {
              tmem_ld32(s_at + 32 * c, s0);
              tmem_ld_wait();
            }
            weigh(s0, c);
          }
          tmem_st_wait();
        }
        ++count;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full0 + 8 * t);
      }
      // ---- the rows' results, or this CTA's part of them
      if (t < tiles) row_wait(p_empty0 + 8 * t, (count & 1u) ^ 1u);
      tc_fence_after();
      if (ok && band) {
        using Part = KaPart<HD, TC_ROWS, true>;
        float* part = scratch.part + (2 * (int64_t)blockIdx.x + (it.from == 0)) * Part::FLOATS;
        KaRow mine{};
        if (live && it.whole()) mine = finish_row(a, it.row0, it.g * rep, it.first, rep, row, m, l);
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          __syncwarp();
          tmem_ld32(o_at + 32 * c, o);
          tmem_ld_wait();
          if (!live) continue;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 x = make_float4(f32(o[i]), f32(o[i + 1]), f32(o[i + 2]), f32(o[i + 3]));
            if (it.whole())
              finish4<HD>(a, mine, 32 * c + i, x);
            else
              *reinterpret_cast<float4*>(part + Part::four(row, 8 * c + i / 4)) = x;
          }
        }
        if (live && !it.whole()) *reinterpret_cast<float2*>(part + Part::ml(row)) = make_float2(m, l);
      }
      if (!it.whole()) {
        int c0, c1;
        line.sharers(walk, it, c0, c1);
        __syncwarp();
        rows_bar();
        if (threadIdx.x == 0) {
          __threadfence();  // (the rows' writes, which the barrier ordered before)
          const int done = atomicAdd(&scratch.count[c0], 1);
          if (done == c1 - c0) {  // the last to come joins the parts, when it is through with its own
            scratch.count[c0] = 0;
            todo[todo[0].rows++ ? 2 : 1] = KaJoin{it.row0, it.g * rep, it.first, it.rows, c0, c1 - c0 + 1};
          }
          __threadfence();
        }
        __syncwarp();  // (aligned instructions follow)
      }
    }
  }
  tc_fence_before();
  __syncwarp();
  __syncthreads();
  tc_fence_after();
  if (warp == 16) tmem_dealloc(tmem, 512);
  for (int i = 0; i < todo[0].rows; ++i) {
    const KaJoin j = todo[1 + i];
    const int some = min(TC_ROWS, TC_JOIN / j.parts);  // rows whose weights fit
    for (int r0 = 0; r0 < j.rows; r0 += some) {
      KaJoin k = j;
      k.first += r0;
      k.rows = min(some, j.rows - r0);
      join_parts<HD, TC_ROWS, TC_THREADS, true>(a, k, r0, rep, scratch.part,
                                          reinterpret_cast<float2*>(smem + TC_ROWS * 8), reinterpret_cast<KaRow*>(smem),
                                          threadIdx.x, [] { __syncthreads(); });
      __syncthreads();
    }
  }
}

template <int HD, bool FP8>
cudaError_t launch_as(const KvPool& kv, const KvAttn& a, const KaScratch& s, int ctas, int* err, cudaStream_t stream) {
  using C = TcCfg<HD, FP8>;
  static_assert((size_t)2 * TC_ROWS * (HD + 4) * 4 <= KV_ATTN_TC_PART_BYTES, "scratch per CTA");
  auto kern = kv_attention_tc_kernel<HD, FP8>;
  static const cudaError_t set = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
  if (set != cudaSuccess) return set;
  kern<<<ctas, TC_THREADS, C::SMEM, stream>>>(kv, a, s, err);
  return cudaGetLastError();
}

}  // namespace

size_t kv_attention_tc_scratch(int sms) { return KV_ATTN_COUNTERS + (size_t)std::min(sms, 152) * KV_ATTN_TC_PART_BYTES; }

cudaError_t kv_attention_tc_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream) {
  sms = std::min(sms, 152);
  KaScratch s{reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + KV_ATTN_COUNTERS), static_cast<int*>(scratch)};
  if (kv.hd == 128) return kv.fp8 ? launch_as<128, true>(kv, a, s, sms, err, stream) : launch_as<128, false>(kv, a, s, sms, err, stream);
  return kv.fp8 ? launch_as<64, true>(kv, a, s, sms, err, stream) : launch_as<64, false>(kv, a, s, sms, err, stream);
}

}  // namespace dcl
