// Attention of many new positions of every sequence over its paged keys and values, on the tcgen05
// tensor cores: the rows of an item (up to 256: new positions x the query heads of one kv head)
// fill one or two tiles of 128, and one pass over the keys serves them all.
//
// Per unit of 128 keys: S = Q K^T into TMEM, P = exp2(S scaled + e - m) in fp16 through shared memory,
// O += P V in TMEM.  P, m, l and the exponents e of the values are those of kv_attention.cu; a
// thread owns a row, so its statistics need no exchange.
//
// FP8 pages.  Four warps copy codes into shared memory (16-byte asynchronous copies, one unit
// ahead) and widen them into the fp16 operand tiles: keys times 2^(e_j - e_max), e_max the unit's
// largest exponent (a key more than 2^15 below the unit's largest loses low bits that its scores,
// so much smaller, do not show), values as they are (e_j enters P).  bf16 pages: keys are copied
// straight into their tile and multiplied in bf16; a value is scaled by the power of two of its
// largest component into fp16, in place (exact but for components below 2^-14 of that one).
// V's tile is [key][hd], the transposed ("MN-major") form of the B operand, as it comes.
//
// The reference m moves only when a score passes it by more than 8: a pass over a unit takes m as it
// is, and is repeated with a larger one if a row's maximum shows that (the scores are still in
// TMEM); O is scaled then.  A unit's first pass is nearly always its last.
//
// What bounds it: shared memory, per unit of two tiles 256 KB of operand reads, 64 KB of P, and for
// FP8 96 KB of widening (about 3500 cycles), against 2200 of tensor time.
//
// Roles (512 threads): warps 0-3 copy and widen; warp 4 allocates TMEM and issues the MMAs; warps
// 8-11 and 12-15 have the rows of the two tiles.  Every wait is bounded (DERR_WAIT_TIMEOUT).
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kv_cache.cuh"
#include "kv_share.cuh"
#include "tc_ptx.cuh"

namespace dcl {
namespace {

constexpr int TC_ROWS = 256;      // rows of an item
constexpr int TC_THREADS = 512;
constexpr int TC_BOX = 128 * 128; // 128 rows of 128 bytes, swizzled
constexpr int TC_JOIN = 64;       // rows joined at a time

template <int HD, bool FP8>
struct TcCfg {
  static constexpr int KB = HD / 64;                  // boxes along hd
  static constexpr int TILE = KB * TC_BOX;            // 128 rows of q, keys or values, 16 bits each
  static constexpr int NS = FP8 ? 2 : 3;              // operand tiles of keys and values, in turn
  static constexpr int P = 2 * TILE;                  // after q: P of two tiles [128][128 keys]
  static constexpr int KV = P + 4 * TC_BOX;
  static constexpr int RAW = KV + NS * TILE;          // FP8: codes of a unit's keys, then of its values
  static constexpr int EXP = RAW + (FP8 ? 2 * 128 * HD : 0);  // [2 units][e, 2^-e][128] floats
  static constexpr int SCALE = EXP + 2 * 2 * 128 * 4; // [2 units] 2^e_max
  static constexpr int BAR = SCALE + 8;
  static constexpr int NBARS = 2 * NS + 4 * 2 + 1;
  static constexpr int HOLDER = BAR + 8 * NBARS;      // TMEM address, abort flag
  static constexpr int WALK = HOLDER + 8;
  static constexpr int TODO = WALK + (int)sizeof(KaWalk);
  static constexpr size_t SMEM = TODO + 3 * sizeof(KaJoin);
  static_assert(SMEM <= 232448, "shared memory per CTA");
  static_assert(TC_JOIN * 152 * 8 + TC_JOIN * 8 <= KV, "a join's weights take the place of q and P");
};

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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t widen(uint32_t w, int half) {  // two E4M3 codes to two fp16
  uint32_t r;
  if (half)
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  else
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t times(uint32_t x, __half2 f) {
  __half2 y = __hmul2(*reinterpret_cast<__half2*>(&x), f);
  return *reinterpret_cast<uint32_t*>(&y);
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
  const KaLine<TC_ROWS> line(kv, a);

  if (warp == 0) line.begin(&shared_walk, err);
  if (warp == 4) {
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

  if (warp < 4) {
    // ================================================================ copies, widening
    // A unit's keys: lane l knows of keys 4 l .. 4 l + 3 (their page and exponents); this warp copies
    // groups 2 warp and 2 warp + 1 of 16 keys.  Chunks of 16 bytes: K's and V's alike.
    constexpr int CH = FP8 ? HD / 16 : HD / 8;       // chunks of a vector
    constexpr int PER = 16 * CH / 32;                // of a group, per lane
    const int shift = kv.page_shift, P = kv.page_len();
    uint32_t seq = 0;  // operand tiles so far (keys and values in turn): stage seq % NS
    bool ok = true;
    // (lane -> key and chunk of a group: eight lanes store into two rows of one box)
    auto key_of = [&](int i) { return (lane >> 2) + 8 * (i / (CH / 4)); };
    auto chunk_of = [&](int i) { return (lane & 3) + 4 * (i % (CH / 4)); };
    while (ok && line.next(walk, it)) {
      const int stop = min(it.len, it.until * KA_UNIT), n = it.until - it.from, key0 = it.from * KA_UNIT;
      const int* table = a.table + (int64_t)it.b * a.max_pages;
      auto page_at = [&](int unit) {  // of this lane's keys; negative: no key of them is to be read
        const int key = key0 + unit * KA_UNIT + 4 * lane;
        if (unit >= n || key >= stop) return -1;
        const int page = table[key >> shift];
        if (page < 0 || page >= kv.pages) {
          report_error(err, DERR_KV_RANGE);
          return -1;
        }
        return page;
      };
      auto vec_of = [&](int page, int key) { return kv.vector_of((page << shift) + (key & (P - 1)), it.g); };
      // copies of this warp's groups of a unit into `dst` (K or V: what follows the pool's pointer)
      auto issue = [&](int unit, int pages, const void* pool, uint32_t dst) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int gr = 2 * warp + h, page = __shfl_sync(0xffffffffu, pages, 4 * gr);
          if (page < 0) continue;
          const uint8_t* src = static_cast<const uint8_t*>(pool) + vec_of(page, key0 + unit * KA_UNIT + 16 * gr) * (CH * 16);
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int k = key_of(i), c = chunk_of(i);
            const uint32_t to = FP8 ? dst + (uint32_t)((16 * gr + k) * CH + c) * 16
                                    : dst + (uint32_t)(c >> 3) * TC_BOX + swz(16 * gr + k, c & 7);
            copy16(to, src + (k * CH + c) * 16);
          }
        }
        copy_commit();
      };
      auto exps_at = [&](int unit, int page, const int8_t* exps) -> uint32_t {
        if (!FP8 || page < 0) return 0;
        return *reinterpret_cast<const uint32_t*>(exps + vec_of(page, key0 + unit * KA_UNIT + 4 * lane));
      };
      auto stage_of = [&](uint32_t s) { return base + C::KV + (s % C::NS) * C::TILE; };
      auto wait_empty = [&](uint32_t s) { return wait(empty0 + 8 * (s % C::NS), ((s / C::NS) & 1u) ^ 1u); };
      auto ready = [&](uint32_t s) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(full0 + 8 * (s % C::NS));
      };
      const uint32_t raw = base + C::RAW;
      int pages = page_at(0), pages2 = page_at(1);
      uint32_t ek = exps_at(0, pages, kv.k_exp), ev = exps_at(0, pages, kv.v_exp);
      if (FP8) {
        issue(0, pages, kv.k, raw);
        issue(0, pages, kv.v, raw + 128 * HD);
      } else {
        ok = wait_empty(seq);
        if (ok) issue(0, pages, kv.k, stage_of(seq));
        if (ok) ok = wait_empty(seq + 1);
        if (ok) issue(0, pages, kv.v, stage_of(seq + 1));
      }
      for (int u = 0; ok && u < n; ++u) {
        const uint32_t blk = seq >> 1;
        const int live = min(KA_UNIT, stop - key0 - u * KA_UNIT);  // keys of the unit
        // (a key is there if it lies before `live` and its page is the cache's)
        auto there = [&](int key) { return __shfl_sync(0xffffffffu, pages, key >> 2) >= 0 && key < live; };
        const int next_page = pages2;
        uint32_t next_ek = 0, next_ev = 0;
        // ---- keys
        copy_wait<1>();
        __syncwarp();
        if (FP8) {
          int top = -128;  // the largest exponent of the keys there
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (pages >= 0 && 4 * lane + i < live) top = max(top, (int)(int8_t)(ek >> (8 * i)));
          top = __reduce_max_sync(0xffffffffu, top);
          if (warp == 0) {
            float e[4], inv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool in = pages >= 0 && 4 * lane + i < live;
              const int y = max(-126, (int)(int8_t)(ev >> (8 * i)));
              e[i] = in ? (float)y : -INFINITY;
              inv[i] = in ? kv_pow2(-y) : 0.f;
            }
            float4* to = reinterpret_cast<float4*>(smem + C::EXP + (blk & 1) * 1024) + lane;
            to[0] = make_float4(e[0], e[1], e[2], e[3]);
            to[32] = make_float4(inv[0], inv[1], inv[2], inv[3]);
            if (lane == 0) *reinterpret_cast<float*>(smem + C::SCALE + 4 * (blk & 1)) = kv_pow2(top);
          }
          ok = wait_empty(seq);
          if (!ok) break;
          const uint32_t dst = stage_of(seq);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 x[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) x[i] = lds128(raw + (uint32_t)((32 * warp + 16 * h + key_of(i)) * CH + chunk_of(i)) * 16);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int k = 32 * warp + 16 * h + key_of(i), c = chunk_of(i);
              const int e = (int)(int8_t)(__shfl_sync(0xffffffffu, ek, k >> 2) >> (8 * (k & 3)));
              const bool in = there(k);
              const __half2 f = __float2half2_rn(in ? kv_pow2(e - top) : 0.f);
              const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
              uint32_t y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = in ? times(widen(w[j >> 1], j & 1), f) : 0u;
              const uint32_t row = dst + (uint32_t)(c >> 2) * TC_BOX;
              st_shared_v4(row + swz(k, 2 * (c & 3)), y[0], y[1], y[2], y[3]);
              st_shared_v4(row + swz(k, 2 * (c & 3) + 1), y[4], y[5], y[6], y[7]);
            }
          }
        } else {
          const uint32_t dst = stage_of(seq);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int k = 32 * warp + 16 * h + key_of(i), c = chunk_of(i);
              if (!there(k)) st_shared_v4(dst + (uint32_t)(c >> 3) * TC_BOX + swz(k, c & 7), 0, 0, 0, 0);
            }
        }
        ready(seq);
        if (FP8) {
          next_ek = exps_at(u + 1, next_page, kv.k_exp);
          next_ev = exps_at(u + 1, next_page, kv.v_exp);
          issue(u + 1, u + 1 < n ? next_page : -1, kv.k, raw);
        } else {
          if (u + 1 < n) ok = wait_empty(seq + 2);
          if (!ok) break;
          issue(u + 1, u + 1 < n ? next_page : -1, kv.k, stage_of(seq + 2));
        }
        ++seq;
        // ---- values
        copy_wait<1>();
        __syncwarp();
        if (FP8) {
          ok = wait_empty(seq);
          if (!ok) break;
          const uint32_t dst = stage_of(seq);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint4 x[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i)
              x[i] = lds128(raw + 128 * HD + (uint32_t)((32 * warp + 16 * h + key_of(i)) * CH + chunk_of(i)) * 16);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int k = 32 * warp + 16 * h + key_of(i), c = chunk_of(i);
              const bool in = there(k);
              const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
              uint32_t y[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = in ? widen(w[j >> 1], j & 1) : 0u;
              const uint32_t row = dst + (uint32_t)(c >> 2) * TC_BOX;
              st_shared_v4(row + swz(k, 2 * (c & 3)), y[0], y[1], y[2], y[3]);
              st_shared_v4(row + swz(k, 2 * (c & 3) + 1), y[4], y[5], y[6], y[7]);
            }
          }
        } else {
          const uint32_t dst = stage_of(seq);
          constexpr int PK = CH / 4;  // this lane's chunks of a key
#pragma unroll
          for (int h = 0; h < 4; ++h) {  // eight keys at a time: key (lane >> 2) + 8 h of the warp's 32
            const int k = 32 * warp + 8 * h + (lane >> 2);
            const bool in = there(k);
            uint4 x[PK];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < PK; ++i) {
              const int c = (lane & 3) + 4 * i;
              x[i] = in ? lds128(dst + (uint32_t)(c >> 3) * TC_BOX + swz(k, c & 7)) : make_uint4(0, 0, 0, 0);
              const uint32_t* w = &x[i].x;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
                top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
              }
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = top ? max(-100, min(126, (int)(top >> 7) - 127)) : 0;
            const float f = kv_pow2(-e);
#pragma unroll
            for (int i = 0; i < PK; ++i) {
              const int c = (lane & 3) + 4 * i;
              uint32_t* w = &x[i].x;
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = pack_f16x2(bf16_lo(w[j]) * f, bf16_hi(w[j]) * f);
              st_shared_v4(dst + (uint32_t)(c >> 3) * TC_BOX + swz(k, c & 7), w[0], w[1], w[2], w[3]);
            }
            if ((lane & 3) == 0) {
              float* to = reinterpret_cast<float*>(smem + C::EXP + (blk & 1) * 1024) + k;
              to[0] = in ? (float)e : -INFINITY;
              to[128] = in ? f : 0.f;
            }
          }
        }
        ready(seq);
        if (FP8) {
          issue(u + 1, u + 1 < n ? next_page : -1, kv.v, raw + 128 * HD);
        } else {
          if (u + 1 < n) ok = wait_empty(seq + 2);
          if (!ok) break;
          issue(u + 1, u + 1 < n ? next_page : -1, kv.v, stage_of(seq + 2));
        }
        ++seq;
        pages = next_page;
        ek = next_ek;
        ev = next_ev;
        pages2 = page_at(u + 2);
      }
      copy_wait<0>();
    }
    copy_wait<0>();
    if (!ok) gave_up();
  } else if (warp == 4) {
    // ================================================================ MMAs
    constexpr uint32_t idesc_s = FP8 ? make_idesc_f16(128, 128) : make_idesc(128, 128);
    constexpr uint32_t idesc_o = make_idesc_f16(128, HD) | IDESC_B_MN;
    const bool leader = elect_one();
    uint32_t seq = 0, items[2] = {0, 0}, count[2] = {0, 0};  // items and units of each tile
    bool ok = true;
    auto issue_s = [&](int t, uint32_t tile) {
      const uint64_t dq = sw128_desc(base + t * C::TILE), dk = sw128_desc(tile);
      if (leader) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          umma_bf16(tmem + 128u * t, dq + (k >> 2) * (TC_BOX >> 4) + 2 * (k & 3), dk + (k >> 2) * (TC_BOX >> 4) + 2 * (k & 3),
                    idesc_s, k > 0 ? 1u : 0u);
        umma_commit(s_full0 + 8 * t);
      }
      __syncwarp();
    };
    auto full = [&](uint32_t s) { return wait(full0 + 8 * (s % C::NS), (s / C::NS) & 1u); };
    auto tile_at = [&](uint32_t s) { return base + C::KV + (s % C::NS) * C::TILE; };
    while (ok && line.next(walk, it)) {
      const int n = it.until - it.from, tiles = it.rows > 128 ? 2 : 1;
      ok = full(seq);
      for (int t = 0; ok && t < tiles; ++t) ok = wait(q_full0 + 8 * t, items[t]++ & 1u);
      if (!ok) break;
      tc_fence_after();
      for (int t = 0; t < tiles; ++t) issue_s(t, tile_at(seq));
      if (leader) umma_commit(empty0 + 8 * (seq % C::NS));
      __syncwarp();
      for (int u = 0; ok && u < n; ++u, seq += 2) {
        ok = full(seq + 1) && (u + 1 == n || full(seq + 2));
        for (int t = 0; ok && t < tiles; ++t) {
          ok = wait(p_full0 + 8 * t, count[t] & 1u);
          if (!ok) break;
          ++count[t];
          tc_fence_after();
          const uint64_t dp = sw128_desc(base + C::P + t * 2 * TC_BOX), dv = sw128_desc_mn(tile_at(seq + 1));
          if (leader) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              umma_bf16(tmem + 256u + (uint32_t)(HD * t), dp + (k >> 2) * (TC_BOX >> 4) + 2 * (k & 3), dv + k * (2048 >> 4),
                        idesc_o, (u > 0 || k > 0) ? 1u : 0u);
            umma_commit(p_empty0 + 8 * t);
            if (t + 1 == tiles) umma_commit(empty0 + 8 * ((seq + 1) % C::NS));
          }
          __syncwarp();
          if (u + 1 < n) {
            issue_s(t, tile_at(seq + 2));
            if (leader && t + 1 == tiles) umma_commit(empty0 + 8 * ((seq + 2) % C::NS));
            __syncwarp();
          }
        }
      }
    }
    if (!ok) gave_up();
    if (leader) umma_commit(drain);  // every MMA issued here completes before the end
    __syncwarp();
    volatile int no_abort = 0;
    mbar_wait(drain, 0, &no_abort);
  } else if (warp >= 8) {
    // ================================================================ rows
    const int t = (warp - 8) >> 2, quarter = warp & 3, r = 32 * quarter + lane;  // row r of tile t
    const uint32_t s_at = tmem + 128u * t + ((uint32_t)(32 * quarter) << 16);
    const uint32_t o_at = tmem + 256u + (uint32_t)(HD * t) + ((uint32_t)(32 * quarter) << 16);
    const uint32_t p_row = base + C::P + t * 2 * TC_BOX;
    auto rows_bar = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
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
      const int rr = it.first + row, tok = rr / rep, h = it.g * rep + rr - tok * rep;
      float qa = a.scale * kLog2e;
      // ---- q: this thread's row into its tile
      if (ok && t < tiles) {
        const uint4* src = reinterpret_cast<const uint4*>(a.q + (it.row0 + tok) * a.q_stride + (int64_t)h * HD);
        uint4 x[HD / 8];
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) x[c] = live ? src[c] : make_uint4(0, 0, 0, 0);
        if (FP8) {
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < HD / 8; ++c) {
            const uint32_t* w = &x[c].x;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(bf16_lo(w[j])), fabsf(bf16_hi(w[j]))));
          }
          const int e = max(-120, min(120, (int)(__float_as_uint(top) >> 23) - 127));
          const float down = kv_pow2(-e);
          qa *= kv_pow2(e);
#pragma unroll
          for (int c = 0; c < HD / 8; ++c) {
            uint32_t* w = &x[c].x;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_f16x2(bf16_lo(w[j]) * down, bf16_hi(w[j]) * down);
          }
        }
#pragma unroll
        for (int c = 0; c < HD / 8; ++c)
          st_shared_v4(base + t * C::TILE + (uint32_t)(c >> 3) * TC_BOX + swz(r, c & 7), x[c].x, x[c].y, x[c].z, x[c].w);
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
        // (bf16: the values' exponents come with their tile)
        if (!FP8 && !row_wait(full0 + 8 * ((seq + 1) % C::NS), ((seq + 1) / C::NS) & 1u)) break;
        if (u > 0 && !row_wait(p_empty0 + 8 * t, (count & 1u) ^ 1u)) break;  // P and O of the unit before are done with
        tc_fence_after();
        if (band) {
          const uint32_t exps = base + C::EXP + (blk & 1) * 1024;
          const float qf = FP8 ? qa * *reinterpret_cast<volatile float*>(smem + C::SCALE + 4 * (blk & 1)) : qa;
          float sum;
          for (;;) {
            const float ref = m == -INFINITY ? 0.f : m;
            float top = -INFINITY;
            sum = 0.f;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              uint32_t s[32];
              tmem_ld32(s_at + 32 * c, s);
              tmem_ld_wait();
              uint32_t w[16];
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 e = ld_shared_v4(exps + 4 * (32 * c + i)), f = ld_shared_v4(exps + 512 + 4 * (32 * c + i));
                const float x0 = fmaf(f32(s[i]), qf, e.x) - ref, x1 = fmaf(f32(s[i + 1]), qf, e.y) - ref;
                const float x2 = fmaf(f32(s[i + 2]), qf, e.z) - ref, x3 = fmaf(f32(s[i + 3]), qf, e.w) - ref;
                top = fmaxf(top, fmaxf(fmaxf(x0, x1), fmaxf(x2, x3)));
                const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
                sum = fmaf(p0, f.x, sum);
                sum = fmaf(p1, f.y, sum);
                sum = fmaf(p2, f.z, sum);
                sum = fmaf(p3, f.w, sum);
                w[i / 2] = pack_f16x2(p0, p1);
                w[i / 2 + 1] = pack_f16x2(p2, p3);
              }
#pragma unroll
              for (int k = 0; k < 4; ++k)
                st_shared_v4(p_row + (uint32_t)(c >> 1) * TC_BOX + swz(r, (c & 1) * 4 + k), w[4 * k], w[4 * k + 1], w[4 * k + 2],
                             w[4 * k + 3]);
            }
            // a larger reference where a row's maximum passes it by more than 8, or is its first
            const bool grew = m == -INFINITY ? top > -INFINITY : top > 8.f;
            if (!__any_sync(0xffffffffu, grew)) break;
            const float mn = grew ? ref + top : m, alpha = grew ? (m == -INFINITY ? 0.f : ex2_approx(m - mn)) : 1.f;
            m = mn;
            l *= alpha;
            if (u > 0) {
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
              tmem_st_wait();
            }
          }
          l += sum;
        }
        ++count;
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full0 + 8 * t);
      }
      // ---- the rows' results, or this CTA's part of them
      if (t < tiles) row_wait(p_empty0 + 8 * t, (count & 1u) ^ 1u);
      tc_fence_after();
      if (ok && band) {
        float* part = scratch.part + ((2 * (int64_t)blockIdx.x + (it.from == 0)) * TC_ROWS + row) * (HD + 4);
        const int64_t at = (int64_t)(it.row0 + tok) * a.H + h;
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(o_at + 32 * c, o);
          tmem_ld_wait();
          if (!live) continue;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 x = make_float4(f32(o[i]), f32(o[i + 1]), f32(o[i + 2]), f32(o[i + 3]));
            if (it.whole())
              finish4(a, at, HD, 32 * c + i, make_float2(m, l), x);
            else
              *reinterpret_cast<float4*>(part + 32 * c + i) = x;
          }
        }
        if (live && !it.whole()) *reinterpret_cast<float2*>(part + HD) = make_float2(m, l);
      }
      if (!it.whole()) {
        int c0, c1;
        line.sharers(walk, it, c0, c1);
        rows_bar();
        if (threadIdx.x == 256) {
          __threadfence();  // (the rows' writes, which the barrier ordered before)
          const int done = atomicAdd(&scratch.count[c0], 1);
          if (done == c1 - c0) {  // the last to come joins the parts, when it is through with its own
            scratch.count[c0] = 0;
            todo[todo[0].rows++ ? 2 : 1] = KaJoin{it.row0, it.g * rep, it.first, it.rows, c0, c1 - c0 + 1};
          }
          __threadfence();
        }
      }
    }
    rows_bar();
    for (int i = 0; i < todo[0].rows; ++i) {
      const KaJoin j = todo[1 + i];
      for (int r0 = 0; r0 < j.rows; r0 += TC_JOIN) {
        KaJoin k = j;
        k.first += r0;
        k.rows = min(TC_JOIN, j.rows - r0);
        join_parts<HD, TC_ROWS, 256>(a, k, rep, scratch.part + (int64_t)r0 * (HD + 4), reinterpret_cast<float2*>(smem + TC_JOIN * 8),
                                     reinterpret_cast<float2*>(smem), (int)threadIdx.x - 256, rows_bar);
        rows_bar();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, 512);
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

size_t kv_attention_tc_scratch(int sms) { return (size_t)std::min(sms, 152) * (KV_ATTN_TC_PART_BYTES + sizeof(int)); }

cudaError_t kv_attention_tc_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream) {
  sms = std::min(sms, 152);
  KaScratch s{static_cast<float*>(scratch),
              reinterpret_cast<int*>(static_cast<uint8_t*>(scratch) + (size_t)sms * KV_ATTN_TC_PART_BYTES)};
  if (kv.hd == 128) return kv.fp8 ? launch_as<128, true>(kv, a, s, sms, err, stream) : launch_as<128, false>(kv, a, s, sms, err, stream);
  return kv.fp8 ? launch_as<64, true>(kv, a, s, sms, err, stream) : launch_as<64, false>(kv, a, s, sms, err, stream);
}

}  // namespace dcl
