// Attention of a few new positions of every sequence over its paged keys and values:
// out = softmax(scale q k^T) v over the sequence's cached positions.
//
// The rows of one kv head (new positions x the query heads that share it) form row tiles of 8, 16 or
// 32, the most that one pass over the keys serves.  A warp takes 16 or 32 keys at a time: S = q k^T and
// O += P v as m16n8k16 products with the rows on the M side, its own running maximum m, sum l and
// O in registers, its own ring of key / value tiles in shared memory (16-byte asynchronous copies;
// no barrier in the loop).  The tensor work is far below its limit as long as the keys arrive from
// memory, which is what bounds a call of few rows.  With FP8 pages, 28 / 4 heads of 128, one row a
// sequence: 2 sequences of 131071 positions (271 MB) in 57.2 us, 4.7 TB/s over the whole launch, of
// which beginning takes 2, joining 38 parts an item 7 to 9; 64 ragged sequences to 4096 (140 MB) in
// 37 us, 3.8 TB/s: beginning 3.4, the keys 24 on average and 31 in the last CTA, joins 2; one of 512 positions,
// 32 heads, 8.9 us, all latency (32 CTAs have an item: 1.9 to begin, 5.9 for its keys).  bf16 pages, 8
// sequences of 1536, 32 heads, 32 rows each (201 MB): 50 us, 4.1 TB/s, the products' issue (P in two parts) as near its limit as memory.
//
// Work is shared out in units of 128 keys of one (sequence, kv head, row tile), all of a launch in
// one line, every CTA an equal part of it: a long sequence is spread over many CTAs, many short
// ones share one, and no CTA waits for another's longer sequence.  A CTA's warps join their
// (m, l, O) in shared memory; where a line's cut falls inside an item its CTAs leave them in
// scratch, and the one that comes last joins them in the order of the keys, so that a result does
// not depend on which that was.
//
// FP8 pages.  Codes are widened to fp16, which holds them exactly, q is scaled per row by a power of
// two into fp16 (its 8 bits fit; what falls below fp16's range is 2^-24 of the row's largest).  A
// key's exponent scales its score.  A value's exponent e_j goes into the exponent of its
// probability: P_j = exp2(s_j + e_j - m) with m near the running maximum of s_j + e_j, so that P is
// bounded whatever the values' sizes; l = sum exp2(s_j - m), an exponential of its own, as P_j 2^-e_j
// loses weights where exponents lie 100 apart.  A vector of zeros is stored with exponent 0 whatever the
// others' sizes and has no term to bound: where one would move m it is given an exponent far down.
//
// P is given in two parts, fp16 with FP8 pages (2^-21 of itself; 2^-32 of the largest term where that is
// more) and bf16 with bf16 pages (2^-16; the instruction wants both operands of one type).  One part
// would leave up to 2^-11 or 2^-8 of a result, beside 2^-8 of the output's own rounding.  Up to 8 rows
// fill half of a product's 16, and the other half takes the second part, so that it costs no product;
// for more it is a product of its own.
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kv_cache.cuh"
#include "kv_share.cuh"

namespace dcl {
namespace {

constexpr int KA_START = 3;   // units of keys that beginning an item takes
constexpr int KA_CTAS = 2;    // CTAs of an SM: one loads while the other begins or ends an item
constexpr int KA_MOST = 304;  // most CTAs of a launch
static_assert(KA_MOST * sizeof(int) <= KV_ATTN_COUNTERS, "a counter per CTA");

// RS: rows of an item that a lane has (quad + 8 i), 8 rows of the item each.
template <int HD, bool FP8, int RS>
struct KaCfg {
  static constexpr int ES = FP8 ? 1 : 2;
  static constexpr int MT = RS == 1 ? 1 : RS / 2;   // tiles of 16 rows (or of 8 and the second parts of their weights)
  static constexpr int WARPS = MT == 1 ? 6 : 4;     // (with KA_CTAS of them on an SM as many as the registers allow)
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int KT = FP8 && MT == 1 ? 32 : 16;  // keys that a warp takes at a time
  static constexpr int NK = KT / 8;                 // column tiles of S
  static constexpr int ROWS = 8 * RS;               // rows of an item
  static constexpr int ROWB = HD * ES;              // bytes of a key
  static constexpr int TILE = KT * ROWB;            // the keys (or values) of a step
  static constexpr int STAGE = 2 * TILE + (FP8 ? 2 * KT : 0);
  static constexpr int LIMIT = 220 * 1024 / KA_CTAS / WARPS / STAGE;
  static constexpr int STAGES = LIMIT > 12 ? 12 : LIMIT;
  static constexpr int RING = STAGES * STAGE;       // one warp's
  // a warp's O takes the ring's place: [ROWS][O_PITCH] floats, a lane's runs of components 4 apart
  // from the next lane's, so that 16-byte stores meet all the banks
  static constexpr int O_PITCH = FP8 ? HD + 36 : HD + HD / 2 + 4;
  static constexpr int RING_B = RING > ROWS * O_PITCH * 4 ? RING : ROWS * O_PITCH * 4;
  static constexpr int ML = WARPS * RING_B;         // {m, l} [warp][ROWS]
  static constexpr int WT = ML + WARPS * ROWS * 8;  // weights of the warps' parts [ROWS][8], then {m, l} of the rows
  static constexpr int QF = WT + ROWS * (8 * 4 + 8);  // q fragments [MT][HD / 16][lane] of 16 bytes
  static constexpr int SC = QF + MT * (HD / 16) * 32 * 16;  // what the keys' exponents give [warp][2][KT] floats
  static constexpr int HEAD = SC + (FP8 ? WARPS * 2 * KT * 4 : 0);  // the walk's variables
  static constexpr int TODO = HEAD + 48;            // joins left to this CTA: their number, and two at most
  static constexpr size_t SMEM = TODO + 3 * 24;
  static_assert(ML >= ROWS * KA_MOST * 8, "the weights of an item's parts take the rings' place");
  static_assert(STAGES >= 2, "a step in flight");
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts32(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <bool FP8>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (FP8)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk c of row r of a tile.  The order of a row's chunks depends on the row,
// so that the eight lanes of a 16-byte load (two keys x four places, or four keys x two) meet
// all the banks.
template <int ROWB>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  return (uint32_t)(r * ROWB + ((c ^ (ROWB == 64 ? (r >> 1) & 3 : r & 7)) << 4));
}
// The order in which hd enters the two products is free as long as q and k, and v and the output,
// agree: a lane's operands are taken from whole 16-byte chunks.  k_chunk: the i-th chunk of 8
// components of q that lane place t covers.  v_comp: the component of column n of product tile j.
template <int HD, bool FP8>
__device__ __forceinline__ int k_chunk(int t, int i) {
  if (FP8) return t * (HD / 32) + i;
  return 2 * t + (i & 1) + 8 * (i >> 1);
}
template <int HD, bool FP8>
__device__ __forceinline__ int v_comp(int n, int j) {
  if (FP8) return n * (HD / 8) + j;
  return (j >> 3) * 64 + 8 * n + (j & 7);
}

// Values of a tile that are no numbers: whether this lane's share of its chunks holds any, the value of
// one component, and zeros in their place.
template <bool FP8>
__device__ __forceinline__ uint32_t nonfinite_bits(uint32_t w) {  // all ones in each such element
  if (FP8) return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu);
  return __vcmpeq2(w & 0x7f807f80u, 0x7f807f80u);
}
template <bool FP8>
__device__ __noinline__ bool has_nonfinite(uint32_t tile, int bytes, int lane) {
  uint32_t any = 0;
  for (int c = 16 * lane; c < bytes; c += 512) {
    const uint4 w = lds128(tile + c);
    any |= nonfinite_bits<FP8>(w.x) | nonfinite_bits<FP8>(w.y) | nonfinite_bits<FP8>(w.z) | nonfinite_bits<FP8>(w.w);
  }
  return any != 0;
}
template <bool FP8>
__device__ __noinline__ void clear_nonfinite(uint32_t tile, int bytes, int lane) {
  for (int c = 16 * lane; c < bytes; c += 512) {
    const uint4 w = lds128(tile + c);
    sts128(tile + c, make_uint4(w.x & ~nonfinite_bits<FP8>(w.x), w.y & ~nonfinite_bits<FP8>(w.y),
                                w.z & ~nonfinite_bits<FP8>(w.z), w.w & ~nonfinite_bits<FP8>(w.w)));
  }
}
// Keys of a step whose values are nothing but zeros (stored with exponent 0) get the exponent KA_ZERO in ev,
// the step's values' exponents; whether there are any.
constexpr float KA_ZERO = -90.f;  // (l holds their weights up to 2^97 times those that m is taken from)
template <int ROWB, int KT>
__device__ __noinline__ bool lower_zeros(uint32_t tile, uint32_t ev, int lane) {
  bool zero = lane < KT && lds_f32(ev + 4 * (lane & (KT - 1))) == 0.f;
  if (zero) {
    uint32_t any = 0;
    for (int c = 0; c < ROWB / 16; ++c) {
      const uint4 w = lds128(tile + chunk_at<ROWB>(lane, c));
      any |= w.x | w.y | w.z | w.w;
    }
    zero = (any & 0x7f7f7f7fu) == 0;
    if (zero) sts32(ev + 4 * lane, KA_ZERO);
  }
  return __any_sync(0xffffffffu, zero);
}
template <int ROWB, bool FP8>
__device__ __forceinline__ float value_at(uint32_t tile, int row, int comp) {
  const int byte = comp * (FP8 ? 1 : 2);
  const uint32_t two = lds_u16(tile + chunk_at<ROWB>(row, byte >> 4) + (byte & 14));
  if (!FP8) return __uint_as_float(two << 16);
  const uint32_t code = byte & 1 ? two >> 8 : two & 0xffu;
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}

// Where component c of a row of O stands in a warp's part of shared memory.
template <int HD, bool FP8>
__device__ __forceinline__ int o_place(int c) {
  if (FP8) return c + 4 * (c / (HD / 8));
  return (c >> 6) * 96 + ((c >> 3) & 7) * 12 + (c & 7);
}
template <int HD, bool FP8, int RS>
__global__ void __launch_bounds__(KaCfg<HD, FP8, RS>::THREADS, KA_CTAS) kv_attention_kernel(KvPool kv, KvAttn a, KaScratch scratch, int* err) {
  using C = KaCfg<HD, FP8, RS>;
  constexpr int MT = C::MT;
  constexpr bool OWN_LO = RS > 1;  // the weights' second parts are products of their own
  constexpr float ABOVE = FP8 ? -7.f : 32.f, SLACK = 8.f;  // the reference above the largest score, and how far that may be passed
  constexpr int KS = HD / 16;  // k steps of S, and pairs of column tiles of O
  constexpr int NT = HD / 8;   // column tiles of O
  constexpr int KT = C::KT, NK = C::NK;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, place = lane & 3;
  const int rep = a.H / kv.G, P = kv.page_len();
  const uint32_t ring = smem_addr(smem) + warp * C::RING_B;
  float2* ml = reinterpret_cast<float2*>(smem + C::ML);

  const KaLine<C::ROWS, KA_START> line(kv, a);

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

    // ---- this lane's rows: quad + 8 i of the tile; asked for before the keys, which would be in the way
    int lim[RS];  // keys each sees
    float qa[RS];  // scale * log2(e) * the power of two that q was divided by
    uint4 raw[RS][HD / 32];
#pragma unroll
    for (int i = 0; i < RS; ++i) {
      const int r = 8 * i + quad, rr = it.first + r;
      const bool live = r < it.rows;
      const int tok = rr / rep, h = it.g * rep + rr - tok * rep;
      lim[i] = !live ? 0 : a.causal ? min(it.len, it.len - it.nq + tok + 1) : it.len;
      const __nv_bfloat16* src = a.q + (it.row0 + tok) * a.q_stride + (int64_t)h * HD;
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        raw[i][c] = make_uint4(0, 0, 0, 0);
        if (live) raw[i][c] = *reinterpret_cast<const uint4*>(src + 8 * k_chunk<HD, FP8>(place, c));
      }
    }

    // ---- this warp's steps: keys key0 + KT warp on, then every WARPS-th
    const int stop = min(key1, lim_max);
    const int* table = a.table + (int64_t)it.b * a.max_pages;
    int next = key0 + KT * warp;  // first key of the next step to copy
    uint32_t bad = 0;             // two bits a stage: 16 keys whose page is not the cache's
    int slot = 0;
    int page[KT / 16];
    auto look_up = [&]() {
#pragma unroll
      for (int h = 0; h < KT / 16; ++h) page[h] = next + 16 * h < stop ? table[(next + 16 * h) >> kv.page_shift] : 0;
    };
    look_up();
    auto issue = [&]() {
      if (next < stop) {
        bad &= ~(3u << (2 * slot));
#pragma unroll
        for (int h = 0; h < KT / 16; ++h) {
          const int key = next + 16 * h;
          if (key >= stop) break;
          if (page[h] >= 0 && page[h] < kv.pages) {
            const int64_t vec = kv.vector_of((page[h] << kv.page_shift) + (key & (P - 1)), it.g);
            const uint8_t* k = static_cast<const uint8_t*>(kv.k) + vec * C::ROWB + 16 * lane;
            const uint8_t* v = static_cast<const uint8_t*>(kv.v) + vec * C::ROWB + 16 * lane;
            const uint32_t dst = ring + slot * C::STAGE;
#pragma unroll
            for (int i = 0; i < C::ROWB / 32; ++i) {
              const int c = i * 32 + lane;
              const uint32_t at = chunk_at<C::ROWB>(16 * h + c / (C::ROWB / 16), c % (C::ROWB / 16));
              copy16(dst + at, k + 512 * i);
              copy16(dst + C::TILE + at, v + 512 * i);
            }
            if (FP8 && lane < 2) copy16(dst + 2 * C::TILE + KT * lane + 16 * h, (lane ? kv.v_exp : kv.k_exp) + vec);
          } else {
            bad |= 1u << (2 * slot + h);
            if (lane == 0) report_error(err, DERR_KV_RANGE);
          }
        }
        next += KT * C::WARPS;
        look_up();
      }
      copy_commit();
      slot = slot + 1 == C::STAGES ? 0 : slot + 1;
    };
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s) issue();

    // q as the product's operand
    {
      uint32_t(*qs)[32][4] = reinterpret_cast<uint32_t(*)[32][4]>(smem + C::QF);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int i = 0; i < (RS > 1 ? 2 : 1); ++i) {
          uint4(&rq)[HD / 32] = raw[2 * mt + i];
          float up = 1.f;
          if (FP8) {
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) {
              const uint32_t w[4] = {rq[c].x, rq[c].y, rq[c].z, rq[c].w};
#pragma unroll
              for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(w[j])), fabsf(bf16_hi(w[j]))));
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            const int x = max(-120, min(120, (int)(__float_as_uint(amax) >> 23) - 127));
            up = kv_pow2(x);
            const float down = kv_pow2(-x);
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) {
              uint32_t* w = &rq[c].x;
#pragma unroll
              for (int j = 0; j < 4; ++j) w[j] = pack_f16x2(bf16_lo(w[j]) * down, bf16_hi(w[j]) * down);
            }
          }
          qa[2 * mt + i] = a.scale * kLog2e * up;
        }
        if (warp == 0) {
#pragma unroll
          for (int s = 0; s < KS; ++s) {  // step s: components 4 s .. 4 s + 3 of this lane's
            const uint32_t* w0 = &raw[2 * mt][s >> 1].x + 2 * (s & 1);
            const uint32_t* w1 = &raw[RS > 1 ? 2 * mt + 1 : 0][s >> 1].x + 2 * (s & 1);
            *reinterpret_cast<uint4*>(qs[mt * KS + s][lane]) =
                RS > 1 ? make_uint4(w0[0], w1[0], w0[1], w1[1]) : make_uint4(w0[0], 0, w0[1], 0);
          }
        }
      }
      __syncthreads();
    }
    const uint32_t qs_addr = smem_addr(smem) + C::QF + lane * 16;

    float o[MT][NT][4], m[RS], l[RS];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][j][k] = 0.f;
#pragma unroll
    for (int i = 0; i < RS; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }

    int cur = 0;
    const uint32_t sc = smem_addr(smem) + C::SC + warp * 2 * KT * 4;
    for (int key = key0 + KT * warp; key < stop; key += KT * C::WARPS) {
      issue();  // into the stage that the last step left
      copy_wait<C::STAGES - 1>();
      __syncwarp();
      const uint32_t sk = ring + cur * C::STAGE, sv = sk + C::TILE, se = sv + C::TILE;
      const uint32_t skip = bad >> (2 * cur) & 3u;
      cur = cur + 1 == C::STAGES ? 0 : cur + 1;
      {
        const bool masked = key + KT > lim_min || skip;
        if (key + KT > lim_max || skip) {  // values that no row sees may be anything: 0 * NaN
          for (int c = lane; c < C::TILE / 16; c += 32) {
            const int r = c / (C::ROWB / 16);
            if (key + r >= lim_max || (skip >> (r >> 4) & 1))
              sts128(sv + chunk_at<C::ROWB>(r, c % (C::ROWB / 16)), make_uint4(0, 0, 0, 0));
          }
        }
        if (FP8) {  // what a key's exponents give: 2^e of the key, e of the value
          if (KT == 32 || lane < KT) {
            const int x = (int)(int8_t)lds_u8(se + lane), y = max(-126, (int)(int8_t)lds_u8(se + KT + lane));
            sts32(sc + 4 * lane, kv_pow2(x));
            sts32(sc + 4 * (KT + lane), (float)y);
          }
        }
        __syncwarp();
        // S = q k^T: column tiles of 8 keys
        float s[MT][NK][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NK; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[i][j][k] = 0.f;
        constexpr int KCH = FP8 ? HD / 64 : HD / 32;  // 16-byte chunks of a key per lane
        constexpr int SPC = FP8 ? 4 : 2;              // k steps of a chunk
#pragma unroll
        for (int c = 0; c < KCH; ++c) {
          uint4 w[NK];
#pragma unroll
          for (int j = 0; j < NK; ++j)
            w[j] = lds128(sk + chunk_at<C::ROWB>(8 * j + quad, FP8 ? place * KCH + c : k_chunk<HD, FP8>(place, c)));
#pragma unroll
          for (int x = 0; x < SPC; ++x) {
            const int st = c * SPC + x;
            uint32_t qreg[MT][4];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              const uint4 q4 = lds128(qs_addr + (i * KS + st) * 512);
              qreg[i][0] = q4.x;
              qreg[i][1] = q4.y;
              qreg[i][2] = q4.z;
              qreg[i][3] = q4.w;
            }
#pragma unroll
            for (int j = 0; j < NK; ++j) {
              const uint32_t* ww = &w[j].x;
              const uint32_t b0 = FP8 ? widen_lo(ww[x]) : ww[2 * (x & 1)];
              const uint32_t b1 = FP8 ? widen_hi(ww[x]) : ww[2 * (x & 1) + 1];
#pragma unroll
              for (int i = 0; i < MT; ++i) mma16816<FP8>(s[i][j], qreg[i], b0, b1);
            }
          }
        }
        // scores in units of log2, and what FP8 values add to the exponent of their weight
        float2 ev[NK];
        auto exponents = [&]() {
#pragma unroll
          for (int j = 0; j < NK; ++j) ev[j] = lds_f2(sc + 4 * (KT + 8 * j + 2 * place));
        };
        auto term = [](float x, float e) { return FP8 ? x + e : x; };
        if (FP8) exponents();
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          float2 kf;
          if (FP8) kf = lds_f2(sc + 4 * (8 * j + 2 * place));
#pragma unroll
          for (int i = 0; i < RS; ++i) {
            float &x0 = s[i >> 1][j][2 * (i & 1)], &x1 = s[i >> 1][j][2 * (i & 1) + 1];
            x0 *= FP8 ? qa[i] * kf.x : qa[i];
            x1 *= FP8 ? qa[i] * kf.y : qa[i];
          }
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < RS; ++i)
#pragma unroll
            for (int j = 0; j < NK; ++j)
#pragma unroll
              for (int k = 0; k < 2; ++k)
                if (key + 8 * j + 2 * place + k >= lim[i] || (skip >> (j >> 1) & 1)) s[i >> 1][j][2 * (i & 1) + k] = -INFINITY;
        }
        // The reference m of a row is taken ABOVE its largest score and moves only when a later one passes
        // that by more than SLACK, so that most steps neither exchange maxima nor scale O.  FP8: below it, P <=
        // 2^15 fills fp16's range, for the sake of small ones that carry large values.  bf16: far above, so that
        // P times the largest values, and their sums, do not overflow.
        float top[RS];
        auto grew = [&]() {
          bool any = false;
#pragma unroll
          for (int i = 0; i < RS; ++i) {
            top[i] = -INFINITY;
#pragma unroll
            for (int j = 0; j < NK; ++j)
              top[i] = fmaxf(top[i], fmaxf(term(s[i >> 1][j][2 * (i & 1)], ev[j].x), term(s[i >> 1][j][2 * (i & 1) + 1], ev[j].y)));
            any |= top[i] > m[i] - (ABOVE - SLACK);
          }
          return __any_sync(0xffffffffu, any);
        };
        bool grown = grew();
        if (FP8 && grown && lower_zeros<C::ROWB, KT>(sv, sc + 4 * KT, lane)) {
          __syncwarp();
          exponents();
          grown = grew();
        }
        if (grown) {
#pragma unroll
          for (int i = 0; i < RS; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            const float mn = fmaxf(m[i], top[i] + ABOVE);
            // (in two steps: l may be as far above 1 as the factor is below it)
            const float half = exp2_fast(0.5f * (m[i] - (mn == -INFINITY ? 0.f : mn))), alpha = half * half;
            m[i] = mn;
            l[i] = l[i] * half * half;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              o[i >> 1][j][2 * (i & 1)] *= alpha;
              o[i >> 1][j][2 * (i & 1) + 1] *= alpha;
              if (!OWN_LO) {
                o[0][j][2] *= alpha;
                o[0][j][3] *= alpha;
              }
            }
          }
        }
        uint32_t p[NK / 2][MT][4], p_lo[OWN_LO ? NK / 2 : 1][MT][4];
#pragma unroll
        for (int i = 0; i < RS; ++i) {
          const float ref = m[i] == -INFINITY ? 0.f : m[i];  // (nothing seen yet: exp2(-inf) = 0)
#pragma unroll
          for (int j = 0; j < NK; ++j) {
            const float s0 = s[i >> 1][j][2 * (i & 1)], s1 = s[i >> 1][j][2 * (i & 1) + 1];
            const float x0 = exp2_fast(term(s0, ev[j].x) - ref), x1 = exp2_fast(term(s1, ev[j].y) - ref);
            // (fp16: 11 bits cut off, so that what they leave needs no widening)
            const float h0 = __uint_as_float(__float_as_uint(x0) & 0xffffe000u), h1 = __uint_as_float(__float_as_uint(x1) & 0xffffe000u);
            const uint32_t hi = FP8 ? pack_f16x2(h0, h1) : upper_halves(x0, x1);
            const uint32_t lo = FP8 ? pack_f16x2(x0 - h0, x1 - h1)
                                    : pack_bf16x2(fmaf(x0, BF16_LO, minus_upper(x0)), fmaf(x1, BF16_LO, minus_upper(x1)));
            l[i] += FP8 ? exp2_fast(s0 - ref) + exp2_fast(s1 - ref) : x0 + x1;
            p[j >> 1][i >> 1][2 * (j & 1) + (i & 1)] = hi;
            if (OWN_LO)
              p_lo[OWN_LO ? j >> 1 : 0][i >> 1][2 * (j & 1) + (i & 1)] = lo;
            else
              p[j >> 1][0][2 * (j & 1) + 1] = lo;
          }
        }
        // A value that is no number and that only some of the rows see (0 * NaN): it is added to the
        // rows that do, one by one, and out of the product.
        if (masked && a.causal && __any_sync(0xffffffffu, has_nonfinite<FP8>(sv, C::TILE, lane))) {
#pragma unroll
          for (int half = 0; half < NK / 2; ++half)
#pragma unroll 1
            for (int jj = 0; jj < 16; ++jj) {
#pragma unroll
              for (int i = 0; i < RS; ++i) {
                const uint32_t pair = __shfl_sync(0xffffffffu, jj < 8 ? p[half][i >> 1][i & 1] : p[half][i >> 1][2 + (i & 1)],
                                                  4 * quad + ((jj & 7) >> 1));
                if (key + 16 * half + jj >= lim[i]) continue;
                const uint32_t bits = jj & 1 ? pair >> 16 : pair & 0xffffu;
                const float pj = FP8 ? __half2float(__ushort_as_half((unsigned short)bits)) : __uint_as_float(bits << 16);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                  for (int k = 0; k < 2; ++k) {
                    const float v = value_at<C::ROWB, FP8>(sv, 16 * half + jj, v_comp<HD, FP8>(2 * place + k, j));
                    if (!isfinite(v)) o[i >> 1][j][2 * (i & 1) + k] += pj * v;
                  }
              }
            }
          __syncwarp();
          clear_nonfinite<FP8>(sv, C::TILE, lane);
          __syncwarp();
        }
        // O += P v, 16 keys at a time
#pragma unroll
        for (int half = 0; half < NK / 2; ++half) {
          if (FP8) {
            constexpr int W = HD / 32;  // 4-code words of a value per lane
            uint32_t v[4][W];
#pragma unroll
            for (int r = 0; r < 4; ++r) {  // keys 2 place, 2 place + 1, and 8 on
              const int row = 16 * half + 2 * place + (r & 1) + 8 * (r >> 1);
              if (W == 4) {
                const uint4 x = lds128(sv + chunk_at<C::ROWB>(row, quad));
                v[r][0] = x.x;
                v[r][1] = x.y;
                v[r][W - 2] = x.z;
                v[r][W - 1] = x.w;
              } else {
                const uint2 x = lds64(sv + chunk_at<C::ROWB>(row, quad >> 1) + 8 * (quad & 1));
                v[r][0] = x.x;
                v[r][1] = x.y;
              }
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
              const uint32_t x0 = __byte_perm(v[0][w], v[1][w], 0x5140), x1 = __byte_perm(v[0][w], v[1][w], 0x7362);
              const uint32_t y0 = __byte_perm(v[2][w], v[3][w], 0x5140), y1 = __byte_perm(v[2][w], v[3][w], 0x7362);
              const uint32_t b0[4] = {widen_lo(x0), widen_hi(x0), widen_lo(x1), widen_hi(x1)};
              const uint32_t b1[4] = {widen_lo(y0), widen_hi(y0), widen_lo(y1), widen_hi(y1)};
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                  mma16816<FP8>(o[i][4 * w + j], p[half][i], b0[j], b1[j]);
                  if (OWN_LO) mma16816<FP8>(o[i][4 * w + j], p_lo[OWN_LO ? half : 0][i], b0[j], b1[j]);
                }
            }
          } else {
#pragma unroll
            for (int c = 0; c < HD / 64; ++c) {
              uint4 v[4];
#pragma unroll
              for (int r = 0; r < 4; ++r)
                v[r] = lds128(sv + chunk_at<C::ROWB>(16 * half + 2 * place + (r & 1) + 8 * (r >> 1), quad + 8 * c));
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const uint32_t *v0 = &v[0].x, *v1 = &v[1].x, *v2 = &v[2].x, *v3 = &v[3].x;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  const uint32_t sel = x ? 0x7632 : 0x5410;
                  const uint32_t b0 = __byte_perm(v0[w], v1[w], sel), b1 = __byte_perm(v2[w], v3[w], sel);
#pragma unroll
                  for (int i = 0; i < MT; ++i) {
                    mma16816<FP8>(o[i][8 * c + 2 * w + x], p[half][i], b0, b1);
                    if (OWN_LO) mma16816<FP8>(o[i][8 * c + 2 * w + x], p_lo[OWN_LO ? half : 0][i], b0, b1);
                  }
                }
              }
            }
          }
        }
      }
      __syncwarp();
    }
    copy_wait<0>();
    __syncwarp();

    // ---- join the warps
#pragma unroll
    for (int i = 0; i < RS; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      if (place == 0) ml[warp * C::ROWS + 8 * i + quad] = make_float2(m[i], l[i]);
    }
    if (key0 + KT * warp < stop) {
      float* mine = reinterpret_cast<float*>(smem + warp * C::RING_B);
      if (!OWN_LO) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          o[0][j][0] += o[0][j][2];
          o[0][j][1] += o[0][j][3];
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; j += 4)
#pragma unroll
          for (int k = 0; k < (RS > 1 ? 4 : 2); ++k)
            *reinterpret_cast<float4*>(mine + (16 * i + quad + 8 * (k >> 1)) * C::O_PITCH +
                                       o_place<HD, FP8>(v_comp<HD, FP8>(2 * place + (k & 1), j))) =
                make_float4(o[i][j][k], o[i][j + 1][k], o[i][j + 2][k], o[i][j + 3][k]);
    }
    __syncthreads();
    // a row's weights by a thread, then four components of a row a thread
    float* wt = reinterpret_cast<float*>(smem + C::WT);
    KaRow* row = reinterpret_cast<KaRow*>(smem + C::WT + C::ROWS * 32);
    float* part = scratch.part + (2 * (int64_t)blockIdx.x + (it.from == 0)) * C::ROWS * (HD + 4);
    if (threadIdx.x < it.rows) {
      const int r = threadIdx.x;
      float2 x[C::WARPS];
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < C::WARPS; ++w) {
        x[w] = ml[w * C::ROWS + r];
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
#pragma unroll 4
    for (int t = threadIdx.x; t < it.rows * Q; t += C::THREADS) {
      const int r = t / Q, c = 4 * (t % Q);
      const float* o_row = reinterpret_cast<const float*>(smem) + r * C::O_PITCH + o_place<HD, FP8>(c);
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
        __threadfence();  // (the block's writes, which the barrier ordered before)
        const int done = atomicAdd(&scratch.count[c0], 1);
        if (done == c1 - c0) {  // the last to come joins the parts, when it is through with its own
          scratch.count[c0] = 0;
          todo[todo[0].rows++ ? 2 : 1] = KaJoin{it.row0, it.g * rep, it.first, it.rows, c0, c1 - c0 + 1};
        }
        __threadfence();
      }
    }
    __syncthreads();
  }
  for (int i = 0; i < todo[0].rows; ++i) {
    const KaJoin j = todo[1 + i];
    join_parts<HD, C::ROWS, C::THREADS, false>(a, j, 0, rep, scratch.part, reinterpret_cast<float2*>(smem),
                                        reinterpret_cast<KaRow*>(smem + C::WT + C::ROWS * 32), threadIdx.x,
                                        [] { __syncthreads(); });
    __syncthreads();
  }
}

template <int HD, bool FP8, int RS>
cudaError_t launch_as(const KvPool& kv, const KvAttn& a, const KaScratch& s, int ctas, int* err, cudaStream_t stream) {
  using C = KaCfg<HD, FP8, RS>;
  static_assert(KA_CTAS * (C::SMEM + 1024) <= 233472, "shared memory of an SM");
  static_assert(2 * C::ROWS * (HD + 4) * 4 <= KV_ATTN_PART_BYTES, "scratch per CTA");
  auto kern = kv_attention_kernel<HD, FP8, RS>;
  static const cudaError_t set =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
  if (set != cudaSuccess) return set;
  kern<<<ctas, C::THREADS, C::SMEM, stream>>>(kv, a, s, err);
  return cudaGetLastError();
}

template <int HD, bool FP8>
cudaError_t launch_rows(const KvPool& kv, const KvAttn& a, const KaScratch& s, int ctas, int* err, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.max_new * (a.H / kv.G);
  if (rows <= 8) return launch_as<HD, FP8, 1>(kv, a, s, ctas, err, stream);
  if (rows <= 16) return launch_as<HD, FP8, 2>(kv, a, s, ctas, err, stream);
  return launch_as<HD, FP8, 4>(kv, a, s, ctas, err, stream);
}

}  // namespace

// Which kernel: the one that passes over the keys once for every 32 rows, or tcgen05 for every 256, where
// beginning an item and joining its parts (32 rows' worth here, up to 256 there) take longer.  In
// thousandths of a us of the whole GPU a unit of 128 keys takes about 10 for 32 rows here; there 15 for up to
// 128 rows, 18 for 256, and on top 5 us an item of a CTA and 0.0175 us a row and part.  Measured, us here /
// there, FP8, 28 / 4 heads of 128: 16 x 8192 positions, 224 rows a kv head 301 / 105; 8 x 3000: 63 rows
// 35 / 34, 112 53 / 37, 224 74 / 48; 4 x 8192 (ten parts an item): 63 rows 50 / 45, 112 61 / 54, 224 90 / 79;
// 1 x 16384, 224 rows 62 / 123; 2 x 1000, 224 rows 24 / 35.  Over 276 shapes (four head layouts, both formats) the rule
// takes 0.8 % longer than the better kernel on average, more than 7 % longer in 13.  Lengths are known to the
// device only: the page table's width stands for them.
bool kv_attention_many_rows(const KvPool& kv, const KvAttn& a) {
  const int64_t rows = (int64_t)a.max_new * (a.H / kv.G);
  if (a.causal || rows <= 32) return false;
  const double units = (double)a.batch * kv.G * (((int64_t)a.max_pages * kv.page_len() + KA_UNIT - 1) / KA_UNIT);
  const int64_t rest = rows % 256;
  const double here = 10.0 * (double)((rows + 31) / 32), there = 18.0 * (double)(rows / 256) + (rest > 128 ? 18 : rest ? 15 : 0);
  const double items = (double)a.batch * kv.G * (double)((rows + 255) / 256), ctas = KA_MOST / KA_CTAS;
  return (here - there) * units > 17.5 * (double)std::min<int64_t>(rows, 256) * (ctas / items + 1) + 5000.0 * items / ctas;
}

size_t kv_attention_scratch(int sms) { return KV_ATTN_COUNTERS + (size_t)KA_CTAS * sms * KV_ATTN_PART_BYTES; }

cudaError_t kv_attention_launch(const KvPool& kv, const KvAttn& a, void* scratch, int sms, int* err, cudaStream_t stream) {
  sms = std::min(sms, KA_MOST / KA_CTAS);
  KaScratch s{reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + KV_ATTN_COUNTERS), static_cast<int*>(scratch)};
  if (kv.hd == 128) return kv.fp8 ? launch_rows<128, true>(kv, a, s, KA_CTAS * sms, err, stream) : launch_rows<128, false>(kv, a, s, KA_CTAS * sms, err, stream);
  return kv.fp8 ? launch_rows<64, true>(kv, a, s, KA_CTAS * sms, err, stream) : launch_rows<64, false>(kv, a, s, KA_CTAS * sms, err, stream);
}

}  // namespace dcl
