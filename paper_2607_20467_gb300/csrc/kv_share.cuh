// How the kernels of kv_attention.cu, kv_attention_q4.cu and kv_attention_tc.cu share their work out, and what
// else they have in common.
//
// An item is the rows of one row tile (new positions x the query heads of one kv head) of one
// sequence; its keys come in units of 128.  All items of a launch stand in one line, each with
// a few positions for its beginning and one for every unit; every CTA takes an equal part of the
// line, so that a long sequence is spread over many CTAs, many short ones share one, and none waits
// for another's longer sequence.
#pragma once

#include <limits.h>

#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KA_UNIT = 128;  // keys of a unit of work
// The kernels for up to 32 rows, which have one scratch:
constexpr int KA_CTAS = 2;    // CTAs of an SM: one loads while the other begins or ends an item
constexpr int KA_MOST = 304;  // most CTAs of a launch
static_assert(3 * KA_MOST * sizeof(int) <= KV_ATTN_COUNTERS, "a counter per CTA, and two for groups of parts");
// START: units that beginning an item takes.  Sharing an item costs each of its CTAs the writing of a
// part and one of them the join (for up to 32 rows 3 and 4 to 20 thousand cycles; a unit of 16 rows
// takes about 1500).  So a cut that falls less than START + 3 positions after an item's beginning or
// START + 1 before its end (KA_FINE: START + 1, 2) goes there, and a CTA has at least KA_LEAST positions where the
// launch is small.
constexpr int KA_LEAST = 4;
// 4 bits, up to 32 rows: finer, as few units of work take long beside what a cut costs.  us with the others' cuts /
// these, 28 / 4 heads: one row, 1 x 1000 10.9 / 8.8, 1 x 4096 11.9 / 9.8, 1 x 16384 17.3 / 13.9, 16 x 1000 14.5 / 11.2; 28
// rows, 1 x 1000 22.6 / 16.7, 1 x 16384 33.6 / 28.6, 20 ragged to 1500 26.8 / 19.7; 64 ragged to 4096, one row 32.7 / 32.5.  (Shares of one unit: 28 rows, 1 x 16384 39; cuts a unit before an end: 1 x 2000, 28 rows 22.7 for 18.5.)
constexpr int KA_FINE = 2;
template <int START, int LEAST>
struct KaCut {
  static constexpr int LOW = START + (LEAST < KA_LEAST ? 1 : 3), HIGH = LEAST < KA_LEAST ? 2 : START + 1;
  static __device__ __forceinline__ int at(int pos, int line) {
    if (line < LOW + HIGH) return 2 * pos < line ? 0 : line;
    return pos < LOW ? 0 : pos > line - HIGH ? line : pos;
  }
};

// The line in equal parts: CTA c of n has positions [start(c), start(c + 1)), each end moved as KaCut
// says.
struct KaShare {
  int64_t each;
  int extra, n;
  __device__ KaShare(int64_t total, int ctas, int least) {
    n = (int)min((int64_t)ctas, (total + least - 1) / least);  // (CTAs past it have nothing)
    if (total < (1ll << 31)) {
      each = n ? (int)total / n : 0;
    } else {
      each = total / n;
    }
    extra = (int)(total - each * n);
  }
  __device__ int64_t start(int c) const { return c >= n ? each * n + extra : each * c + min(c, extra); }
  __device__ int owner(int64_t u) const {
    const int64_t big = extra * (each + 1);
    const int64_t at = u < big ? u : u - big, size = u < big ? each + 1 : each;
    const int c = at < (1ll << 31) && size < (1ll << 31) ? (int)at / (int)size : (int)(at / size);
    return u < big ? c : extra + c;
  }
};

// The rows of one row tile of kv head g of sequence b, and this CTA's units of its keys.
struct KaItem {
  int b, g, first, rows;  // its rows [first, first + rows) of the nq * rep of the sequence's kv head
  int row0, nq, len;      // the sequence's first row of q, its new positions, its cached ones
  int from, until, units; // units [from, until) of those there are
  int line;               // its positions
  int64_t item0;          // its first position
  __device__ __forceinline__ bool whole() const { return from == 0 && until == units; }
};
// An item whose parts are all there: `parts` of them, from CTA c0 on.
struct KaJoin {
  int row0, head0, first, rows, c0, parts;
};

struct KaWalk {
  int64_t u, end, total, before;  // this CTA's part of the line; positions of the sequences before b
  int b;
};

// How much longer than a share items may be that are not cut, where all of them are about as long: a cut costs two
// CTAs a beginning and an end, and a join.  4 bits, us cut / whole: 64 sequences of 1024, 28 / 4 heads, one row
// 20.8 / 17.8; 8 of 1536, 32 heads, one row 24.1 / 21.2, 16 rows 36.3 / 30.0, 32 rows 47.7 / 44.4; 16 of 1024,
// 28 / 4 heads, 448 rows 48.6 / 40.0.  (6: 16 sequences of 1024, one row 14.3 / 15.3.  Other formats are always cut.)
constexpr int KA_KEEP = 5;
// ROWS of an item; positions for its beginning (START); SEQS: sequences, in 32s, of which a lane keeps the positions
// while it looks for its CTA's part.  A second look at the lengths of the others takes as long as all the rest, but what is
// kept adds to the registers of a kernel whose loop has none left: 9 rows and more of FP8 and bf16 pages keep 32.  us, 32 kept
// / 128: FP8, one row, 120 sequences 22.6 / 21.5; FP8, 32 heads, 8 of 1536, 16 rows 35.9 / 37.6; causal 4 x 8192, 64 new
// 160.2 / 165.1; bf16, 32 heads, 8 of 1536, 32 rows 50.0 / 50.9; tcgen05, FP8, 16 x 8192, 224 rows 112.2 / 113.7.
template <int ROWS, int START, int KEEP = 0, int LEAST = KA_LEAST, int SEQS = 4>
struct KaLine {
  const KvAttn& a;
  int G, rep, room;
  __device__ KaLine(const KvPool& kv, const KvAttn& a_)
      : a(a_), G(kv.G), rep(a_.H / kv.G), room(a_.max_pages << kv.page_shift) {}
  __device__ __forceinline__ int seq_rows(int b, int& row0) const {
    row0 = min(max(a.q_start[b], 0), a.rows);
    return min(max(a.q_start[b + 1], row0), a.rows) - row0;
  }
  __device__ __forceinline__ int seq_len(int b) const { return min(max(a.lens[b], 0), room); }
  __device__ __forceinline__ int tiles_of(int nq) const { return (int)(((int64_t)nq * rep + ROWS - 1) / ROWS); }
  // (at least one unit: the rows of a sequence without keys are still written)
  __device__ __forceinline__ int line_of(int len) const { return START + max(1, (len + KA_UNIT - 1) / KA_UNIT); }

  // This CTA's part (a warp; lane 0 writes it).
  __device__ __forceinline__ void begin(KaWalk* walk, int* err) const {
    const int lane = threadIdx.x & 31;
    int least = INT_MAX, most = 0;  // an item's positions
    auto scan = [&](int b0, int64_t& own) {  // positions of sequences b0 .. b0 + 31: inclusive prefix
      int row0;
      const int b = b0 + lane;
      own = 0;
      if (b < a.batch) {
        const int raw = a.lens[b], nq = seq_rows(b, row0);
        if (raw != min(max(raw, 0), room) && blockIdx.x == 0) report_error(err, DERR_KV_RANGE);
        if (nq) {
          const int line = line_of(min(max(raw, 0), room));
          own = (int64_t)G * tiles_of(nq) * line;
          least = min(least, line);
          most = max(most, line);
        }
      }
      int64_t upto = own;
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
      }
      return upto;
    };
    int64_t total = 0, owns[SEQS], uptos[SEQS];
    if constexpr (SEQS == 1) {
      uptos[0] = 0;
      for (int b0 = 0; b0 < a.batch; b0 += 32) {
        uptos[0] = scan(b0, owns[0]);
        total += __shfl_sync(0xffffffffu, uptos[0], 31);
      }
    } else {
#pragma unroll
      for (int i = 0; i < SEQS; ++i) {
        owns[i] = uptos[i] = 0;
        if (32 * i < a.batch) {
          uptos[i] = scan(32 * i, owns[i]);
          total += __shfl_sync(0xffffffffu, uptos[i], 31);
        }
      }
      for (int b0 = 32 * SEQS; b0 < a.batch; b0 += 32) {
        int64_t own;
        total += __shfl_sync(0xffffffffu, scan(b0, own), 31);
      }
    }
    const KaShare share(total, gridDim.x, LEAST);
    // no longer than a share and KEEP (and no shorter, so that no CTA has two): a CTA each
    const bool whole = KEEP && (int)__reduce_min_sync(0xffffffffu, (unsigned)least) >= share.each + (share.extra > 0) &&
                       (int)__reduce_max_sync(0xffffffffu, (unsigned)most) <= share.each + KEEP;
    // where the cut before CTA c goes: the position, its sequence and the positions before that
    auto cut = [&](int c, int& b, int64_t& before) -> int64_t {
      const int64_t u = share.start(c);
      before = 0;
      auto here = [&](int b0, int64_t upto, int64_t own, int64_t& at) {  // whether it is among sequences b0 .. b0 + 31
        const unsigned hit = __ballot_sync(0xffffffffu, u < before + upto);
        if (!hit) {
          before += __shfl_sync(0xffffffffu, upto, 31);
          return false;
        }
        const int l = __ffs(hit) - 1;
        b = b0 + l;
        before += __shfl_sync(0xffffffffu, upto - own, l);
        const int line = line_of(seq_len(b));
        const int64_t in = u - before;
        const int pos = in < (1ll << 31) ? (int)in % line : (int)(in % line);
        at = u - pos + (whole ? (2 * pos < line ? 0 : line) : KaCut<START, LEAST>::at(pos, line));
        return true;
      };
      int64_t at;
      if constexpr (SEQS == 1) {
        for (int b0 = 0; b0 < a.batch; b0 += 32) {
          if (a.batch > 32) uptos[0] = scan(b0, owns[0]);
          if (here(b0, uptos[0], owns[0], at)) return at;
        }
      } else {
#pragma unroll
        for (int i = 0; i < SEQS; ++i)
          if (32 * i < a.batch && here(32 * i, uptos[i], owns[i], at)) return at;
        for (int b0 = 32 * SEQS; b0 < a.batch; b0 += 32) {
          int64_t own;
          const int64_t upto = scan(b0, own);
          if (here(b0, upto, own, at)) return at;
        }
      }
      b = a.batch;
      return total;
    };
    int b = 0, b_end;
    int64_t before = 0, before_end, u = 0, end = 0;
    if ((int)blockIdx.x < share.n) {
      u = cut(blockIdx.x, b, before);
      end = cut(blockIdx.x + 1, b_end, before_end);
    }
    if (lane == 0) *walk = KaWalk{u, end, total, before, b};
  }

  // The next item of the part; false at its end.  (it.b < 0 before the first)
  __device__ __forceinline__ bool next(KaWalk& w, KaItem& it) const {
    while (w.u < w.end) {
      if (it.b != w.b) {
        it.b = w.b;
        it.nq = seq_rows(w.b, it.row0);
        it.len = seq_len(w.b);
      }
      const int line = line_of(it.len), nt = tiles_of(it.nq);
      if (it.nq == 0 || w.u - w.before >= (int64_t)G * nt * line) {
        if (it.nq) w.before += (int64_t)G * nt * line;
        ++w.b;
        continue;
      }
      const int64_t in = w.u - w.before;
      const int which = in < (1ll << 31) ? (int)in / line : (int)(in / line);
      it.item0 = w.before + (int64_t)which * line;
      it.line = line;
      it.units = line - START;
      const int64_t upto = min(w.end, it.item0 + line);
      it.from = max(0, (int)(w.u - it.item0) - START);
      it.until = (int)(upto - it.item0) - START;
      w.u = upto;
      if (it.until <= it.from) continue;  // (this part of the line holds the item's beginning only)
      it.g = which / nt;
      it.first = (which - it.g * nt) * ROWS;
      it.rows = min(ROWS, it.nq * rep - it.first);
      return true;
    }
    return false;
  }
  // The CTAs c0 .. c1 that share an item that is not whole.
  __device__ __forceinline__ void sharers(const KaWalk& w, const KaItem& it, int& c0, int& c1) const {
    const KaShare share(w.total, gridDim.x, LEAST);
    c0 = share.owner(it.item0 + KaCut<START, LEAST>::LOW - 1);
    c1 = share.owner(it.item0 + it.line - KaCut<START, LEAST>::HIGH);
  }
};

// Where a part of an item's rows has four components of a row, and its {m, l}: row by row, or
// (BY_FOUR) rows next to one another, for writers that have a row a thread.
template <int HD, int ROWS, bool BY_FOUR>
struct KaPart {
  static constexpr int FLOATS = ROWS * (HD + 4);
  static __device__ __forceinline__ int four(int r, int q) { return BY_FOUR ? (q * ROWS + r) * 4 : r * (HD + 4) + 4 * q; }
  static __device__ __forceinline__ int ml(int r) { return BY_FOUR ? HD * ROWS + 2 * r : r * (HD + 4) + HD; }
};

// Scratch of a launch: the parts of shared items, and how many of each have come.
struct KaScratch {
  float* part;  // [2 * CTAs] of KaPart: O, m, l (a CTA's items that it does not begin, and does)
  int* count;   // [CTAs], by the CTA that begins the item; zero between launches
};

// How an item's parts are joined: of more than `one` in groups of about their number's root, each group by its
// last CTA to come, and the groups' by the last of those (one SM reads parts at about 26 bytes a cycle).  A group's
// counter, beside an item's: of the CTA where it begins, which is an item's first (k = 0) or not.
struct KaGroups {
  int n, size, groups;
  __device__ __forceinline__ KaGroups(int n_, int one) : n(n_), size(n_), groups(1) {
    if (n <= one) return;
    size = (int)ceilf(sqrtf((float)n));
    groups = (n + size - 1) / size;
  }
  __device__ __forceinline__ int of(int part) const { return groups > 1 ? part / size : 0; }
  __device__ __forceinline__ int parts(int k) const { return min(size, n - k * size); }
};
// Whether this is the last of n to come (one thread of a block, after a barrier).  The block's writes come before it,
// what a join reads after; the counter is zero again.
__device__ __forceinline__ bool ka_come(int* count, int n) {
  int done;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(done) : "l"(count) : "memory");
  if (done == n - 1) *count = 0;
  return done == n - 1;
}

// A joined row: 1 / l (0 for a row that sees nothing), and its place in the output.
struct KaRow {
  float inv;
  int at;
};
// Row r of an item (its first of the sequence's kv head: first), {m, l} joined: what its components need,
// and its log-sum-exp.
__device__ __forceinline__ KaRow finish_row(const KvAttn& a, int row0, int head0, int first, int rep, int r, float m, float l) {
  const int tok = (first + r) / rep, at = (row0 + tok) * a.H + head0 + first + r - tok * rep;
  if (a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  return KaRow{l == 0.f ? 0.f : 1.f / l, at};
}
template <int HD>
__device__ __forceinline__ void finish4(const KvAttn& a, const KaRow& row, int c, const float4& o) {
  const float f = row.inv;
  *reinterpret_cast<uint2*>(a.out + (int64_t)row.at * HD + c) = make_uint2(pack_bf16x2(o.x * f, o.y * f), pack_bf16x2(o.z * f, o.w * f));
}
__device__ __forceinline__ void add_scaled(float4& acc, const float4& y, float f) {
  acc.x = fmaf(y.x, f, acc.x);
  acc.y = fmaf(y.y, f, acc.y);
  acc.z = fmaf(y.z, f, acc.z);
  acc.w = fmaf(y.w, f, acc.w);
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Copies of pages: 16 bytes a time, asynchronously.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts8(uint32_t a, uint32_t v) { asm volatile("st.shared.u8 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
// two E4M3 codes to two fp16
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
// Byte offset of 16-byte chunk c of row r of a tile of 4-bit codes.  Rows change places, as a value's operand
// takes 8 (HD = 128) or 4 bytes of every other row: a half-warp's 8-byte loads, or a warp's 4-byte ones, then
// meet all the banks, and a key's (16 or 8 bytes of neighbouring rows) as well.  8 rows on is 512 or 128 bytes
// further, 16 rows 16 rows.
template <int ROWB>
__device__ __forceinline__ uint32_t chunk4_at(int r, int c) {
  if (ROWB == 64) {
    const int x = r & 1 ? 4 + ((r >> 1 & 3) ^ 1) : r >> 1 & 3;
    return (uint32_t)(((r & ~7) + x) * 64 + ((c ^ (x & 2)) << 4));
  }
  const int x = r & 1 ? 8 + ((r >> 1 & 7) ^ 2) : r >> 1 & 7;
  return (uint32_t)(((r & ~15) + x) * 32 + (c << 4));
}
// Two bf16 parts of a weight p: its upper half (8 bits), and what that leaves of p (1 + 2^-17).  The factor, the
// same for all weights and half of what the parts may be off by, keeps the second above zero where the
// first is: an infinite value then gives the infinity, where a part of zero would make it no number.
constexpr float BF16_LO = 1.f + 1.f / 131072.f;
__device__ __forceinline__ float minus_upper(float p) { return __uint_as_float((__float_as_uint(p) & 0xffff0000u) | 0x80000000u); }
__device__ __forceinline__ uint32_t upper_halves(float p0, float p1) {
  return __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
}
// The root of a part's weight, the largest reference top: l is scaled by it twice, as l may be as far above
// 1 as the weight is below it (values' exponents, which the references hold and l does not).
__device__ __forceinline__ float part_half(float m, float top) { return m == -INFINITY ? 0.f : exp2_fast(0.5f * (m - top)); }

// The parts of an item, left by its CTAs, joined by THREADS threads (tid of them; sync: their barrier):
// every part's {m, l} into shared memory (w, [rows][parts]) at once, a row's weights by a thread or
// a warp (what its components need in row); then four components of a row a thread, 12 to 16 loads in
// flight (one takes about 1000 cycles here: a warp per row, part after part, took 35000 for 38
// parts and 17000 for two parts of 32 rows).  it's rows begin at row r0 of the parts.  STEPS: of some of the parts, into
// the first of them (a group) or the rows' results.
struct KaSome {
  int c0, stride, n;  // those of every stride-th CTA from c0 on
  bool group;
};
template <int HD, int ROWS, int THREADS, bool BY_FOUR, bool STEPS, typename Sync>
__device__ __forceinline__ void join_parts(const KvAttn& a, const KaJoin& it, int r0, int rep, float* parts, float2* w,
                                           KaRow* row, int tid, Sync sync, const KaSome& some = {}) {
  using P = KaPart<HD, ROWS, BY_FOUR>;
  constexpr int Q = HD / 4;
  const int warp = tid >> 5, lane = tid & 31, n = STEPS ? some.n : it.parts;
  // (the item's first CTA's part is its second, the others' their first)
  const int c0 = STEPS ? some.c0 : it.c0, begins = !STEPS || c0 == it.c0;
  float* first = parts + (2 * (int64_t)c0 + begins) * P::FLOATS;
  auto part_at = [&](int c) { return (int64_t)max(2 * c * (STEPS ? some.stride : 1) - begins, 0) * P::FLOATS; };
  auto part_of = [&](int c) { return first + part_at(c); };
  auto done = [&](int r, float top, float sum) {
    if (STEPS && some.group) *reinterpret_cast<float2*>(first + P::ml(r0 + r)) = make_float2(top, sum);
    else row[r] = finish_row(a, it.row0, it.head0, it.first, rep, r, top, sum);
  };
  for (int i = tid; i < it.rows * n; i += THREADS) {
    const int c = i / it.rows, r = i - c * it.rows;
    w[r * n + c] = __ldcg(reinterpret_cast<const float2*>(part_of(c) + P::ml(r0 + r)));
  }
  sync();
  if (n <= 8) {
    for (int r = tid; r < it.rows; r += THREADS) {
      float2* wr = w + r * n;
      float top = -INFINITY, sum = 0.f;
      for (int c = 0; c < n; ++c) top = fmaxf(top, wr[c].x);
      for (int c = 0; c < n; ++c) {
        const float2 x = wr[c];
        const float half = part_half(x.x, top);
        wr[c].x = half * half;
        sum = fmaf(x.y * half, half, sum);
      }
      done(r, top, sum);
    }
  } else {
    for (int r = warp; r < it.rows; r += THREADS / 32) {
      float2* wr = w + r * n;
      float top = -INFINITY, sum = 0.f;
      for (int c = lane; c < n; c += 32) top = fmaxf(top, wr[c].x);
      top = warp_max(top);
      for (int c = lane; c < n; c += 32) {
        const float2 x = wr[c];
        const float half = part_half(x.x, top);
        wr[c].x = half * half;
        sum = fmaf(x.y * half, half, sum);
      }
      sum = warp_sum(sum);
      if (lane == 0) done(r, top, sum);
    }
  }
  sync();
  // (by fours: a warp has eight rows of four neighbouring fours, whole sectors to read and to write)
  auto row_of = [&](int t) { return BY_FOUR ? t / (8 * Q) * 8 + (t >> 2 & 7) : t / Q; };
  auto four_of = [&](int t) { return BY_FOUR ? (t / 32) % (Q / 4) * 4 + (t & 3) : t % Q; };
  const int all = (BY_FOUR ? (it.rows + 7) / 8 * 8 : it.rows) * Q;
  auto tasks = [&](auto tasks_, auto parts_) {
    constexpr int T = decltype(tasks_)::value, U = decltype(parts_)::value;
#pragma unroll 1
    for (int t0 = tid; t0 < all; t0 += T * THREADS) {
      float4 acc[T];
      const float* from[T];
      const float2* wr[T];
#pragma unroll
      for (int k = 0; k < T; ++k) {
        const int t = min(t0 + k * THREADS, all - 1), r = min(row_of(t), it.rows - 1);
        acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        from[k] = first + P::four(r0 + r, four_of(t));
        wr[k] = w + r * n;
      }
#pragma unroll 1
      for (int c = 0; c < n; c += U) {
        float4 y[T][U];
#pragma unroll
        for (int i = 0; i < U; ++i)  // (past the end: the last again, without weight)
#pragma unroll
          for (int k = 0; k < T; ++k)
            y[k][i] = __ldcg(reinterpret_cast<const float4*>(from[k] + part_at(min(c + i, n - 1))));
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
          for (int k = 0; k < T; ++k)
            if (c + i < n) add_scaled(acc[k], y[k][i], wr[k][c + i].x);
      }
#pragma unroll
      for (int k = 0; k < T; ++k) {
        const int t = t0 + k * THREADS;
        if (t >= all) break;
        if (STEPS && some.group) *reinterpret_cast<float4*>(first + P::four(r0 + row_of(t), four_of(t))) = acc[k];
        else if (!BY_FOUR || row_of(t) < it.rows) finish4<HD>(a, row[row_of(t)], 4 * four_of(t), acc[k]);
      }
    }
  };
  if (n == 2)  // (most often; what a thread has is loaded at once)
    tasks(std::integral_constant<int, 6>{}, std::integral_constant<int, 2>{});
  else if (n <= 4)
    tasks(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
  else
    tasks(std::integral_constant<int, 2>{}, std::integral_constant<int, 8>{});
}

}  // namespace
}  // namespace dcl
