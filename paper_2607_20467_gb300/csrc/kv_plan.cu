// The plan of a step over a paged cache: from how many positions every sequence keeps and how many new
// ones it gets, its pages, and the slots and positions of the step's rows, without the host.
//
//   need_b = ceil((start_b + new_b) / page_len)            pages past it go back, in order of (b, place)
//   lack_b = max(0, need_b - held_b)                       given where lack_0 + .. + lack_b <= pages free
//   q_start_b = new_0 + .. + new_(b - 1)                   of the sequences that got theirs
//   slot = table[b][pos / page_len] * page_len + pos % page_len,  pos = start_b + row - q_start_b
//
// One CTA: prefix sums over the sequences, in pieces of as many as it has threads, a warp for a
// sequence's pages, a thread for a row (its sequence by bisection in q_start).
#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KP_THREADS = 512;
constexpr int KP_WARPS = KP_THREADS / 32;

// A sequence's numbers; one that is not within its table gets no rows and keeps what it has.
struct KpSeq {
  int start, rows, held, need;
  bool bad;
  __device__ __forceinline__ int back() const { return max(0, held - need); }
  __device__ __forceinline__ int lack() const { return max(0, need - held); }
};
__device__ __forceinline__ KpSeq kp_seq(const KvPlan& a, int b) {
  KpSeq s{0, 0, 0, 0, false};
  if (b >= a.batch) return s;
  const int held = a.held[b];
  s.start = a.start[b];
  s.rows = a.rows_new[b];
  s.held = min(max(held, 0), a.max_pages);
  s.bad = held != s.held || s.start < 0 || s.rows < 0 || (int64_t)s.start + s.rows > (int64_t)a.max_pages << a.page_shift;
  if (s.bad) {
    s.start = s.rows = 0;
    s.need = s.held;
  } else {
    s.need = (int)(((int64_t)s.start + s.rows + (1 << a.page_shift) - 1) >> a.page_shift);
  }
  return s;
}

// Inclusive prefix sum over the block's threads; total: of all of them.
__device__ __forceinline__ int64_t kp_scan(int64_t x, int64_t* sums, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // (the last scan's sums are read)
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  int64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < KP_WARPS; ++w) {
    const int64_t y = sums[w];
    if (w < warp) before += y;
    total += y;
  }
  return x + before;
}

__global__ void __launch_bounds__(KP_THREADS) kv_plan_kernel(KvPlan a, int* err) {
  __shared__ int64_t sums[KP_WARPS];
  __shared__ int64_t off[KP_THREADS];            // where a sequence's pages go to, or come from
  __shared__ int first[KP_THREADS], count[KP_THREADS];  // its first page to give or take, and how many
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, P = 1 << a.page_shift;
  const int there = a.batch ? *a.n_free : 0;  // (no sequences: nothing but rows of none)
  int64_t returned = 0, total;
  for (int b0 = 0; b0 < a.batch; b0 += KP_THREADS) {
    const KpSeq s = kp_seq(a, b0 + threadIdx.x);
    if (s.bad) report_error(err, DERR_KV_RANGE);
    kp_scan(s.back(), sums, total);
    returned += total;
  }
  // (a stack that is not one: nothing is planned)
  const bool broken = there < 0 || there + returned > a.n_pages;
  if (broken && threadIdx.x == 0) report_error(err, DERR_KV_RANGE);
  const int64_t pages = there + returned;

  // ---- pages go back
  int64_t carry = 0;
  for (int b0 = 0; !broken && returned && b0 < a.batch; b0 += KP_THREADS) {
    const KpSeq s = kp_seq(a, b0 + threadIdx.x);
    const int64_t upto = carry + kp_scan(s.back(), sums, total);
    off[threadIdx.x] = there + upto - s.back();
    first[threadIdx.x] = s.need;
    count[threadIdx.x] = s.back();
    __syncthreads();
    for (int i = warp; i < KP_THREADS && b0 + i < a.batch; i += KP_WARPS) {
      int* row = a.table + (int64_t)(b0 + i) * a.max_pages + first[i];
      for (int j = lane; j < count[i]; j += 32) {
        a.free[off[i] + j] = row[j];
        row[j] = -1;
      }
    }
    carry += total;
  }
  __syncthreads();

  // ---- pages that are lacking, and the rows' starts
  int64_t lacked = 0, rows = 0, taken = 0;
  for (int b0 = 0; b0 < a.batch; b0 += KP_THREADS) {
    const int b = b0 + threadIdx.x;
    const KpSeq s = kp_seq(a, b);
    const int64_t upto = lacked + kp_scan(s.lack(), sums, total);
    lacked += total;
    const bool ok = !broken && !s.bad && (s.lack() == 0 || upto <= pages);
    const int64_t end = rows + kp_scan(ok ? s.rows : 0, sums, total);
    rows += total;
    off[threadIdx.x] = pages - 1 - (upto - s.lack());
    first[threadIdx.x] = s.held;
    count[threadIdx.x] = ok ? s.lack() : 0;
    kp_scan(count[threadIdx.x], sums, total);  // (orders the writes above, too)
    taken += total;
    if (b < a.batch) {
      a.q_start[b + 1] = (int)min(end, (int64_t)a.n_rows);
      a.seq_len[b] = ok ? s.start + s.rows : s.start;
    }
    for (int i = warp; i < KP_THREADS && b0 + i < a.batch; i += KP_WARPS) {
      int* row = a.table + (int64_t)(b0 + i) * a.max_pages + first[i];
      for (int j = lane; j < count[i]; j += 32) row[j] = a.free[off[i] - j];
    }
    __syncthreads();
    if (b < a.batch && !broken && !s.bad && (ok || s.back())) a.held[b] = s.need;
  }
  if (threadIdx.x == 0) {
    a.q_start[0] = 0;
    if (a.batch && !broken) *a.n_free = (int)(pages - taken);
    if (rows > a.n_rows) report_error(err, DERR_KV_RANGE);
  }
  __syncthreads();

  // ---- rows
  const int live = (int)min(rows, (int64_t)a.n_rows);
  for (int r = threadIdx.x; r < a.n_rows; r += KP_THREADS) {
    int slot = -1, pos = -1;
    if (r < live) {
      int lo = 0, hi = a.batch - 1;  // the first sequence that ends past r
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.q_start[mid + 1] > r) hi = mid;
        else lo = mid + 1;
      }
      pos = a.start[lo] + r - a.q_start[lo];
      const int page = a.table[(int64_t)lo * a.max_pages + (pos >> a.page_shift)];
      if (page >= 0 && page < a.n_pages) slot = (page << a.page_shift) + (pos & (P - 1));
      else report_error(err, DERR_KV_RANGE);
    }
    a.slot[r] = slot;
    a.pos[r] = pos;
  }
}

}  // namespace

cudaError_t kv_plan_launch(const KvPlan& a, int* err, cudaStream_t stream) {
  kv_plan_kernel<<<1, KP_THREADS, 0, stream>>>(a, err);
  return cudaGetLastError();
}

}  // namespace dcl
