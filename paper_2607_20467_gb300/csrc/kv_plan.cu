// The plan of a step over a paged cache: from how many positions every sequence keeps and how many new
// ones it gets, its pages, and the slots and positions of the step's rows, without the host.
//
//   need_b = ceil((start_b + new_b) / page_len)            pages past it go back, in order of (b, place)
//   lack_b = max(0, need_b - held_b)                       given where lack_0 + .. + lack_b <= pages free
//   q_start_b = new_0 + .. + new_(b - 1)                   of the sequences that got theirs
//   slot = table[b][pos / page_len] * page_len + pos % page_len,  pos = start_b + row - q_start_b
//
// A few numbers a sequence, a slot and a position a row: a call is bound by the chain of its steps.  Prefix
// sums over the sequences in pieces of a CTA's threads; a warp for a sequence's pages; a thread for a few
// rows (their sequence by bisection in q_start).  Steps of many rows or sequences: a cluster of 8 CTAs for the
// pages, each of which has the sums for itself, and a second kernel for the rows, launched as the first
// begins.  In a graph, where no page moves: 8 sequences of 32 rows 3.6 us, of which the launch is about 2; 256 prompts of
// up to 1536 positions (172 thousand rows, 1.4 MB) 7.7 (one CTA for all 96; the cluster's CTAs for the rows, too, 16.5: ten of
// them were the rows' instructions on 8 SMs; 16 rows a thread there 20.6).  Pages add a warp's two dependent looks at memory
// for each sequence it has: of a call that takes them and one that returns them, together, 8 sequences' 8 pages 0.6 us, 64
// sequences' 64 2 to 3, the prompts' 10875 3.1 (with the prompts' rows and without: 7.7 + 6.0, and 16.8 with the pages).
#include "common.cuh"
#include "kv_cache.cuh"

namespace dcl {
namespace {

constexpr int KP_CLUSTER = 8;
constexpr int KP_ONE_SEQS = 256, KP_ONE_ROWS = 4096;  // most of a step that one block lays out (kv_plan_launch)
constexpr int KP_STARTS = 2048;  // sequences whose first rows and positions the rows' kernel keeps in shared memory
constexpr int KP_ROW_THREADS = 256;

// A sequence's numbers; one that is not within its table gets no rows and keeps what it has: its pages, and its
// start, which is 0 only where that is no position of the table.
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
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  s.bad = held != s.held || s.start < 0 || s.rows < 0 || (int64_t)s.start + s.rows > room;
  if (s.bad) {
    if (s.start < 0 || s.start > room) s.start = 0;
    s.rows = 0;
    s.need = s.held;
  } else {
    s.need = (int)(((int64_t)s.start + s.rows + (1 << a.page_shift) - 1) >> a.page_shift);
  }
  return s;
}

// Inclusive prefix sum over the block's threads, and the sum of all.  Calls in turn take sums of their own.
template <int T>
__device__ __forceinline__ int64_t kp_scan(int64_t x, int64_t (&sums)[T / 32], int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  int64_t upto = lane < T / 32 ? sums[lane] : 0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  total = __shfl_sync(0xffffffffu, upto, 31);
  const int64_t before = __shfl_sync(0xffffffffu, upto, max(warp - 1, 0));
  return warp ? x + before : x;
}

// What a sequence that got its rows keeps: start is what seq_len tells, which may have taken its place.
__device__ __forceinline__ int kp_kept(const KvPlan& a, int b) { return __ldcg(a.seq_len + b) - a.rows_new[b]; }

// Slots and positions of rows first .. first + 3 and every step after; starts, keeps: q_start and what the sequences
// keep in shared memory, or NULL.
__device__ __forceinline__ void kp_rows(const KvPlan& a, const int* starts, const int* keeps, int64_t first, int64_t step, int* err) {
  const int P = 1 << a.page_shift;
  const bool wide = ((reinterpret_cast<uintptr_t>(a.slot) | reinterpret_cast<uintptr_t>(a.pos)) & 15) == 0;
  auto start_of = [&](int b) { return starts ? starts[b] : __ldcg(a.q_start + b); };
  auto kept_of = [&](int b) { return starts ? keeps[b] : kp_kept(a, b); };
  const int live = start_of(a.batch);
  for (; first < a.n_rows; first += step) {
    const int r0 = (int)first;
    int slot[4] = {-1, -1, -1, -1}, pos[4] = {-1, -1, -1, -1};
    if (r0 < live) {
      int lo = 0, hi = a.batch - 1;  // the first sequence that ends past r0
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start_of(mid + 1) > r0) hi = mid;
        else lo = mid + 1;
      }
      int q0 = start_of(lo), q1 = start_of(lo + 1), at = kept_of(lo), have = -1, base = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= live - r0) break;  // (r0 + 3 may pass 2^31)
        const int r = r0 + i;
        if (r >= q1) {
          do {
            q0 = q1;
            q1 = start_of(++lo + 1);
          } while (r >= q1);
          at = kept_of(lo);
          have = -1;
        }
        pos[i] = at + r - q0;
        if (have != pos[i] >> a.page_shift) {
          have = pos[i] >> a.page_shift;
          base = __ldcg(a.table + (int64_t)lo * a.max_pages + have);
          if (base < 0 || base >= a.n_pages) {
            report_error(err, DERR_KV_RANGE);
            base = -1;
          }
        }
        slot[i] = base < 0 ? -1 : (base << a.page_shift) + (pos[i] & (P - 1));
      }
    }
    if (wide && first + 4 <= a.n_rows) {
      *reinterpret_cast<int4*>(a.slot + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      *reinterpret_cast<int4*>(a.pos + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (first + i < a.n_rows) {
          a.slot[r0 + i] = slot[i];
          a.pos[r0 + i] = pos[i];
        }
    }
  }
}

template <int T, int CTAS, bool ROWS_TOO>
__global__ void __launch_bounds__(T) kv_plan_kernel(KvPlan a, int* err) {
  __shared__ int64_t sums[2][T / 32];
  __shared__ int64_t off[T];             // where a sequence's pages go to, or come from
  __shared__ int first[T], count[T];     // its first page to give or take, and how many
  constexpr int KEPT = ROWS_TOO ? KP_ONE_SEQS : 0;  // what the rows here need of the sequences
  __shared__ int starts[KEPT + 1], keeps[KEPT + 1];
  __shared__ int most;                   // pages taken
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = CTAS > 1 ? (int)blockIdx.x : 0, warp = rank * (T / 32) + (tid >> 5);  // (one cluster is the grid)
  auto meet = [] {  // what was written before is there for all CTAs
    if (CTAS > 1) {
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      __syncthreads();
    }
  };
  if (!ROWS_TOO) pdl_launch_dependents();
  static_assert(KEPT <= T, "all sequences of a block's step at once");
  const bool one = ROWS_TOO || a.batch <= T;
  const int there = a.batch ? *a.n_free : 0;  // (no sequences: nothing but rows of none)
  const KpSeq mine = kp_seq(a, tid);
  auto seq = [&](int b0) { return one ? mine : kp_seq(a, b0 + tid); };
  auto both = [](const KpSeq& s) { return (int64_t)s.back() << 32 | s.lack(); };  // (sums of either are below 2^31)
  if (tid == 0) most = 0;

  // ---- pages that come back; of at most T sequences all sums at once
  int64_t total, sum = 0;
  int64_t returned = 0;
  for (int b0 = 0, i = 0; b0 < a.batch; b0 += T, i ^= 1) {
    const KpSeq s = seq(b0);
    if (s.bad && rank == 0) report_error(err, DERR_KV_RANGE);
    sum = kp_scan<T>(both(s), sums[i], total);
    returned += total >> 32;
  }
  // (a stack that is not one: nothing is planned)
  const bool broken = there < 0 || there + returned > a.n_pages;
  if (broken && tid == 0 && rank == 0) report_error(err, DERR_KV_RANGE);
  const int64_t pages = there + returned;

  if (!broken && returned) {
    int64_t carry = 0;
    for (int b0 = 0; b0 < a.batch; b0 += T) {
      const KpSeq s = seq(b0);
      __syncthreads();
      if (!one) sum = kp_scan<T>(both(s), sums[0], total);
      off[tid] = there + carry + (sum >> 32) - s.back();
      first[tid] = s.need;
      count[tid] = s.back();
      __syncthreads();
      for (int i = warp; i < T && b0 + i < a.batch; i += CTAS * (T / 32)) {
        int* row = a.table + (int64_t)(b0 + i) * a.max_pages + first[i];
        for (int j = lane; j < count[i]; j += 32) {
          a.free[off[i] + j] = row[j];
          row[j] = -1;
        }
      }
      carry += total >> 32;
    }
    meet();
  }

  // ---- pages that are lacking, and the rows' starts
  int64_t lacked = 0, rows = 0;
  for (int b0 = 0; b0 < a.batch; b0 += T) {
    const int b = b0 + tid;
    const KpSeq s = seq(b0);
    if (!one) {
      __syncthreads();
      sum = kp_scan<T>(both(s), sums[0], total);
    }
    const int64_t upto = lacked + (sum & 0xffffffff);
    lacked += total & 0xffffffff;
    const bool ok = !broken && !s.bad && (s.lack() == 0 || upto <= pages);
    const int taken = (int)__reduce_max_sync(0xffffffffu, ok && s.lack() ? (unsigned)upto : 0u);  // (they ascend)
    off[tid] = pages - 1 - (upto - s.lack());
    first[tid] = s.held;
    count[tid] = ok ? s.lack() : 0;
    const int64_t end = rows + kp_scan<T>(ok ? s.rows : 0, sums[1], total);
    rows += total;
    if (lane == 0 && taken) atomicMax(&most, taken);
    if (b < a.batch) {
      const int q = (int)min(end, (int64_t)a.n_rows);
      if (ROWS_TOO) {
        starts[b + 1] = q;
        keeps[b] = s.start;
      }
      if (rank == 0) a.q_start[b + 1] = q;
    }
    meet();  // (every CTA has read what the sequences hold and keep)
    for (int i = warp; i < T && b0 + i < a.batch; i += CTAS * (T / 32)) {
      int* row = a.table + (int64_t)(b0 + i) * a.max_pages + first[i];
      for (int j = lane; j < count[i]; j += 32) row[j] = __ldcg(a.free + off[i] - j);
    }
    if (rank == 0 && b < a.batch) {
      a.seq_len[b] = ok ? s.start + s.rows : s.start;
      if (ok) a.held[b] = s.need;  // (one with pages to return lacks none)
    }
  }
  if (tid == 0) {
    if (ROWS_TOO) starts[0] = 0;
    if (rank == 0) {
      a.q_start[0] = 0;
      if (rows > a.n_rows) report_error(err, DERR_KV_RANGE);
    }
  }
  meet();
  if (rank == 0 && tid == 0 && a.batch && !broken) *a.n_free = (int)(pages - most);
  if (ROWS_TOO) kp_rows(a, starts, keeps, 4 * tid, 4 * T, err);
}

// The rows of a step that has many of them, by CTAs all over the GPU.
__global__ void __launch_bounds__(KP_ROW_THREADS) kv_plan_rows_kernel(KvPlan a, int* err) {
  __shared__ int starts[KP_STARTS + 1], keeps[KP_STARTS];
  pdl_wait();
  const bool kept = a.batch <= KP_STARTS;
  for (int i = threadIdx.x; kept && i <= a.batch; i += KP_ROW_THREADS) {
    starts[i] = a.q_start[i];
    if (i < a.batch) keeps[i] = kp_kept(a, i);
  }
  __syncthreads();
  kp_rows(a, kept ? starts : nullptr, keeps, 4 * ((int64_t)blockIdx.x * KP_ROW_THREADS + threadIdx.x), 4 * (int64_t)gridDim.x * KP_ROW_THREADS, err);
}

}  // namespace

cudaError_t kv_plan_launch(const KvPlan& a, int sms, int* err, cudaStream_t stream) {
  // One kernel while the rows are a few a thread, in us, one / two, no page moved: 256 rows of 8 sequences 3.2 / 5.7,
  // 4096 of 8 4.2 / 6.0, 4096 of 64 4.6 / 6.3, 256 of 256 5.2 / 7.7, 4096 of 256 5.7 / 7.0, 32000 of 16 14.8 / 6.0.  A call that
  // takes a page for every sequence and one that returns them, together: 8 sequences 6.3 / 11.5, 64 10.0 / 12.8, 128
  // 11.3 / 13.7, 256 18.3 / 14.9 (16 a warp, one after another; most steps of decoding move a page for few).
  if (a.n_rows <= KP_ONE_ROWS && a.batch <= KP_ONE_SEQS) {
    kv_plan_kernel<512, 1, true><<<1, 512, 0, stream>>>(a, err);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(KP_CLUSTER);
  cfg.blockDim = dim3(1024);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = KP_CLUSTER;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_plan_kernel<1024, KP_CLUSTER, false>, a, err);
  if (e != cudaSuccess || a.n_rows == 0) return e;
  const int64_t ctas = ((int64_t)a.n_rows + 4 * KP_ROW_THREADS - 1) / (4 * KP_ROW_THREADS), most = 8 * (int64_t)sms;
  return launch_pdl(kv_plan_rows_kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(KP_ROW_THREADS), 0, stream, a, err);
}

}  // namespace dcl
