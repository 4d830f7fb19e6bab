// Page tables of one stream that live on the device: lengths, page ids, the free pages as a stack.
// A step's bookkeeping (how many pages every sequence takes or gives back, which ones, and the slot
// of every new token) is prefix sums over the batch, held in shared memory, so a step can be captured
// into a graph and replayed while its sequences grow.
//
//   have_i = ceil(len_i / P), want_i = ceil((len_i + new_i) / P), first_i = sum_{j<i} (want_j - have_j)
//   page (have_i + c) of sequence i = free[n_free - 1 - first_i - c]
//   start_i = sum_{j<i} new_j;  token i of the call: slot = page * P + position % P
//
// Trimming is the inverse: what it gives back is taken again in the same order.  Nothing is changed
// when the call cannot be carried out as a whole.  What bounds a step of single tokens is the launch and
// three dependent trips to the L2 (ids, lengths, free pages); the bytes (some KB) do not count.  Where
// many pages or slots may be written, a cluster of eight blocks shares them out: each makes the sums for itself,
// and none writes before all have read (64 sequences of 500 to 9 000 tokens released and taken in: 105 us with
// one block, 16.6 so).

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

constexpr int kTableMaxBatch = QC_TABLE_MAX_BATCH;
constexpr int kTableMaxSeqs = QC_TABLE_MAX_SEQS;
constexpr int kCluster = 8;
constexpr int kManySlots = 4096;      // from so many slots (or entries of the rows released) on a cluster
constexpr int kRun = 8;               // rounds of 32 adjacent slots that a warp writes before it looks for its place again

struct TableArgs {
  int32_t* pages;
  int32_t* lens;
  int32_t* free;
  int32_t* state;
  const int32_t* ids;      // null: 0, 1, ...
  const int32_t* count;    // new tokens, or tokens to keep; null: 1 each, or none
  int32_t* starts;
  int32_t* slots;
  int32_t n_seqs, max_seqs, max_pages, page_shift, n_pages, max_slots;
};

struct Sums {
  int64_t pages, tokens;
};

// Sums of a thread block's values, of which the first n_warps warps have any: before is what the threads before this one
// have, the result is the total.
__device__ __forceinline__ Sums block_scan(Sums v, Sums& before, Sums* warp_sums, int n_warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums x = v;
  if (warp < n_warps) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t p = __shfl_up_sync(0xffffffffu, x.pages, o), k = __shfl_up_sync(0xffffffffu, x.tokens, o);
      if (lane >= o) x.pages += p, x.tokens += k;
    }
  }
  __syncthreads();   // warp_sums may still be read from the sum before
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  Sums base{0, 0}, total{0, 0};
  for (int w = 0; w < n_warps; ++w) {
    if (w < warp) base.pages += warp_sums[w].pages, base.tokens += warp_sums[w].tokens;
    total.pages += warp_sums[w].pages, total.tokens += warp_sums[w].tokens;
  }
  before = Sums{base.pages + x.pages - v.pages, base.tokens + x.tokens - v.tokens};
  return total;
}

// One sequence of the call.
struct __align__(16) Seq {
  int32_t id, len;     // row of the table, tokens before the call
  int32_t first;       // pages that the sequences before it take or give back
  int32_t start;       // tokens of the sequences before it; TRIM: tokens that stay
};

// the last of n sequences whose `first` (FIRST) or `start` is <= i; both ascend from 0
template <bool FIRST>
__device__ __forceinline__ int last_not_above(const Seq* s, int n, int32_t i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((FIRST ? s[mid].first : s[mid].start) <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One block, or a cluster of them.  TRIM: give back what lies behind the tokens to keep; else take pages for the new tokens.
template <bool TRIM>
__global__ void __launch_bounds__(1024) table_kernel(const TableArgs T) {
  extern __shared__ __align__(16) uint8_t shared[];
  Seq* seqs = reinterpret_cast<Seq*>(shared);                          // [n_seqs]
  uint32_t* seen = reinterpret_cast<uint32_t*>(seqs + T.n_seqs);       // [max_seqs / 32] ids met (where ids are given)
  __shared__ Sums warp_sums[32];
  __shared__ int32_t error, free_pages;
  const int n_seqs = T.n_seqs, shift = T.page_shift, up = (1 << shift) - 1;
  const int thread = blockIdx.x * blockDim.x + threadIdx.x, n_threads = gridDim.x * blockDim.x;
  if (threadIdx.x == 0) error = 0;
  if (T.ids)
    for (int i = threadIdx.x; i < (T.max_seqs + 31) / 32; i += blockDim.x) seen[i] = 0;
  pdl_wait();
  if (threadIdx.x == 0) free_pages = T.state[0];      // (one read: all threads go the same way whatever happens to it meanwhile)
  __syncthreads();
  const int32_t n_free = free_pages;

  Sums all{0, 0};
  for (int i0 = 0; i0 < n_seqs; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    Sums mine{0, 0};
    Seq s{};
    if (i < n_seqs) {
      const int32_t count = T.count ? T.count[i] : (TRIM ? 0 : 1);
      s.id = T.ids ? T.ids[i] : i;
      int bad = 0;
      if (s.id < 0 || s.id >= T.max_seqs || count < 0) bad = QC_ERR_INVALID_ARG;
      else if (T.ids && (atomicOr(&seen[s.id >> 5], 1u << (s.id & 31)) >> (s.id & 31)) & 1u) bad = QC_ERR_STATE;
      else {
        s.len = T.lens[s.id];
        const int64_t room = static_cast<int64_t>(T.max_pages) << shift, old = s.len;
        if (old < 0 || old > room) bad = QC_ERR_STATE;
        else if (!TRIM && old + count > room) bad = QC_ERR_OOM_PAGES;
        else {
          const int64_t now = TRIM ? min(old, static_cast<int64_t>(count)) : old + count;
          const int64_t a = (old + up) >> shift, b = (now + up) >> shift;
          mine.pages = TRIM ? a - b : b - a;
          mine.tokens = TRIM ? 0 : count;
          s.start = static_cast<int32_t>(now);      // (TRIM)
        }
      }
      if (bad) atomicMax(&error, bad);
    }
    Sums before;
    const Sums sum = block_scan(mine, before, warp_sums, (min(n_seqs - i0, static_cast<int>(blockDim.x)) + 31) >> 5);
    s.first = static_cast<int32_t>(min(all.pages + before.pages, static_cast<int64_t>(INT32_MAX)));
    if (!TRIM) s.start = static_cast<int32_t>(min(all.tokens + before.tokens, static_cast<int64_t>(INT32_MAX)));
    if (i < n_seqs) seqs[i] = s;
    all.pages += sum.pages, all.tokens += sum.tokens;
  }
  __syncthreads();
  int bad = error;
  if (!bad) {
    if (n_free < 0 || n_free > T.n_pages) bad = QC_ERR_STATE;
    else if (TRIM && n_free + all.pages > T.n_pages) bad = QC_ERR_STATE;   // more pages than there are
    else if (!TRIM && all.pages > n_free) bad = QC_ERR_OOM_PAGES;
    else if (!TRIM && all.tokens > T.max_slots) bad = QC_ERR_INVALID_ARG;
  }
  if (bad) {      // (every block finds the same)
    if (thread == 0) atomicMax(&T.state[1], bad);
    if (!TRIM) {
      for (int i = thread; i <= n_seqs; i += n_threads) T.starts[i] = 0;
      for (int i = thread; i < T.max_slots; i += n_threads) T.slots[i] = -1;
    }
    return;
  }
  if (gridDim.x > 1) cluster_barrier();      // all have read
  const int32_t n_moved = static_cast<int32_t>(all.pages), n_tokens = static_cast<int32_t>(all.tokens);
  // pages, in one row over all sequences
  for (int k = thread; k < n_moved; k += n_threads) {
    const Seq s = seqs[last_not_above<true>(seqs, n_seqs, k)];
    const int32_t stay = ((TRIM ? s.start : s.len) + up) >> shift;
    int32_t* entry = T.pages + static_cast<size_t>(s.id) * T.max_pages + stay + (k - s.first);
    if (TRIM) {
      T.free[n_free + n_moved - 1 - k] = *entry;
      *entry = -1;
    } else {
      *entry = T.free[n_free - 1 - k];
    }
  }
  for (int i = thread; i < n_seqs; i += n_threads) {
    const Seq s = seqs[i];
    if (TRIM) {
      if (s.start != s.len) T.lens[s.id] = s.start;
    } else {      // (the counts may lie in the table: they are not read again)
      T.lens[s.id] = s.len + ((i + 1 < n_seqs ? seqs[i + 1].start : n_tokens) - s.start);
      T.starts[i] = s.start;
    }
  }
  if (thread == 0) {
    T.state[0] = n_free + (TRIM ? n_moved : -n_moved);
    if (!TRIM) T.starts[n_seqs] = n_tokens;
  }
  if (TRIM) return;
  // slots: a page that was there is in the table, one that is new among the free ones (which stay as they are)
  const auto slot_of = [&](int i, const Seq& s) {
    const int32_t pos = s.len + (i - s.start), page = pos >> shift, have = (s.len + up) >> shift;
    const int32_t id = page < have ? T.pages[static_cast<size_t>(s.id) * T.max_pages + page] : T.free[n_free - 1 - s.first - (page - have)];
    return (id << shift) + (pos & up);
  };
  if (gridDim.x == 1) {
    for (int i = thread; i < T.max_slots; i += n_threads) T.slots[i] = i < n_tokens ? slot_of(i, seqs[last_not_above<false>(seqs, n_seqs, i)]) : -1;
    return;
  }
  const int lane = threadIdx.x & 31;
  for (int run = thread >> 5; run * (32 * kRun) < T.max_slots; run += n_threads >> 5) {
    int i = run * (32 * kRun) + lane, seq = i < n_tokens ? last_not_above<false>(seqs, n_seqs, i) : 0;
#pragma unroll
    for (int k = 0; k < kRun; ++k, i += 32) {
      if (i < n_tokens)
        while (seq + 1 < n_seqs && seqs[seq + 1].start <= i) ++seq;
      if (i < T.max_slots) T.slots[i] = i < n_tokens ? slot_of(i, seqs[seq]) : -1;
    }
  }
}

__global__ void __launch_bounds__(256) table_reset_kernel(const TableArgs T) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x, at = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t entries = static_cast<int64_t>(T.max_seqs) * T.max_pages;
  for (int64_t i = at; i < entries; i += step) T.pages[i] = -1;
  for (int64_t i = at; i < T.max_seqs; i += step) T.lens[i] = 0;
  for (int64_t i = at; i < T.n_pages; i += step) T.free[i] = static_cast<int32_t>(T.n_pages - 1 - i);
  if (at == 0) {
    T.state[0] = T.n_pages;
    T.state[1] = T.state[2] = T.state[3] = 0;
  }
}

int32_t check_table(const qc_table* t, TableArgs& a) {
  if (!t || !t->pages_dev || !t->lens_dev || !t->free_dev || !t->state_dev) return QC_ERR_INVALID_ARG;
  if (t->page_size != 16 && t->page_size != 32 && t->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (t->max_seqs < 1 || t->max_pages < 1 || t->n_pages < 1) return QC_ERR_INVALID_ARG;
  if (t->max_seqs > kTableMaxSeqs) return QC_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(t->n_pages) * t->page_size > INT32_MAX || static_cast<int64_t>(t->max_pages) * t->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  const void* ptrs[4] = {t->pages_dev, t->lens_dev, t->free_dev, t->state_dev};
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) & 3) return QC_ERR_INVALID_ARG;
  a = TableArgs{};
  a.pages = t->pages_dev, a.lens = t->lens_dev, a.free = t->free_dev, a.state = t->state_dev;
  a.max_seqs = t->max_seqs, a.max_pages = t->max_pages, a.n_pages = t->n_pages;
  a.page_shift = t->page_size == 16 ? 4 : t->page_size == 32 ? 5 : 6;
  return QC_OK;
}

int32_t check_batch(const TableArgs& a, int32_t n_seqs, const int32_t* ids, const int32_t* count) {
  if (n_seqs < 1 || (!ids && n_seqs > a.max_seqs)) return QC_ERR_INVALID_ARG;
  if (n_seqs > kTableMaxBatch) return QC_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(ids) | reinterpret_cast<uintptr_t>(count)) & 3) return QC_ERR_INVALID_ARG;
  return QC_OK;
}

// One block of as many threads as there is work for, or a cluster; behind the launch before it, whose end it waits for.
template <bool TRIM>
int32_t launch_table(const TableArgs& a, bool many, void* cuda_stream) {
  const size_t smem = static_cast<size_t>(a.n_seqs) * sizeof(Seq) + (a.ids ? (a.max_seqs + 31) / 32 * 4 : 0);
  // 48 KB are there for a call's lists and the kernel's own variables (528 bytes) together; a longer list asks for more, well before
  // that.  (Always the most, so that two calls at once cannot take it from one another.)
  constexpr int kMost = kTableMaxBatch * static_cast<int>(sizeof(Seq)) + kTableMaxSeqs / 8;
  if (smem > 32 * 1024)
    if (const int32_t bad = status_of(cudaFuncSetAttribute(table_kernel<TRIM>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost))) return bad;
  const int32_t work = a.max_slots > a.n_seqs ? a.max_slots : a.n_seqs;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(many ? kCluster : 1);
  cfg.blockDim = dim3(many || work > 512 ? 1024 : work > 256 ? 512 : 256);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = many ? 2 : 1;
  return status_of(cudaLaunchKernelEx(&cfg, table_kernel<TRIM>, a));
}

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_table_reset(int32_t device, void* cuda_stream, const qc_table* table) {
  TableArgs a;
  if (const int32_t bad = check_table(table, a)) return bad;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  const int64_t entries = static_cast<int64_t>(a.max_seqs) * a.max_pages;
  const int64_t most = entries > a.n_pages ? entries : a.n_pages;
  const int blocks = static_cast<int>(most / 256 + 1 < 1184 ? most / 256 + 1 : 1184);
  cudaLaunchConfig_t cfg{};      // (its own status: the last error may be another call's)
  cfg.gridDim = dim3(blocks), cfg.blockDim = dim3(256), cfg.stream = static_cast<cudaStream_t>(cuda_stream);
  return status_of(cudaLaunchKernelEx(&cfg, table_reset_kernel, a));
}

extern "C" int32_t qc_table_extend(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                                   const int32_t* n_new_dev, int32_t max_slots, int32_t* starts_dev, int32_t* slots_dev) {
  TableArgs a;
  if (const int32_t bad = check_table(table, a)) return bad;
  if (const int32_t bad = check_batch(a, n_seqs, seq_ids_dev, n_new_dev)) return bad;
  if (!starts_dev || max_slots < 0 || (max_slots > 0 && !slots_dev)) return QC_ERR_INVALID_ARG;
  if (max_slots > QC_QUANT_MAX_TOKENS) return QC_ERR_UNSUPPORTED;      // (indexes of 32 bits go beyond the last one)
  if ((reinterpret_cast<uintptr_t>(starts_dev) | reinterpret_cast<uintptr_t>(slots_dev)) & 3) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  a.n_seqs = n_seqs, a.ids = seq_ids_dev, a.count = n_new_dev, a.starts = starts_dev, a.slots = slots_dev, a.max_slots = max_slots;
  return launch_table<false>(a, max_slots >= kManySlots, cuda_stream);
}

extern "C" int32_t qc_table_trim(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                                 const int32_t* n_keep_dev) {
  TableArgs a;
  if (const int32_t bad = check_table(table, a)) return bad;
  if (const int32_t bad = check_batch(a, n_seqs, seq_ids_dev, n_keep_dev)) return bad;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  a.n_seqs = n_seqs, a.ids = seq_ids_dev, a.count = n_keep_dev;
  // a release may give back every page of its rows; drafts that are turned down give back a few
  return launch_table<true>(a, !n_keep_dev && static_cast<int64_t>(n_seqs) * a.max_pages >= kManySlots, cuda_stream);
}
