// Page tables of one stream that live on the device: lengths, page ids, the free pages as a stack.
// A step's bookkeeping (how many pages every sequence takes or gives back, which ones, and the slot
// of every new token) is prefix sums over the batch, done by one thread block that holds the whole
// batch's numbers in shared memory, so a step can be captured into a graph and replayed while its
// sequences grow.
//
//   have_i = ceil(len_i / P), want_i = ceil((len_i + new_i) / P), first_i = sum_{j<i} (want_j - have_j)
//   page (have_i + c) of sequence i = free[n_free - 1 - first_i - c]
//   start_i = sum_{j<i} new_j;  token i of the call: slot = page * P + position % P
//
// Trimming is the inverse: what it gives back is taken again in the same order.  Nothing is changed
// when the call cannot be carried out as a whole.  What bounds it is the launch and three dependent
// trips to the L2 (ids, lengths, free pages); the bytes (some KB) do not count.

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

constexpr int kTableMaxBatch = QC_TABLE_MAX_BATCH;
constexpr int kTableMaxSeqs = QC_TABLE_MAX_SEQS;
constexpr int kSlotsInBlock = 8192;   // more slots than that are written by a launch of their own

struct TableArgs {
  int32_t* pages;
  int32_t* lens;
  int32_t* free;
  int32_t* state;
  const int32_t* ids;      // null: 0, 1, ...
  const int32_t* count;    // new tokens, or tokens to keep; null: 1 each, or none
  int32_t* starts;
  int32_t* slots;
  int32_t n_seqs, max_seqs, max_pages, page, n_pages, max_slots;
};

// Sums of a thread block's values: *before is what the threads before this one have, the result is the total.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* before, int64_t* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();   // warp_sums may still be read from the sum before
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int64_t base = 0, total = 0;
  for (int w = 0; w < n_warps; ++w) {
    if (w < warp) base += warp_sums[w];
    total += warp_sums[w];
  }
  *before = base + x - v;
  return total;
}

// the last index whose entry is <= i, of n entries in ascending order (entry 0 is 0)
__device__ __forceinline__ int last_not_above(const int32_t* a, int n, int32_t i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int32_t slot_of(const TableArgs& T, int seq, int32_t len, int32_t end, int32_t i) {
  const int32_t id = T.ids ? T.ids[seq] : seq;
  const int32_t pos = len - (end - i);
  return T.pages[static_cast<size_t>(id) * T.max_pages + pos / T.page] * T.page + pos % T.page;
}

// One block.  TRIM: give back what lies behind the tokens to keep; else take pages for the new tokens.
template <bool TRIM>
__global__ void __launch_bounds__(1024) table_kernel(const TableArgs T) {
  extern __shared__ int32_t shared[];
  int32_t* first = shared;                       // [n_seqs] pages that the sequences before take or give back
  int32_t* keep = first + T.n_seqs;              // [n_seqs] pages that stay, or are there before
  int32_t* start = keep + T.n_seqs;              // [n_seqs] tokens of the sequences before (not TRIM)
  uint32_t* seen = reinterpret_cast<uint32_t*>(start + (TRIM ? 0 : T.n_seqs));   // [max_seqs / 32] ids met (where ids are given)
  __shared__ int64_t warp_sums[32];
  __shared__ int32_t error;
  const int n_seqs = T.n_seqs, page = T.page;
  if (threadIdx.x == 0) error = 0;
  if (T.ids)
    for (int i = threadIdx.x; i < (T.max_seqs + 31) / 32; i += blockDim.x) seen[i] = 0;
  pdl_wait();
  __syncthreads();
  const int32_t n_free = T.state[0];

  int64_t pages_total = 0, tokens_total = 0;
  for (int i0 = 0; i0 < n_seqs; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    int64_t moved = 0, tokens = 0;
    if (i < n_seqs) {
      const int32_t id = T.ids ? T.ids[i] : i, count = T.count ? T.count[i] : (TRIM ? 0 : 1);
      int bad = 0;
      if (id < 0 || id >= T.max_seqs || count < 0) bad = QC_ERR_INVALID_ARG;
      else if (T.ids && (atomicOr(&seen[id >> 5], 1u << (id & 31)) >> (id & 31)) & 1u) bad = QC_ERR_STATE;
      else {
        const int64_t old = T.lens[id], room = static_cast<int64_t>(T.max_pages) * page;
        if (old < 0 || old > room) bad = QC_ERR_STATE;
        else if (!TRIM && old + count > room) bad = QC_ERR_OOM_PAGES;
        else {
          const int64_t now = TRIM ? min(old, static_cast<int64_t>(count)) : old + count;
          const int64_t a = (old + page - 1) / page, b = (now + page - 1) / page;
          moved = TRIM ? a - b : b - a;
          keep[i] = static_cast<int32_t>(TRIM ? b : a);
          tokens = TRIM ? 0 : count;
        }
      }
      if (bad) atomicMax(&error, bad);
    }
    int64_t before;
    const int64_t sum = block_scan(moved, &before, warp_sums);
    if (i < n_seqs) first[i] = static_cast<int32_t>(min(pages_total + before, static_cast<int64_t>(INT32_MAX)));
    pages_total += sum;
    if (!TRIM) {
      const int64_t more = block_scan(tokens, &before, warp_sums);
      if (i < n_seqs) start[i] = static_cast<int32_t>(min(tokens_total + before, static_cast<int64_t>(INT32_MAX)));
      tokens_total += more;
    }
  }
  __syncthreads();
  int bad = error;
  if (!bad) {
    if (n_free < 0 || n_free > T.n_pages) bad = QC_ERR_STATE;
    else if (TRIM && n_free + pages_total > T.n_pages) bad = QC_ERR_STATE;   // more pages than there are
    else if (!TRIM && pages_total > n_free) bad = QC_ERR_OOM_PAGES;
    else if (!TRIM && tokens_total > T.max_slots) bad = QC_ERR_INVALID_ARG;
  }
  if (bad) {
    if (threadIdx.x == 0) atomicMax(&T.state[1], bad);
    if (!TRIM) {
      for (int i = threadIdx.x; i <= n_seqs; i += blockDim.x) T.starts[i] = 0;
      if (T.max_slots <= kSlotsInBlock)
        for (int i = threadIdx.x; i < T.max_slots; i += blockDim.x) T.slots[i] = -1;
    }
    return;
  }
  // pages, in one row over all sequences
  for (int k = threadIdx.x; k < static_cast<int>(pages_total); k += blockDim.x) {
    const int i = last_not_above(first, n_seqs, k);
    const int32_t id = T.ids ? T.ids[i] : i;
    int32_t* entry = T.pages + static_cast<size_t>(id) * T.max_pages + keep[i] + (k - first[i]);
    if (TRIM) {
      T.free[n_free + static_cast<int>(pages_total) - 1 - k] = *entry;
      *entry = -1;
    } else {
      *entry = T.free[n_free - 1 - k];
    }
  }
  for (int i = threadIdx.x; i < n_seqs; i += blockDim.x) {
    const int32_t id = T.ids ? T.ids[i] : i;
    if (TRIM) {
      const int32_t count = T.count ? T.count[i] : 0;
      if (count < T.lens[id]) T.lens[id] = count;
    } else {
      T.lens[id] += T.count ? T.count[i] : 1;
      T.starts[i] = start[i];
    }
  }
  if (threadIdx.x == 0) {
    T.state[0] = n_free + static_cast<int32_t>(TRIM ? pages_total : -pages_total);
    if (!TRIM) T.starts[n_seqs] = static_cast<int32_t>(tokens_total);
  }
  if (TRIM || T.max_slots > kSlotsInBlock) return;
  __syncthreads();   // this block wrote the pages and lengths that the slots are made from
  for (int i = threadIdx.x; i < T.max_slots; i += blockDim.x) {
    int32_t slot = -1;
    if (i < tokens_total) {
      const int seq = last_not_above(start, n_seqs, i);
      slot = slot_of(T, seq, T.lens[T.ids ? T.ids[seq] : seq], seq + 1 < n_seqs ? start[seq + 1] : static_cast<int32_t>(tokens_total), i);
    }
    T.slots[i] = slot;
  }
}

// The slots of a long call, from what table_kernel has left (no tokens where it refused).
__global__ void __launch_bounds__(256) slots_kernel(const TableArgs T) {
  pdl_wait();
  const int32_t total = T.starts[T.n_seqs];
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < T.max_slots; i += gridDim.x * blockDim.x) {
    int32_t slot = -1;
    if (i < total) {
      const int seq = last_not_above(T.starts, T.n_seqs, i);
      slot = slot_of(T, seq, T.lens[T.ids ? T.ids[seq] : seq], T.starts[seq + 1], i);
    }
    T.slots[i] = slot;
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
  a.max_seqs = t->max_seqs, a.max_pages = t->max_pages, a.page = t->page_size, a.n_pages = t->n_pages;
  return QC_OK;
}

int32_t check_batch(const TableArgs& a, int32_t n_seqs, const int32_t* ids, const int32_t* count) {
  if (n_seqs < 1 || (!ids && n_seqs > a.max_seqs)) return QC_ERR_INVALID_ARG;
  if (n_seqs > kTableMaxBatch) return QC_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(ids) | reinterpret_cast<uintptr_t>(count)) & 3) return QC_ERR_INVALID_ARG;
  return QC_OK;
}

int threads_for(int32_t n) { return n <= 256 ? 256 : n <= 512 ? 512 : 1024; }

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
  table_reset_kernel<<<blocks, 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? QC_OK : QC_ERR_CUDA;
}

extern "C" int32_t qc_table_extend(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                                   const int32_t* n_new_dev, int32_t max_slots, int32_t* starts_dev, int32_t* slots_dev) {
  TableArgs a;
  if (const int32_t bad = check_table(table, a)) return bad;
  if (const int32_t bad = check_batch(a, n_seqs, seq_ids_dev, n_new_dev)) return bad;
  if (!starts_dev || max_slots < 0 || (max_slots > 0 && !slots_dev)) return QC_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(starts_dev) | reinterpret_cast<uintptr_t>(slots_dev)) & 3) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  a.n_seqs = n_seqs, a.ids = seq_ids_dev, a.count = n_new_dev, a.starts = starts_dev, a.slots = slots_dev, a.max_slots = max_slots;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const size_t smem = static_cast<size_t>(n_seqs) * 12 + (seq_ids_dev ? (a.max_seqs + 31) / 32 * 4 : 0);
  if (smem > 48 * 1024 && cudaFuncSetAttribute(table_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) return QC_ERR_CUDA;
  const int32_t work = max_slots <= kSlotsInBlock && max_slots > n_seqs ? max_slots : n_seqs;
  if (launch_pdl(table_kernel<false>, dim3(1), dim3(threads_for(work)), smem, stream, a) != cudaSuccess) return QC_ERR_CUDA;
  if (max_slots > kSlotsInBlock) {
    const int blocks = max_slots / 256 + 1 < 1184 ? max_slots / 256 + 1 : 1184;
    if (launch_pdl(slots_kernel, dim3(blocks), dim3(256), 0, stream, a) != cudaSuccess) return QC_ERR_CUDA;
  }
  return QC_OK;
}

extern "C" int32_t qc_table_trim(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                                 const int32_t* n_keep_dev) {
  TableArgs a;
  if (const int32_t bad = check_table(table, a)) return bad;
  if (const int32_t bad = check_batch(a, n_seqs, seq_ids_dev, n_keep_dev)) return bad;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  a.n_seqs = n_seqs, a.ids = seq_ids_dev, a.count = n_keep_dev;
  const size_t smem = static_cast<size_t>(n_seqs) * 8 + (seq_ids_dev ? (a.max_seqs + 31) / 32 * 4 : 0);
  if (smem > 48 * 1024 && cudaFuncSetAttribute(table_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) return QC_ERR_CUDA;
  return launch_pdl(table_kernel<true>, dim3(1), dim3(threads_for(n_seqs)), smem, static_cast<cudaStream_t>(cuda_stream), a) == cudaSuccess ? QC_OK : QC_ERR_CUDA;
}
