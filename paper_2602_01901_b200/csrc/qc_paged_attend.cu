// Attention of a step's queries over bf16 pages, where adjacent sequences of a batch share a prefix.
//
//   out = softmax(scale [q_shared K_prefix ; q_own K_own]) [V_prefix ; V_own]

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

struct StreamArgs {
  const uint16_t* q;
  int64_t q_stride;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* pages;
  const int32_t* lens;
  int32_t max_pages, n_pages, rows;
};

struct AttendArgs {
  StreamArgs stream[2];   // own, shared
  const int32_t* ids;
  const int32_t* starts;
  const int32_t* groups;
  const int32_t* shared_ids;
  uint16_t* out;
  float* lse;
  int32_t* plan;          // [1] whether the batch is computed
  int32_t* status;
  int32_t hq, hkv, group, page, page_shift;
  int32_t n_seqs, n_groups, n_tokens, max_queries, causal;
  float scale_log2;
};

__device__ __forceinline__ void report(const AttendArgs& A, int code) {
  if (A.status) atomicMax(A.status, code);
}

__device__ __forceinline__ int length_of(const AttendArgs& A, const StreamArgs& S, int row) {
  const int64_t len = __ldg(S.lens + row), room = static_cast<int64_t>(S.max_pages) << A.page_shift;
  if (len >= 0 && len <= room) return static_cast<int>(len);
  report(A, QC_ERR_PLAN);
  return len < 0 ? 0 : static_cast<int>(room);
}

struct Seq {
  int32_t token0, queries, row;
};
__device__ __forceinline__ bool seq_of(const AttendArgs& A, int i, Seq& s) {
  int64_t a = i, b = i + 1;
  if (A.starts) a = __ldg(A.starts + i), b = __ldg(A.starts + i + 1);
  s.token0 = static_cast<int32_t>(a), s.queries = static_cast<int32_t>(b - a), s.row = A.ids ? __ldg(A.ids + i) : i;
  return a >= 0 && b >= a && b <= A.n_tokens && b - a <= A.max_queries && s.row >= 0 && s.row < A.stream[0].rows;
}

struct Group {
  int32_t first, last, row;
};
__device__ __forceinline__ bool group_of(const AttendArgs& A, int g, Group& u) {
  u.first = A.groups ? __ldg(A.groups + g) : 0, u.last = A.groups ? __ldg(A.groups + g + 1) : A.n_seqs;
  u.row = A.shared_ids ? __ldg(A.shared_ids + g) : g;
  return u.first >= 0 && u.last >= u.first && u.last <= A.n_seqs && u.row >= 0 && u.row < A.stream[1].rows;
}

__global__ void __launch_bounds__(256) paged_plan_kernel(const __grid_constant__ AttendArgs A) {
  pdl_wait();
  bool fine = true;
  Seq s;
  Group u;
  for (int i = threadIdx.x; i < A.n_seqs; i += 256) fine &= seq_of(A, i, s);
  for (int i = threadIdx.x; i < A.n_groups; i += 256) fine &= group_of(A, i, u);
  fine = __syncthreads_and(fine);
  if (threadIdx.x == 0) {
    A.plan[0] = fine;
    if (!fine) report(A, QC_ERR_INVALID_ARG);
  }
}

// One warp per row: a key at a time.
template <int D>
__device__ __forceinline__ void sweep(const AttendArgs& A, const StreamArgs& S, int row, int kvh, int64_t token, int head, int seen, float (&o)[D / 32], float& m,
                                      float& l, int lane) {
  float q[D / 32], k[D / 32];
  const auto load = [&](const uint16_t* p, float (&f)[D / 32]) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const float2 x = bf16x2_to_f32(__ldg(reinterpret_cast<const uint32_t*>(p) + i * 32 + lane));
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  };
  load(S.q + token * S.q_stride + static_cast<int64_t>(head) * D, q);
  for (int j = 0; j < seen; ++j) {
    const int32_t id = __ldg(S.pages + static_cast<int64_t>(row) * S.max_pages + (j >> A.page_shift));
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(S.n_pages)) {
      report(A, QC_ERR_BAD_PAGE);
      continue;
    }
    const int64_t at = (((static_cast<int64_t>(id) * A.hkv + kvh) << A.page_shift) + (j & (A.page - 1))) * D;
    load(S.k_pool + at, k);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= A.scale_log2;
    const float top = fmaxf(m, s);
    if (s == -INFINITY) continue;      // (weighs nothing)
    const float before = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(m - top), p = exp2f(s - (top == -INFINITY ? 0.f : top));   // (a score that is no number has no place in an order)
    load(S.v_pool + at, k);
    l = fmaf(l, before, p);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = fmaf(o[i], before, p * k[i]);
    m = top;
  }
}

// Grid: (sequences, query heads).
template <int D>
__global__ void __launch_bounds__(128) paged_attend_kernel(const __grid_constant__ AttendArgs A) {
  pdl_wait();
  if (!A.plan[0]) return;
  const int seq = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, kvh = head / A.group;
  Seq s;
  seq_of(A, seq, s);
  int prefix = 0, shared_row = 0;
  for (int g = 0; g < A.n_groups; ++g) {
    Group u;
    group_of(A, g, u);
    if (seq >= u.first && seq < u.last) prefix = length_of(A, A.stream[1], u.row), shared_row = u.row;
  }
  const int len = length_of(A, A.stream[0], s.row);
  for (int i = threadIdx.x >> 5; i < s.queries; i += 4) {
    float o[D / 32] = {}, m = -INFINITY, l = 0.f;
    const int64_t token = s.token0 + i;
    if (prefix) sweep<D>(A, A.stream[1], shared_row, kvh, token, head, prefix, o, m, l, lane);
    sweep<D>(A, A.stream[0], s.row, kvh, token, head, A.causal ? len - (s.queries - 1 - i) : len, o, m, l, lane);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const size_t row = token * A.hq + head;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) reinterpret_cast<uint32_t*>(A.out + row * D)[x * 32 + lane] = pack_bf16x2(o[2 * x] * inv, o[2 * x + 1] * inv);
    if (A.lse && lane == 0) A.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

bool off(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

int32_t check_stream(const qc_paged_stream* s, const qc_paged_attend_args* a, StreamArgs& d) {
  if (!s->q_dev || !s->k_pool_dev || !s->v_pool_dev || !s->pages_dev || !s->lens_dev) return QC_ERR_INVALID_ARG;
  if (off(s->q_dev, 16) || off(s->k_pool_dev, 16) || off(s->v_pool_dev, 16) || off(s->pages_dev, 4) || off(s->lens_dev, 4)) return QC_ERR_INVALID_ARG;
  if (s->q_stride < 0 || s->q_stride % 8 || s->max_pages < 1 || s->n_pages < 1 || s->rows < 1) return QC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(s->max_pages) * a->page_size > INT32_MAX - 4096 || static_cast<int64_t>(s->n_pages) * a->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(s->n_pages) * a->page_size * a->n_kv_heads > INT32_MAX) return QC_ERR_UNSUPPORTED;      // (a tile copy's row is a number of 32 bits)
  d = {static_cast<const uint16_t*>(s->q_dev), s->q_stride, static_cast<const uint16_t*>(s->k_pool_dev), static_cast<const uint16_t*>(s->v_pool_dev),
       s->pages_dev, s->lens_dev, s->max_pages, s->n_pages, s->rows};
  return QC_OK;
}

bool has_stream(const qc_paged_stream& s) { return s.q_dev || s.k_pool_dev || s.v_pool_dev || s.pages_dev || s.lens_dev; }

int32_t check_sizes(const qc_paged_attend_args* a) {
  if (!a) return QC_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (a->page_size != 16 && a->page_size != 32 && a->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (a->n_kv_heads < 1 || a->n_q_heads < 1 || a->n_q_heads % a->n_kv_heads || a->n_seqs < 1 || a->n_tokens < 0 || a->max_queries < 1 || a->n_groups < 0)
    return QC_ERR_INVALID_ARG;
  if (a->n_kv_heads > QC_PAGED_MAX_HEADS || a->n_q_heads > QC_PAGED_MAX_HEADS || a->n_seqs > QC_PAGED_MAX_SEQS || a->max_queries > QC_PAGED_MAX_QUERIES ||
      a->n_groups > QC_PAGED_MAX_SEQS)
    return QC_ERR_UNSUPPORTED;
  if (a->n_tokens > QC_PAGED_MAX_TOKENS) return QC_ERR_UNSUPPORTED;
  return QC_OK;
}

size_t workspace_bytes(const qc_paged_attend_args* a) { return 256; }

// Whether the rows written lie over rows of queries.
bool over_queries(const qc_paged_stream& s, const qc_paged_attend_args* a) {
  const uint64_t row = static_cast<uint64_t>(a->n_q_heads) * a->head_dim * 2, n = a->n_tokens;
  const uint64_t q = reinterpret_cast<uint64_t>(s.q_dev), out = reinterpret_cast<uint64_t>(a->out_dev);
  return q < out + row * n && out < q + static_cast<uint64_t>(s.q_stride) * 2 * (n - 1) + row;
}

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_paged_workspace_bytes(const qc_paged_attend_args* args, size_t* bytes) {
  if (!bytes) return QC_ERR_INVALID_ARG;
  if (const int32_t bad = check_sizes(args)) return bad;
  *bytes = workspace_bytes(args);
  return QC_OK;
}

extern "C" int32_t qc_paged_attend(int32_t device, void* cuda_stream, const qc_paged_attend_args* args) {
  if (const int32_t bad = check_sizes(args)) return bad;
  if (!args->out_dev || off(args->out_dev, 16) || off(args->lse_out_dev, 4) || off(args->status_dev, 4) || off(args->seq_ids_dev, 4) || off(args->starts_dev, 4) ||
      off(args->groups_dev, 4) || off(args->shared_ids_dev, 4) || off(args->workspace_dev, 16))
    return QC_ERR_INVALID_ARG;
  if (!(args->softmax_scale >= 0.f) || !isfinite(args->softmax_scale)) return QC_ERR_INVALID_ARG;
  if (!args->starts_dev && args->n_tokens < args->n_seqs) return QC_ERR_INVALID_ARG;
  AttendArgs A{};
  if (const int32_t bad = check_stream(&args->own, args, A.stream[0])) return bad;
  if (!args->seq_ids_dev && args->n_seqs > args->own.rows) return QC_ERR_INVALID_ARG;
  const bool shared = has_stream(args->shared);
  if (shared) {
    if (const int32_t bad = check_stream(&args->shared, args, A.stream[1])) return bad;
    if (!args->groups_dev && args->n_groups != 1) return QC_ERR_INVALID_ARG;
    if (!args->shared_ids_dev && args->n_groups > args->shared.rows) return QC_ERR_INVALID_ARG;
  } else if (args->n_groups != 0 || args->groups_dev || args->shared_ids_dev) {
    return QC_ERR_INVALID_ARG;
  }
  if (args->workspace_bytes < workspace_bytes(args) || !args->workspace_dev) return QC_ERR_INVALID_ARG;
  if (args->n_tokens == 0) return QC_OK;
  if (over_queries(args->own, args) || (shared && over_queries(args->shared, args))) return QC_ERR_INVALID_ARG;
  A.ids = args->seq_ids_dev, A.starts = args->starts_dev, A.groups = args->groups_dev, A.shared_ids = args->shared_ids_dev;
  A.out = static_cast<uint16_t*>(args->out_dev), A.lse = args->lse_out_dev, A.status = args->status_dev;
  A.plan = static_cast<int32_t*>(args->workspace_dev);
  A.hq = args->n_q_heads, A.hkv = args->n_kv_heads, A.group = A.hq / A.hkv, A.page = args->page_size;
  A.page_shift = A.page == 16 ? 4 : A.page == 32 ? 5 : 6;
  A.n_seqs = args->n_seqs, A.n_groups = args->n_groups, A.n_tokens = args->n_tokens, A.max_queries = args->max_queries, A.causal = args->causal != 0;
  const float scale = args->softmax_scale > 0.f ? args->softmax_scale : 1.0f / sqrtf(static_cast<float>(args->head_dim));
  A.scale_log2 = scale * 1.4426950408889634f;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (const int32_t bad = status_of(launch_pdl(paged_plan_kernel, dim3(1), dim3(256), 0, stream, A))) return bad;
  return status_of(launch_pdl(args->head_dim == 128 ? paged_attend_kernel<128> : paged_attend_kernel<64>, dim3(A.n_seqs, A.hq), dim3(128), 0, stream, A));
}
