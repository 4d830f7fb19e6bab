// Rows of queries and keys normalised and turned by their positions, to a tensor or to their places in a cache's pages.
//
//   y = x / sqrt(mean x^2 + eps) * w, then (a, b) -> (a cos - b sin, b cos + a sin) for pair i by positions[axis of i] * freqs[i]
//
// Bound by its bytes (a row in, a row out).  The angles are a token's, not a head's: a block works them out once for its
// tokens, a thread per pair, and its warps turn all heads with them.  An angle is counted in turns, as a fraction of 64 bits:
// freq / 2 pi modulo 1 once, times the position modulo 2^64, so a far position loses nothing (in fp32 position 100 000 is 6e-3
// radians off), and sine and cosine are taken of a number in [-1, 1) half turns.
// A row is held by D / 16 lanes, two 16-byte vectors each: those whose pairs the lane turns, so that no element changes lanes.
// The squares' sum takes 3 exchanges.

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

constexpr int kRowThreads = 256;
constexpr int kMaxTokens = 16;      // tokens of a block

struct Rows {                       // q, k or v
  const uint16_t* x;
  int64_t stride;
  uint16_t* out;                    // null: to the pool
  int64_t out_stride;
  const void* norm;
};

struct RotateArgs {
  Rows q, k, v;
  uint16_t* k_pool;
  uint16_t* v_pool;
  const float* freqs;
  const int32_t* axes;
  const int32_t* positions;
  int64_t position_stride;
  const int32_t* slots;
  int32_t n_tokens, hq, hk, hv;     // heads of q, k and v that there are
  int32_t heads, rows;              // heads of the pools; hq + hk + hv
  int32_t pairs, n_axes, norm_f32;
  int32_t page_shift, n_slots;
  int32_t tokens, chunk;            // of a block: tokens, and rows of a token
  float inv_chunk, eps;
};

// The angle of a pair at a position, as (cos, sin).
__device__ __forceinline__ float2 turn_of(float freq, int32_t position) {
  const double turns = static_cast<double>(freq) * 0.15915494309189533577;
  const unsigned long long part = __double2ull_rn((turns - floor(turns)) * 18446744073709551616.0);
  const unsigned long long at = part * static_cast<unsigned long long>(static_cast<long long>(position));
  float2 cs;
  sincospif(static_cast<float>(static_cast<int32_t>(at >> 32)) * 4.656612873077392578125e-10f, &cs.y, &cs.x);   // 2^-31
  return isfinite(freq) ? cs : make_float2(NAN, NAN);
}

// Where a lane's pair i (of 8) of the block's token is: pairs (i, i + 1) of all lanes follow one another, so that the lanes of a
// row read 16 bytes each from adjacent places.
template <int D>
__device__ __forceinline__ int place_of(int token, int pair) {
  constexpr int kLanes = D / 16;
  return token * (D / 2) + ((pair % 8) / 2 * kLanes + pair / 8) * 2 + pair % 2;
}

__device__ __forceinline__ void weights_of(const void* norm, int f32, int vector, float (&w)[8]) {
  if (f32) {
    const float4* p = static_cast<const float4*>(norm) + 2 * vector;
    const float4 a = __ldg(p), b = __ldg(p + 1);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  } else {
    bf16x8_to_f32(__ldg(static_cast<const uint4*>(norm) + vector), w);
  }
}

// Grid: (tokens / T.tokens, rows of a token / T.chunk).  ADJ: pairs are neighbours.
template <int D, bool ADJ>
__global__ void __launch_bounds__(kRowThreads, 4) rotate_kernel(const __grid_constant__ RotateArgs T) {
  constexpr int kLanes = D / 16, kPass = kRowThreads / kLanes;      // rows of a pass of the block
  __shared__ __align__(16) float2 turns[kMaxTokens * (D / 2)];
  pdl_wait();
  const int token0 = blockIdx.x * T.tokens, tokens = min(T.tokens, T.n_tokens - token0);
  const int row0 = blockIdx.y * T.chunk, chunk = min(T.chunk, T.rows - row0), n = tokens * chunk;
  const int j = threadIdx.x % kLanes;
  // the lane's two vectors: those with its pairs, or what is left of a row that turns in part
  const int turning = T.pairs / 8;
  const bool turns_here = j < turning;
  const int a = ADJ || !turns_here ? 2 * j : j, b = ADJ || !turns_here ? 2 * j + 1 : turning + j;

  struct Row {
    uint4 x, y;
    int token, row;
  };
  const auto fetch = [&](Row& r, int i) {
    // (a short last chunk divides by another number)
    r.token = chunk == T.chunk ? static_cast<int>((static_cast<float>(i) + 0.5f) * T.inv_chunk) : i / chunk;
    r.row = row0 + i - r.token * chunk;
    const Rows& s = r.row < T.hq ? T.q : r.row < T.hq + T.hk ? T.k : T.v;
    const int head = r.row < T.hq ? r.row : r.row < T.hq + T.hk ? r.row - T.hq : r.row - T.hq - T.hk;
    const uint4* p = reinterpret_cast<const uint4*>(s.x + (token0 + r.token) * s.stride + static_cast<int64_t>(head) * D);
    r.x = p[a], r.y = p[b];
  };
  Row next{};
  int i = threadIdx.x / kLanes;
  if (i < n) fetch(next, i);

  for (int e = threadIdx.x; e < tokens * T.pairs; e += kRowThreads) {
    const int token = e / T.pairs, pair = e - token * T.pairs, axis = T.axes ? __ldg(T.axes + pair) : 0;
    float2 cs = make_float2(NAN, NAN);
    if (static_cast<uint32_t>(axis) < static_cast<uint32_t>(T.n_axes))
      cs = turn_of(__ldg(T.freqs + pair), __ldg(T.positions + axis * T.position_stride + token0 + token));
    turns[place_of<D>(token, pair)] = cs;
  }
  __syncthreads();

#pragma unroll 1
  for (; i - threadIdx.x / kLanes < n; i += kPass) {      // (all lanes of a warp: they exchange sums)
    const Row r = next;
    const bool there = i < n;
    if (i + kPass < n) fetch(next, i + kPass);
    const bool is_q = r.row < T.hq, is_v = r.row >= T.hq + T.hk;
    uint4 x = r.x, y = r.y;
    const void* norm = is_q ? T.q.norm : T.k.norm;
    float f[16];
    bf16x8_to_f32(x, f);
    bf16x8_to_f32(y, f + 8);
    float scale = 1.f;
    if (T.q.norm || T.k.norm) {
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int c = 0; c < 16; c += 4) {
        s0 = fma2(make_float2(f[c], f[c + 1]), make_float2(f[c], f[c + 1]), s0);
        s1 = fma2(make_float2(f[c + 2], f[c + 3]), make_float2(f[c + 2], f[c + 3]), s1);
      }
      float sum = (s0.x + s0.y) + (s1.x + s1.y);
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      scale = rsqrtf(sum * (1.f / D) + T.eps);
    }
    if (!there) continue;
    if (!is_v) {
      if (norm) {
        float w[8];
        weights_of(norm, T.norm_f32, a, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) f[c] *= scale * w[c];
        weights_of(norm, T.norm_f32, b, w);
#pragma unroll
        for (int c = 0; c < 8; ++c) f[8 + c] *= scale * w[c];
      }
      if (turns_here) {
        const float4* cs = reinterpret_cast<const float4*>(turns + r.token * (D / 2)) + j;
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          const float4 t = cs[c / 2 * kLanes];
          float &u0 = f[ADJ ? 2 * c : c], &v0 = f[ADJ ? 2 * c + 1 : 8 + c], &u1 = f[ADJ ? 2 * c + 2 : c + 1], &v1 = f[ADJ ? 2 * c + 3 : 9 + c];
          const float p0 = u0, q0 = v0, p1 = u1, q1 = v1;
          u0 = p0 * t.x - q0 * t.y, v0 = q0 * t.x + p0 * t.y;
          u1 = p1 * t.z - q1 * t.w, v1 = q1 * t.z + p1 * t.w;
        }
      }
      x = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
      y = make_uint4(pack_bf16x2(f[8], f[9]), pack_bf16x2(f[10], f[11]), pack_bf16x2(f[12], f[13]), pack_bf16x2(f[14], f[15]));
    }
    const int head = is_q ? r.row : is_v ? r.row - T.hq - T.hk : r.row - T.hq;
    uint16_t* to;
    if (is_q || (!is_v && T.k.out)) {
      const Rows& s = is_q ? T.q : T.k;
      to = s.out + (token0 + r.token) * s.out_stride + static_cast<int64_t>(head) * D;
    } else {
      const int32_t slot = __ldg(T.slots + token0 + r.token);
      if (static_cast<uint32_t>(slot) >= static_cast<uint32_t>(T.n_slots)) continue;
      const int32_t page = slot >> T.page_shift, in_page = slot & ((1 << T.page_shift) - 1);
      to = (is_v ? T.v_pool : T.k_pool) + (((static_cast<int64_t>(page) * T.heads + head) << T.page_shift) + in_page) * D;
    }
    reinterpret_cast<uint4*>(to)[a] = x;
    reinterpret_cast<uint4*>(to)[b] = y;
  }
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

// Memory as `count` runs of `bytes`, `stride` bytes apart.
struct Span {
  uint64_t at, bytes, stride, count;
  uint64_t end() const { return at + stride * (count - 1) + bytes; }
};
Span rows_span(const void* p, int64_t stride, int32_t heads, int32_t head_dim, int32_t n) {
  return {reinterpret_cast<uint64_t>(p), static_cast<uint64_t>(heads) * head_dim * 2, static_cast<uint64_t>(stride) * 2, static_cast<uint64_t>(n)};
}
Span flat_span(const void* p, uint64_t bytes) { return {reinterpret_cast<uint64_t>(p), bytes, 0, 1}; }

// Whether two such have a byte in common (runs that lie between those of another with the same stride have none; with
// different strides what lies between counts as theirs).
bool meet(const Span& a, const Span& b) {
  if (!a.at || !b.at || a.end() <= b.at || b.end() <= a.at) return false;
  if (a.count == 1 || b.count == 1 || a.stride != b.stride) {
    const Span &one = a.count == 1 ? a : b, &many = a.count == 1 ? b : a;
    if (one.count != 1 || many.count == 1 || many.stride == 0) return true;
    if (one.at < many.at) return true;                               // (they meet as wholes, so it reaches into the first run)
    const uint64_t in = (one.at - many.at) % many.stride;
    return in < many.bytes || in + one.bytes > many.stride;
  }
  if (a.stride == 0) return true;
  const uint64_t apart = (a.at < b.at ? b.at - a.at : a.at - b.at) % a.stride;
  const uint64_t first = a.at < b.at ? a.bytes : b.bytes, second = a.at < b.at ? b.bytes : a.bytes;
  return apart < first || apart + second > a.stride;
}

int32_t check_rotate(const qc_rotate_args* a, bool to_pool, RotateArgs& T) {
  if (!a) return QC_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (a->n_tokens < 0 || a->n_q_heads < 0 || a->n_kv_heads < 0) return QC_ERR_INVALID_ARG;
  if (a->n_tokens > QC_PAGED_MAX_TOKENS || a->n_q_heads > QC_PAGED_MAX_HEADS || a->n_kv_heads > QC_PAGED_MAX_HEADS) return QC_ERR_UNSUPPORTED;
  if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 16) return QC_ERR_INVALID_ARG;
  if ((a->q_dev && a->n_q_heads < 1) || (a->k_dev && a->n_kv_heads < 1) || (!a->q_dev) != (!a->q_out_dev)) return QC_ERR_INVALID_ARG;
  if (to_pool ? a->k_out_dev != nullptr : (!a->k_dev) != (!a->k_out_dev)) return QC_ERR_INVALID_ARG;
  if (off16(a->q_dev) || off16(a->q_out_dev) || off16(a->k_dev) || off16(a->k_out_dev) || off16(a->q_norm_dev) || off16(a->k_norm_dev)) return QC_ERR_INVALID_ARG;
  const int64_t q_row = static_cast<int64_t>(a->n_q_heads) * a->head_dim, k_row = static_cast<int64_t>(a->n_kv_heads) * a->head_dim;
  const auto bad_stride = [&](const void* p, int64_t stride, int64_t least) { return p && (stride < 0 || stride % 8 || (a->n_tokens > 1 && stride < least)); };
  if (bad_stride(a->q_dev, a->q_stride, 0) || bad_stride(a->k_dev, a->k_stride, 0) || bad_stride(a->q_out_dev, a->q_out_stride, q_row) ||
      bad_stride(a->k_out_dev, a->k_out_stride, k_row))
    return QC_ERR_INVALID_ARG;
  if (!(a->eps >= 0.f) || !isfinite(a->eps)) return QC_ERR_INVALID_ARG;
  if (a->rotary_dim && (a->q_dev || a->k_dev)) {
    if (a->n_axes < 1 || !a->freqs_dev || off4(a->freqs_dev) || off4(a->axes_dev) || off4(a->positions_dev) || (!a->positions_dev && a->n_tokens)) return QC_ERR_INVALID_ARG;
    if (a->n_axes > QC_ROTATE_MAX_AXES) return QC_ERR_UNSUPPORTED;
    if (a->n_axes > 1 && a->position_stride < 0) return QC_ERR_INVALID_ARG;
    T.pairs = a->rotary_dim / 2;
  }
  T.freqs = a->freqs_dev, T.axes = a->axes_dev, T.positions = a->positions_dev, T.position_stride = a->position_stride;
  T.q = {static_cast<const uint16_t*>(a->q_dev), a->q_stride, static_cast<uint16_t*>(a->q_out_dev), a->q_out_stride, a->q_dev ? a->q_norm_dev : nullptr};
  T.k = {static_cast<const uint16_t*>(a->k_dev), a->k_stride, static_cast<uint16_t*>(a->k_out_dev), a->k_out_stride, a->k_dev ? a->k_norm_dev : nullptr};
  T.hq = a->q_dev ? a->n_q_heads : 0, T.hk = a->k_dev ? a->n_kv_heads : 0, T.heads = a->n_kv_heads;
  T.n_tokens = a->n_tokens, T.n_axes = a->n_axes, T.norm_f32 = a->norm_f32 != 0, T.eps = a->eps;
  return QC_OK;
}

// Whether what a call writes lies over anything but its own input.
bool overlaps(const qc_rotate_args* a, const Span* more, int n_more) {
  const int n = a->n_tokens, d = a->head_dim;
  const Span q = rows_span(a->q_dev, a->q_stride, a->n_q_heads, d, n), q_out = rows_span(a->q_out_dev, a->q_out_stride, a->n_q_heads, d, n);
  const Span k = rows_span(a->k_dev, a->k_stride, a->n_kv_heads, d, n), k_out = rows_span(a->k_out_dev, a->k_out_stride, a->n_kv_heads, d, n);
  const auto same = [&](const Span& x, const Span& y) { return x.at == y.at && (x.stride == y.stride || n == 1); };
  if (meet(q_out, k_out) || meet(q_out, k) || meet(k_out, q)) return true;
  if ((meet(q_out, q) && !same(q_out, q)) || (meet(k_out, k) && !same(k_out, k))) return true;
  for (int i = 0; i < n_more; ++i)
    if (meet(q_out, more[i]) || meet(k_out, more[i])) return true;
  return false;
}

int32_t launch_rotate(RotateArgs& T, int32_t head_dim, bool adjacent, cudaStream_t stream) {
  const int pass = kRowThreads / (head_dim / 16);
  T.rows = T.hq + T.hk + T.hv;
  // Few rows: a block per pass of rows, so that none waits for another.  Many: all rows of as many tokens as make some eight passes,
  // whose angles are worked out together.
  if (static_cast<int64_t>(T.n_tokens) * T.rows <= 148 * 8 * pass) {
    T.tokens = 1, T.chunk = min(T.rows, pass);
  } else {
    T.tokens = max(1, min(kMaxTokens, 8 * pass / T.rows)), T.chunk = min(T.rows, 16 * pass);
  }
  T.inv_chunk = 1.f / T.chunk;
  const dim3 grid((T.n_tokens + T.tokens - 1) / T.tokens, (T.rows + T.chunk - 1) / T.chunk);
  const auto kernel = head_dim == 128 ? (adjacent ? rotate_kernel<128, true> : rotate_kernel<128, false>) : (adjacent ? rotate_kernel<64, true> : rotate_kernel<64, false>);
  return status_of(launch_pdl(kernel, grid, dim3(kRowThreads), 0, stream, T));
}

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_rotate(int32_t device, void* cuda_stream, const qc_rotate_args* args) {
  RotateArgs T{};
  if (const int32_t bad = check_rotate(args, false, T)) return bad;
  if (!args->q_dev && !args->k_dev) return QC_ERR_INVALID_ARG;
  if (args->n_tokens == 0) return QC_OK;
  if (overlaps(args, nullptr, 0)) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  return launch_rotate(T, args->head_dim, args->adjacent != 0, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int32_t qc_paged_append(int32_t device, void* cuda_stream, const qc_paged_append_args* args) {
  if (!args) return QC_ERR_INVALID_ARG;
  const qc_rotate_args* r = &args->rows;
  RotateArgs T{};
  if (const int32_t bad = check_rotate(r, true, T)) return bad;
  if (args->page_size != 16 && args->page_size != 32 && args->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (args->n_pages < 1 || r->n_kv_heads < 1) return QC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(args->n_pages) * args->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  if ((!r->k_dev) != (!args->k_pool_dev) || (!args->v_dev) != (!args->v_pool_dev) || (!r->k_dev && !args->v_dev)) return QC_ERR_INVALID_ARG;
  if (off16(args->v_dev) || off16(args->k_pool_dev) || off16(args->v_pool_dev) || off4(args->slots_dev)) return QC_ERR_INVALID_ARG;
  if (args->v_dev && (args->v_stride < 0 || args->v_stride % 8)) return QC_ERR_INVALID_ARG;
  if (r->n_tokens == 0) return QC_OK;
  if (!args->slots_dev) return QC_ERR_INVALID_ARG;
  const uint64_t pool = static_cast<uint64_t>(args->n_pages) * args->page_size * r->n_kv_heads * r->head_dim * 2;
  const Span kp = flat_span(args->k_pool_dev, pool), vp = flat_span(args->v_pool_dev, pool);
  const Span ins[3] = {rows_span(r->q_dev, r->q_stride, r->n_q_heads, r->head_dim, r->n_tokens), rows_span(r->k_dev, r->k_stride, r->n_kv_heads, r->head_dim, r->n_tokens),
                       rows_span(args->v_dev, args->v_stride, r->n_kv_heads, r->head_dim, r->n_tokens)};
  for (const Span& s : ins)
    if (meet(kp, s) || meet(vp, s)) return QC_ERR_INVALID_ARG;
  const Span more[3] = {ins[2], kp, vp};
  if (meet(kp, vp) || overlaps(r, more, 3)) return QC_ERR_INVALID_ARG;
  T.v = {static_cast<const uint16_t*>(args->v_dev), args->v_stride, nullptr, 0, nullptr};
  T.hv = args->v_dev ? r->n_kv_heads : 0;
  T.k_pool = static_cast<uint16_t*>(args->k_pool_dev), T.v_pool = static_cast<uint16_t*>(args->v_pool_dev);
  T.slots = args->slots_dev;
  T.page_shift = args->page_size == 16 ? 4 : args->page_size == 32 ? 5 : 6;
  T.n_slots = args->n_pages * args->page_size;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  return launch_rotate(T, r->head_dim, r->adjacent != 0, static_cast<cudaStream_t>(cuda_stream));
}
