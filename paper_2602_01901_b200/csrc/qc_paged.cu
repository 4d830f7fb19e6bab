// Rows of queries and keys normalised and turned by their positions, to a tensor or to their places in a cache's pages.
//
//   y = x / sqrt(mean x^2 + eps) * w, then (a, b) -> (a cos - b sin, b cos + a sin) for pair i by positions[axis of i] * freqs[i]
//
// Bound by its bytes, a row in and a row out.  The angles are a token's, not a head's: a warp works them out once for its token, a lane per
// pair or two, multiplies the norm's weights in, and turns all heads with these factors, which it keeps in shared memory.  Occupancy
// decides, since rows under way are what hides the memory: 48 registers, 40 warps an SM.  10 813 tokens of 64 heads of 128 take 59.8 us, 92 % of
// what a copy moves (factors in registers, 96 of them, 78 us; blocks of some tokens that share angles, weights read for each row,
// 71); with V into pages 88.7 us of 82.3.  One token takes 3.2 us in a graph, a launch's latency.
// An angle is counted in turns, as a fraction of 64 bits: freq / 2 pi modulo 1 once, times the position modulo 2^64, and sine and cosine are taken of
// a number in [-1, 1) half turns.  The fraction is off by less than 2^-64, a position's angle by 2^-33 turns; its rounding to fp32, 2^-26
// turns at most, is all that is seen (in fp32 throughout position 100 000 is 6e-3 radians off; with freq / 2 pi in one double position 2^31 was off by
// 4e-6 turns for frequencies to 100).
// A row is held by D / 16 lanes, two 16-byte vectors each: those whose pairs the lane turns, so that no element changes lanes.
// The squares' sum takes 3 exchanges.

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

constexpr int kRowThreads = 128, kRowBlocks = 10;

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
  int32_t chunk;                    // rows of a token that a warp takes
  float eps;
};

// The angle of a pair at a position, as (cos, sin).
__device__ __forceinline__ float2 turn_of(float freq, int32_t position) {
  // freq / 2 pi in two doubles: what the first leaves off counts too, times the position
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57, k64 = 18446744073709551616.0;
  const double f = freq, turns = f * kTurn, rest = fma(f, kTurnRest, fma(f, kTurn, -turns));
  const unsigned long long part = __double2ull_rn((turns - floor(turns)) * k64) + static_cast<unsigned long long>(__double2ll_rn(rest * k64));
  const unsigned long long at = part * static_cast<unsigned long long>(static_cast<long long>(position));
  float2 cs;
  sincospif(static_cast<float>(static_cast<int32_t>(at >> 32)) * 4.656612873077392578125e-10f, &cs.y, &cs.x);   // 2^-31
  return isfinite(freq) ? cs : make_float2(NAN, NAN);
}

// A lane's 16 elements as pairs (p[i], q[i]).
template <bool ADJ>
__device__ __forceinline__ void pairs_of(const uint4& x, const uint4& y, float2 (&p)[4], float2 (&q)[4]) {
  if constexpr (ADJ) {
    float e[16];
    bf16x8_to_f32(x, e), bf16x8_to_f32(y, e + 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = make_float2(e[4 * i], e[4 * i + 2]), q[i] = make_float2(e[4 * i + 1], e[4 * i + 3]);
  } else {
    bf16x8_to_f32x2(x, p), bf16x8_to_f32x2(y, q);
  }
}
template <bool ADJ>
__device__ __forceinline__ void pairs_of(const uint4 (&raw)[4], float2 (&p)[4], float2 (&q)[4]) {      // of fp32
  float4 e[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = make_float4(__uint_as_float(raw[i].x), __uint_as_float(raw[i].y), __uint_as_float(raw[i].z), __uint_as_float(raw[i].w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (ADJ) p[i] = make_float2(e[i].x, e[i].z), q[i] = make_float2(e[i].y, e[i].w);
    else if (i < 2) p[2 * i] = make_float2(e[i].x, e[i].y), p[2 * i + 1] = make_float2(e[i].z, e[i].w);
    else q[2 * i - 4] = make_float2(e[i].x, e[i].y), q[2 * i - 3] = make_float2(e[i].z, e[i].w);
  }
}

// A warp per chunk of a token's rows: q's, then k's, then v's.  ADJ: pairs are neighbours.
template <int D, bool ADJ>
__global__ void __launch_bounds__(kRowThreads, kRowBlocks) rotate_kernel(const __grid_constant__ RotateArgs T) {
  constexpr int kLanes = D / 16, kPass = 32 / kLanes, kMine = D / 64;      // rows of a pass of the warp; pairs that a lane finds the angle of
  struct Kind {                     // rows of q, k or v as if they began at row 0, `step` elements apart where they go
    const uint16_t* from;
    uint16_t* to;                   // null: nowhere
    int64_t step;
  };
  struct Warp {
    // of rows of q, of k: (p, q) -> (p * x + q * y, q * x' + p * y'), for two pairs a float4 of x and y, then one of x' and y'; those of a row's lanes
    // follow one another
    float4 factors[2][8 * kLanes];
    float2 turns[D / 2];
    Kind kinds[3];
  };
  __shared__ __align__(16) Warp warps[kRowThreads / 32];
  pdl_wait();
  Warp& W = warps[threadIdx.x / 32];
  const int lane = threadIdx.x % 32, j = lane % kLanes;
  const int token = blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32;
  if (token >= T.n_tokens) return;
  const int row_end = min(T.rows, static_cast<int>(blockIdx.y + 1) * T.chunk), hqk = T.hq + T.hk;
  int r = blockIdx.y * T.chunk + lane / kLanes;
  // the lane's two vectors: those with its pairs, or what is left of a row that turns in part
  const int turning = T.pairs / 8;
  const bool turns_here = j < turning;
  const int a = ADJ || !turns_here ? 2 * j : j, b = ADJ || !turns_here ? 2 * j + 1 : turning + j;
  const auto kind_of = [&](int r) { return r < T.hq ? 0 : r < hqk ? 1 : 2; };

  struct Row {
    uint4 x, y;
  };
  const auto fetch = [&](Row& row, const uint16_t* from) {
    const uint4* const p = reinterpret_cast<const uint4*>(from);
    row.x = p[a], row.y = p[b];
  };
  const auto begin_of = [&](int kind) {
    const Rows& s = kind == 0 ? T.q : kind == 1 ? T.k : T.v;
    return s.x + (token * s.stride - static_cast<int64_t>(kind == 0 ? 0 : kind == 1 ? T.hq : hqk) * D);
  };
  // All that a warp begins with is asked for before any of it is waited for, the longest chain first.  The lanes of the first row
  // find the factors of q, those of the second k's.
  const int of = lane / kLanes;
  const void* const weights = of == 0 ? T.q.norm : of == 1 ? T.k.norm : nullptr;
  int axis[kMine];
  float freq[kMine];
  int32_t position[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int pair = lane + 32 * i;
    axis[i] = pair < T.pairs && T.axes ? __ldg(T.axes + pair) : 0, freq[i] = pair < T.pairs ? __ldg(T.freqs + pair) : 0.f;
  }
  const int32_t slot = T.slots ? __ldg(T.slots + token) : -1;
  Row next{};
  if (r < row_end) fetch(next, begin_of(kind_of(r)) + r * D);
  uint4 raw[4] = {};
  if (weights) {
    const uint4* const p = static_cast<const uint4*>(weights);
    if (T.norm_f32) raw[0] = __ldg(p + 2 * a), raw[1] = __ldg(p + 2 * a + 1), raw[2] = __ldg(p + 2 * b), raw[3] = __ldg(p + 2 * b + 1);
    else raw[0] = __ldg(p + a), raw[1] = __ldg(p + b);
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const bool there = lane + 32 * i < T.pairs && static_cast<uint32_t>(axis[i]) < static_cast<uint32_t>(T.n_axes);
    position[i] = there ? __ldg(T.positions + axis[i] * T.position_stride + token) : 0, freq[i] = there ? freq[i] : NAN;
  }

#pragma unroll
  for (int i = 0; i < kMine; ++i)
    if (lane + 32 * i < T.pairs) W.turns[lane + 32 * i] = turn_of(freq[i], position[i]);
  if (lane < 3) {
    Kind k{begin_of(lane), lane == 2 ? T.v_pool : lane == 1 ? T.k_pool : T.q.out, D};
    if (lane == 0 || (lane == 1 && T.k.out)) {
      const Rows& s = lane ? T.k : T.q;
      k.to = s.out + (token * s.out_stride - (lane ? T.hq : 0) * D);
    } else if (T.slots) {
      const int32_t page = slot >> T.page_shift, in_page = slot & ((1 << T.page_shift) - 1);
      k.step = static_cast<int64_t>(D) << T.page_shift;
      const int64_t at = ((static_cast<int64_t>(page) * T.heads << T.page_shift) + in_page) * D - (lane == 1 ? T.hq : hqk) * k.step;
      k.to = static_cast<uint32_t>(slot) < static_cast<uint32_t>(T.n_slots) ? k.to + at : nullptr;
    }
    W.kinds[lane] = k;
  }
  float2 pp[4], qq[4];
  if (!weights) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pp[i] = qq[i] = make_float2(1.f, 1.f);
  } else if (T.norm_f32) {
    pairs_of<ADJ>(raw, pp, qq);
  } else {
    pairs_of<ADJ>(raw[0], raw[1], pp, qq);
  }
  __syncwarp();
  if (of < 2) {
    float4* const to = W.factors[of] + j;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 t = turns_here ? *reinterpret_cast<const float4*>(W.turns + 8 * j + 2 * i) : make_float4(1.f, 0.f, 1.f, 0.f);
      to[2 * i * kLanes] = make_float4(pp[i].x * t.x, pp[i].y * t.z, qq[i].x * -t.y, qq[i].y * -t.w);
      to[(2 * i + 1) * kLanes] = make_float4(qq[i].x * t.x, qq[i].y * t.z, pp[i].x * t.y, pp[i].y * t.w);
    }
  }
  __syncwarp();

#pragma unroll 1
  for (; r - lane / kLanes < row_end; r += kPass) {      // (all lanes of a warp: they exchange sums)
    Row row = next;
    if (r + kPass < row_end) fetch(next, W.kinds[kind_of(r + kPass)].from + (r + kPass) * D);
    const int kind = kind_of(r);
    float2 p[4], q[4];
    pairs_of<ADJ>(row.x, row.y, p, q);
    float scale = 1.f;
    if (T.q.norm || T.k.norm) {
      float2 s0 = mul2(p[0], p[0]), s1 = mul2(q[0], q[0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) s0 = fma2(p[i], p[i], s0), s1 = fma2(q[i], q[i], s1);
      s0 = add2(s0, s1);
      float sum = s0.x + s0.y;
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (kind ? T.k.norm : T.q.norm) scale = rsqrtf(sum * (1.f / D) + T.eps);
    }
    if (r >= row_end) continue;
    if (kind < 2) {
      const float4* const f = W.factors[kind] + j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 t0 = f[2 * i * kLanes], t1 = f[(2 * i + 1) * kLanes];
        float2 u = mul2(p[i], make_float2(t0.x, t0.y)), v = mul2(q[i], make_float2(t1.x, t1.y));
        if (turns_here) u = fma2(q[i], make_float2(t0.z, t0.w), u), v = fma2(p[i], make_float2(t1.z, t1.w), v);
        p[i] = mul2(u, make_float2(scale, scale)), q[i] = mul2(v, make_float2(scale, scale));
      }
      if constexpr (ADJ) {
        row.x = make_uint4(pack_bf16x2(p[0].x, q[0].x), pack_bf16x2(p[0].y, q[0].y), pack_bf16x2(p[1].x, q[1].x), pack_bf16x2(p[1].y, q[1].y));
        row.y = make_uint4(pack_bf16x2(p[2].x, q[2].x), pack_bf16x2(p[2].y, q[2].y), pack_bf16x2(p[3].x, q[3].x), pack_bf16x2(p[3].y, q[3].y));
      } else {
        row.x = make_uint4(pack_bf16x2(p[0].x, p[0].y), pack_bf16x2(p[1].x, p[1].y), pack_bf16x2(p[2].x, p[2].y), pack_bf16x2(p[3].x, p[3].y));
        row.y = make_uint4(pack_bf16x2(q[0].x, q[0].y), pack_bf16x2(q[1].x, q[1].y), pack_bf16x2(q[2].x, q[2].y), pack_bf16x2(q[3].x, q[3].y));
      }
    }
    const Kind& k = W.kinds[kind];
    if (!k.to) continue;
    uint4* const to = reinterpret_cast<uint4*>(k.to + r * k.step);
    to[a] = row.x, to[b] = row.y;
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

// Whether a run of memory that a call writes lies over what it reads besides rows.
bool over_tables(const qc_rotate_args* a, const Span& out) {
  const uint64_t pairs = a->q_dev || a->k_dev ? a->rotary_dim / 2 : 0, weights = static_cast<uint64_t>(a->head_dim) * (a->norm_f32 ? 4 : 2);
  const auto over = [&](const void* p, uint64_t bytes) { return bytes && meet(out, flat_span(p, bytes)); };
  for (int axis = 0; pairs && axis < a->n_axes; ++axis)
    if (over(a->positions_dev + axis * a->position_stride, static_cast<uint64_t>(a->n_tokens) * 4)) return true;
  return over(a->freqs_dev, pairs * 4) || over(a->axes_dev, pairs * 4) || (a->q_dev && over(a->q_norm_dev, weights)) || (a->k_dev && over(a->k_norm_dev, weights));
}

// Whether what a call writes lies over anything but its own input.
bool overlaps(const qc_rotate_args* a, const Span* more, int n_more) {
  const int n = a->n_tokens, d = a->head_dim;
  const Span q = rows_span(a->q_dev, a->q_stride, a->n_q_heads, d, n), q_out = rows_span(a->q_out_dev, a->q_out_stride, a->n_q_heads, d, n);
  const Span k = rows_span(a->k_dev, a->k_stride, a->n_kv_heads, d, n), k_out = rows_span(a->k_out_dev, a->k_out_stride, a->n_kv_heads, d, n);
  const auto same = [&](const Span& x, const Span& y) { return x.at == y.at && (x.stride == y.stride || n == 1); };
  if (meet(q_out, k_out) || meet(q_out, k) || meet(k_out, q)) return true;
  if ((meet(q_out, q) && !same(q_out, q)) || (meet(k_out, k) && !same(k_out, k))) return true;
  if (over_tables(a, q_out) || over_tables(a, k_out)) return true;
  for (int i = 0; i < n_more; ++i)
    if (meet(q_out, more[i]) || meet(k_out, more[i])) return true;
  return false;
}

int32_t launch_rotate(RotateArgs& T, int32_t head_dim, bool adjacent, cudaStream_t stream) {
  const int pass = 512 / head_dim;
  T.rows = T.hq + T.hk + T.hv;
  // A warp per pass of rows where they are few, so that none waits for another; where they are many, as many rows as leave 20 warps for each of
  // 148 SMs, up to 24 passes (against 8: 1 % less of 10 813 tokens' time)
  const int passes = (T.rows + pass - 1) / pass;
  const int each = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(24, static_cast<int64_t>(T.n_tokens) * passes / (148 * 20))));
  const int chunks = (passes + each - 1) / each;
  T.chunk = (passes + chunks - 1) / chunks * pass;
  constexpr int kWarps = kRowThreads / 32;
  const dim3 grid((T.n_tokens + kWarps - 1) / kWarps, chunks);
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
  const Span more[4] = {ins[2], kp, vp, flat_span(args->slots_dev, static_cast<uint64_t>(r->n_tokens) * 4)};
  if (meet(kp, vp) || meet(kp, more[3]) || meet(vp, more[3]) || over_tables(r, kp) || over_tables(r, vp) || overlaps(r, more, 4)) return QC_ERR_INVALID_ARG;
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
