// Attention of a step's queries over a cache in 4 bits.
//
// A row of K or V stands for lo + s c (s = 1 / r, codes c in 0..15), that is mid + s (c - 8) with mid = lo + 8 s, so
//   q . k_j       = s_j sum_d q_d (c_jd - 8) + mid_j sum_d q_d
//   sum_j p_j v_j = sum_j (p_j s_j)(c_jd - 8) + sum_j p_j mid_j
// and the only large sums run over codes, which are exact in 16 bits: a code becomes an fp16 number by an AND and an
// OR into the mantissa of 1024 (1024 + c, or 1024 + 16 c from the upper half of a byte) and one packed operation that
// takes the constant off.  The queries are exact in fp16 as well once a power of two has brought the unit's
// largest element below 2^12 (bf16 has fewer bits; what is 2^-25 of the largest loses bits, which no score shows).  The
// weights p_j s_j are rounded to fp16 (2^-12) after a division by a power of two not below the warp's largest s.
// Everything else is fp32.
//
// Products are m16n8k16 with the keys (for K) and the elements (for V) as rows and up to eight query rows as columns:
// the heads of a group times the sequence's queries.  The pages are laid out for this (qc_quant.cuh): operands come
// from global memory in whole 16-byte vectors in lane order, and a product's scores become the next one's weights by
// two transposes in registers.

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.cuh"
#include "qc_quant.h"

#include <cuda_fp16.h>

namespace qc {
namespace {

constexpr int kTile = 64;            // keys that a warp takes at a time
constexpr int kAttWarps = 4;
constexpr float kLeastStep = 3.9443045261050590e-31f;   // 2^-101, below every step but 0

struct StreamArgs {
  const uint16_t* q;
  int64_t q_stride;
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  const int32_t* pages;
  const int32_t* lens;
  int32_t max_pages, n_pages;
};

struct AttendArgs {
  StreamArgs text, visual;
  const int32_t* ids;
  const int32_t* starts;
  uint16_t* out;
  float* lse;
  float* part;          // [splits][units][8 * NT][D + 2]
  int32_t* status;
  int32_t hq, hkv, group, page, page_shift;
  int32_t n_seqs, max_seqs, n_tokens, max_queries, causal, has_visual;
  int32_t n_splits, row_tiles;
  int64_t page_bytes;
  float scale_log2;
};

__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// Bits 0-3 and 16-19 (lower) or 4-7 and 20-23 (upper) of x as two fp16 numbers c - 8.
__device__ __forceinline__ uint32_t lower_codes(uint32_t x) { return sub_h2((x & 0x000f000fu) | 0x64006400u, 0x64086408u); }   // 1024 + c - 1032
__device__ __forceinline__ uint32_t upper_codes(uint32_t x) {
  return fma_h2((x & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);   // (1024 + 16 c) / 16 - 72
}
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The codes of a block of 16 tokens that a lane holds: for K the words of its even and its odd token, for V the
// words of its element pairs.
template <int D>
struct Block {
  uint4 w[D / 64];
};
template <int D>
__device__ __forceinline__ void load_block(Block<D>& b, const uint8_t* p, int lane, bool on) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
    b.w[i] = on ? __ldg(reinterpret_cast<const uint4*>(p + i * 512 + lane * 16)) : make_uint4(0, 0, 0, 0);
}

// One unit: up to 8 * NT query rows of one (sequence, KV head) that share their keys.  A warp's running state.
template <int D, int NT>
struct Rows {
  float acc[NT][D / 16][4];
  float m[NT][2], l[NT][2], z[NT][2];
  float n;                 // the power of two that the weights were divided by
};

template <int D, int NT>
struct Query {
  uint32_t b[NT][D / 16][2];   // operands of the score products
  float sum[NT][2];            // sum of the elements, for the columns 2 t and 2 t + 1
  float scale;                 // softmax scale * log2 e * the power of two that was taken out
};

// Row r of the unit is query r / group of the sequence, head r % group of the KV head.
template <int D, int NT>
__device__ __forceinline__ void load_query(Query<D, NT>& Q, const AttendArgs& A, const StreamArgs& S, int64_t token0, int head0, int row0,
                                           int n_rows, int lane) {
  const int g = lane >> 2, t = lane & 3;
  uint4 raw[NT][D / 32];
  float top = 0.f;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row0 + nt * 8 + g;
    const bool on = r < n_rows;
    const uint16_t* q = S.q + (token0 + r / A.group) * S.q_stride + static_cast<int64_t>(head0 + r % A.group) * D + t * (D / 4);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      raw[nt][i] = on ? __ldg(reinterpret_cast<const uint4*>(q) + i) : make_uint4(0, 0, 0, 0);
      float f[8];
      bf16x8_to_f32(raw[nt][i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  // 2^e with top * 2^-e in [2^11, 2^12); a zero or subnormal top counts as 2^-100, an infinite one as 2^127
  const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100), 127) - 11;
  const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);   // -111 <= e <= 116
  Q.scale = A.scale_log2 * __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      float f[8];
      bf16x8_to_f32(raw[nt][i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = __half2float(__float2half_rn(f[j] * down));
        sum += f[j];
      }
      Q.b[nt][2 * i][0] = pack_f16x2(f[0], f[4]);
      Q.b[nt][2 * i][1] = pack_f16x2(f[1], f[5]);
      Q.b[nt][2 * i + 1][0] = pack_f16x2(f[2], f[6]);
      Q.b[nt][2 * i + 1][1] = pack_f16x2(f[3], f[7]);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    Q.sum[nt][0] = __shfl_sync(0xffffffffu, sum, t * 8);
    Q.sum[nt][1] = __shfl_sync(0xffffffffu, sum, t * 8 + 4);
  }
}

// Scores of a block: c[0], c[1] the lane's even token for columns 2 t and 2 t + 1, c[2], c[3] its odd one.
template <int D, int NT>
__device__ __forceinline__ void score_block(const Block<D>& k, const Query<D, NT>& Q, float (&c)[NT][4]) {
  uint32_t even[D / 32], odd[D / 32];
  if constexpr (D == 128) {
    even[0] = k.w[0].x, even[1] = k.w[0].y, even[2] = k.w[0].z, even[3] = k.w[0].w;
    odd[0] = k.w[1].x, odd[1] = k.w[1].y, odd[2] = k.w[1].z, odd[3] = k.w[1].w;
  } else {
    even[0] = k.w[0].x, even[1] = k.w[0].y, odd[0] = k.w[0].z, odd[1] = k.w[0].w;
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t xe = h ? even[w] >> 8 : even[w], xo = h ? odd[w] >> 8 : odd[w];
      const uint32_t a0 = lower_codes(xe), a1 = lower_codes(xo), a2 = upper_codes(xe), a3 = upper_codes(xo);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16_16816(c[nt], a0, a1, a2, a3, Q.b[nt][2 * w + h][0], Q.b[nt][2 * w + h][1]);
    }
  }
}

// One tile of keys from key0 on; `len` keys are there, column x of tile nt sees those before lim[nt][x].
template <int D, int NT>
__device__ __forceinline__ void attend_tile(Rows<D, NT>& R, const Query<D, NT>& Q, const AttendArgs& A, const StreamArgs& S, const int32_t* table,
                                            int kvh, int key0, int len, const int32_t (&lim)[NT][2], int least_lim, int lane) {
  constexpr int kBlocks = kTile / 16;
  const int g = lane >> 2;
  Block<D> kb[kBlocks], vb[kBlocks];
  uint2 kp[kBlocks], vp[kBlocks];
  bool on[kBlocks];
  const size_t code_bytes = static_cast<size_t>(A.hkv) * A.page * (D / 2);
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const int key = key0 + 16 * b;
    on[b] = key < len;
    const int32_t id = on[b] ? table[key >> A.page_shift] : 0;
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(S.n_pages)) {   // not followed
      if (lane == 0 && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_BAD_PAGE));
      on[b] = false;
    }
    const int in_page = key & (A.page - 1);
    const size_t base = static_cast<size_t>(on[b] ? id : 0) * A.page_bytes;
    const size_t code = base + (static_cast<size_t>(kvh) * A.page + in_page) * (D / 2);
    const size_t word = base + code_bytes + (static_cast<size_t>(kvh) * A.page + in_page + 2 * g) * 4;
    load_block<D>(kb[b], S.k_pool + code, lane, on[b]);
    kp[b] = on[b] ? __ldg(reinterpret_cast<const uint2*>(S.k_pool + word)) : make_uint2(0, 0);
    load_block<D>(vb[b], S.v_pool + code, lane, on[b]);
    vp[b] = on[b] ? __ldg(reinterpret_cast<const uint2*>(S.v_pool + word)) : make_uint2(0, 0);
  }

  float s[kBlocks][NT][4];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    score_block<D, NT>(kb[b], Q, s[b]);
    const float s0 = quant_step(kp[b].x), s1 = quant_step(kp[b].y);
    const float m0 = fmaf(8.f, s0, __uint_as_float(kp[b].x << 16)) * Q.scale, m1 = fmaf(8.f, s1, __uint_as_float(kp[b].y << 16)) * Q.scale;
    const float f0 = s0 * Q.scale, f1 = s1 * Q.scale;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      s[b][nt][0] = fmaf(f0, s[b][nt][0], m0 * Q.sum[nt][0]);
      s[b][nt][1] = fmaf(f0, s[b][nt][1], m0 * Q.sum[nt][1]);
      s[b][nt][2] = fmaf(f1, s[b][nt][2], m1 * Q.sum[nt][0]);
      s[b][nt][3] = fmaf(f1, s[b][nt][3], m1 * Q.sum[nt][1]);
    }
  }
  const bool all_on = on[0] && on[1] && on[2] && on[3];
  const bool masked = key0 + kTile > least_lim || !all_on;   // the same for the whole warp
  if (masked) {
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (!on[b] || key0 + 16 * b + 2 * g + (x >> 1) >= lim[nt][x & 1]) s[b][nt][x] = -INFINITY;
  }
  // a row that no column sees has no part in anything: its parameters may be whatever was there before
  float step[kBlocks][2], mid[kBlocks][2];
  uint32_t top = 0;
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t p = i ? vp[b].y : vp[b].x;
      step[b][i] = quant_step(p);
      mid[b][i] = fmaf(8.f, step[b][i], __uint_as_float(p << 16));
      if (masked && (!on[b] || key0 + 16 * b + 2 * g + i >= len)) step[b][i] = mid[b][i] = 0.f;
      top = max(top, __float_as_uint(fminf(step[b][i], 1e38f)));
    }
  top = __reduce_max_sync(0xffffffffu, top);
  // larger scores or steps than before: everything so far is put on the new reference
  bool more = __uint_as_float(top) > R.n;
  float high[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float h = s[0][nt][x];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) h = fmaxf(h, fmaxf(s[b][nt][x], s[b][nt][x + 2]));
      high[nt][x] = h;
      more |= h > R.m[nt][x];
    }
  if (__any_sync(0xffffffffu, more)) {
    const float n_new = fmaxf(R.n, __uint_as_float((top & 0x7f800000u) + 0x00800000u));
    const float down = R.n / n_new;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float h = high[nt][x];
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 4));
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 8));
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 16));
        h = fmaxf(h, R.m[nt][x]);
        const float corr = h == R.m[nt][x] ? 1.f : exp2f(R.m[nt][x] - h);   // (both minus infinity: nothing so far)
        R.m[nt][x] = h;
        R.l[nt][x] *= corr;
        R.z[nt][x] *= corr;
        const float f = corr * down;
#pragma unroll
        for (int mb = 0; mb < D / 16; ++mb) R.acc[nt][mb][x] *= f, R.acc[nt][mb][x + 2] *= f;
      }
    R.n = n_new;
  }
  // weights
  const float up = 32768.f / R.n;      // p s / n <= 1: the largest weight is 2^15
  uint32_t w[kBlocks][NT][2];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const float u0 = step[b][0] * up, u1 = step[b][1] * up;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float m = R.m[nt][x & 1];
        p[x] = ex2_approx(s[b][nt][x] - (m == -INFINITY ? 0.f : m));
        R.l[nt][x & 1] += p[x];
        // (a value that is no number counts only where it is seen)
        R.z[nt][x & 1] = fmaf(p[x], masked && p[x] == 0.f ? 0.f : mid[b][x >> 1], R.z[nt][x & 1]);
      }
      w[b][nt][0] = movmatrix_trans(pack_f16x2(p[0] * u0, p[1] * u0));
      w[b][nt][1] = movmatrix_trans(pack_f16x2(p[2] * u1, p[3] * u1));
    }
  }
#pragma unroll
  for (int mb = 0; mb < D / 16; ++mb)
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const uint4& v = vb[b].w[mb / 4];
      const uint32_t x = mb % 4 == 0 ? v.x : mb % 4 == 1 ? v.y : mb % 4 == 2 ? v.z : v.w;
      const uint32_t a0 = lower_codes(x), a1 = upper_codes(x), a2 = lower_codes(x >> 8), a3 = upper_codes(x >> 8);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16_16816(R.acc[nt][mb], a0, a1, a2, a3, w[b][nt][0], w[b][nt][1]);
    }
}

// Writes D finished elements of a row: lane g's run of D / 8.
template <int D>
__device__ __forceinline__ void store_run(uint16_t* row, int g, const float (&o)[D / 8]) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
    reinterpret_cast<uint4*>(row + g * (D / 8))[i] = make_uint4(pack_bf16x2(o[8 * i], o[8 * i + 1]), pack_bf16x2(o[8 * i + 2], o[8 * i + 3]),
                                                                pack_bf16x2(o[8 * i + 4], o[8 * i + 5]), pack_bf16x2(o[8 * i + 6], o[8 * i + 7]));
}

// What a part with reference ms and a sum counts for on reference m.  Minus infinity with a sum means that its scores were
// no numbers.
__device__ __forceinline__ float weight_of(float ms, float m) { return ms == -INFINITY ? NAN : exp2f(ms - m); }

struct UnitPlace {
  int64_t token0;    // the sequence's first query
  int32_t n_rows;    // query rows of the (sequence, KV head); 0: nothing to do
  int32_t queries;
  int32_t row;       // row of the page tables
};

__device__ __forceinline__ UnitPlace place_of(const AttendArgs& A, int seq, bool report) {
  UnitPlace u{0, 0, 0, 0};
  int64_t a = seq, b = seq + 1;
  if (A.starts) a = A.starts[seq], b = A.starts[seq + 1];
  u.row = A.ids ? A.ids[seq] : seq;
  if (a < 0 || b < a || b > A.n_tokens || b - a > A.max_queries || u.row < 0 || u.row >= A.max_seqs) {
    if (report && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_INVALID_ARG));
    return u;
  }
  u.token0 = a;
  u.queries = static_cast<int32_t>(b - a);
  u.n_rows = u.queries * A.group;
  return u;
}

__device__ __forceinline__ int length_of(const AttendArgs& A, const StreamArgs& S, int row, bool report) {
  const int64_t len = S.lens[row], room = static_cast<int64_t>(S.max_pages) << A.page_shift;
  if (len >= 0 && len <= room) return static_cast<int>(len);
  if (report && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_PLAN));
  return len < 0 ? 0 : static_cast<int>(room);
}

// Grid: (splits, KV heads x row tiles, sequences).
template <int D, int NT>
__global__ void __launch_bounds__(kAttWarps * 32) quant_attend_kernel(const __grid_constant__ AttendArgs A) {
  __shared__ float sm_acc[kAttWarps][8 * NT][D];
  __shared__ float sm_m[kAttWarps][8 * NT], sm_l[kAttWarps][8 * NT];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, kvh = blockIdx.y / A.row_tiles, row0 = blockIdx.y % A.row_tiles * (8 * NT), seq = blockIdx.z;
  pdl_launch_dependents();
  const UnitPlace u = place_of(A, seq, threadIdx.x == 0);
  if (row0 >= u.n_rows) return;
  const int len_t = length_of(A, A.text, u.row, threadIdx.x == 0);
  const int len_v = A.has_visual ? length_of(A, A.visual, u.row, threadIdx.x == 0) : 0;
  const int tiles_v = (len_v + kTile - 1) / kTile, tiles = tiles_v + (len_t + kTile - 1) / kTile;
  const int per = (tiles + A.n_splits - 1) / A.n_splits;
  const int first = split * per, last = min(tiles, first + per);

  Rows<D, NT> R;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int x = 0; x < 2; ++x) R.m[nt][x] = -INFINITY, R.l[nt][x] = R.z[nt][x] = 0.f;
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) R.acc[nt][mb][0] = R.acc[nt][mb][1] = R.acc[nt][mb][2] = R.acc[nt][mb][3] = 0.f;
  }
  R.n = kLeastStep;
  int tile = first + warp;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const bool visual = part == 0;
    const int begin = visual ? 0 : tiles_v, end = min(last, visual ? tiles_v : tiles);
    if (tile >= end) continue;
    const StreamArgs& S = visual ? A.visual : A.text;
    const int len = visual ? len_v : len_t;
    Query<D, NT> Q;
    load_query<D, NT>(Q, A, S, u.token0, kvh * A.group, row0, u.n_rows, lane);
    int32_t lim[NT][2], least = INT32_MAX;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = row0 + nt * 8 + 2 * t + x;
        lim[nt][x] = !visual && A.causal && r < u.n_rows ? len - (u.queries - 1 - r / A.group) : len;
        least = min(least, lim[nt][x]);
      }
    least = min(least, __shfl_xor_sync(0xffffffffu, least, 1));
    least = min(least, __shfl_xor_sync(0xffffffffu, least, 2));
    const int32_t* table = S.pages + static_cast<size_t>(u.row) * S.max_pages;
    for (; tile < end; tile += kAttWarps)
      attend_tile<D, NT>(R, Q, A, S, table, kvh, (tile - begin) * kTile, len, lim, least, lane);
  }
  // the warps' sums meet in shared memory
  const float unit = R.n * (1.f / 32768.f);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float l = R.l[nt][x], z = R.z[nt][x];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o), z += __shfl_xor_sync(0xffffffffu, z, o);
      const int col = nt * 8 + 2 * t + x;
      if (g == 0) sm_m[warp][col] = R.m[nt][x], sm_l[warp][col] = l;
#pragma unroll
      for (int mb = 0; mb < D / 16; ++mb) {
        sm_acc[warp][col][g * (D / 8) + 2 * mb] = fmaf(R.acc[nt][mb][x], unit, z);
        sm_acc[warp][col][g * (D / 8) + 2 * mb + 1] = fmaf(R.acc[nt][mb][x + 2], unit, z);
      }
    }
  __syncthreads();
  const int n_here = min(8 * NT, u.n_rows - row0);
  for (int col = warp; col < n_here; col += kAttWarps) {
    float m = -INFINITY, l = 0.f, o[D / 32] = {};
#pragma unroll
    for (int w = 0; w < kAttWarps; ++w) m = fmaxf(m, sm_m[w][col]);
#pragma unroll
    for (int w = 0; w < kAttWarps; ++w) {
      if (sm_l[w][col] == 0.f) continue;
      const float f = weight_of(sm_m[w][col], m);
      l = fmaf(sm_l[w][col], f, l);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] = fmaf(sm_acc[w][col][i * 32 + lane], f, o[i]);
    }
    const int r = row0 + col;
    if (A.n_splits == 1) {
      const size_t row = static_cast<size_t>(u.token0 + r / A.group) * A.hq + kvh * A.group + r % A.group;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) A.out[row * D + i * 32 + lane] = f32_to_bf16_rne(o[i] * inv);
      if (A.lse && lane == 0) A.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
    } else {
      const size_t row = (static_cast<size_t>(split) * A.n_tokens * A.hq) + static_cast<size_t>(u.token0 + r / A.group) * A.hq + kvh * A.group + r % A.group;
      float* dst = A.part + row * (D + 2);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dst[i * 32 + lane] = o[i];
      if (lane == 0) dst[D] = m, dst[D + 1] = l;
    }
  }
}

// One warp per output row: the splits' sums on a common reference.
template <int D>
__global__ void __launch_bounds__(128) quant_merge_kernel(const __grid_constant__ AttendArgs A) {
  const int lane = threadIdx.x & 31, seq = blockIdx.y;
  const int i = blockIdx.x * 4 + (threadIdx.x >> 5);   // (query, head) of the sequence
  pdl_wait();
  const UnitPlace u = place_of(A, seq, false);
  if (i >= u.queries * A.hq) return;
  const size_t row = static_cast<size_t>(u.token0) * A.hq + i, step = static_cast<size_t>(A.n_tokens) * A.hq * (D + 2);
  const float* src = A.part + row * (D + 2);
  float m = -INFINITY, l = 0.f, o[D / 32] = {};
  for (int s = 0; s < A.n_splits; ++s) m = fmaxf(m, src[s * step + D]);
  for (int s = 0; s < A.n_splits; ++s) {
    const float ms = src[s * step + D], ls = src[s * step + D + 1];
    if (ls == 0.f) continue;
    const float f = weight_of(ms, m);
    l = fmaf(ls, f, l);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) o[j] = fmaf(src[s * step + j * 32 + lane], f, o[j]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < D / 32; ++j) A.out[row * D + j * 32 + lane] = f32_to_bf16_rne(o[j] * inv);
  if (A.lse && lane == 0) A.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

bool off(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

int32_t check_stream(const qc_quant_stream* s, const qc_quant_attend_args* a, StreamArgs& d) {
  if (!s->q_dev || !s->k_pool_dev || !s->v_pool_dev || !s->pages_dev || !s->lens_dev) return QC_ERR_INVALID_ARG;
  if (off(s->q_dev, 16) || off(s->k_pool_dev, 16) || off(s->v_pool_dev, 16) || off(s->pages_dev, 4) || off(s->lens_dev, 4)) return QC_ERR_INVALID_ARG;
  if (s->q_stride < 0 || s->q_stride % 8 || s->max_pages < 1 || s->n_pages < 1) return QC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(s->max_pages) * a->page_size > INT32_MAX - kTile || static_cast<int64_t>(s->n_pages) * a->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  d.q = static_cast<const uint16_t*>(s->q_dev), d.q_stride = s->q_stride;
  d.k_pool = static_cast<const uint8_t*>(s->k_pool_dev), d.v_pool = static_cast<const uint8_t*>(s->v_pool_dev);
  d.pages = s->pages_dev, d.lens = s->lens_dev, d.max_pages = s->max_pages, d.n_pages = s->n_pages;
  return QC_OK;
}

int32_t check_sizes(const qc_quant_attend_args* a) {
  if (!a) return QC_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (a->page_size != 16 && a->page_size != 32 && a->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (a->n_kv_heads < 1 || a->n_q_heads < 1 || a->n_q_heads % a->n_kv_heads || a->n_seqs < 1 || a->max_seqs < 1 || a->n_tokens < 0 || a->max_queries < 1)
    return QC_ERR_INVALID_ARG;
  if (a->n_kv_heads > QC_QUANT_MAX_HEADS || a->n_q_heads > QC_QUANT_MAX_HEADS || a->n_seqs > QC_TABLE_MAX_BATCH || a->max_queries > QC_QUANT_MAX_QUERIES)
    return QC_ERR_UNSUPPORTED;
  return QC_OK;
}

int splits_for(const qc_quant_attend_args* a, int row_tiles) {
  const int64_t units = static_cast<int64_t>(a->n_seqs) * a->n_kv_heads * row_tiles;
  int64_t pages = a->text ? a->text->max_pages : 0;
  if (a->visual) pages += a->visual->max_pages;
  const int64_t tiles = (pages * a->page_size + kTile - 1) / kTile;
  int64_t n = (148 * 4 + units - 1) / units;
  if (n > (tiles + kAttWarps - 1) / kAttWarps) n = (tiles + kAttWarps - 1) / kAttWarps;
  return static_cast<int>(n < 1 ? 1 : n > 64 ? 64 : n);
}

int row_tile_of(const qc_quant_attend_args* a) { return a->max_queries * (a->n_q_heads / a->n_kv_heads) > 8 ? 2 : 1; }

template <int D, int NT>
cudaError_t launch(const AttendArgs& A, cudaStream_t stream) {
  quant_attend_kernel<D, NT><<<dim3(A.n_splits, A.hkv * A.row_tiles, A.n_seqs), kAttWarps * 32, 0, stream>>>(A);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || A.n_splits == 1) return e;
  return launch_pdl(quant_merge_kernel<D>, dim3((A.max_queries * A.hq + 3) / 4, A.n_seqs), dim3(128), 0, stream, A);
}

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_quant_workspace_bytes(const qc_quant_attend_args* args, size_t* bytes) {
  if (!bytes) return QC_ERR_INVALID_ARG;
  if (const int32_t bad = check_sizes(args)) return bad;
  const int nt = row_tile_of(args), group = args->n_q_heads / args->n_kv_heads;
  const int splits = splits_for(args, (args->max_queries * group + 8 * nt - 1) / (8 * nt));
  *bytes = splits == 1 ? 0 : static_cast<size_t>(splits) * args->n_tokens * args->n_q_heads * (args->head_dim + 2) * 4;
  return QC_OK;
}

extern "C" int32_t qc_quant_attend(int32_t device, void* cuda_stream, const qc_quant_attend_args* args) {
  if (const int32_t bad = check_sizes(args)) return bad;
  if (!args->text || !args->out_dev || off(args->out_dev, 16) || off(args->lse_out_dev, 4) || off(args->status_dev, 4) || off(args->seq_ids_dev, 4) ||
      off(args->starts_dev, 4) || off(args->workspace_dev, 16))
    return QC_ERR_INVALID_ARG;
  if (!(args->softmax_scale >= 0.f) || !isfinite(args->softmax_scale)) return QC_ERR_INVALID_ARG;
  if (!args->seq_ids_dev && args->n_seqs > args->max_seqs) return QC_ERR_INVALID_ARG;
  if (!args->starts_dev && args->n_tokens < args->n_seqs) return QC_ERR_INVALID_ARG;
  AttendArgs A{};
  if (const int32_t bad = check_stream(args->text, args, A.text)) return bad;
  if (args->visual)
    if (const int32_t bad = check_stream(args->visual, args, A.visual)) return bad;
  size_t need = 0;
  if (const int32_t bad = qc_quant_workspace_bytes(args, &need)) return bad;
  if (need > args->workspace_bytes || (need && !args->workspace_dev)) return QC_ERR_INVALID_ARG;
  if (args->n_tokens == 0) return QC_OK;
  A.has_visual = args->visual != nullptr;
  A.ids = args->seq_ids_dev, A.starts = args->starts_dev;
  A.out = static_cast<uint16_t*>(args->out_dev), A.lse = args->lse_out_dev, A.part = static_cast<float*>(args->workspace_dev);
  A.status = args->status_dev;
  A.hq = args->n_q_heads, A.hkv = args->n_kv_heads, A.group = A.hq / A.hkv, A.page = args->page_size;
  A.page_shift = A.page == 16 ? 4 : A.page == 32 ? 5 : 6;
  A.n_seqs = args->n_seqs, A.max_seqs = args->max_seqs, A.n_tokens = args->n_tokens, A.max_queries = args->starts_dev ? args->max_queries : 1;
  A.causal = args->causal != 0;
  const int nt = row_tile_of(args);
  A.row_tiles = (args->max_queries * A.group + 8 * nt - 1) / (8 * nt);
  A.n_splits = splits_for(args, A.row_tiles);
  A.page_bytes = quant_page_bytes(A.hkv, args->head_dim, A.page);
  const float scale = args->softmax_scale > 0.f ? args->softmax_scale : 1.0f / sqrtf(static_cast<float>(args->head_dim));
  A.scale_log2 = scale * 1.4426950408889634f;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (args->head_dim == 128) e = nt == 1 ? launch<128, 1>(A, stream) : launch<128, 2>(A, stream);
  else e = nt == 1 ? launch<64, 1>(A, stream) : launch<64, 2>(A, stream);
  return e == cudaSuccess ? QC_OK : QC_ERR_CUDA;
}
