// Attention of a step's queries over a cache in 4 bits.
//
// A row of K or V stands for lo + s c (s = 1 / r, codes c in 0..15), so
//   q . k_j       = s_j sum_d q_d c_jd + lo_j sum_d q_d
//   sum_j p_j v_j = sum_j (p_j s_j)(c_jd - 8) + sum_j p_j (lo_j + 8 s_j)
// and the long sums run over codes, which take next to no conversion: masked out of a word they are fp16 numbers already,
// c * 2^-24 (subnormal ones, whose steps are equal), or 16 times that from the upper half of a byte.  A query row is exact in
// fp16 once a power of two of its own has brought its largest element below 2^15 (bf16 has fewer bits; what is below 2^-21 of the
// largest loses some, 2^-35 of the largest at most), so a row does not depend on those beside it: columns of a product are
// separate sums.  The weights p_j s_j are rounded to fp16 (2^-11) after a division by a power of two not below the
// largest s so far.  Everything else is fp32.  The 8 is taken off tile by tile, as a product with ones: sums of c alone
// would grow with the keys, and the tensor cores' adder, which cuts off, would leave a part of them behind.
//
// That adder lines its addends up by the operands' exponent fields, a subnormal number's being that of 2^-14 (seen with one
// large and one small addend).  So each of a product's 16 addends is cut off at 2^-15 of the largest weight, or query element,
// among them, times one code (2^-19 for upper codes).  At worst that is 2^-9 of the steps of V in an output and 2^-8 of
// a K's step times the query's largest element in a score, 1.4 % of what 4 bits leave of it (step / sqrt(12) times the query's
// length); mostly nothing, as a bf16 element above 2^-7 of the largest, or a weight above 2^-4, has no bits there.  Codes higher
// up in the mantissa would cost three shifts a word instead of one.
//
// Products are m16n8k16 with the keys (for K) and the elements (for V) as rows and up to eight query rows as columns:
// the heads of a group times the sequence's queries.  The pages are laid out for this (qc_quant.cuh): a lane's operands
// are whole 16-byte vectors, and a product's scores become the next one's weights by two transposes in registers.
// With four query rows or fewer the eight columns hold them twice, with two or one four times.  Every lane then has the
// scores of all four blocks of a tile for the same rows, and weighs one half or one quarter of them: each set of columns sums up
// its own blocks, and the sets are put together like the sums of different warps.  (One row, eight sequences of 8 541
// tokens, 32 heads: 68.3 us with eight columns of which one counts, 65.9 so; 16 sequences of 60 to 5 000: 33.4 and 31.4.)
//
// What bounds it: the bytes, 68 per row of 128 elements, would take 45 us of 65.7 (those eight sequences now).  A tile of 64 keys is some
// 950 instructions of a warp, 68 of them products; masks and shifts run at half the rate of other instructions and the products at an
// eighth.  No pipe is full (issue slots 49 %, ALU 50 %, tensor 27 %): the three warps of a scheduler mostly wait for their own dependent
// instructions.  Small batches are bound by a block's start: the plan, page ids, first tiles, sums and the join follow one
// another, 9.6 us for one sequence.

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.cuh"
#include "qc_quant.h"

#include <atomic>
#include <chrono>

namespace qc {
namespace {

constexpr int kTile = 64;            // keys that a warp takes at a time
constexpr int kUnitCost = 4;         // what a unit costs each warp besides its tiles, in tiles (its first tiles' way, the sums; 1: 35.2 us instead of
                                     // 31.4 for 16 sequences of 60 to 5 000 tokens, 32 heads; 71.9 instead of 66.0 for three of 90 000)
// Tiles per warp below which units are shared out among warps.  More rows make more of a unit's pieces: 24 ragged sequences with
// five queries, 8 heads of 4, 64 wide, take 32.3 us with 3 and 26.2 with 6 or 12, 16 sequences of 4 000 tokens with five
// queries, 4 heads of 4, 41.2 with 6 and 35.6 with 12, 16 ragged ones of one row 32.5 with 6 and 30.7 with 3.
template <int ROWS>
constexpr uint32_t kFewTiles = ROWS == 2 ? 3 : 12;
constexpr uint32_t kWholeTiles = 3;  // a unit of so many tiles per warp of a team is not cut (one sequence of 707 tokens, 32 heads: 9.6 us, cut 22.8)
constexpr uint32_t kLeastStep = (127u - 104u) << 23;   // 2^-104, below every step but 0: a range is 15 steps, and 2^-100 at least

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
  StreamArgs stream[2];   // text, visual
  const int32_t* ids;
  const int32_t* starts;
  uint16_t* out;
  float* lse;
  float* part;          // [teams][2][8 * NT * (D + 2)] pieces of units that reach over a border
  unsigned long long* flags;   // [teams][2] a piece is there: holds this launch's number
  unsigned long long* turn;    // counts the launches of a captured call (take_turn)
  unsigned long long nonce;    // another one in every call
  int32_t* status;
  int32_t hq, hkv, group, page, page_shift;
  int32_t n_seqs, max_seqs, n_tokens, max_queries, causal, has_visual;
  float inv_group;
  uint32_t page_units, head_units;   // bytes of a page, and of a head's codes in it, / 64
  uint32_t code_units;               // bytes of a page's codes, / 64
  float scale_log2;
};

__device__ __forceinline__ float4 lds_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts_f4(uint32_t addr, float2 a, float2 b) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y) : "memory");
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const uint8_t* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// D = A B + C, fp16 operands (subnormal ones count), fp32 sums
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                              float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
// C += A B
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
constexpr uint32_t kLower = 0x000f000fu, kUpper = 0x00f000f0u;   // codes as two fp16 numbers: c * 2^-24, and c * 2^-20
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {      // NaN if one is
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// A warp's running state over the keys of one unit: up to 8 * NT query rows of one (sequence, KV head), its columns.
template <int D, int NT>
struct Rows {
  float acc[NT][D / 16][4];  // times 2^-24 (even elements) and 2^-20 (odd ones)
  float ref[NT][2];          // what a column's scores are relative to; 0 before the first key that it sees
  float l[NT][2], z[NT][2];  // this lane's part of sum p and sum p mid
  uint32_t step;             // bits of the power of two that the weights were divided by
  uint32_t seen;             // columns that have seen a key, a bit per (nt, x)
  bool all_seen;             // every column of the warp has
};

template <int D, int NT>
struct Query {
  uint32_t b[NT][D / 16][2];   // operands of the score products: lower codes' elements, and a 16th of the upper ones'
  float sum[NT][2];            // sum of the elements times 2^-24, for the columns 2 t and 2 t + 1
  float scale[NT][2];          // softmax scale * log2 e * the powers of two that were taken out of the column
};

// Row r of a unit is query r / group of the sequence, head r % group of the KV head.
__device__ __forceinline__ int query_of(const AttendArgs& A, int r) { return static_cast<int>((static_cast<float>(r) + 0.5f) * A.inv_group); }

template <int D, int NT>
struct RawQuery {
  uint4 x[NT][D / 32];
};
template <int D, int NT, int REP>
__device__ __forceinline__ void ask_query(RawQuery<D, NT>& raw, const AttendArgs& A, const StreamArgs& S, int64_t token0, int head0, int row0, int n_rows, int lane) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row0 + nt * 8 + (lane >> 2) % (8 / REP), query = query_of(A, r);
    const uint16_t* q = S.q + (token0 + query) * S.q_stride + static_cast<int64_t>(head0 + r - query * A.group) * D + (lane & 3) * (D / 4);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) raw.x[nt][i] = r < n_rows ? __ldg(reinterpret_cast<const uint4*>(q) + i) : make_uint4(0, 0, 0, 0);
  }
}

template <int D, int NT>
__device__ __forceinline__ void make_query(Query<D, NT>& Q, const RawQuery<D, NT>& given, const AttendArgs& A, int lane) {
  const int t = lane & 3;
  const uint4(&raw)[NT][D / 32] = given.x;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 x = raw[nt][i];
      top = max_bf16x2(top, max_bf16x2(max_bf16x2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), max_bf16x2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
    }
    top = max_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int top_exp = static_cast<int>(max(top & 0xffffu, top >> 16) >> 7);      // (of numbers that are not negative, the larger one has the larger bits)
    // 2^e with the row's largest element times 2^-e in [2^14, 2^15); below 2^-90 it counts as that, from 2^101 on it has no scores
    const int e = min(max(top_exp - 127, -90), 100) - 14;
    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);   // -104 <= e <= 86
    const float scale = A.scale_log2 * __uint_as_float(static_cast<uint32_t>(127 + 24 + e) << 23);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      float f[8];
      bf16x8_to_f32(raw[nt][i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= down;
      const float s = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
      sum += s;
      Q.b[nt][2 * i][0] = pack_f16x2(f[0], f[4]);
      Q.b[nt][2 * i][1] = pack_f16x2(f[1] * 0.0625f, f[5] * 0.0625f);
      Q.b[nt][2 * i + 1][0] = pack_f16x2(f[2], f[6]);
      Q.b[nt][2 * i + 1][1] = pack_f16x2(f[3] * 0.0625f, f[7] * 0.0625f);
    }
    if (top_exp > 127 + 100) sum = NAN;      // (an infinity or a NaN among them)
    sum *= 5.9604644775390625e-8f;      // 2^-24
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    Q.sum[nt][0] = __shfl_sync(0xffffffffu, sum, t * 8);
    Q.sum[nt][1] = __shfl_sync(0xffffffffu, sum, t * 8 + 4);
    Q.scale[nt][0] = __shfl_sync(0xffffffffu, scale, t * 8);
    Q.scale[nt][1] = __shfl_sync(0xffffffffu, scale, t * 8 + 4);
  }
}

// ---- tiles on their way -------------------------------------------------------------------------------
//
// A warp fetches its tiles into a ring of its own: two places for the codes of K's tiles and two for V's, and two for the
// parameters (K's, then V's) of a tile, which come with its K.  A lane's 16-byte copies are the vectors that it reads
// later itself; the parameters are read by other lanes.
template <int D>
struct Ring {
  static constexpr int kCodes = kTile * D / 2;
  static constexpr int kParams = kTile * 8;
  static constexpr int kBytes = 4 * kCodes + 2 * kParams;
};

// A run: adjacent tiles of one stream, kBatch of which a lane's worth of page ids covers.
constexpr int kBatch = 32 / (kTile / 16);

// Where the blocks of a batch of tiles are, one per lane, in units of 64 bytes: a block's parameters are one unit.
struct Batch {
  uint32_t codes, params;
  bool there;
};

__device__ __forceinline__ int32_t ask_ids(const AttendArgs& A, const int32_t* table, int tile, int len, int lane) {
  const int key = tile * kTile + lane * 16;
  return key < len ? __ldg(table + (key >> A.page_shift)) : -1;
}

template <int D>
__device__ __forceinline__ Batch batch_of(const AttendArgs& A, const StreamArgs& S, int32_t id, int kvh, int tile, int len, int lane) {
  const int key = tile * kTile + lane * 16, block = (key & (A.page - 1)) >> 4;
  Batch b;
  b.there = static_cast<uint32_t>(id) < static_cast<uint32_t>(S.n_pages);
  if (!b.there && key < len && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_BAD_PAGE));   // a page that is none is not followed
  const uint32_t page = (b.there ? static_cast<uint32_t>(id) : 0u) * A.page_units;   // what is not there is fetched from page 0 and never looked at
  b.codes = page + kvh * A.head_units + block * (D / 8);
  b.params = page + A.code_units + ((kvh * A.page) >> 4) + block;
  return b;
}

// Requests the codes of a tile of K and the parameters of K and V; `at` (0, 4, ..): the tile's blocks in the batch.
template <int D>
__device__ __forceinline__ void fetch_keys(const StreamArgs& S, const Batch& batch, int at, uint32_t codes, uint32_t params, int lane) {
#pragma unroll
  for (int b = 0; b < kTile / 16; ++b) {
    const uint8_t* src = S.k_pool + static_cast<uint64_t>(__shfl_sync(0xffffffffu, batch.codes, at + b)) * 64 + lane * 16;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) cp_async_16(codes + b * (8 * D) + i * 512 + lane * 16, src + i * 512);
  }
  const uint32_t p = __shfl_sync(0xffffffffu, batch.params, at + (lane >> 2 & 3));
  cp_async_16(params + lane * 16, (lane < 16 ? S.k_pool : S.v_pool) + static_cast<uint64_t>(p) * 64 + (lane & 3) * 16);
}

template <int D>
__device__ __forceinline__ void fetch_values(const StreamArgs& S, const Batch& batch, int at, uint32_t codes, int lane) {
#pragma unroll
  for (int b = 0; b < kTile / 16; ++b) {
    const uint8_t* src = S.v_pool + static_cast<uint64_t>(__shfl_sync(0xffffffffu, batch.codes, at + b)) * 64 + lane * 16;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) cp_async_16(codes + b * (8 * D) + i * 512 + lane * 16, src + i * 512);
  }
}

// ---- a tile -----------------------------------------------------------------------------------------------

// The products of block b of a tile of K with the queries: c[nt] for the lane's even token (0, 1: columns 2 t, 2 t + 1) and
// its odd one (2, 3), times 2^-24.
template <int D, int NT>
__device__ __forceinline__ void score_block(float (&c)[NT][4], const Query<D, NT>& Q, uint32_t codes, int b, int lane) {
  uint32_t x[D / 16];      // the words of the even token, then of the odd one
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint4 k = lds128(codes + b * (8 * D) + i * 512 + lane * 16);
    x[4 * i] = k.x, x[4 * i + 1] = k.y, x[4 * i + 2] = k.z, x[4 * i + 3] = k.w;
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
#pragma unroll
  for (int w = 0; w < D / 32; ++w)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t xe = x[w] >> (8 * h), xo = x[D / 32 + w] >> (8 * h);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_f16_16816(c[nt], xe & kLower, xo & kLower, xe & kUpper, xo & kUpper, Q.b[nt][2 * w + h][0], Q.b[nt][2 * w + h][1]);
    }
}

__device__ __forceinline__ float step_of(uint32_t params) {
  const float r = __uint_as_float(params & 0xffff0000u);
  float s;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(r));   // (off by 2^-23 of itself)
  return r == 0.f ? 0.f : s;
}

// What the parameters of a tile's rows say, each worked out by one lane: lane l has the rows 4 l .. 4 l + 3 of 128, K's and then
// V's.  (s, lo) for K, (s, lo + 8 s) for V; those of V rows that are not there may be whatever was there before
// and count as 0.
struct RowValues {
  float2 v[4];
};
__device__ __forceinline__ float rows_of(RowValues& r, uint32_t params, uint32_t on, int left, bool masked, int lane) {
  const uint4 raw = lds128(params + lane * 16);
  const uint32_t p[4] = {raw.x, raw.y, raw.z, raw.w};
  const bool is_v = lane >= 16;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float s = step_of(p[i]);
    const float lo = __uint_as_float(p[i] << 16);
    float m = is_v ? fmaf(8.f, s, lo) : lo;
    if (masked && is_v && (!(on >> (lane >> 2 & 3) & 1u) || (lane & 15) * 4 + i >= left)) s = m = 0.f;
    top = fmaxf(top, s);
    r.v[i] = make_float2(s, m);
  }
  return is_v ? top : 0.f;
}

// Weights of a tile's scores, as operands of the value products.  `rows`: what rows_of found, in shared memory; `top`: the
// largest step that this lane saw.  `masked`: the tile has keys that are not there, or that some column does not see;
// `left` keys are there from its first on, `back` of them are behind the unit's first query.
template <int D, int NT, int REP>
__device__ __forceinline__ void weigh_tile(Rows<D, NT>& R, const float (&scores)[kTile / 16][NT][4], uint32_t (&w)[kTile / 16][NT][2], const Query<D, NT>& Q,
                                           uint32_t rows, float top, uint32_t on, const AttendArgs& A, int left, int row0, int back, bool masked, int lane) {
  constexpr int kMine = kTile / 16 / REP;      // blocks that this lane weighs
  const int g = lane >> 2, t = lane & 3;
  const int first = REP == 1 ? 0 : REP == 2 ? t & 2 : t;
  float c[kMine][NT][4];
#pragma unroll
  for (int b = 0; b < kMine; ++b) {
    const float4 k = lds_f4(rows + (first + b) * 128 + g * 16);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (REP == 1) c[b][nt][x] = scores[b][nt][x];
        else if constexpr (REP == 2) c[b][nt][x] = first ? scores[2 + b][nt][x] : scores[b][nt][x];
        else c[b][nt][x] = t & 2 ? (t & 1 ? scores[3][nt][x] : scores[2][nt][x]) : (t & 1 ? scores[1][nt][x] : scores[0][nt][x]);
      }
      // (s C + lo sum) stays below 2^127, whatever the row of K: |C| <= 15 * 2^15 * 128 * 2^-24
      const float2 sum = make_float2(Q.sum[nt][0], Q.sum[nt][1]), scale = make_float2(Q.scale[nt][0], Q.scale[nt][1]),
                   less = make_float2(-R.ref[nt][0], -R.ref[nt][1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 step = i ? make_float2(k.z, k.z) : make_float2(k.x, k.x), lo = i ? make_float2(k.w, k.w) : make_float2(k.y, k.y);
        const float2 x = fma2(fma2(step, make_float2(c[b][nt][2 * i], c[b][nt][2 * i + 1]), mul2(lo, sum)), scale, less);
        c[b][nt][2 * i] = x.x, c[b][nt][2 * i + 1] = x.y;
      }
    }
  }
  if (masked) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // keys of the tile that the column sees
        const int seen = left - max(0, back - query_of(A, row0 + nt * 8 + (2 * t + x) % (8 / REP)));
#pragma unroll
        for (int b = 0; b < kMine; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (!(on >> (first + b) & 1u) || 16 * (first + b) + 2 * g + i >= seen) c[b][nt][2 * i + x] = -INFINITY;
      }
  }
  // scores above what they are relative to, or larger steps than before: everything so far is put on a new reference
  bool more = !R.all_seen || __float_as_uint(top) > R.step;
  float high[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float h = fmaxf(c[0][nt][x], c[0][nt][x + 2]);
#pragma unroll
      for (int b = 1; b < kMine; ++b) h = max3(h, c[b][nt][x], c[b][nt][x + 2]);
      high[nt][x] = h;
      more |= h > 0.f;
    }
  if (__any_sync(0xffffffffu, more)) {
    // the next power of two; a step that is no number, or beyond 2^126, makes its row's outputs no numbers anyway
    const uint32_t top_bits = __reduce_max_sync(0xffffffffu, __float_as_uint(fminf(top, 8.5e37f)));
    const uint32_t now = max(R.step, top_bits > R.step ? (top_bits & 0x7f800000u) + 0x00800000u : 0u);
    const float down = now - R.step >= (126u << 23) ? 0.f : __uint_as_float((127u << 23) - (now - R.step));   // old / new
    R.step = now;
    bool all = true;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t bit = 1u << (2 * nt + x);
        float h = high[nt][x];
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 4));
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 8));
        h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 16));
        const bool known = R.seen & bit, any = h > -INFINITY;
        const float delta = (known ? h > 0.f : any) ? h : 0.f;
        const float corr = known ? ex2_approx(-delta) : 1.f;      // (nothing so far: nothing to put on another reference)
        R.ref[nt][x] += delta;
        if (any) R.seen |= bit;
        all &= (R.seen & bit) != 0;
        R.l[nt][x] *= corr;
        R.z[nt][x] *= corr;
        const float f = corr * down;
#pragma unroll
        for (int mb = 0; mb < D / 16; ++mb) R.acc[nt][mb][x] *= f, R.acc[nt][mb][x + 2] *= f;
#pragma unroll
        for (int b = 0; b < kMine; ++b) c[b][nt][x] -= delta, c[b][nt][x + 2] -= delta;
      }
    R.all_seen = __all_sync(0xffffffffu, all);
  }
  const float up = __uint_as_float(((127u + 127u + 15u) << 23) - R.step);      // 2^15 / step: the largest weight is 2^15
  uint32_t h[kMine][NT][2];
#pragma unroll
  for (int b = 0; b < kMine; ++b) {
    const float4 v = lds_f4(rows + kTile * 8 + (first + b) * 128 + g * 16);
    const float u0 = v.x * up, u1 = v.z * up, mid[2] = {v.y, v.w};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        p[x] = ex2_approx(c[b][nt][x]);
        R.l[nt][x & 1] += p[x];
      }
      if (!masked) {
#pragma unroll
        for (int x = 0; x < 4; ++x) R.z[nt][x & 1] = fmaf(p[x], mid[x >> 1], R.z[nt][x & 1]);
      } else {      // (a value that is no number counts only where it is seen)
#pragma unroll
        for (int x = 0; x < 4; ++x) R.z[nt][x & 1] = fmaf(p[x], p[x] == 0.f ? 0.f : mid[x >> 1], R.z[nt][x & 1]);
      }
      h[b][nt][0] = pack_f16x2(p[0] * u0, p[1] * u0);
      h[b][nt][1] = pack_f16x2(p[2] * u1, p[3] * u1);
      if constexpr (REP == 1) w[b][nt][0] = transpose_8x8(h[b][nt][0]), w[b][nt][1] = transpose_8x8(h[b][nt][1]);
    }
  }
  // a block's weights in the columns of the lanes that weighed it, 0 in the others
  if constexpr (REP > 1) {
#pragma unroll
    for (int b = 0; b < kTile / 16; ++b)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) w[b][nt][i] = transpose_8x8(b / kMine == (REP == 2 ? t >> 1 : t) ? h[b % kMine][nt][i] : 0u);
  }
}

// The values of a tile, and the scores of the next one (NEXT), side by side: neither waits for the other, and what one warp
// does between its tiles is a chain otherwise.
template <int D, int NT, bool NEXT>
__device__ __forceinline__ void add_values(Rows<D, NT>& R, const uint32_t (&w)[kTile / 16][NT][2], uint32_t codes, float (&c)[kTile / 16][NT][4],
                                           const Query<D, NT>& Q, uint32_t next_codes, int lane) {
  constexpr int kBlocks = kTile / 16;
  // - 8 * the weights' sums, of even elements' codes, and of odd ones' (which are 16 times as large)
  float less[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    less[nt][0] = less[nt][1] = less[nt][2] = less[nt][3] = 0.f;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)      // rows of 8 * 2^-24 and of 128 * 2^-24, negative
      mma_f16_16816(less[nt], 0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u, w[b][nt][0], w[b][nt][1]);
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    uint32_t x[kBlocks][4];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const uint4 v = lds128(codes + b * (8 * D) + i * 512 + lane * 16);
      x[b][0] = v.x, x[b][1] = v.y, x[b][2] = v.z, x[b][3] = v.w;
    }
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += 2) {
      if constexpr (NEXT) {
        constexpr int kShare = kBlocks / (D / 32);
#pragma unroll
        for (int b = 0; b < kShare; ++b) score_block<D, NT>(c[(2 * i + j0 / 2) * kShare + b], Q, next_codes, (2 * i + j0 / 2) * kShare + b, lane);
      }
      float sum[2][NT][4];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t lo = x[b][j0 + j], hi = lo >> 8;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (b == 0) mma_f16_16816(sum[j][nt], lo & kLower, lo & kUpper, hi & kLower, hi & kUpper, w[b][nt][0], w[b][nt][1], less[nt][0], less[nt][1], less[nt][2], less[nt][3]);
            else mma_f16_16816(sum[j][nt], lo & kLower, lo & kUpper, hi & kLower, hi & kUpper, w[b][nt][0], w[b][nt][1]);
          }
        }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) R.acc[nt][4 * i + j0 + j][k] += sum[j][nt][k];
    }
  }
}

// ---- the batch's work as one row -------------------------------------------------------------------------
//
// Sequence after sequence, unit after unit (KV head, then rows of queries), tile after tile (the visual stream's, then the
// text's).  The row is cut into ranges of equal cost, one per team of 1, 2, 4 or all warps of a block, so that the teams end together
// whatever the lengths are; the warps of a team share out a unit's tiles.  A unit costs its tiles and kUnitCost more for
// every warp of the team.  A unit inside one range is finished there; of one that reaches over a border each team leaves
// its sums, a piece, and raises the piece's flag.  Then it looks at the flags of the unit's other pieces: the team that
// finds all of them up puts the pieces together, in the order of the teams, and takes the flags down.  (Each team raises its
// own before it looks, so the last one finds all.  Two may, and write the same.  A flag is up when it holds the launch's
// number of 64 bits, so the workspace needs no clearing.)  Where units are short next to that, or next to a range, a
// team takes those that begin in its range whole, and nothing is left to put together.
//
// Teams of one warp are the even ones: with teams of a whole block, a range of many short units costs more than one of a long
// unit (16 sequences of 60 to 5 000 tokens, 32 heads: 52.2 us with whole blocks, 29.7 with single warps; 40 sequences of
// 33 000, 4 heads of 4: 142 and 135).  Whole blocks only where there are fewer units than blocks, two or four warps
// where the whole batch is small.

struct Place {       // one sequence
  int64_t token0;    // its first query
  int32_t n_rows;    // query rows per KV head; 0: nothing to do
  int32_t queries, row;
  int32_t len[2], tiles_v, tiles;
};

__device__ __forceinline__ int length_of(const AttendArgs& A, const StreamArgs& S, int row, bool report) {
  const int64_t len = __ldg(S.lens + row), room = static_cast<int64_t>(S.max_pages) << A.page_shift;
  if (len >= 0 && len <= room) return static_cast<int>(len);
  if (report && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_PLAN));
  return len < 0 ? 0 : static_cast<int>(room);
}

__device__ __forceinline__ Place place_of(const AttendArgs& A, int seq, bool report) {
  Place u{};
  int64_t a = seq, b = seq + 1;
  if (A.starts) a = __ldg(A.starts + seq), b = __ldg(A.starts + seq + 1);
  u.row = A.ids ? __ldg(A.ids + seq) : seq;
  if (a < 0 || b < a || b > A.n_tokens || b - a > A.max_queries || u.row < 0 || u.row >= A.max_seqs) {
    if (report && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_INVALID_ARG));
    return u;
  }
  u.token0 = a;
  u.queries = static_cast<int32_t>(b - a);
  u.n_rows = u.queries * A.group;
  if (u.n_rows == 0) return u;
  u.len[0] = length_of(A, A.stream[0], u.row, report);
  u.len[1] = A.has_visual ? length_of(A, A.stream[1], u.row, report) : 0;
  u.tiles_v = (u.len[1] + kTile - 1) / kTile;
  u.tiles = max(1, u.tiles_v + (u.len[0] + kTile - 1) / kTile);   // (without any key there still is a row to write)
  return u;
}

// What a part with reference ms and a sum counts for on reference m.  Minus infinity with a sum means that its scores were
// no numbers.
__device__ __forceinline__ float weight_of(float ms, float m) { return ms == -INFINITY ? NAN : ex2_approx(ms - m); }

// Sums (reference, sum, elements) put on one reference, 32 at a time, one per lane.
struct Joined {
  float m = -INFINITY, l = 0.f;
  // This lane's sum counts for what is returned; the elements so far are put on the new reference.
  template <int N>
  __device__ __forceinline__ float join(float2 ml, float (&o)[N]) {
    float top = ml.x;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    top = fmaxf(top, m);
    const float f = ml.y == 0.f ? 0.f : weight_of(ml.x, top), before = l == 0.f ? 0.f : weight_of(m, top);
    float sum = ml.y * f;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
    l = fmaf(l, before, sum);
    m = top;
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] *= before;
    return f;
  }
};

template <int D>
__device__ __forceinline__ void write_row(const AttendArgs& A, size_t row, float m, float l, const float (&o)[D / 32], int lane) {
  float inv, log;      // (off by 2^-23 of themselves, and by 2^-22)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(l));
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(log) : "f"(l));
  if (l == 0.f) inv = 0.f;
  if constexpr (D == 128) {
    reinterpret_cast<uint2*>(A.out + row * D)[lane] = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
  } else {
    reinterpret_cast<uint32_t*>(A.out + row * D)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
  }
  if (A.lse && lane == 0) A.lse[row] = l == 0.f ? -INFINITY : (m + log) * 0.69314718055994531f;
}

// the same from memory that another block wrote in this launch
template <int D>
__device__ __forceinline__ void load_run_l2(const float* p, float (&o)[D / 32], int lane) {
  if constexpr (D == 128) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(p) + lane);
    o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
  } else {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(p) + lane);
    o[0] = v.x, o[1] = v.y;
  }
}

template <int D>
__device__ __forceinline__ void load_run(const float* p, float (&o)[D / 32], int lane) {   // this lane's elements of a row
  if constexpr (D == 128) {
    const float4 v = reinterpret_cast<const float4*>(p)[lane];
    o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
  } else {
    const float2 v = reinterpret_cast<const float2*>(p)[lane];
    o[0] = v.x, o[1] = v.y;
  }
}

// A piece: columns of D elements, then (reference, sum) of each column.
template <int D, int ROWS>
__device__ __forceinline__ float* piece_at(const AttendArgs& A, int team, int place) {
  return A.part + (static_cast<size_t>(team) * 2 + place) * (ROWS * (D + 2));
}

// Puts the pieces of a unit together and writes its rows: columns member, member + warps, ...  Not inlined, so that the
// loop over the tiles keeps its registers.
template <int D, int ROWS>
__device__ __noinline__ void merge_pieces(const AttendArgs& A, uint32_t first_team, uint32_t last_team, uint32_t first_place, int member, int warps, int n_here,
                                          int row0, int64_t token0, int kvh, int lane) {
  constexpr int kCols = 4;      // columns side by side: each one's sums are two trips to the L2 after one another
  for (int col0 = member; col0 < n_here; col0 += kCols * warps) {
    float o[kCols][D / 32] = {};
    Joined J[kCols];
    const auto col_of = [&](int c) { return min(col0 + c * warps, n_here - 1); };
    for (uint32_t i0 = first_team; i0 <= last_team; i0 += 32) {
      const uint32_t i = i0 + lane;
      const int n = min(32u, last_team + 1 - i0);
      float2 ml[kCols];
      float f[kCols];
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
        ml[c] = make_float2(-INFINITY, 0.f);
        if (lane < n) ml[c] = __ldcg(reinterpret_cast<const float2*>(piece_at<D, ROWS>(A, i, i == first_team ? first_place : 0) + ROWS * D) + col_of(c));
      }
#pragma unroll
      for (int c = 0; c < kCols; ++c) f[c] = J[c].join(ml[c], o[c]);
#pragma unroll 2
      for (int k = 0; k < n; ++k) {
        const float* piece = piece_at<D, ROWS>(A, i0 + k, i0 + k == first_team ? first_place : 0);
        float v[kCols][D / 32];
#pragma unroll
        for (int c = 0; c < kCols; ++c) load_run_l2<D>(piece + col_of(c) * D, v[c], lane);
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          const float fk = __shfl_sync(0xffffffffu, f[c], k);
#pragma unroll
          for (int j = 0; j < D / 32; ++j) o[c][j] = fmaf(v[c][j], fk, o[c][j]);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      const int r = row0 + col0 + c * warps, query = query_of(A, r);
      if (col0 + c * warps < n_here)
        write_row<D>(A, static_cast<size_t>(token0 + query) * A.hq + kvh * A.group + r - query * A.group, J[c].m, J[c].l, o[c], lane);
    }
  }
}

__device__ __forceinline__ unsigned long long flag_of(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}

// What this launch's flags hold: the call's number and, as the replays of a captured call all have that, how often it has
// been launched in this workspace.  (Flags that no team found all up stay up: where lengths changed while a call ran, its blocks
// may have shared the batch out in different ways.  A later replay must not take them for its own.)  The upper 44 bits of a word
// are the call's, else it counts from here on; where it begins is the clock's, so that a count that begins again does not repeat the
// one before.  Every block adds 1, once, and all find the same quotient: a launch's blocks have a multiple of the grid's size behind
// them.  The last block of a launch past half of the 20 bits ends the count.
// `begin`: where this block would have the count begin.  Nobody waits for what the exchange finds, but where units are cut
// (number_of; 100 sequences of 100 tokens, 8 heads of 4: 11.1 us, 11.4 if all wait, 10.8 without a count).
constexpr unsigned long long kTurns = (1ull << 20) - 1;
struct Turn {
  unsigned long long w, begin, found;
};
__device__ __forceinline__ void take_turn(Turn& t, unsigned long long* word, unsigned long long call) {
  if ((t.w ^ call) & ~kTurns) {
    t.begin = (call & ~kTurns) | (static_cast<uint32_t>(clock()) % 1024u) * gridDim.x;
    asm volatile("atom.relaxed.gpu.global.cas.b64 %0, [%1], %2, %3;" : "=l"(t.found) : "l"(word), "l"(t.w), "l"(t.begin) : "memory");
  }
  if (((t.w ^ call) & ~kTurns) || (t.w & kTurns) < kTurns / 2) {
    asm volatile("red.relaxed.gpu.global.add.u64 [%0], 1;" ::"l"(word) : "memory");
  } else {
    const uint32_t turn = static_cast<uint32_t>(atomicAdd(word, 1ull) & kTurns);
    if (turn % gridDim.x == gridDim.x - 1) atomicExch(word, 0ull);
  }
}
__device__ __forceinline__ unsigned long long number_of(const Turn& t, unsigned long long call) {
  unsigned long long found = t.w;
  if ((t.w ^ call) & ~kTurns) {
    found = t.found;
    asm volatile("" : "+l"(found));      // (waited for here, and no earlier)
    if (found == t.w) found = t.begin;   // else another block has begun the count
  }
  return (call ^ static_cast<unsigned long long>(static_cast<uint32_t>(found & kTurns) / gridDim.x) << 1) | 1ull;
}

__device__ __forceinline__ void team_barrier(int team, int threads) {
  if (threads == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory");
}

// What a team knows about its range and the unit it is at, found by its first warp.  Kept in shared memory: it is looked at
// once a unit, and the loop over the tiles has no registers to spare for it.
struct Work {
  int64_t token0;
  int32_t n_rows, queries, row, len[2], tiles_v, tiles;                     // the sequence (Place)
  int32_t kvh, row0, first, last;                                           // the unit, and its tiles that are in the range
  uint32_t unit_at, at, end;                                                // where the unit begins, where the next one does, where the range ends
  int32_t seq, whole_units, found, warps;
  uint32_t per, longer, more, per_tile, team;   // cost of a range, ranges that cost one more, cost of a unit besides its tiles, and of a tile
};

// One block per SM, of twelve warps (168 registers a thread; eight with 255 have too little on their way: 71.1 us instead of 65.9
// for eight sequences of 8 541 tokens, 32 heads).  With sixteen rows to a unit eight warps, or its sums would not stay in registers.
template <int NT>
constexpr int kWarpsOf = NT == 1 ? 12 : 8;
template <int D, int NT, int REP>
__global__ void __launch_bounds__(kWarpsOf<NT> * 32, 1) quant_attend_kernel(const __grid_constant__ AttendArgs A) {
  constexpr int kAttWarps = kWarpsOf<NT>;
  using R_ = Ring<D>;
  constexpr int kRow = D + 4;            // of a column's sums in shared memory
  constexpr int kRows = 8 * NT / REP;    // query rows of a unit
  static_assert(8 * NT * kRow * 4 <= R_::kBytes, "a warp's sums take its ring's place");
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint2 scan[kAttWarps];
  __shared__ float sm_m[kAttWarps][8 * NT], sm_l[kAttWarps][8 * NT];
  __shared__ uint32_t longest_;
  __shared__ uint2 sums_;      // tiles and units of the batch
  __shared__ unsigned long long number_;
  __shared__ int sm_all[kAttWarps];
  __shared__ Work work_[kAttWarps];
  __shared__ int2 me_[kAttWarps];      // a warp's team in the block, its place in the team
  uint2* before = reinterpret_cast<uint2*>(smem + kAttWarps * R_::kBytes);   // [n_seqs + 1] tiles and units of the sequences before
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  pdl_wait();
  if (threadIdx.x == 0) before[0] = make_uint2(0, 0), longest_ = 0;
  __syncthreads();
  const bool counts = threadIdx.x == (kAttWarps - 1) * 32;
  Turn turn{};
  if (counts) turn.w = flag_of(A.turn);
  // what a sequence costs, and the sums up to it over a warp
  const auto cost_of = [&](int i, uint32_t& x, uint32_t& n) {
    uint64_t mine = 0;
    n = 0;
    if (i < A.n_seqs) {
      const Place u = place_of(A, i, blockIdx.x == 0);
      n = A.hkv * ((u.n_rows + kRows - 1) / kRows);
      mine = static_cast<uint64_t>(u.tiles) * n;
      if (n) atomicMax(&longest_, static_cast<uint32_t>(u.tiles));
    }
    const bool big = mine > (1u << 22);
    x = big ? 0u : static_cast<uint32_t>(mine);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, x, o), k = __shfl_up_sync(0xffffffffu, n, o);
      if (lane >= o) x += y, n += k;
    }
    return big;
  };
  constexpr uint32_t kMost = 1u << 26;      // tiles of a batch: 2^32 rows
  if (A.n_seqs <= 64) {      // one warp: a small batch is soon done, and what a block does once it waits for, instructions included
    if (warp == 0) {
      uint32_t tiles = 0, units = 0;
      for (int i0 = 0; i0 < A.n_seqs; i0 += 32) {
        uint32_t x, n;
        if (__any_sync(0xffffffffu, cost_of(i0 + lane, x, n))) tiles = kMost + 1;
        if (i0 + lane < A.n_seqs) before[i0 + lane + 1] = make_uint2(tiles + x, units + n);
        tiles += __shfl_sync(0xffffffffu, x, 31), units += __shfl_sync(0xffffffffu, n, 31);
      }
      if (lane == 0) sums_ = make_uint2(tiles, units);
    }
  } else {
    uint2 all = make_uint2(0, 0);
#pragma unroll 1
    for (int i0 = 0; i0 < A.n_seqs; i0 += kAttWarps * 32) {
      const int i = i0 + threadIdx.x;
      uint32_t x, n;
      const bool big = cost_of(i, x, n);
      if (lane == 31) scan[warp] = make_uint2(x, n);
      if (__syncthreads_or(big)) all.x = kMost + 1;
      uint2 base = all;
#pragma unroll 1
      for (int w = 0; w < kAttWarps; ++w) {
        if (w < warp) base.x += scan[w].x, base.y += scan[w].y;
        all.x += scan[w].x, all.y += scan[w].y;
      }
      if (i < A.n_seqs) before[i + 1] = make_uint2(base.x + x, base.y + n);
      all.x = min(all.x, 2 * kMost);
      __syncthreads();
    }
    if (threadIdx.x == 0) sums_ = all;
  }
  if (counts) take_turn(turn, A.turn, A.nonce);
  __syncthreads();
  if (sums_.x > kMost) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && A.status) atomicMax(A.status, static_cast<int>(QC_ERR_PLAN));
    return;
  }
  const uint32_t tiles_all = sums_.x, units = sums_.y, longest = longest_;
  const uint32_t n_warps = gridDim.x * kAttWarps;
  uint32_t team_warps = 1;
  if (units * kAttWarps <= n_warps) team_warps = kAttWarps;
  else if (tiles_all <= n_warps * kFewTiles<kRows>) team_warps = units * 4 <= n_warps ? 4 : units * 2 <= n_warps ? 2 : 1;
  const int shift = team_warps == 2 ? 1 : team_warps == 4 ? 2 : 0;      // (of the teams that are not a whole block)
  const uint32_t n_teams = team_warps == kAttWarps ? gridDim.x : n_warps >> shift;
  // a team for every unit, each one short: one each, whatever they cost.  Else a unit's cost is at most a range's share of the tiles:
  // a whole range would have nothing but a cost to cover (one sequence of 32 000 tokens, 8 heads of 8: 27.0 us without that, 23.9 so)
  const bool one_each = units <= n_teams && longest <= team_warps * kWholeTiles;
  const uint32_t more = one_each ? 1 : max(1u, min(kUnitCost * team_warps, tiles_all / n_teams)), per_tile = one_each ? 0 : 1, cost = tiles_all * per_tile + units * more;
  // ranges of per_team or one more
  uint32_t per_team = cost / n_teams, longer = cost - per_team * n_teams;
  const bool whole_units = longest <= max(team_warps * kWholeTiles, per_team / 8);
  if (!whole_units && per_team < team_warps) per_team = team_warps, longer = 0;
  if (counts && !whole_units) number_ = number_of(turn, A.nonce);
  const auto before_cost = [&](int s) { return before[s].x * per_tile + before[s].y * more; };
  const int in_block = team_warps == kAttWarps ? 0 : warp >> shift, member = team_warps == kAttWarps ? warp : warp & (team_warps - 1);
  volatile Work& W = work_[in_block];
  if (lane == 0) me_[warp] = make_int2(in_block, member);
  if (member == 0 && lane == 0) {
    // where there are more teams than units, those that find nothing to do are spread over the chip (64 sequences of 20 to 100
    // tokens, 8 heads of 8: 10.5 us against 11.7); else adjacent ranges share an SM (16 ragged sequences: 29.5 against 30.6)
    const uint32_t team = one_each ? in_block * gridDim.x + blockIdx.x : blockIdx.x * (kAttWarps / team_warps) + in_block;
    const uint32_t at = min(static_cast<uint64_t>(team) * per_team + min(team, longer), static_cast<uint64_t>(cost));
    W.warps = team_warps, W.team = team, W.per = per_team, W.longer = longer, W.more = more, W.per_tile = per_tile, W.whole_units = whole_units;
    W.at = at, W.end = min(cost, at + per_team + (team < longer ? 1 : 0));
    int lo = 0, hi = A.n_seqs - 1;      // the last sequence that begins at or before the range
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before_cost(mid) <= at) lo = mid;
      else hi = mid - 1;
    }
    W.seq = lo;
  }
  __syncthreads();      // every warp knows its team, and the team's size
  const uint32_t ring = smem_u32(smem) + warp * R_::kBytes;
  while (true) {
    if (me_[warp].y == 0) {   // the team's first warp finds its next unit
      __syncwarp();
      uint32_t at = W.at;
      const uint32_t end = W.end, more = W.more, per_tile = W.per_tile;
      int seq = W.seq, first = 0, last = 0;
      while (at < end && first >= last) {
        while (before[seq + 1].x * per_tile + before[seq + 1].y * more <= at) ++seq;
        const Place u = place_of(A, seq, false);
        const int row_tiles = (u.n_rows + kRows - 1) / kRows, units = A.hkv * row_tiles;
        const uint32_t unit_cost = u.tiles * per_tile + more, seq_at = before[seq].x * per_tile + before[seq].y * more;
        const int unit = (at - seq_at) / unit_cost;
        const uint32_t unit_at = seq_at + unit * unit_cost;
        last = u.tiles;
        if (W.whole_units) {
          if (unit_at < at) last = 0;      // it begins before the range: the next one
        } else {
          first = max(0, static_cast<int>(at - unit_at) - static_cast<int>(more));
          last = min(u.tiles, static_cast<int>(end - unit_at) - static_cast<int>(more));
        }
        if (unit >= units) last = 0;       // (lengths that change under the call: wrong sums, and no more than that)
        at = unit_at + unit_cost;
        if (first < last && lane == 0) {
          const int kvh = row_tiles == 1 ? unit : unit / row_tiles;
          W.unit_at = unit_at, W.first = first, W.last = last, W.kvh = kvh, W.row0 = (unit - kvh * row_tiles) * kRows;
          W.token0 = u.token0, W.n_rows = u.n_rows, W.queries = u.queries, W.row = u.row, W.len[0] = u.len[0], W.len[1] = u.len[1];
          W.tiles_v = u.tiles_v, W.tiles = u.tiles;
        }
      }
      if (lane == 0) W.seq = seq, W.at = at, W.found = first < last;
    }
    team_barrier(me_[warp].x, W.warps * 32);
    if (!W.found) break;

    Rows<D, NT> R;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int x = 0; x < 2; ++x) R.ref[nt][x] = R.l[nt][x] = R.z[nt][x] = 0.f;
#pragma unroll
      for (int mb = 0; mb < D / 16; ++mb) R.acc[nt][mb][0] = R.acc[nt][mb][1] = R.acc[nt][mb][2] = R.acc[nt][mb][3] = 0.f;
    }
    R.step = kLeastStep;
    R.seen = 0;
    R.all_seen = false;

    // this warp's tiles of the unit, adjacent ones: a run in each stream
#pragma unroll 1
    for (int now = 1; now >= 0; --now) {
      const int first = W.first, n = W.last - first, warps = W.warps, member = me_[warp].y, tiles_v = W.tiles_v;
      const int mine0 = first + n * member / warps, mine1 = first + n * (member + 1) / warps;      // (even shares: warps share their units)
      const int shift = now ? 0 : tiles_v;      // the stream's first tile in the unit
      const int run = max(mine0, shift) - shift, stop = (now ? min(mine1, tiles_v) : mine1) - shift;
      if (run >= stop) continue;
      const StreamArgs& S = A.stream[now];
      const int len = W.len[now], back = now || !A.causal ? 0 : W.queries - 1, kvh = W.kvh;
      const int32_t* table = S.pages + static_cast<size_t>(W.row) * S.max_pages;
      // the next tile to ask for: its batch's first tile, the batch, and the next batch's page ids
      int asked = run, at_tile = run;
      int32_t ids = ask_ids(A, table, run, len, lane);
      RawQuery<D, NT> raw;
      ask_query<D, NT, REP>(raw, A, S, W.token0, kvh * A.group, W.row0, W.n_rows, lane);
      Batch batch = batch_of<D>(A, S, ids, kvh, run, len, lane);
      ids = ask_ids(A, table, run + kBatch, len, lane);
      uint32_t there = 0;      // blocks that are there of the next two tiles and the two behind them, 4 bits a tile
      const uint32_t params = ring + 4 * R_::kCodes;
      const auto ask_keys = [&]() {       // of tile `asked`
        if (asked < stop) {
          const int at = (asked - at_tile) * 4;
          there |= (__ballot_sync(0xffffffffu, batch.there) >> at & 15u) << ((asked & 3) * 4);
          fetch_keys<D>(S, batch, at, ring + (asked & 1) * R_::kCodes, params + (asked & 1) * R_::kParams, lane);
        }
        cp_async_commit_group();
      };
      const auto ask_values = [&]() {      // of the same tile; then the next one's turn
        if (asked < stop) fetch_values<D>(S, batch, (asked - at_tile) * 4, ring + (2 + (asked & 1)) * R_::kCodes, lane);
        cp_async_commit_group();
        if (++asked - at_tile == kBatch) {
          at_tile += kBatch;
          batch = batch_of<D>(A, S, ids, kvh, at_tile, len, lane);
          ids = ask_ids(A, table, at_tile + kBatch, len, lane);
        }
      };
      ask_keys();
      ask_values();
      ask_keys();
      ask_values();
      Query<D, NT> Q;
      make_query<D, NT>(Q, raw, A, lane);
      float c[kTile / 16][NT][4];
      cp_async_wait_group<3>();
      __syncwarp();
#pragma unroll
      for (int b = 0; b < kTile / 16; ++b) score_block<D, NT>(c[b], Q, ring + (run & 1) * R_::kCodes, b, lane);
      for (int tile = run; tile < stop; ++tile) {
        const uint32_t on = there >> ((tile & 3) * 4) & 15u;
        there &= ~(15u << ((tile & 3) * 4));
        const int left = len - tile * kTile;
        const bool masked = left - back < kTile || on != 15u;
        const uint32_t scratch = ring + (tile & 1) * R_::kCodes;      // K's place: its codes have been read
        uint32_t w[kTile / 16][NT][2];
        float top;
        __syncwarp();
        {
          RowValues rows;
          top = rows_of(rows, params + (tile & 1) * R_::kParams, on, left, masked, lane);
          sts_f4(scratch + lane * 32, rows.v[0], rows.v[1]);
          sts_f4(scratch + lane * 32 + 16, rows.v[2], rows.v[3]);
        }
        __syncwarp();
        weigh_tile<D, NT, REP>(R, c, w, Q, scratch, top, on, A, left, W.row0, back, masked, lane);
        __syncwarp();
        ask_keys();                  // two tiles on, in this one's places
        cp_async_wait_group<2>();    // the next tile's keys, this one's values
        __syncwarp();
        const uint32_t values = ring + (2 + (tile & 1)) * R_::kCodes, next = ring + ((tile + 1) & 1) * R_::kCodes;
        if (tile + 1 < stop) add_values<D, NT, true>(R, w, values, c, Q, next, lane);
        else add_values<D, NT, false>(R, w, values, c, Q, next, lane);
        __syncwarp();
        ask_values();
      }
      cp_async_wait_all();
      __syncwarp();
    }
    // the team's sums meet in shared memory
    const int in_block = me_[warp].x, member = me_[warp].y, n_rows = W.n_rows, row0 = W.row0, kvh = W.kvh, warps = W.warps, threads = warps * 32, team0 = in_block * warps;
    const int64_t token0 = W.token0;
    const float unit_step = __uint_as_float(R.step) * (1.f / 32768.f);
    constexpr float kEven = 16777216.f, kOdd = 1048576.f;
    float* mine = reinterpret_cast<float*>(smem + warp * R_::kBytes);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float l = R.l[nt][x], z = R.z[nt][x];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o), z += __shfl_xor_sync(0xffffffffu, z, o);
        const int col = nt * 8 + 2 * t + x;
        if (g == 0) sm_m[warp][col] = R.seen >> (2 * nt + x) & 1u ? R.ref[nt][x] : -INFINITY, sm_l[warp][col] = l;
        if (row0 + col % kRows < n_rows) {
          float* dst = mine + col * kRow + g * (D / 8);
#pragma unroll
          for (int mb = 0; mb < D / 16; mb += 2)
            *reinterpret_cast<float4*>(dst + 2 * mb) = make_float4(fmaf(R.acc[nt][mb][x] * kEven, unit_step, z), fmaf(R.acc[nt][mb][x + 2] * kOdd, unit_step, z),
                                                                   fmaf(R.acc[nt][mb + 1][x] * kEven, unit_step, z), fmaf(R.acc[nt][mb + 1][x + 2] * kOdd, unit_step, z));
        }
      }
    const int n_here = min(kRows, n_rows - row0);
    const bool whole = W.first == 0 && W.last == W.tiles;
    // pieces: the first team's is its second one if a unit before this one ends in its range, all others are a team's first
    const uint32_t team = W.team, unit_at = W.unit_at;
    uint32_t first_team = team, last_team = team, first_place = 0;
    if (!whole) {
      const uint32_t per = W.per, longer = W.longer, turn = longer * (per + 1);      // where the shorter ranges begin
      const uint32_t most = gridDim.x * (kAttWarps / warps) - 1;
      const auto team_at = [&](uint32_t p) { return min(most, p < turn ? p / (per + 1) : longer + (p - turn) / per); };
      first_team = team_at(unit_at + W.more), last_team = team_at(unit_at + W.tiles + W.more - 1);
      first_place = unit_at > first_team * per + min(first_team, longer) ? 1 : 0;
    }
    const uint32_t place = team == first_team ? first_place : 0;
    float* piece = piece_at<D, kRows>(A, team, place);
    // four sets of columns of a warp put together first, then the team's warps (the same instructions: they are fetched once)
    constexpr bool kTwice = REP == 4;
    constexpr int kSets = kTwice ? 1 : REP;
#pragma unroll 1
    for (int round = kTwice ? 0 : 1; round < 2; ++round) {
      const bool own = kTwice && round == 0;
      const int w0 = own ? warp : team0, n = own ? REP : warps * kSets;
      const auto ml_at = [&](int i) { return own ? i * kRows : i / kSets * (8 * NT) + i % kSets * kRows; };
      const auto row_at = [&](int i) { return own ? i * (kRows * kRow) : i / kSets * static_cast<int>(R_::kBytes / 4) + i % kSets * (kRows * kRow); };
      if (own) __syncwarp();
      else team_barrier(in_block, threads);
#pragma unroll 1
      for (int col = own ? 0 : member; col < n_here; col += own ? 1 : warps) {
        const int i = ml_at(min(lane, n - 1));
        const float2 ml = lane < n ? make_float2((&sm_m[w0][col])[i], (&sm_l[w0][col])[i]) : make_float2(-INFINITY, 0.f);
        float o[D / 32] = {};
        Joined J;
        const float f = J.join(ml, o);
        const float* row = reinterpret_cast<const float*>(smem + w0 * R_::kBytes) + col * kRow;
#pragma unroll 2
        for (int k = 0; k < n; ++k) {
          const float fk = __shfl_sync(0xffffffffu, f, k);
          float v[D / 32];
          load_run<D>(row + row_at(k), v, lane);
#pragma unroll
          for (int j = 0; j < D / 32; ++j) o[j] = fmaf(v[j], fk, o[j]);
        }
        if (!own && whole) {
          const int r = row0 + col, query = query_of(A, r);
          write_row<D>(A, static_cast<size_t>(token0 + query) * A.hq + kvh * A.group + r - query * A.group, J.m, J.l, o, lane);
        } else {
          float* to = own ? const_cast<float*>(row) : piece + col * D;
          if constexpr (D == 128) reinterpret_cast<float4*>(to)[lane] = make_float4(o[0], o[1], o[2], o[3]);
          else reinterpret_cast<float2*>(to)[lane] = make_float2(o[0], o[1]);
          __syncwarp();
          if (lane == 0) {
            if (own) sm_m[warp][col] = J.m, sm_l[warp][col] = J.l;
            else reinterpret_cast<float2*>(piece + kRows * D)[col] = make_float2(J.m, J.l);
          }
        }
      }
    }
    if (!whole) {
      team_barrier(in_block, threads);
      if (member == 0) {
        asm volatile("fence.acq_rel.gpu;" ::: "memory");      // the piece, which other warps wrote a part of, is there before its flag
        if (lane == 0) atomicExch(A.flags + 2 * team + place, number_);
        __syncwarp();
        asm volatile("fence.sc.gpu;" ::: "memory");
        bool all = true;
        for (uint32_t i = first_team + lane; i <= last_team; i += 32) all &= flag_of(A.flags + 2 * i + (i == first_team ? first_place : 0)) == number_;
        all = __all_sync(0xffffffffu, all);
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
        if (lane == 0) sm_all[in_block] = all;
      }
      team_barrier(in_block, threads);
      if (sm_all[in_block]) {
        merge_pieces<D, kRows>(A, first_team, last_team, first_place, member, warps, n_here, row0, token0, kvh, lane);
        if (member == 0)
          for (uint32_t i = first_team + lane; i <= last_team; i += 32) A.flags[2 * i + (i == first_team ? first_place : 0)] = 0;
      }
    }
    team_barrier(in_block, threads);      // the rings' places, and what is known about the unit, are free again
  }
}

bool off(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

int32_t check_stream(const qc_quant_stream* s, const qc_quant_attend_args* a, StreamArgs& d) {
  if (!s->q_dev || !s->k_pool_dev || !s->v_pool_dev || !s->pages_dev || !s->lens_dev) return QC_ERR_INVALID_ARG;
  if (off(s->q_dev, 16) || off(s->k_pool_dev, 16) || off(s->v_pool_dev, 16) || off(s->pages_dev, 4) || off(s->lens_dev, 4)) return QC_ERR_INVALID_ARG;
  if (s->q_stride < 0 || s->q_stride % 8 || s->max_pages < 1 || s->n_pages < 1) return QC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(s->max_pages) * a->page_size > INT32_MAX - 4096 || static_cast<int64_t>(s->n_pages) * a->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  d.q = static_cast<const uint16_t*>(s->q_dev), d.q_stride = s->q_stride;
  d.k_pool = static_cast<const uint8_t*>(s->k_pool_dev), d.v_pool = static_cast<const uint8_t*>(s->v_pool_dev);
  d.pages = s->pages_dev, d.lens = s->lens_dev, d.max_pages = s->max_pages, d.n_pages = s->n_pages;
  return QC_OK;
}

// Whether the output lies over rows of queries that other blocks may still read.  At the very place of its query each row may be: a
// unit's rows are written by the team that finishes it, when all of its teams have read them, and no other unit reads them.
bool over_queries(const qc_quant_stream* s, const qc_quant_attend_args* a) {
  const uint64_t row = static_cast<uint64_t>(a->n_q_heads) * a->head_dim * 2, stride = static_cast<uint64_t>(s->q_stride) * 2;
  const uint64_t q = reinterpret_cast<uintptr_t>(s->q_dev), out = reinterpret_cast<uintptr_t>(a->out_dev), end = out + row * a->n_tokens;
  if (a->n_tokens < 1 || (q == out && (stride == row || a->n_tokens == 1))) return false;
  if (q >= end) return false;
  if (q + row > out || stride == 0) return q + row > out;
  const uint64_t token = (out - row - q) / stride + 1;      // the first whose row ends behind the output's beginning
  return token < static_cast<uint64_t>(a->n_tokens) && q + token * stride < end;
}

int32_t check_sizes(const qc_quant_attend_args* a) {
  if (!a) return QC_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (a->page_size != 16 && a->page_size != 32 && a->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (a->n_kv_heads < 1 || a->n_q_heads < 1 || a->n_q_heads % a->n_kv_heads || a->n_seqs < 1 || a->max_seqs < 1 || a->n_tokens < 0 || a->max_queries < 1)
    return QC_ERR_INVALID_ARG;
  if (a->n_kv_heads > QC_QUANT_MAX_HEADS || a->n_q_heads > QC_QUANT_MAX_HEADS || a->n_seqs > QC_QUANT_MAX_SEQS || a->max_queries > QC_QUANT_MAX_QUERIES)
    return QC_ERR_UNSUPPORTED;
  return QC_OK;
}

// Query rows of a unit: as many columns of a product as they need.  Sixteen only where they are all taken (16 sequences of 8 000
// tokens, 4 heads of 8, 64 wide, two queries: 34.3 us against 36.3 with units of eight; with one to five queries on 4 heads of
// 4, 128 wide, 30 against 26).
int unit_rows(const qc_quant_attend_args* a) {
  const int64_t rows = static_cast<int64_t>(a->max_queries) * (a->n_q_heads / a->n_kv_heads);
  return rows <= 2 ? 2 : rows <= 4 ? 4 : rows % 16 ? 8 : 16;
}

constexpr int kMostTeams = 2560;   // of one warp each; the workspace is sized for it
constexpr int kFlagWords = kMostTeams * 2 + 16;   // flags and the count of launches; the pieces behind begin at a line of 128 bytes, as the workspace does
                                                  // (16 bytes off: 1 us of 66 for 8 sequences of 8 541 tokens)

static_assert(kMostTeams / 8 * 1024 < (1 << 19), "where the count of launches begins, and the blocks of one, in half of its 20 bits");

// A number that no other call has, nor memory by chance.
unsigned long long next_nonce() {
  static std::atomic<unsigned long long> count{static_cast<unsigned long long>(std::chrono::steady_clock::now().time_since_epoch().count()) * 0x9E3779B97F4A7C15ull ^
                                               static_cast<unsigned long long>(std::chrono::system_clock::now().time_since_epoch().count())};
  unsigned long long x = count.fetch_add(0x9E3779B97F4A7C15ull, std::memory_order_relaxed);   // splitmix64
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  x ^= x >> 31;
  return x ? x : 1;
}

template <int D, int NT, int REP>
cudaError_t launch(AttendArgs& A, int device, cudaStream_t stream) {
  constexpr int kAttWarps = kWarpsOf<NT>;
  const int smem = kAttWarps * Ring<D>::kBytes + (A.n_seqs + 1) * 8;
  constexpr int kMost = kAttWarps * Ring<D>::kBytes + (QC_QUANT_MAX_SEQS + 1) * 8;
  static std::atomic<bool> configured[64] = {};     // per device: the kernel may take that much
  cudaError_t e;
  if (device >= 64 || !configured[device].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(quant_attend_kernel<D, NT, REP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    if (device < 64) configured[device].store(true, std::memory_order_relaxed);
  }
  int sms = 0;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return e;
  int blocks = sms;
  if (blocks > kMostTeams / kAttWarps) blocks = kMostTeams / kAttWarps;
  A.nonce = next_nonce();
  return launch_pdl(quant_attend_kernel<D, NT, REP>, dim3(blocks), dim3(kAttWarps * 32), smem, stream, A);
}

template <int D>
cudaError_t launch_rows(AttendArgs& A, int rows, int device, cudaStream_t stream) {
  return rows == 2 ? launch<D, 1, 4>(A, device, stream) : rows == 4 ? launch<D, 1, 2>(A, device, stream) : rows == 8 ? launch<D, 1, 1>(A, device, stream)
                                                                                                                   : launch<D, 2, 1>(A, device, stream);
}

size_t workspace_bytes(const qc_quant_attend_args* a) {
  return kFlagWords * sizeof(unsigned long long) + static_cast<size_t>(kMostTeams) * 2 * unit_rows(a) * (a->head_dim + 2) * 4;
}

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_quant_workspace_bytes(const qc_quant_attend_args* args, size_t* bytes) {
  if (!bytes) return QC_ERR_INVALID_ARG;
  if (const int32_t bad = check_sizes(args)) return bad;
  *bytes = workspace_bytes(args);
  return QC_OK;
}

extern "C" int32_t qc_quant_attend(int32_t device, void* cuda_stream, const qc_quant_attend_args* args) {
  if (const int32_t bad = check_sizes(args)) return bad;
  if (!args->out_dev || off(args->out_dev, 16) || off(args->lse_out_dev, 4) || off(args->status_dev, 4) || off(args->seq_ids_dev, 4) ||
      off(args->starts_dev, 4) || off(args->workspace_dev, 16))
    return QC_ERR_INVALID_ARG;
  if (!(args->softmax_scale >= 0.f) || !isfinite(args->softmax_scale)) return QC_ERR_INVALID_ARG;
  if (!args->seq_ids_dev && args->n_seqs > args->max_seqs) return QC_ERR_INVALID_ARG;
  if (!args->starts_dev && args->n_tokens < args->n_seqs) return QC_ERR_INVALID_ARG;
  AttendArgs A{};
  if (const int32_t bad = check_stream(&args->text, args, A.stream[0])) return bad;
  const qc_quant_stream& v = args->visual;
  A.has_visual = v.q_dev || v.k_pool_dev || v.v_pool_dev || v.pages_dev || v.lens_dev;
  if (A.has_visual)
    if (const int32_t bad = check_stream(&v, args, A.stream[1])) return bad;
  if (over_queries(&args->text, args) || (A.has_visual && over_queries(&v, args))) return QC_ERR_INVALID_ARG;
  if (args->workspace_bytes < workspace_bytes(args) || !args->workspace_dev) return QC_ERR_INVALID_ARG;
  if (args->n_tokens == 0) return QC_OK;
  A.ids = args->seq_ids_dev, A.starts = args->starts_dev;
  A.out = static_cast<uint16_t*>(args->out_dev), A.lse = args->lse_out_dev;
  A.flags = static_cast<unsigned long long*>(args->workspace_dev), A.turn = A.flags + 2 * kMostTeams, A.part = reinterpret_cast<float*>(A.flags + kFlagWords);
  A.status = args->status_dev;
  A.hq = args->n_q_heads, A.hkv = args->n_kv_heads, A.group = A.hq / A.hkv, A.page = args->page_size;
  A.page_shift = A.page == 16 ? 4 : A.page == 32 ? 5 : 6;
  A.n_seqs = args->n_seqs, A.max_seqs = args->max_seqs, A.n_tokens = args->n_tokens, A.max_queries = args->starts_dev ? args->max_queries : 1;
  A.causal = args->causal != 0;
  A.inv_group = 1.f / A.group;
  A.head_units = static_cast<uint32_t>(A.page * (args->head_dim / 2) / 64), A.code_units = A.hkv * A.head_units;
  A.page_units = static_cast<uint32_t>(quant_page_bytes(A.hkv, args->head_dim, A.page) / 64);
  if (static_cast<int64_t>(args->text.n_pages) * A.page_units > UINT32_MAX || static_cast<int64_t>(A.has_visual ? v.n_pages : 0) * A.page_units > UINT32_MAX)
    return QC_ERR_UNSUPPORTED;
  const float scale = args->softmax_scale > 0.f ? args->softmax_scale : 1.0f / sqrtf(static_cast<float>(args->head_dim));
  A.scale_log2 = scale * 1.4426950408889634f;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int rows = unit_rows(args);
  const cudaError_t e = args->head_dim == 128 ? launch_rows<128>(A, rows, device, stream) : launch_rows<64>(A, rows, device, stream);
  return status_of(e);
}
