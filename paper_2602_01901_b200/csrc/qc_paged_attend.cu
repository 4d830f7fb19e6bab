// Attention of a step's queries over bf16 pages, where adjacent sequences of a batch share a prefix.
//
//   out = softmax(scale [q_shared K_prefix ; q_own K_own]) [V_prefix ; V_own]
//
// A prefix's keys are scored by all query rows of its group at once (its tokens times the query heads of a KV head), a sequence's
// own by its own rows: both are units of at most 128 rows over a run of keys, and one kernel takes them all, on the tensor
// cores.  What a unit finds of a row is (largest score, sum, weighted values); a second kernel puts a row's parts together.
//
// The batch is one row of units, prefixes first, whose costs (tiles of 64 keys, and a constant for a unit) are laid end to
// end and cut into equal ranges, one per block, two blocks an SM.  A unit inside one range leaves its rows at their queries' places; one that a border
// cuts leaves a piece per block.  Every number of this plan comes from the lists and lengths on the device.
//
// Per tile: S[128 x 64] = Q K^T and O[128 x D] += P V by tcgen05.mma, Q, K and V in shared memory (K and V by tensor-map copies of
// pages), S, P and O in tensor memory.  Four warps hold a row per thread, one issues products, one fetches.
// Units of few rows hold them two or four times (rows r and r + 64, or r + 32 and so on): every copy weighs another half or quarter of
// a tile's keys, so that all four warps take part in the exponentials; the copies are added up when the unit ends.

#include "../../include/qc.h"
#include "qc_quant.h"
#include "qc_umma.cuh"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace qc {
namespace {

constexpr int kRows = 128;       // query rows of a unit
constexpr int kKeys = 64;        // keys of a tile
constexpr int kBlock = kRows + 64;
constexpr int kUnits = 4;        // units that are known to the block at a time
constexpr int kMeta = 8;         // tiles whose places are
constexpr uint32_t kScoresAt = 0, kOutAt = 128, kColumns = 256;   // tensor memory: two score buffers of 64 columns, D of the sums
constexpr float kRescale = 8.f;  // the reference of a row moves when its scores have grown by 2^8
constexpr uint32_t kUnitCost = 2;
constexpr uint32_t kApart = 32, kLeastPiece = 4, kPieceShare = 4;
constexpr uint32_t kMostCost = 1u << 27;
constexpr int kSlim = 8;         // rows of a unit that four threads each hold in every warp
constexpr int kMostHeld = 2048;  // items that a block keeps in shared memory while it looks for its range

struct StreamArgs {
  const uint16_t* q;
  int64_t q_stride;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* pages;
  const int32_t* lens;
  int32_t max_pages, n_pages, rows;
};

// What the second kernel knows of a prefix or a sequence.
struct Record {
  uint32_t base;           // where its costs begin
  int32_t tiles, token0, queries;
  int32_t group;           // a sequence's prefix, or -1
  int32_t spare[3];
};

// A row of costs, cut into ranges: the first `longer` workers have `per` + 1, the others `per`.
struct Line {
  uint32_t begin, per, longer, workers;
  int32_t least;           // tiles of a piece
};
// Whether the batch is computed, and its rows of costs: prefixes and sequences in one, or in one each.
struct Plan {
  Line line[2];
  int32_t fine, lines;
};

struct AttendArgs {
  CUtensorMap map[2][2];  // K and V of own and shared pages: a copy brings a page's tokens of a head, 64 elements of K or all of V
  StreamArgs stream[2];   // own, shared
  const int32_t* ids;
  const int32_t* starts;
  const int32_t* groups;
  const int32_t* shared_ids;
  uint16_t* out;
  float* lse;
  Plan* plan;
  Record* records;        // [groups + sequences]
  float* rows;            // [kinds][tokens * heads][D] sums of whole units
  float2* row_ml;         // [kinds][tokens * heads]
  float* pieces;          // [workers][lines][2][128 * (D + 2)]
  int32_t* status;
  int32_t hq, hkv, group, page, page_shift;
  int32_t n_seqs, n_groups, n_tokens, max_queries, causal;
  float scale_log2, inv_group;
};

__device__ __forceinline__ void report(const AttendArgs& A, int code) {
  if (A.status) atomicMax(A.status, code);
}

__device__ __forceinline__ int length_of(const AttendArgs& A, const StreamArgs& S, int row, bool tell) {
  const int64_t len = __ldg(S.lens + row), room = static_cast<int64_t>(S.max_pages) << A.page_shift;
  if (len >= 0 && len <= room) return static_cast<int>(len);
  if (tell) report(A, QC_ERR_PLAN);
  return len < 0 ? 0 : static_cast<int>(room);
}

// A prefix (items 0 .. n_groups - 1) or a sequence's own tokens.
struct Item {
  int32_t token0, queries, row, len, tiles;
  uint32_t units, per_head;      // units; those of a KV head
  bool fine;
};
struct Held {
  int32_t token0, queries, row, len;
};
__device__ __forceinline__ void count_units(const AttendArgs& A, Item& u) {
  u.tiles = (u.len + kKeys - 1) / kKeys;
  u.per_head = static_cast<uint32_t>((static_cast<int64_t>(u.queries) * A.group + kRows - 1) / kRows);
  u.units = u.tiles ? min(static_cast<uint64_t>(u.per_head) * A.hkv, static_cast<uint64_t>(kMostCost)) : 0;
}
__device__ __forceinline__ Item item_from(const AttendArgs& A, const Held& h) {
  Item u{};
  u.token0 = h.token0, u.queries = h.queries, u.row = h.row, u.len = h.len, u.fine = true;
  if (u.queries) count_units(A, u);
  return u;
}
__device__ __forceinline__ Item item_of(const AttendArgs& A, int i, bool tell) {
  Item u{};
  const bool shared = i < A.n_groups;
  int64_t a, b;
  if (shared) {
    a = A.groups ? __ldg(A.groups + i) : 0, b = A.groups ? __ldg(A.groups + i + 1) : A.n_seqs;
    u.row = A.shared_ids ? __ldg(A.shared_ids + i) : i;
    u.fine = a >= 0 && b >= a && b <= A.n_seqs;
    if (u.fine && A.starts) a = __ldg(A.starts + a), b = __ldg(A.starts + b);
  } else {
    const int seq = i - A.n_groups;
    a = seq, b = seq + 1;
    if (A.starts) a = __ldg(A.starts + seq), b = __ldg(A.starts + seq + 1);
    u.row = A.ids ? __ldg(A.ids + seq) : seq;
    u.fine = b - a <= A.max_queries;
  }
  const StreamArgs& S = A.stream[shared];
  u.fine = u.fine && a >= 0 && b >= a && b <= A.n_tokens && u.row >= 0 && u.row < S.rows;
  if (!u.fine) return u;
  u.token0 = static_cast<int32_t>(a), u.queries = static_cast<int32_t>(b - a);
  if (u.queries == 0) return u;
  u.len = length_of(A, S, u.row, tell);
  count_units(A, u);
  return u;
}
__device__ __forceinline__ uint32_t unit_cost(int tiles) { return kUnitCost + tiles; }
// kMostCost + 1: too much
__device__ __forceinline__ uint32_t cost_of(const Item& u) {
  return static_cast<uint32_t>(min(static_cast<uint64_t>(u.units) * unit_cost(u.tiles), static_cast<uint64_t>(kMostCost) + 1));
}

// Every range is as long as a tile at least.
__device__ __forceinline__ Line line_of(uint32_t begin, uint32_t cost, uint32_t most) {
  const uint32_t workers = max(1u, min(most, cost));
  const uint32_t per = cost / workers;
  return Line{begin, per, cost % workers, workers, static_cast<int32_t>(max(1u, min(kLeastPiece, per / kPieceShare)))};
}
// Where a border at tile t of a unit is: never so near to its first or last tile that a piece would hardly be worth its start.
__device__ __forceinline__ int border(int least, int t, int tiles) {
  if (tiles < 2 * least) return t <= tiles / 2 ? 0 : tiles;
  return t < least ? 0 : t > tiles - least ? tiles : t;
}
__device__ __forceinline__ uint32_t range_begin(const Line& p, uint32_t w) { return p.begin + w * p.per + min(w, p.longer); }
__device__ __forceinline__ uint32_t worker_at(const Line& p, uint32_t at) {
  at -= p.begin;
  const uint32_t turn = p.longer * (p.per + 1);
  return at < turn ? at / (p.per + 1) : p.longer + (at - turn) / p.per;
}

struct Unit {
  int32_t token0;                // the token of its first row
  int32_t head0;                 // and that row's head inside the KV head's group
  int32_t query0, queries;       // the query of its first row among the item's
  int32_t n_here, kvh, shared, row, first, tiles, len;
  int32_t all_see;               // keys that every row sees
  int32_t place;                 // of a piece: worker * 4 + line * 2, + 1 where the unit begins in the range; -1: the unit is whole
};

// How often a unit's rows are held, every 32, 64 or 128 rows: as often as the copies' sums, 32 elements at a time, fit the place where
// they meet.
__device__ __forceinline__ int copies_of(int n_here) { return n_here <= 30 ? 4 : n_here <= 60 ? 2 : 1; }

struct Meta {
  int32_t y[4];                  // of a tile's pages: the first row in the pool, -1: the page is not there
  int32_t on, shared;            // blocks of 16 keys that are there
};

template <int D>
struct Shape {
  static constexpr int kRing = D == 128 ? 2 : 4;      // tiles of K, and of V, under way
  static constexpr uint32_t kTile = kKeys * D * 2, kHalf = kKeys * 128, kQ = kRows * D * 2, kQHalf = kRows * 128;
  // where the copies' sums meet, their references behind them
  static constexpr uint32_t kMeet = kQ + 2 * kRing * kTile, kMeetBytes = 15616, kRefs = kMeet + kMeetBytes;
  static constexpr uint32_t kTiles = kRefs + kRows * 8;
};

struct Control {
  uint64_t s[2], p[2], o[2], k[4], v[4], k_free[4], v_free[4], full[kUnits], empty[kUnits], q;
  uint64_t sums[8];
  Unit units[kUnits];
  Meta meta[kMeta];
  uint32_t tmem, beat, redo[4];
  int32_t failed;
};
static_assert(2 * (Shape<128>::kTiles + sizeof(Control) + 1024) <= 228 * 1024, "two blocks share an SM");

// O (+)= P V for one tile: a product for 16 keys, the weights 8 columns of tensor memory and the values at b0 .. b3.
__device__ __forceinline__ void values(uint32_t tmem_d, uint32_t tmem_p, uint64_t b0, uint64_t b1, uint64_t b2, uint64_t b3, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, pa, po;\n\t.reg .b32 ta;\n\t"
      "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 pa, %7, 0;\n\tsetp.eq.b32 po, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %6, pa;\n\t"
      "add.u32 ta, %1, 8;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], %3, %6, po;\n\t"
      "add.u32 ta, %1, 16;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], %4, %6, po;\n\t"
      "add.u32 ta, %1, 24;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], %5, %6, po;\n\t}" ::"r"(tmem_d),
      "r"(tmem_p), "l"(b0), "l"(b1), "l"(b2), "l"(b3), "r"(idesc), "r"(accumulate)
      : "memory");
}
template <int D>
__device__ __forceinline__ void scores(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc) {
  if constexpr (D == 128) {
    umma_scores<kRows * 128, kKeys * 128>(tmem_d, a, b, idesc);
  } else {
    asm volatile(
        "{\n\t.reg .pred e, pz, po;\n\t.reg .b64 da, db;\n\t"
        "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 pz, 0, 0;\n\tsetp.eq.b32 po, 0, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, pz;\n\t"
        "add.u64 da, %1, 2;\n\tadd.u64 db, %2, 2;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, po;\n\t"
        "add.u64 da, %1, 4;\n\tadd.u64 db, %2, 4;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, po;\n\t"
        "add.u64 da, %1, 6;\n\tadd.u64 db, %2, 6;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, po;\n\t}"
        ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc) : "memory");
  }
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
// Rows 0-15 of a warp's lanes, a row shared out among four threads: 8 columns at a time, thread l has columns 2 (l % 4) and the next one of row
// l / 4 (registers 0 and 1) and of the row 8 below (2 and 3); or 4 columns at a time, column l % 4 of row l / 4 and of the row 8 below.
__device__ __forceinline__ void tmem_ld_quads16(uint32_t taddr, uint32_t (&r)[8]) {      // 16 columns
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_quads64(uint32_t taddr, uint32_t (&r)[32]) {      // 64 columns
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_quads64(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
               : "memory");
}
__device__ __forceinline__ void tmem_st_fours32(uint32_t taddr, const uint32_t (&r)[16]) {      // 32 columns
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Whether all rows' threads say so.  Rows' warps go on together or not at all, so that none waits at a barrier for
// one that has given up.
__device__ __forceinline__ bool rows_all(bool x) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"(static_cast<uint32_t>(x)), "n"(kRows) : "memory");
  return all != 0;
}
__device__ __forceinline__ bool rows_any(bool x) { return !rows_all(!x); }
__device__ __forceinline__ void rows_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kRows) : "memory"); }

// Keys [from, to) of a table row for one query, by one warp, a key at a time: what the tensor cores cannot give where a value that is
// infinite or no number stands behind a weight of 0 (0 times it is no number).  Replaces those of the row's sums that are no finite
// numbers, on the row's reference.
template <int D>
__device__ __noinline__ void sweep(const AttendArgs& A, const StreamArgs& S, int row, int kvh, int64_t token, int head, int from, int to, float* sums, const float2* ml,
                                   uint32_t* beat, int lane) {
  float o[D / 32] = {}, m = -INFINITY, l = 0.f, q[D / 32];
  const auto load = [&](const uint16_t* p, float (&f)[D / 32]) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const float2 x = bf16x2_to_f32(__ldg(reinterpret_cast<const uint32_t*>(p) + i * 32 + lane));
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  };
  load(S.q + token * S.q_stride + static_cast<int64_t>(head) * D, q);
#pragma unroll 2
  for (int j = from; j < to; ++j) {
    if (lane == 0 && (j & 63) == 0) atomicAdd(beat, 1u);
    const int32_t id = __ldg(S.pages + static_cast<int64_t>(row) * S.max_pages + (j >> A.page_shift));
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(S.n_pages)) continue;
    const int64_t at = (((static_cast<int64_t>(id) * A.hkv + kvh) << A.page_shift) + (j & (A.page - 1))) * D;
    float k[D / 32], v[D / 32];
    load(S.k_pool + at, k);
    load(S.v_pool + at, v);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= A.scale_log2;
    if (s == -INFINITY) continue;      // (weighs nothing)
    const float top = fmaxf(m, s), before = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(m - top), p = exp2f(s - (top == -INFINITY ? 0.f : top));
    l = fmaf(l, before, p);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = fmaf(o[i], before, p * v[i]);
    m = top;
  }
  const float scale = m == -INFINITY && l == 0.f ? 0.f : exp2f(m - ml->x);
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float* const to_here = sums + (i * 32 + lane) * 2 + e;
      if (!isfinite(*to_here)) *to_here = l == 0.f ? 0.f : o[2 * i + e] * scale;
    }
}

__device__ __forceinline__ void store_32(float* p, const uint32_t* r) {      // 32 bytes, a sector
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// Warps 0-3: a query row per thread; warp 4 issues products; warp 5 finds units and fetches.  Hand-offs (mbarriers, all waits bounded):
//   full[u], empty[u]   warp 5 -> the others: unit u % 4 is described; back: its place is free
//   q                   rows -> warp 4: the unit's queries are in shared memory
//   k[i], v[i]          copies -> warp 4 (and v to rows that clear what no token has): a tile has landed
//   s[b]                tensor core -> rows: scores of tile t in buffer b = t & 1
//   p[b]                rows -> warp 4: its weights are there, over the scores
//   o[b]                tensor core -> warp 4, rows: its value products are done
//   k_free[i], v_free[i]  tensor core -> warp 5: the tile's place may be written (rings of two: s and o say so)
// No barrier runs two completions ahead of a waiter: the next completion needs something that the waiter does after it has seen
// the one before.  Tiles are counted through all units of the block.
template <int D>
__global__ void __launch_bounds__(kBlock, 2) paged_attend_kernel(const __grid_constant__ AttendArgs A) {
  using Z = Shape<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sQ = smem_u32(smem), sK = sQ + Z::kQ, sV = sK + Z::kRing * Z::kTile, sMeet = sQ + Z::kMeet;
  Control& C = *reinterpret_cast<Control*>(smem + Z::kTiles);
  volatile int32_t& failed = C.failed;
  constexpr bool kLong = Z::kRing > 2;      // rings of two are free when the score buffer, or its weights, are
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (sQ & 1023u) {      // (there is no static shared memory, so it begins at a multiple of 1024; products never run on a misplaced tile)
    if (threadIdx.x == 0) report(A, QC_ERR_PLAN);
    return;
  }
  if (warp == 5) {
    if (lane == 0) {
      for (int i = 0; i < 2; ++i) mbar_init(&C.s[i], 1), mbar_init(&C.p[i], kRows), mbar_init(&C.o[i], 1);
      for (int i = 0; i < 4; ++i) mbar_init(&C.k[i], 1), mbar_init(&C.v[i], 1), mbar_init(&C.k_free[i], 1), mbar_init(&C.v_free[i], 1);
      for (int i = 0; i < kUnits; ++i) mbar_init(&C.full[i], 1), mbar_init(&C.empty[i], kRows + 1);
      mbar_init(&C.q, kRows);
      fence_mbar_init();
      C.failed = 0, C.beat = 0;
      for (int i = 0; i < 4; ++i) C.redo[i] = 0;
    }
  } else if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&C.tmem)), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();

  // ---- the plan: costs of the items before each one, in the tiles' place until they come
  uint32_t* const before = reinterpret_cast<uint32_t*>(smem);      // [items]
  const int n_items = A.n_groups + A.n_seqs;
  Held* const held = reinterpret_cast<Held*>(smem + kMostHeld * 8);      // [items], where there are no more than that
  const bool holds = n_items <= kMostHeld;
  uint32_t total = 0;
  bool fine = true;
  for (int i0 = 0; i0 < n_items; i0 += kBlock) {
    const int i = i0 + threadIdx.x;
    uint32_t x = 0;
    Item u{};
    if (i < n_items) {
      u = item_of(A, i, blockIdx.x == 0);
      x = cost_of(u);
      fine &= u.fine;
    }
    const uint32_t mine = x;
    uint64_t sum = x;      // (a warp's sum may pass 32 bits)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    if (lane == 31) C.sums[warp] = sum;
    __syncthreads();
    uint64_t base = total, all = total;
#pragma unroll
    for (int w = 0; w < kBlock / 32; ++w) base += w < warp ? C.sums[w] : 0, all += C.sums[w];
    total = static_cast<uint32_t>(min(all, static_cast<uint64_t>(kMostCost) + 1));
    const uint32_t at = static_cast<uint32_t>(min(base + sum - mine, static_cast<uint64_t>(kMostCost) + 1));
    if (i < n_items) {
      before[i] = at;
      if (holds) held[i] = Held{u.token0, u.queries, u.row, u.len};
      if (blockIdx.x == 0) {
        int group = -1;
        if (i >= A.n_groups && A.n_groups) {      // the last group that begins at or before the sequence, if it reaches it
          const int seq = i - A.n_groups;
          if (A.groups) {
            int lo = 0, hi = A.n_groups;
            while (lo < hi) {
              const int mid = (lo + hi) >> 1;
              if (__ldg(A.groups + mid + 1) > seq) hi = mid;
              else lo = mid + 1;
            }
            if (lo < A.n_groups && __ldg(A.groups + lo) <= seq) group = lo;
          } else {
            group = 0;
          }
        }
        A.records[i] = Record{at, u.units ? u.tiles : 0, u.token0, u.queries, group, {}};
      }
    }
    __syncthreads();
  }
  fine = __syncthreads_and(fine);
  const bool few = total <= kMostCost;
  // Prefixes and sequences apart where every block has some of both
  const uint32_t cut = A.n_groups < n_items ? before[A.n_groups] : total;
  Plan plan{{}, fine && few, 1};
  if (cut >= kApart * gridDim.x && total - cut >= kApart / 4 * gridDim.x) {
    plan.lines = 2;
    plan.line[0] = line_of(0, cut, gridDim.x), plan.line[1] = line_of(cut, total - cut, gridDim.x);
  } else {
    plan.line[0] = line_of(0, total, gridDim.x);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *A.plan = plan;
    if (!fine) report(A, QC_ERR_INVALID_ARG);
    else if (!few) report(A, QC_ERR_PLAN);
  }
  const bool works = plan.fine && total && (blockIdx.x < plan.line[0].workers || (plan.lines == 2 && blockIdx.x < plan.line[1].workers));
  tc5_fence_before();
  __syncthreads();
  tc5_fence_after();
  const uint32_t tmem = C.tmem;

  if (works && warp == 5) {
    // ------------------------------------------------------------------ units and tiles
    // The block's ranges: of one row of costs, or of both; the second half of the blocks, which share their SMs with the first, begin with
    // the sequences', so that prefixes' products and sequences' copies go side by side.
    struct Range {
      uint32_t at, end, item_at, begin;
      int item, line, least;
    };
    const auto range_of = [&](int line) -> Range {
      Range r{};
      const Line p = line ? plan.line[1] : plan.line[0];
      r.line = line, r.least = p.least;
      if (blockIdx.x >= p.workers) return r;
      r.at = r.begin = range_begin(p, blockIdx.x), r.end = range_begin(p, blockIdx.x + 1);
      int lo = 0, hi = n_items - 1;      // the last item that begins at or before the range
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (before[mid] <= r.at) lo = mid;
        else hi = mid - 1;
      }
      r.item = lo, r.item_at = before[lo];
      return r;
    };
    const int begins_with = plan.lines == 2 && blockIdx.x >= gridDim.x / 2 ? 1 : 0;
    Range range = range_of(begins_with), other{};
    if (plan.lines == 2) other = range_of(1 - begins_with);
    if (range.at >= range.end) range = other, other = Range{};
    // 32 items, one per lane, from `first_held` on
    Held mine{};
    int first_held = range.item;
    const auto hold = [&](int from) {
      first_held = from;
      if (from + lane < n_items) {
        const Item x = item_of(A, from + lane, false);
        mine = Held{x.token0, x.queries, x.row, x.len};
      }
    };
    const auto held_at = [&](int item) -> Item {
      const int from = item - first_held;
      return item_from(A, Held{__shfl_sync(0xffffffffu, mine.token0, from), __shfl_sync(0xffffffffu, mine.queries, from), __shfl_sync(0xffffffffu, mine.row, from),
                               __shfl_sync(0xffffffffu, mine.len, from)});
    };
    if (!holds) hold(range.item);
    else if (range.item + lane < n_items) mine = held[range.item + lane];
    __syncwarp();
    fence_proxy_async();      // (the costs have been read before copies take their place)
    Item u = held_at(range.item);
    // the next unit
    const auto find = [&](Unit& w) -> bool {
      while (true) {
        if (range.at >= range.end) {
          if (other.at >= other.end) return false;
          range = other, other = Range{};
          hold(range.item);
          u = held_at(range.item);
        }
        const uint32_t cost = cost_of(u), one = unit_cost(u.tiles);
        if (u.units == 0 || range.at >= range.item_at + cost) {
          if (++range.item >= n_items) {
            range.at = range.end;
            continue;
          }
          range.item_at += cost;
          if (range.item == first_held + 32) hold(range.item);
          u = held_at(range.item);
          if (range.at < range.item_at) range.at = range.item_at;
          continue;
        }
        const uint32_t unit = (range.at - range.item_at) / one, unit_at = range.item_at + unit * one, tiles_at = unit_at + kUnitCost;
        const int first = border(range.least, static_cast<int>(range.begin - tiles_at), u.tiles), last = border(range.least, static_cast<int>(range.end - tiles_at), u.tiles);
        range.at = unit_at + one;
        if (first >= last) continue;
        const int kvh = unit / u.per_head, part = unit - kvh * u.per_head;
        const int64_t row0 = static_cast<int64_t>(part) * kRows, rows = static_cast<int64_t>(u.queries) * A.group;
        w.n_here = static_cast<int32_t>(min(static_cast<int64_t>(kRows), rows - row0));
        w.query0 = part ? static_cast<int32_t>(row0 / A.group) : 0, w.head0 = part ? static_cast<int32_t>(row0 - static_cast<int64_t>(w.query0) * A.group) : 0;
        w.token0 = u.token0 + w.query0, w.queries = u.queries, w.kvh = kvh, w.shared = range.item < A.n_groups, w.row = u.row, w.first = first, w.tiles = last - first, w.len = u.len;
        w.all_see = w.shared || !A.causal ? u.len : max(0, u.len - (u.queries - 1 - w.query0));
        w.place = first == 0 && last == u.tiles ? -1 : static_cast<int>(blockIdx.x) * 4 + range.line * 2 + (first == 0 ? 1 : 0);
        return true;
      }
    };
    const int per_tile = kKeys >> A.page_shift;
    // a unit, whether there is one, and page ids, one per lane: from page `batch` of its row on, and the 32 behind them
    struct Ahead {
      Unit w;
      bool has;
      int32_t batch, ids, next_ids;
    };
    const auto ask = [&](const Unit& w, int from) -> int32_t {
      const int page = from + lane;
      const StreamArgs& S = A.stream[w.shared];
      return static_cast<int64_t>(page) << A.page_shift < w.len ? __ldg(S.pages + static_cast<int64_t>(w.row) * S.max_pages + page) : -1;
    };
    const auto look = [&](Ahead& x) {
      x.has = find(x.w);
      if (!x.has) return;
      x.batch = x.w.first * per_tile;
      x.ids = ask(x.w, x.batch), x.next_ids = ask(x.w, x.batch + 32);
    };
    Ahead now{}, then{};      // the unit at hand, and the next one, whose page ids are on their way
    look(now);
    bool looked = false;      // for the next one: behind the first copy
    bool stopped = false, described = false;
    uint32_t n_units = 0;      // described
    int tile = 0;              // of the unit, next to be fetched
    uint32_t k_next = 0, v_next = 0;
    constexpr int kHalves = D / 64;
    const int half = lane % kHalves, page_of_tile = lane / kHalves;
    const auto copy_keys = [&](const Meta& m, uint32_t dst, uint64_t* bar) {
      const int y = page_of_tile < per_tile ? m.y[page_of_tile] : -1;
      const uint32_t n = __popc(__ballot_sync(0xffffffffu, y >= 0));
      if (lane == 0) mbar_expect_tx(bar, n * A.page * 128);
      __syncwarp();
      if (y >= 0) tensor_g2s_2d(dst + half * Z::kHalf + page_of_tile * A.page * 128, &A.map[m.shared][0], half * 64, y, bar);
    };
    const auto copy_values = [&](const Meta& m, uint32_t dst, uint64_t* bar) {
      const int y = lane < per_tile ? m.y[lane] : -1;
      const uint32_t n = __popc(__ballot_sync(0xffffffffu, y >= 0));
      if (lane == 0) mbar_expect_tx(bar, n * A.page * (D * 2));
      __syncwarp();
      if (y >= 0) tensor_g2s_3d(dst + lane * A.page * (D * 2), &A.map[m.shared][1], 0, y, 0, bar);
    };
    uint32_t idle = 0, beat = 0;
    bool ok = true;
    while (ok && (!stopped || v_next < k_next)) {
      bool progress = false;
      if (!stopped && !described) {      // tell the others about the unit, or that there is none
        const uint32_t slot = n_units % kUnits;
        if (n_units < kUnits || __all_sync(0xffffffffu, mbar_test_wait(&C.empty[slot], (n_units / kUnits - 1) & 1u))) {
          if (lane == 0) {
            Unit& d = C.units[slot];
            d = now.w;
            if (!now.has) d.tiles = 0;
            mbar_arrive(&C.full[slot]);
          }
          __syncwarp();
          ++n_units;
          progress = true;
          if (now.has) described = true, tile = 0;
          else stopped = true;
        }
      }
      if (described) {
        const uint32_t i = k_next % Z::kRing;
        if (k_next < Z::kRing || __all_sync(0xffffffffu, mbar_test_wait(kLong ? &C.k_free[i] : &C.s[i], (k_next / Z::kRing - 1) & 1u))) {
          const Unit& w = now.w;
          const int t = w.first + tile, page0 = t * per_tile;
          if (page0 - now.batch >= 32) now.batch += 32, now.ids = now.next_ids, now.next_ids = ask(w, now.batch + 32);
          const int32_t id = __shfl_sync(0xffffffffu, now.ids, min(31, page0 - now.batch + page_of_tile));
          const bool exists = page_of_tile < per_tile && static_cast<int64_t>(page0 + page_of_tile) << A.page_shift < w.len;
          const bool there = exists && static_cast<uint32_t>(id) < static_cast<uint32_t>(A.stream[w.shared].n_pages);
          if (exists && !there) report(A, QC_ERR_BAD_PAGE);
          Meta& m = C.meta[k_next % kMeta];
          const uint32_t pages = __ballot_sync(0xffffffffu, there && half == 0);
          if (half == 0 && page_of_tile < 4) m.y[page_of_tile] = there ? (id * A.hkv + w.kvh) << A.page_shift : -1;
          if (lane == 0) {
            int on = 0;
            for (int b = 0; b < kKeys / 16; ++b) on |= (pages >> ((b * 16 >> A.page_shift) * kHalves) & 1) << b;
            m.on = on, m.shared = w.shared;
          }
          __syncwarp();
          copy_keys(m, sK + i * Z::kTile, &C.k[i]);
          ++k_next;
          progress = true;
          if (++tile == w.tiles) {
            if (!looked) look(then);
            described = false;
            now = then, looked = !now.has;
          }
        }
      }
      if (v_next < k_next) {
        const uint32_t i = v_next % Z::kRing;
        if (v_next < Z::kRing || __all_sync(0xffffffffu, mbar_test_wait(kLong ? &C.v_free[i] : &C.o[i], (v_next / Z::kRing - 1) & 1u))) {
          copy_values(C.meta[v_next % kMeta], sV + i * Z::kTile, &C.v[i]);
          ++v_next;
          progress = true;
        }
      }
      if (progress) {
        idle = 0;
      } else if (described && !looked) {      // the next unit is looked for while there is nothing else to do
        look(then), looked = true;
      } else if (++idle > (1u << 20) || ((idle & 1023u) == 0 && failed)) {
        const uint32_t now = *reinterpret_cast<volatile uint32_t*>(&C.beat);
        if (failed || now == beat) ok = false;
        beat = now, idle = 0;
      }
    }
    if (!ok) failed = 1;
  } else if (works && warp == 4) {
    // ------------------------------------------------------------------ products
    constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((kKeys >> 3) << 17) | ((kRows >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((D >> 3) << 17) | ((kRows >> 4) << 24);
    bool ok = true;
    const auto wait_on = [&](uint64_t* bar, uint32_t parity) {      // warp-uniform, bounded: as long as something moves
      if (!ok || __all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
      uint32_t beat = *reinterpret_cast<volatile uint32_t*>(&C.beat);
      while (!__all_sync(0xffffffffu, bounded_wait(bar, parity))) {
        const uint32_t now = *reinterpret_cast<volatile uint32_t*>(&C.beat);
        if (failed || __all_sync(0xffffffffu, now == beat)) {
          ok = false;
          break;
        }
        beat = now;
      }
    };
    const uint64_t qd = umma_desc(sQ, 16, 1024);
    // keys 16, 32 and 48 of a tile of values (pages one after the other, a page's halves of 64 elements too), in 16 bytes
    uint32_t v_step[3];
#pragma unroll
    for (int j = 1; j < 4; ++j) v_step[j - 1] = ((16 * j >> A.page_shift) * A.page * (D * 2) + (16 * j & (A.page - 1)) * 128) >> 4;
    uint32_t s_next = 0, o_next = 0;      // tiles
    const auto issue_scores = [&]() {
      const uint32_t b = s_next & 1u, i = s_next % Z::kRing;
      // the buffer holds the weights of the tile before the last one until their products are done (products with different sums are
      // not documented to run in the order of their issue)
      if (s_next >= 2) wait_on(&C.o[b], (s_next / 2 - 1) & 1u);
      wait_on(&C.k[i], (s_next / Z::kRing) & 1u);
      if (!ok) return;
      tc5_fence_after();
      scores<D>(tmem + kScoresAt + b * kKeys, qd, umma_desc(sK + i * Z::kTile, 16, 1024), kIdescS);
      umma_commit(&C.s[b]);
      if (kLong) umma_commit(&C.k_free[i]);
      ++s_next;
    };
    for (uint32_t n = 0; ok; ++n) {
      const uint32_t slot = n % kUnits;
      wait_on(&C.full[slot], (n / kUnits) & 1u);
      if (!ok) break;
      const int tiles = *reinterpret_cast<volatile int32_t*>(&C.units[slot].tiles);
      if (tiles == 0) break;
      wait_on(&C.q, n & 1u);
      for (int t = 0; t < 2 && t < tiles && ok; ++t) issue_scores();
      for (int t = 0; t < tiles && ok; ++t) {
        const uint32_t b = o_next & 1u, i = o_next % Z::kRing;
        wait_on(&C.p[b], (o_next / 2) & 1u);
        wait_on(&C.v[i], (o_next / Z::kRing) & 1u);
        if (!ok) break;
        tc5_fence_after();
        const uint64_t vd = umma_desc(sV + i * Z::kTile, A.page * 128, 1024);
        values(tmem + kOutAt, tmem + kScoresAt + b * kKeys, vd, vd + v_step[0], vd + v_step[1], vd + v_step[2], kIdescO, t > 0 ? 1u : 0u);
        umma_commit(&C.o[b]);
        if (kLong) umma_commit(&C.v_free[i]);
        ++o_next;
        if (t + 2 < tiles) issue_scores();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&C.empty[slot]);
    }
    // (nothing arrives behind the block's end)
    if (kLong && s_next) wait_on(&C.k_free[(s_next - 1) % Z::kRing], ((s_next - 1) / Z::kRing) & 1u);
    if (kLong && o_next) wait_on(&C.v_free[(o_next - 1) % Z::kRing], ((o_next - 1) / Z::kRing) & 1u);
    if (!ok) failed = 1;
    __syncwarp();
  } else if (works) {
    // ------------------------------------------------------------------ rows
    const uint32_t t_row = tmem + (static_cast<uint32_t>(warp * 32) << 16);   // this warp's 32 lanes of tensor memory
    bool ok = true;
    const auto wait_on = [&](uint64_t* bar, uint32_t parity) {
      if (!ok || __all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return;
      uint32_t beat = *reinterpret_cast<volatile uint32_t*>(&C.beat);
      while (!__all_sync(0xffffffffu, bounded_wait(bar, parity))) {
        const uint32_t now = *reinterpret_cast<volatile uint32_t*>(&C.beat);
        if (failed || __all_sync(0xffffffffu, now == beat)) {
          ok = false;
          break;
        }
        beat = now;
      }
    };
    uint32_t t0 = 0;      // tiles of the units before
    // rows of a unit are its first query's heads from head0 on, then the next query's
    const auto query_of = [&](const Unit& u, int row) { return static_cast<int>((static_cast<float>(u.head0 + row) + 0.5f) * A.inv_group); };
    // a unit as this thread sees it: its row, of n_here that are held `copies` times
    struct Mine {
      int n_here, tiles, first, len, all_see, shared;
      int copies, row, copy, seen;
      bool real;
    };
    const auto take = [&](uint32_t n, Mine& x) {
      const Unit& u = C.units[n % kUnits];
      x.n_here = u.n_here, x.tiles = u.tiles, x.first = u.first, x.len = u.len, x.all_see = u.all_see, x.shared = u.shared;
      x.copies = copies_of(x.n_here);
      x.copy = threadIdx.x >> (x.copies == 4 ? 5 : x.copies == 2 ? 6 : 7), x.row = threadIdx.x & (x.copies == 4 ? 31 : x.copies == 2 ? 63 : 127);
      if (x.n_here <= kSlim) x.row = lane >> 2;      // four threads a row
      x.real = x.row < x.n_here;
      x.seen = x.shared || !A.causal ? x.len : max(0, x.len - (u.queries - 1 - u.query0 - query_of(u, x.row)));
    };
    // the unit's queries, from their places straight into shared memory: a thread per row, or per 16 bytes where there are few; rows that are
    // none keep what was there
    const auto ask_query = [&](uint32_t n) {
      const Unit& u = C.units[n % kUnits];
      const StreamArgs& S = A.stream[u.shared];
      constexpr int kChunks = D / 8;
      const int n_here = u.n_here, copies = copies_of(n_here);
      const bool slim = n_here <= kSlim;
      const int row = slim ? threadIdx.x / kChunks : threadIdx.x & (kRows / copies - 1), query = query_of(u, row);
      const uint16_t* p = S.q + (u.token0 + query) * S.q_stride + static_cast<int64_t>(u.kvh * A.group + u.head0 + row - query * A.group) * D;
      if (row >= n_here) return;
      const auto bring = [&](uint32_t to, const uint16_t* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); };
      if (slim) {      // (kSlim rows are no more than the threads)
        const int chunk = threadIdx.x % kChunks;
        const uint32_t to = sQ + (chunk >> 3) * Z::kQHalf + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);      // (copies are multiples of 8 rows apart)
#pragma unroll
        for (int c = 0; c < 4; ++c) bring(to + c * (kRows / 4) * 128, p + chunk * 8);
      } else {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) bring(sQ + (i >> 3) * Z::kQHalf + threadIdx.x * 128 + (((i & 7) ^ (threadIdx.x & 7)) << 4), p + i * 8);
      }
    };
    const auto put_query = [&]() {
      cp_async_wait_all();
      fence_proxy_async();
      mbar_arrive(&C.q);
    };
    Mine x;
    wait_on(&C.full[0], 0u);
    if (ok && C.units[0].tiles) ask_query(0), put_query();
    for (uint32_t n = 0;; ++n) {
      if (!rows_all(ok)) break;
      take(n, x);
      if (x.tiles == 0) break;
      float ref = -INFINITY, sum = 0.f;
      bool more = false;      // units
      const bool idle = x.copies == 1 && warp * 32 >= x.n_here;      // a warp without rows
      const auto weigh = [&](auto tag, int t, uint32_t gt, uint32_t on, bool masked) {
        constexpr int REP = decltype(tag)::value, N = kKeys / REP;
        const uint32_t at = t_row + kScoresAt + (gt & 1u) * kKeys;
        const int col0 = REP == 1 ? 0 : x.copy * N;
        float p[N];
        if constexpr (REP == 1) {
          uint32_t r0[32], r1[32];
          tmem_ld32_nowait(at, r0);
          tmem_ld32_nowait(at + 32, r1);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 32; ++j) p[j] = __uint_as_float(r0[j]), p[32 + j] = __uint_as_float(r1[j]);
        } else if constexpr (REP == 2) {
          uint32_t r[32];
          tmem_ld32(at + col0, r);
#pragma unroll
          for (int j = 0; j < 32; ++j) p[j] = __uint_as_float(r[j]);
        } else {
          uint32_t r[16];
          tmem_ld16(at + col0, r);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; ++j) p[j] = __uint_as_float(r[j]);
        }
        if (masked) {
          const int left = x.seen - (t * kKeys + col0);
          const uint32_t here = on >> (col0 / 16);
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (j >= left || !(here >> (j / 16) & 1u)) p[j] = -INFINITY;
        }
        float mx[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
        for (int j = 4; j < N; j += 2) mx[(j >> 1) & 3] = max3(mx[(j >> 1) & 3], p[j], p[j + 1]);
        const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * A.scale_log2;   // (the scale is positive)
        float corr = 1.f;
        if ((top > ref + kRescale || ref == -INFINITY) && top != -INFINITY) {
          corr = exp2f(ref - top);      // 0 on the first keys
          ref = top;
        }
        const float less = ref == -INFINITY ? 0.f : -ref;
        float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          const float2 y = fma2(make_float2(p[j], p[j + 1]), make_float2(A.scale_log2, A.scale_log2), make_float2(less, less));
          p[j] = ex2_approx(y.x);
          p[j + 1] = ex2_approx(y.y);
          ps[(j >> 1) & 1] = add2(ps[(j >> 1) & 1], make_float2(p[j], p[j + 1]));
        }
        sum = sum * corr + ((ps[0].x + ps[0].y) + (ps[1].x + ps[1].y));
        if (gt != t0 && __any_sync(0xffffffffu, corr != 1.f)) {      // rare: the sums so far go to the new reference
          wait_on(&C.o[(gt - 1) & 1u], ((gt - 1) / 2) & 1u);
          if (!ok) return;
          tc5_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t r[32];
            tmem_ld32(t_row + kOutAt + c, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * corr);
            tmem_st32(t_row + kOutAt + c, r);
          }
          tmem_wait_st();
        }
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          constexpr int kEach = N / 2;
          const uint32_t y = pack_bf16x2(p[j % kEach * 2], p[j % kEach * 2 + 1]);
          w[j] = REP == 1 || j / kEach == x.copy ? y : 0u;      // (the other copies' keys weigh nothing in this one)
        }
        tmem_st32(at, w);
        tmem_wait_st();
      };
      // the same for units of few rows: a warp's quarter of the keys, four of them a thread
      const auto weigh_slim = [&](int t, uint32_t gt, uint32_t on, bool masked) {
        const uint32_t at = t_row + kScoresAt + (gt & 1u) * kKeys;
        const int key = warp * 16 + 2 * (lane & 3);      // and the next one, and those 8 behind
        uint32_t r[8];
        tmem_ld_quads16(at + warp * 16, r);
        tmem_wait_ld();
        float p[4] = {__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[4]), __uint_as_float(r[5])};
        if (masked) {
          const int left = x.seen - (t * kKeys + key);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if ((j & 1) + (j >> 1) * 8 >= left || !(on >> warp & 1u)) p[j] = -INFINITY;
        }
        float top = fmaxf(max3(p[0], p[1], p[2]), p[3]);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)) * A.scale_log2;
        float corr = 1.f;
        if ((top > ref + kRescale || ref == -INFINITY) && top != -INFINITY) {
          corr = exp2f(ref - top);
          ref = top;
        }
        const float less = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = ex2_approx(fmaf(p[j], A.scale_log2, less));
        sum = sum * corr + ((p[0] + p[1]) + (p[2] + p[3]));
        if (gt != t0 && __any_sync(0xffffffffu, corr != 1.f)) {
          wait_on(&C.o[(gt - 1) & 1u], ((gt - 1) / 2) & 1u);
          if (!ok) return;
          tc5_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 64) {
            uint32_t o[32];
            tmem_ld_quads64(t_row + kOutAt + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * corr);      // (no row is 8 below one)
            tmem_st_quads64(t_row + kOutAt + c, o);
          }
          tmem_wait_st();
        }
        const uint32_t near = pack_bf16x2(p[0], p[1]), far = pack_bf16x2(p[2], p[3]);
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = j / 4 != warp || (j & 1) ? 0u : j & 2 ? far : near;
        tmem_st_fours32(at, w);
        tmem_wait_st();
      };
      for (int i = 0; i < x.tiles && ok; ++i) {
        const uint32_t gt = t0 + i;
        const int t = x.first + i;
        wait_on(&C.s[gt & 1u], (gt / 2) & 1u);
        if (!ok) break;
        tc5_fence_after();
        if (i + 1 == x.tiles) {      // the queries have been read for the last time: the next unit's are on their way while this one ends
          wait_on(&C.full[(n + 1) % kUnits], ((n + 1) / kUnits) & 1u);
          if (!ok) break;
          more = C.units[(n + 1) % kUnits].tiles != 0;
          if (more) ask_query(n + 1);
        }
        const uint32_t on = *reinterpret_cast<volatile int32_t*>(&C.meta[gt % kMeta].on);
        const int left = x.len - t * kKeys;
        if (!idle) {
          const bool masked = on != 15u || (t + 1) * kKeys > x.all_see;
          if (x.n_here <= kSlim) weigh_slim(t, gt, on, masked);
          else if (x.copies == 4) weigh(std::integral_constant<int, 4>{}, t, gt, on, masked);
          else if (x.copies == 2) weigh(std::integral_constant<int, 2>{}, t, gt, on, masked);
          else weigh(std::integral_constant<int, 1>{}, t, gt, on, masked);
        }
        if (on != 15u || left < kKeys) {      // values that no token has may be anything: a weight of 0 does not cancel a NaN
          const uint32_t v = gt % Z::kRing;
          wait_on(&C.v[v], (gt / Z::kRing) & 1u);
          const int key = threadIdx.x & 63, h = threadIdx.x >> 6;
          if (ok && h < D / 64 && (key >= left || !(on >> (key / 16) & 1u))) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
              sts128(sV + v * Z::kTile + (key >> A.page_shift) * A.page * (D * 2) + (h * A.page + (key & (A.page - 1))) * 128 + c * 16, make_uint4(0, 0, 0, 0));
          }
          fence_proxy_async();
        }
        if (!ok) break;
        tc5_fence_before();
        mbar_arrive(&C.p[gt & 1u]);
      }
      t0 += x.tiles;
      if (more) put_query();
      wait_on(&C.o[(t0 - 1) & 1u], ((t0 - 1) / 2) & 1u);
      if (!rows_all(ok)) {
        ok = false;
        break;
      }
      tc5_fence_after();

      // ---- the unit's rows: to their queries' places, or as a piece
      const Unit& u = C.units[n % kUnits];
      const size_t rows0 = static_cast<size_t>(u.shared) * A.n_tokens;
      const auto place_of = [&](int row) -> size_t {      // of whole units
        const int query = query_of(u, row);
        return (rows0 + u.token0 + query) * A.hq + u.kvh * A.group + u.head0 + row - query * A.group;
      };
      float* const piece = A.pieces + static_cast<size_t>(u.place) * (kRows * (D + 2));
      const auto sums_of = [&](int row) -> float* { return u.place < 0 ? A.rows + place_of(row) * D : piece + row * D; };
      const auto ml_of = [&](int row) -> float2* { return u.place < 0 ? A.row_ml + place_of(row) : reinterpret_cast<float2*>(piece + kRows * D) + row; };
      bool strange = false;      // a sum that is no finite number although its row's weights are numbers
      const auto flag = [&](int row) { atomicOr(&C.redo[row >> 5], 1u << (row & 31)), strange = true; };
      if (x.copies == 1) {
        bool found = false;
        if (!idle) {
          float* const to = sums_of(x.real ? x.row : 0);
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t r[32];
            tmem_ld32(t_row + kOutAt + c, r);
            float2 none[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};      // (0 times what is no finite number is no number)
#pragma unroll
            for (int j = 0; j < 32; j += 2)
              none[j / 2 & 1] = fma2(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), make_float2(0.f, 0.f), none[j / 2 & 1]);
            found |= !((none[0].x + none[0].y) + (none[1].x + none[1].y) == 0.f);
            if (x.real)
#pragma unroll
              for (int j = 0; j < 32; j += 8) store_32(to + c + j, r + j);
          }
          if (x.real) *ml_of(x.row) = make_float2(ref, sum);
        }
        if (found && x.real && isfinite(sum)) flag(x.row);
      } else {
        // The copies' sums meet in shared memory: whole rows, halves or quarters of all rows at a time, as they fit.
        const int held = x.copies * x.n_here, mine = x.copy * x.n_here + x.row;
        float2* const refs = reinterpret_cast<float2*>(smem + (x.n_here <= kSlim ? Z::kMeet + 4 * kSlim * 512 : Z::kRefs));      // [copies][n_here]
        // elements c0 to c0 + kCols of all rows, from all copies
        const auto gather = [&](auto cols_tag, auto copies_tag, int c0) {
          constexpr int kCols = decltype(cols_tag)::value, kChunks = kCols / 4, kCopies = decltype(copies_tag)::value;
          for (int i = threadIdx.x; i < x.n_here * kChunks; i += kRows) {
            const int row = i / kChunks, chunk = i % kChunks;
            float2 z[kCopies];
            uint4 v[kCopies];
            float top = -INFINITY, all = 0.f;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
              const int at = k * x.n_here + row;
              z[k] = refs[at], v[k] = lds128(sMeet + at * (kCols * 4) + ((chunk ^ (at & 7)) << 4));
              top = fmaxf(top, z[k].x);
            }
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
              const float f = z[k].x == -INFINITY ? 1.f : ex2_approx(z[k].x - top);      // (a sum on no reference is no number)
              if (z[k].y != 0.f) {
                all = fmaf(z[k].y, f, all);
                y.x = fmaf(__uint_as_float(v[k].x), f, y.x), y.y = fmaf(__uint_as_float(v[k].y), f, y.y);
                y.z = fmaf(__uint_as_float(v[k].z), f, y.z), y.w = fmaf(__uint_as_float(v[k].w), f, y.w);
              }
            }
            reinterpret_cast<float4*>(sums_of(row) + c0)[chunk] = y;
            if (c0 + chunk == 0) *ml_of(row) = make_float2(top, all);
            if (!(isfinite(y.x) && isfinite(y.y) && isfinite(y.z) && isfinite(y.w)) && isfinite(all)) flag(row);
          }
        };
        const auto meet = [&](auto cols_tag, auto copies_tag, int c0) {
          constexpr int kCols = decltype(cols_tag)::value, kStep = kCols < 64 ? kCols : 64;
#pragma unroll 1
          for (int c = 0; c < kCols; c += kStep) {
            uint32_t r[kStep / 32][32];
#pragma unroll
            for (int i = 0; i < kStep / 32; ++i) tmem_ld32_nowait(t_row + kOutAt + c0 + c + i * 32, r[i]);
            tmem_wait_ld();
            if (x.real) {
#pragma unroll
              for (int j = 0; j < kStep / 4; ++j)
                sts128(sMeet + mine * (kCols * 4) + (((c / 4 + j) ^ (mine & 7)) << 4), make_uint4(r[j / 8][j % 8 * 4], r[j / 8][j % 8 * 4 + 1], r[j / 8][j % 8 * 4 + 2], r[j / 8][j % 8 * 4 + 3]));
            }
          }
          rows_barrier();
          gather(cols_tag, copies_tag, c0);
        };
        const auto meet_all = [&](auto copies_tag) {
          if (held * D * 4 <= static_cast<int>(Z::kMeetBytes)) {
            meet(std::integral_constant<int, D>{}, copies_tag, 0);
          } else {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              if (c) rows_barrier();      // (what was there has been read)
              meet(std::integral_constant<int, 32>{}, copies_tag, c);
            }
          }
        };
        if (x.n_here <= kSlim) {
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          if (x.real && (lane & 3) == 0) refs[mine] = make_float2(ref, sum);
#pragma unroll 1
          for (int c = 0; c < D; c += 64) {
            uint32_t r[32];
            tmem_ld_quads64(t_row + kOutAt + c, r);
            tmem_wait_ld();
            if (x.real) {
#pragma unroll
              for (int j = 0; j < 8; ++j) {      // elements c + 8 j + 2 (lane % 4) and the next one
                const uint32_t to = sMeet + mine * (D * 4) + (((c / 4 + 2 * j + ((lane & 3) >> 1)) ^ (mine & 7)) << 4) + (lane & 1) * 8;
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(r[4 * j]), "r"(r[4 * j + 1]) : "memory");
              }
            }
          }
          rows_barrier();
          gather(std::integral_constant<int, D>{}, std::integral_constant<int, 4>{}, 0);
        } else {
          if (x.real) refs[mine] = make_float2(ref, sum);
          if (x.copies == 4) meet_all(std::integral_constant<int, 4>{});
          else meet_all(std::integral_constant<int, 2>{});
        }
      }
      if (rows_any(strange)) {      // rare: rows whose sums a value behind a weight of 0 may have spoiled, by hand
        for (int row = warp; row < x.n_here; row += 4) {
          if (!(C.redo[row >> 5] >> (row & 31) & 1u)) continue;
          const int query = query_of(u, row), head = u.kvh * A.group + u.head0 + row - query * A.group;
          const int seen = x.shared || !A.causal ? x.len : max(0, x.len - (u.queries - 1 - u.query0 - query));
          sweep<D>(A, A.stream[x.shared], u.row, u.kvh, u.token0 + query, head, x.first * kKeys, min(seen, (x.first + x.tiles) * kKeys), sums_of(row), ml_of(row), &C.beat, lane);
        }
        rows_barrier();
        if (threadIdx.x < 4) C.redo[threadIdx.x] = 0;
      }
      tc5_fence_before();
      mbar_arrive(&C.empty[n % kUnits]);
    }
    if (!ok) failed = 1;
  }
  __syncwarp();
  tc5_fence_before();
  __syncthreads();
  if (works && failed && threadIdx.x == 0) report(A, QC_ERR_TIMEOUT);
  if (warp == 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns) : "memory");
}

// What a part with reference m and a sum counts for on reference top.  Minus infinity with a sum means that its scores were no numbers.
__device__ __forceinline__ float weight_of(float2 ml, float top) { return ml.y == 0.f ? 0.f : ml.x == -INFINITY ? NAN : exp2f(ml.x - top); }

// Puts the parts of each row together: a warp per row, a part's reference and sum per lane.  Grid: (sequences, parts of their rows).
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const __grid_constant__ AttendArgs A) {
  pdl_wait();
  const Plan plan = *A.plan;
  if (!plan.fine) return;
  const int lane = threadIdx.x & 31, step = gridDim.y * 8;
  const Record own = A.records[A.n_groups + blockIdx.x];
  Record prefix{};
  if (own.group >= 0) prefix = A.records[own.group];
  const size_t heads = static_cast<size_t>(A.n_tokens) * A.hq;
  for (int r = blockIdx.y * 8 + (threadIdx.x >> 5); r < own.queries * A.hq; r += step) {
    const int query = r / A.hq, head = r - query * A.hq, kvh = head / A.group;
    const int64_t token = own.token0 + query;
    const size_t at = token * A.hq + head;
    float m = -INFINITY, l = 0.f, o[D / 32] = {};
#pragma unroll 1
    for (int kind = own.group >= 0 ? 1 : 0; kind >= 0; --kind) {
      const Record& u = kind ? prefix : own;
      if (u.tiles == 0) continue;
      const int64_t flat = (token - u.token0) * A.group + head - kvh * A.group;
      const uint32_t per_head = static_cast<uint32_t>((static_cast<int64_t>(u.queries) * A.group + kRows - 1) / kRows);
      const uint32_t tiles_at = u.base + (kvh * per_head + static_cast<uint32_t>(flat / kRows)) * unit_cost(u.tiles) + kUnitCost;
      const int line = plan.lines == 2 && kind == 0 ? 1 : 0;
      const Line p = line ? plan.line[1] : plan.line[0];
      const bool cut = u.tiles >= 2 * p.least;
      const uint32_t first = worker_at(p, tiles_at + (cut ? p.least - 1 : u.tiles / 2)), last = worker_at(p, tiles_at + (cut ? u.tiles - p.least : u.tiles / 2));
      const int row = static_cast<int>(flat % kRows);
      const auto part = [&](uint32_t w) -> const float* {
        return first == last ? A.rows + (kind * heads + at) * D : A.pieces + (static_cast<size_t>(w) * 4 + line * 2 + (w == first ? 1 : 0)) * (kRows * (D + 2)) + row * D;
      };
      for (uint32_t w0 = first; w0 <= last; w0 += 32) {
        const uint32_t w = w0 + lane;
        const int n = min(32u, last + 1 - w0);
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < n)
          ml = __ldcg(first == last ? A.row_ml + kind * heads + at
                                    : reinterpret_cast<const float2*>(A.pieces + (static_cast<size_t>(w) * 4 + line * 2 + (w == first ? 1 : 0)) * (kRows * (D + 2)) + kRows * D) + row);
        float top = ml.x;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        top = fmaxf(top, m);
        const float f = weight_of(ml, top), old = weight_of(make_float2(m, l), top);
        float sum = ml.y * f;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        l = l * old + sum, m = top;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) o[k] = old == 0.f ? 0.f : o[k] * old;
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
          const float fk = __shfl_sync(0xffffffffu, f, k);
          const float* from = part(w0 + k);
          float v[D / 32];
          if constexpr (D == 128) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(from) + lane);
            v[0] = y.x, v[1] = y.y, v[2] = y.z, v[3] = y.w;
          } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(from) + lane);
            v[0] = y.x, v[1] = y.y;
          }
#pragma unroll
          for (int e = 0; e < D / 32; ++e) o[e] += fk == 0.f ? 0.f : v[e] * fk;
        }
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if constexpr (D == 128) reinterpret_cast<uint2*>(A.out + at * D)[lane] = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    else reinterpret_cast<uint32_t*>(A.out + at * D)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
    if (A.lse && lane == 0) A.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
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

// The workspace: plan and records, then the sums of whole units' rows, then pieces, each part at a multiple of 256 bytes.
constexpr int kMostWorkers = 296;
struct Layout {
  size_t records, rows, row_ml, pieces, bytes;
};
Layout layout_of(const qc_paged_attend_args* a) {
  const auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
  const size_t heads = static_cast<size_t>(a->n_tokens) * a->n_q_heads * (a->n_groups ? 2 : 1);
  Layout w{};
  w.records = 256;
  w.rows = w.records + up(static_cast<size_t>(a->n_groups + a->n_seqs) * sizeof(Record));
  w.row_ml = w.rows + up(heads * a->head_dim * 4);
  w.pieces = w.row_ml + up(heads * 8);
  w.bytes = w.pieces + static_cast<size_t>(kMostWorkers) * 4 * kRows * (a->head_dim + 2) * 4;
  return w;
}
size_t workspace_bytes(const qc_paged_attend_args* a) { return layout_of(a).bytes; }

// A pool as rows of D elements, from which a copy brings 64 of each token of a page and head; or the halves of the rows as a dimension of
// their own, and a copy brings all of them, one half after the other.  With the 128-byte swizzle.
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int32_t make_map(CUtensorMap* out, const void* pool, const qc_paged_attend_args* a, int32_t n_pages, bool values) {
  static const EncodeFn encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) fn = nullptr;
    return reinterpret_cast<EncodeFn>(fn);
  }();
  if (!encode) return QC_ERR_CUDA;
  const cuuint64_t d = a->head_dim, rows = static_cast<cuuint64_t>(n_pages) * a->n_kv_heads * a->page_size;
  const cuuint32_t page = a->page_size, steps[3] = {1, 1, 1};
  const cuuint64_t flat[2] = {d, rows}, halves[3] = {64, rows, d / 64}, strides[2] = {d * 2, 128};
  const cuuint32_t box2[2] = {64, page}, box3[3] = {64, page, static_cast<cuuint32_t>(d / 64)};
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, values ? 3 : 2, const_cast<void*>(pool), values ? halves : flat, strides, values ? box3 : box2, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? QC_OK
             : QC_ERR_CUDA;
}

template <int D>
cudaError_t launch(const AttendArgs& A, int device, cudaStream_t stream) {
  constexpr int kBytes = Shape<D>::kTiles + sizeof(Control);
  static std::atomic<bool> configured[64] = {};     // per device: the kernel may take that much
  cudaError_t e;
  if (device >= 64 || !configured[device].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(paged_attend_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    if (device < 64) configured[device].store(true, std::memory_order_relaxed);
  }
  int sms = 0;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return e;
  if ((e = launch_pdl(paged_attend_kernel<D>, dim3(min(2 * sms, kMostWorkers)), dim3(kBlock), kBytes, stream, A)) != cudaSuccess) return e;
  const int64_t rows = static_cast<int64_t>(A.starts ? A.max_queries : 1) * A.hq;
  return launch_pdl(paged_join_kernel<D>, dim3(A.n_seqs, static_cast<unsigned>(min((rows + 7) / 8, static_cast<int64_t>(65535)))), dim3(256), 0, stream, A);
}

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
      off(args->groups_dev, 4) || off(args->shared_ids_dev, 4) || off(args->workspace_dev, 256))
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
  uint8_t* const work = static_cast<uint8_t*>(args->workspace_dev);
  const Layout w = layout_of(args);
  A.plan = reinterpret_cast<Plan*>(work), A.records = reinterpret_cast<Record*>(work + w.records), A.rows = reinterpret_cast<float*>(work + w.rows);
  A.row_ml = reinterpret_cast<float2*>(work + w.row_ml), A.pieces = reinterpret_cast<float*>(work + w.pieces);
  A.hq = args->n_q_heads, A.hkv = args->n_kv_heads, A.group = A.hq / A.hkv, A.page = args->page_size;
  A.page_shift = A.page == 16 ? 4 : A.page == 32 ? 5 : 6;
  A.n_seqs = args->n_seqs, A.n_groups = args->n_groups, A.n_tokens = args->n_tokens, A.max_queries = args->max_queries, A.causal = args->causal != 0;
  const float scale = args->softmax_scale > 0.f ? args->softmax_scale : 1.0f / sqrtf(static_cast<float>(args->head_dim));
  A.scale_log2 = scale * 1.4426950408889634f, A.inv_group = 1.f / A.group;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  for (int i = 0; i <= (shared ? 1 : 0); ++i) {
    const qc_paged_stream& s = i ? args->shared : args->own;
    if (const int32_t bad = make_map(&A.map[i][0], s.k_pool_dev, args, s.n_pages, false)) return bad;
    if (const int32_t bad = make_map(&A.map[i][1], s.v_pool_dev, args, s.n_pages, true)) return bad;
  }
  return status_of(args->head_dim == 128 ? launch<128>(A, device, stream) : launch<64>(A, device, stream));
}
