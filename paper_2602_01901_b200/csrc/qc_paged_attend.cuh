// The plan of qc_paged_attend, as its kernels see it.
//
// A batch is items: prefixes (of groups) and sequences.  An item's rows (query tokens times the query heads of a KV head) that score the same
// keys are units: at most 128 rows, which a block takes with the tensor cores' large products (qc_paged_attend.cu), or, where an item has no
// more than kFew, all of them, which a warp takes (qc_paged_few.cuh).  The blocks of the launch are shared out between the two
// kinds by what each has to do.  The costs of a kind's units (tiles of keys, and a constant for a unit) are laid end to end and cut into
// equal ranges, one per worker: a block, or a warp.  A unit inside one range leaves its rows' sums at their queries' places; of
// one that a border cuts each worker leaves a piece.  A second kernel puts together what there is of a row.
// Every number of the plan comes from the lists and lengths on the device, and all blocks find the same.
#pragma once

#include "../../include/qc.h"
#include "qc_device.cuh"

namespace qc {
namespace paged {

// Rows of an item that a warp takes.  With 8 in its place, so that blocks take 9 to 16: the five images' chats 54.1 us instead of 50.4; one long
// prefix (16 rows of 32 heads, 8 541 keys) 47.3 and 48.0, 64 sequences of 500 keys with 12 rows on each of 4 KV heads 28.0 and 27.9; the 24 drafted
// sequences, 64 wide with up to 20 rows, 33.5 and 38.1.  So the border lies where rows of 128 elements want it.  (Of these rows, 16 columns of 128
// elements, some 190 bytes a thread are written to local memory and read back: the only such ones in the kernel.)
constexpr int kFew = 16;
constexpr int kBlock = 192;       // threads of a block of either kernel
constexpr int kMostHeld = 2048;   // items that a block keeps in shared memory while it looks for its range
constexpr uint32_t kMostCost = 1u << 30;      // of a kind's units: sums of two such, and of one and a difference, fit in 32 bits

struct Stream {
  const uint16_t* q;
  int64_t q_stride;
  const uint16_t* k_pool;
  const uint16_t* v_pool;
  const int32_t* pages;
  const int32_t* lens;
  int32_t max_pages, n_pages, rows;
};

// What the second kernel knows of an item: where its costs begin among those of its kind, its tiles (0: no units), tokens.
struct Record {
  uint32_t base;
  int32_t tiles, token0, queries;
};

// A row of costs, cut into ranges: the first `longer` workers have `per` + 1, the others `per`.
struct Line {
  uint32_t per, longer, workers;
  int32_t least;           // tiles of a piece
};
// Lines of units of many and of few rows; the first `many` blocks take the former.
struct Plan {
  Line line[2];
  uint32_t many;
  int32_t fine;            // whether the batch is computed
};

struct Args {
  CUtensorMap map[2][2];   // many rows: K and V of own and shared pages: a copy brings a page's tokens of a head, 64 elements of K or all of V
  Stream stream[2];        // own, shared
  const int32_t* ids;
  const int32_t* starts;
  const int32_t* groups;
  const int32_t* shared_ids;
  uint16_t* out;
  float* lse;
  Plan* plan;
  Record* records;         // [sequences][2] its own tokens, its prefix
  float* rows;             // [kinds][tokens * heads][D] sums of whole units
  float2* row_ml;          // [kinds][tokens * heads] their references and sums of weights
  float* pieces;           // [workers][2][128][D] of many rows
  float2* piece_ml;        // [workers][2][128]: side by side, since they are read first
  float* few_pieces;       // [workers][2][kFew][D]
  float2* few_piece_ml;    // [workers][2][kFew]
  int32_t* status;
  int32_t hq, hkv, group, page, page_shift;
  int32_t n_seqs, n_groups, n_tokens, max_queries, causal;
  float scale_log2, inv_group;
};

#ifdef __CUDACC__

__device__ __forceinline__ void report(const Args& A, int code) {
  if (A.status) atomicMax(A.status, code);
}

__device__ __forceinline__ int length_of(const Args& A, const Stream& S, int row, bool tell) {
  const int64_t len = __ldg(S.lens + row), room = static_cast<int64_t>(S.max_pages) << A.page_shift;
  if (len >= 0 && len <= room) return static_cast<int>(len);
  if (tell) report(A, QC_ERR_PLAN);
  return len < 0 ? 0 : static_cast<int>(room);
}

// The two kinds of units: rows of a unit, keys of a tile, what a unit costs besides its tiles, and the least tiles of a range and (as long as
// ranges are not much longer) of a piece.  With these values one sequence takes 12.6 us, the five images' chats 50.4, the 24 drafted sequences 38.1,
// the video's questions 158; with another one in the place of one of them:
//   a unit of many rows costs 2 tiles: at 0 images 53.7, drafts 38.4, video 161; at 6 images 50.5, drafts 39.2, video 158;
//   of few rows 6: at 2 images 51.5, drafts 40.5, video 162, but one sequence 12.4;
//   a range of few rows has 2 tiles or more: at 1 one sequence 12.7, video 160, the others as here; at 4 one sequence 15.5, drafts 35.9;
//   a piece of many rows has 4: at 1 video 160, the others as here; of few rows 3: at 8 images 51.3, long own sequences 181 (180).
struct Many {
  static constexpr int kRows = 128, kKeys = 64;
  static constexpr bool kIsFew = false;
  static constexpr uint32_t kUnitCost = 2, kRange = 1, kPiece = 4;
};
struct Few {
  static constexpr int kRows = kFew, kKeys = 16;
  static constexpr bool kIsFew = true;
  static constexpr uint32_t kUnitCost = 6, kRange = 2, kPiece = 3;
};
// What a tile of many rows takes a block, in tiles that the warps of a block take together: so much alone, and more beside the others, which keep
// the memory busy (images 50.4 us, 78.2 without it; drafts 38.1 and 37.5, video 158 and 158; with 5 alone 61.5, 37.6 and 165).
constexpr float kManyTile = 3.f, kManyMore = 6.f;

// An item as it is held while units are looked for.
struct Held {
  int32_t token0, queries, row, len;
};
struct Item {
  int32_t token0, queries, row, len, tiles;
  uint32_t units, per_head;      // units; those of a KV head
};

__device__ __forceinline__ bool is_few(const Args& A, int queries) { return static_cast<int64_t>(queries) * A.group <= kFew; }

template <typename K>
__device__ __forceinline__ Item item_from(const Args& A, const Held& h) {
  Item u{h.token0, h.queries, h.row, h.len, 0, 0, 1};
  if (u.queries == 0 || is_few(A, u.queries) != K::kIsFew) return u;
  u.tiles = (u.len + K::kKeys - 1) / K::kKeys;
  u.per_head = static_cast<uint32_t>((static_cast<int64_t>(u.queries) * A.group + K::kRows - 1) / K::kRows);
  u.units = u.tiles ? static_cast<uint32_t>(min(static_cast<uint64_t>(u.per_head) * A.hkv, static_cast<uint64_t>(kMostCost))) : 0u;
  return u;
}

// Items 0 .. n_groups - 1 are prefixes, the others sequences.  `fine`: the numbers on the device fit.
__device__ __forceinline__ Held item_of(const Args& A, int i, bool tell, bool& fine) {
  Held h{};
  const bool shared = i < A.n_groups;
  int64_t a, b;
  if (shared) {
    a = A.groups ? __ldg(A.groups + i) : 0, b = A.groups ? __ldg(A.groups + i + 1) : A.n_seqs;
    h.row = A.shared_ids ? __ldg(A.shared_ids + i) : i;
    fine = a >= 0 && b >= a && b <= A.n_seqs;
    if (fine && A.starts) a = __ldg(A.starts + a), b = __ldg(A.starts + b);
  } else {
    const int seq = i - A.n_groups;
    a = seq, b = seq + 1;
    if (A.starts) a = __ldg(A.starts + seq), b = __ldg(A.starts + seq + 1);
    h.row = A.ids ? __ldg(A.ids + seq) : seq;
    fine = b - a <= A.max_queries;
  }
  const Stream& S = A.stream[shared];
  fine = fine && a >= 0 && b >= a && b <= A.n_tokens && h.row >= 0 && h.row < S.rows;
  if (!fine) return Held{};
  h.token0 = static_cast<int32_t>(a), h.queries = static_cast<int32_t>(b - a);
  if (h.queries) h.len = length_of(A, S, h.row, tell);
  return h;
}

template <typename K>
__device__ __forceinline__ uint32_t unit_cost(int tiles) { return K::kUnitCost + tiles; }
template <typename K>
__device__ __forceinline__ uint32_t cost_of(const Item& u) {      // kMostCost + 1: too much
  return static_cast<uint32_t>(min(static_cast<uint64_t>(u.units) * unit_cost<K>(u.tiles), static_cast<uint64_t>(kMostCost) + 1));
}

__device__ __forceinline__ uint32_t range_begin(const Line& p, uint32_t w) { return w * p.per + min(w, p.longer); }
__device__ __forceinline__ uint32_t worker_at(const Line& p, uint32_t at) {
  const uint32_t turn = p.longer * (p.per + 1);
  return at < turn ? at / (p.per + 1) : p.longer + (at - turn) / p.per;
}
// Where a border at tile t of a unit is: never so near to its first or last tile that a piece would hardly be worth its start.
__device__ __forceinline__ int border(int least, int t, int tiles) {
  if (tiles < 2 * least) return t <= tiles / 2 ? 0 : tiles;
  return t < least ? 0 : t > tiles - least ? tiles : t;
}
// The workers of a unit whose tiles begin at `tiles_at`.
__device__ __forceinline__ void workers_of(const Line& p, uint32_t tiles_at, int tiles, uint32_t& first, uint32_t& last) {
  const bool cut = tiles >= 2 * p.least;
  first = worker_at(p, tiles_at + (cut ? p.least - 1 : tiles / 2));
  last = cut ? worker_at(p, tiles_at + (tiles - p.least)) : first;
}

// What all blocks find out first, with all of their threads: the costs of the items of each kind before each item, and the items (where they are
// no more than kMostHeld), in shared memory.
struct Found {
  uint32_t before[2][2 * QC_PAGED_MAX_SEQS];
  Held held[kMostHeld];
};
__device__ __forceinline__ Line line_of(uint32_t cost, uint32_t most, uint32_t range, uint32_t piece) {
  Line p{};
  p.workers = max(1u, min(most, cost / range));
  p.per = cost / p.workers, p.longer = cost - p.per * p.workers;
  p.least = static_cast<int32_t>(max(range, min(piece, p.per / 4)));
  return p;
}
// `sums`: [kBlock / 32].
__device__ __forceinline__ Plan plan_of(const Args& A, Found& found, uint64_t* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_items = A.n_groups + A.n_seqs;
  constexpr uint32_t kTooMuch = kMostCost + 1;
  bool fine = true;
  uint32_t total[2] = {0, 0};
  for (int i0 = 0; i0 < n_items; i0 += kBlock) {
    const int i = i0 + threadIdx.x;
    uint32_t mine[2] = {0, 0};
    Held h{};
    if (i < n_items) {
      bool ok;
      h = item_of(A, i, blockIdx.x == 0, ok);
      if (is_few(A, h.queries)) mine[1] = cost_of<Few>(item_from<Few>(A, h));
      else mine[0] = cost_of<Many>(item_from<Many>(A, h));
      fine &= ok;
    }
    uint32_t sum[2] = {mine[0], mine[1]};      // (what is too much stays kTooMuch; the costs before an item are of no use then)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, sum[k], o);
        if (lane >= o) sum[k] = min(kTooMuch, sum[k] + y);
      }
    if (lane == 31) sums[warp] = static_cast<uint64_t>(sum[1]) << 32 | sum[0];
    __syncthreads();
    uint32_t at[2] = {min(kTooMuch, total[0] + (sum[0] - mine[0])), min(kTooMuch, total[1] + (sum[1] - mine[1]))};
#pragma unroll
    for (int w = 0; w < kBlock / 32; ++w)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t x = static_cast<uint32_t>(sums[w] >> (32 * k));
        if (w < warp) at[k] = min(kTooMuch, at[k] + x);
        total[k] = min(kTooMuch, total[k] + x);
      }
    if (i < n_items) {
      found.before[0][i] = at[0], found.before[1][i] = at[1];
      if (n_items <= kMostHeld) found.held[i] = h;
    }
    __syncthreads();
  }
  fine = __syncthreads_and(fine);
  const bool small = total[0] <= kMostCost && total[1] <= kMostCost;
  // All that can go side by side does, where there are blocks enough (or nearly so); else they are shared out by the time they take.  Either kind has
  // a block at least.
  const uint32_t blocks = gridDim.x, warps = kBlock / 32;
  uint32_t many = min(blocks, total[0] / Many::kRange);
  const uint32_t few = (min(blocks * warps, max(1u, total[1] / Few::kRange)) + warps - 1) / warps;
  if (total[1] && total[0] && many + few / 2 > blocks) {
    const float share = total[1] / (kManyTile * total[0] + total[1]), tile = kManyTile + kManyMore * share;
    many = max(1u, min(blocks - 1, static_cast<uint32_t>(blocks * (tile * total[0] / (tile * total[0] + total[1])) + 0.5f)));
  }
  if (total[1]) many = min(many, blocks - 1);
  Plan p{};
  p.many = many;
  p.line[0] = line_of(total[0], max(1u, many), Many::kRange, Many::kPiece);
  p.line[1] = line_of(total[1], max(1u, blocks - many) * warps, Few::kRange, Few::kPiece);
  p.fine = fine && small;
  if (blockIdx.x == 0 && threadIdx.x == 0 && !p.fine) report(A, fine ? QC_ERR_PLAN : QC_ERR_INVALID_ARG);
  if (total[0] == 0) p.line[0].workers = 0;
  if (total[1] == 0) p.line[1].workers = 0;
  return p;
}

// What the second kernel needs, by one block.
__device__ __forceinline__ void write_down(const Args& A, const Plan& plan, const Found& found) {
  if (threadIdx.x == 0) *A.plan = plan;
  const bool holds = A.n_groups + A.n_seqs <= kMostHeld;
  const auto record = [&](int i) -> Record {
    bool fine;
    const Held h = holds ? found.held[i] : item_of(A, i, false, fine);
    const bool few = is_few(A, h.queries);
    const Item u = few ? item_from<Few>(A, h) : item_from<Many>(A, h);
    return Record{found.before[few][i], u.units ? u.tiles : 0, h.token0, h.queries};
  };
  for (int seq = threadIdx.x; seq < A.n_seqs; seq += kBlock) {
    int group = -1;
    if (A.n_groups) {      // the group that the sequence is in: the first that ends behind it, if it begins by then
      int lo = 0, hi = A.groups ? A.n_groups : 0;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(A.groups + mid + 1) > seq) hi = mid;
        else lo = mid + 1;
      }
      if (!A.groups || (lo < A.n_groups && __ldg(A.groups + lo) <= seq)) group = lo;
    }
    A.records[2 * seq] = record(A.n_groups + seq);
    A.records[2 * seq + 1] = group >= 0 ? record(group) : Record{};
  }
}

struct Unit {
  int32_t token0;                // the token of its first row
  int32_t head0;                 // and that row's head inside the KV head's group
  int32_t query0, queries;       // the query of its first row among the item's
  int32_t n_here, kvh, shared, row, first, tiles, len;
  int32_t all_see;               // keys that every row sees
  int32_t place;                 // of a piece: worker * 2, + 1 where the unit begins in the range; -1: the unit is whole
};

// A warp's way through its worker's range, unit by unit.  32 items are held, one per lane.
template <typename K>
struct Walk {
  uint32_t at, begin, end, item_at;
  int item, least, first_held, worker;
  Held mine;
  Item u;

  __device__ __forceinline__ void hold(const Args& A, int from, int lane) {
    first_held = from;
    bool fine;
    if (from + lane < A.n_groups + A.n_seqs) mine = item_of(A, from + lane, false, fine);
  }
  __device__ __forceinline__ void turn_to(const Args& A, int i) {
    const int from = i - first_held;
    u = item_from<K>(A, Held{__shfl_sync(0xffffffffu, mine.token0, from), __shfl_sync(0xffffffffu, mine.queries, from),
                                         __shfl_sync(0xffffffffu, mine.row, from), __shfl_sync(0xffffffffu, mine.len, from)});
  }
  // (reads what plan_of has found for the last time)
  __device__ __forceinline__ void start(const Args& A, const Line& p, int w, const Found& found, int lane) {
    const int n_items = A.n_groups + A.n_seqs;
    worker = w, least = p.least;
    at = begin = range_begin(p, w), end = range_begin(p, w + 1);
    int lo = 0, hi = n_items - 1;      // the last item that begins at or before the range
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (found.before[K::kIsFew][mid] <= at) lo = mid;
      else hi = mid - 1;
    }
    item = lo, item_at = found.before[K::kIsFew][lo];
    mine = Held{};
    if (n_items > kMostHeld) hold(A, item, lane);
    else if (first_held = item, item + lane < n_items) mine = found.held[item + lane];
    turn_to(A, item);
  }
  // The next unit, if there is one.
  __device__ __forceinline__ bool find(const Args& A, Unit& w, int lane) {
    const int n_items = A.n_groups + A.n_seqs;
    while (at < end) {
      const uint32_t cost = cost_of<K>(u), one = unit_cost<K>(u.tiles);
      if (u.units == 0 || at >= item_at + cost) {
        if (++item >= n_items) return false;
        item_at += cost;
        if (item == first_held + 32) hold(A, item, lane);
        turn_to(A, item);
        if (at < item_at) at = item_at;
        continue;
      }
      const uint32_t unit = (at - item_at) / one, unit_at = item_at + unit * one, tiles_at = unit_at + K::kUnitCost;
      const int first = border(least, static_cast<int>(begin - tiles_at), u.tiles), last = border(least, static_cast<int>(end - tiles_at), u.tiles);
      at = unit_at + one;
      if (first >= last) continue;
      int kvh = unit, part = 0;
      if (!K::kIsFew) kvh = unit / u.per_head, part = unit - kvh * u.per_head;
      const int64_t row0 = static_cast<int64_t>(part) * K::kRows, rows = static_cast<int64_t>(u.queries) * A.group;
      w.n_here = static_cast<int32_t>(min(static_cast<int64_t>(K::kRows), rows - row0));
      w.query0 = part ? static_cast<int32_t>(row0 / A.group) : 0, w.head0 = part ? static_cast<int32_t>(row0 - static_cast<int64_t>(w.query0) * A.group) : 0;
      w.token0 = u.token0 + w.query0, w.queries = u.queries, w.kvh = kvh, w.shared = item < A.n_groups, w.row = u.row, w.first = first, w.tiles = last - first, w.len = u.len;
      w.all_see = w.shared || !A.causal ? u.len : max(0, u.len - (u.queries - 1 - w.query0));
      w.place = first == 0 && last == u.tiles ? -1 : worker * 2 + (first == 0 ? 1 : 0);
      return true;
    }
    return false;
  }
};

// Rows of a unit are its first query's heads from head0 on, then the next query's.
__device__ __forceinline__ int query_of(const Args& A, const Unit& u, int row) { return static_cast<int>((static_cast<float>(u.head0 + row) + 0.5f) * A.inv_group); }
__device__ __forceinline__ int head_of(const Args& A, const Unit& u, int row, int query) { return u.kvh * A.group + u.head0 + row - query * A.group; }
__device__ __forceinline__ int seen_by(const Args& A, const Unit& u, int query) {
  return u.shared || !A.causal ? u.len : max(0, u.len - (u.queries - 1 - u.query0 - query));
}
// Where a row's sums go where its unit is whole.
__device__ __forceinline__ size_t place_of(const Args& A, const Unit& u, int row) {
  const int query = query_of(A, u, row);
  return (static_cast<size_t>(u.shared) * A.n_tokens + u.token0 + query) * A.hq + head_of(A, u, row, query);
}

// Page ids of a unit's row, one per lane, from page `from` on.
__device__ __forceinline__ int32_t ask_ids(const Args& A, const Unit& w, int from, int lane) {
  const int page = from + lane;
  const Stream& S = A.stream[w.shared];
  return static_cast<int64_t>(page) << A.page_shift < w.len ? __ldg(S.pages + static_cast<int64_t>(w.row) * S.max_pages + page) : -1;
}

// Keys [from, to) of a table row for one query, by one warp, a key at a time: what the tensor cores cannot give where a value that is
// infinite or no number stands behind a weight of 0 (0 times it is no number).  Replaces those of the row's sums that are no finite
// numbers, on the row's reference.
template <int D>
__device__ __noinline__ void sweep(const Args& A, const Unit& u, int row, int from, int to, float* sums, const float2* ml, uint32_t* beat, int lane) {
  const Stream& S = A.stream[u.shared];
  const int query = query_of(A, u, row), head = head_of(A, u, row, query);
  to = min(to, seen_by(A, u, query));
  float o[D / 32] = {}, m = -INFINITY, l = 0.f, q[D / 32];
  const auto load = [&](const uint16_t* p, float (&f)[D / 32]) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const float2 x = bf16x2_to_f32(__ldg(reinterpret_cast<const uint32_t*>(p) + i * 32 + lane));
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  };
  load(S.q + (u.token0 + query) * S.q_stride + static_cast<int64_t>(head) * D, q);
#pragma unroll 2
  for (int j = from; j < to; ++j) {
    if (beat && lane == 0 && (j & 63) == 0) atomicAdd(beat, 1u);
    const int32_t id = __ldg(S.pages + static_cast<int64_t>(u.row) * S.max_pages + (j >> A.page_shift));
    if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(S.n_pages)) continue;
    const int64_t at = (((static_cast<int64_t>(id) * A.hkv + u.kvh) << A.page_shift) + (j & (A.page - 1))) * D;
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
  // (by the two sums, not the two references: these are scores, and where scores are large they are apart by their roundings)
  const float scale = l == 0.f ? 0.f : ml->y / l;
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float* const to_here = sums + (i * 32 + lane) * 2 + e;
      if (!isfinite(*to_here)) *to_here = l == 0.f ? 0.f : o[2 * i + e] * scale;
    }
}

#endif  // __CUDACC__

}  // namespace paged
}  // namespace qc
