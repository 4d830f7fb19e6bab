// Attention over bf16 pages for units of few rows: a sequence's own keys, or a prefix that few share.
//
// Such a unit reads its keys and values for 16 rows at most: some flops a byte, far below what the tensor cores need, so it is bound by
// the bytes as long as enough of them are under way.  Each warp works on its own: it walks its range of the plan (qc_paged_attend.cuh)
// and fetches tiles of 16 keys into a ring of its own, so that an SM has twelve independent chains of copies, products and
// softmax.  Eight sequences of 8 541 keys of 32 heads take 180 us, 0.97 of what a copy moves.  Short units are latency: a tile takes some 1 000 cycles
// alone and 3 400 where all warps fetch, a unit's start and end 3 000 to 7 500.  (As units of many rows, one chain of three hand-offs per
// block, 48 sequences of 64 tokens of 32 heads took the first kernel 25.5 us instead of 13.2.)
//
// Products are mma.sync m16n8k16 with the keys (for K) and the elements (for V) as rows and eight query rows as columns, once or
// twice:  S^T[16 keys x 8] = K Q^T,  O^T[D x 8] += V^T P^T.  Scores leave the first with a key per lane group; a transpose in registers
// makes them the second's operand.  Weights are rounded to bf16 there (2^-8 of themselves at most, the operand type; their sum is not), everything else is fp32.
// (In two bf16 parts, qc_paged_attend.cu says why not, they take one sequence from 12.5 to 13.1 us, long own sequences from 180 to 182, the video's
// questions from 158 to 162.)
// Rows of K and V lie in shared memory as in their page, 16 bytes at a time turned by the row, so that both ldmatrix
// patterns meet no bank twice.

#pragma once

#include "qc_paged_attend.cuh"

namespace qc {
namespace paged {

constexpr float kRescale = 8.f;      // the reference of a row moves when its scores have grown by 2^8

template <int D>
struct Ring {
  static constexpr int kStages = 256 / D;                   // 2 or 4 tiles
  static constexpr uint32_t kTile = Few::kKeys * D * 2;          // of K or of V
  static constexpr uint32_t kBytes = kStages * 2 * kTile;   // a warp's
};

// A tile's rows of K and V: row r at r * 2 D bytes, its 16-byte vector c at (c ^ r % 8).
template <int D>
__device__ __forceinline__ void ask_tile(const Args& A, const Stream& S, int32_t id, bool there, int kvh, int tile, int left, uint32_t to, int lane) {
  constexpr int kVectors = D / 8, kRowsAtOnce = 32 / kVectors;
  const int in_page = tile * Few::kKeys & (A.page - 1);
  const size_t at = there ? (((static_cast<size_t>(id) * A.hkv + kvh) << A.page_shift) + in_page) * D : 0;
  const uint16_t* const k = S.k_pool + at + lane * 8;
  const uint16_t* const v = S.v_pool + at + lane * 8;
  const int row0 = lane / kVectors, c = lane % kVectors;
#pragma unroll
  for (int i = 0; i < Few::kKeys / kRowsAtOnce; ++i) {
    const int row = i * kRowsAtOnce + row0;
    const uint32_t place = to + row * (D * 2) + ((c ^ (row & 7)) << 4);
    const int bytes = there && row < left ? 16 : 0;      // (the rest are zeros: what no token has may be anything)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(place), "l"(k + i * 256), "r"(bytes) : "memory");
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(place + Ring<D>::kTile), "l"(v + i * 256), "r"(bytes) : "memory");
  }
}

// Pages of a unit's row: ids one per lane from page `batch` on, and the 32 behind them.
struct Ahead {
  Unit w;
  bool has;
  int32_t batch, ids, next_ids;
};

// One unit: its rows in NT times eight columns.
template <int D, int NT>
__device__ __forceinline__ void take_unit(const Args& A, Ahead& x, uint32_t ring, int lane) {
  using R = Ring<D>;
  const Unit& w = x.w;
  const Stream& S = A.stream[w.shared];
  const int g = lane >> 2, t = lane & 3, stop = w.first + w.tiles;
  int asked = w.first;
  const auto ask = [&]() {
    if (asked < stop) {
      const int page = asked * Few::kKeys >> A.page_shift;
      if (page - x.batch >= 32) x.batch += 32, x.ids = x.next_ids, x.next_ids = ask_ids(A, w, x.batch + 32, lane);
      const int32_t id = __shfl_sync(0xffffffffu, x.ids, page - x.batch);
      const bool there = static_cast<uint32_t>(id) < static_cast<uint32_t>(S.n_pages);
      if (!there && lane == 0) report(A, QC_ERR_BAD_PAGE);
      ask_tile<D>(A, S, id, there, w.kvh, asked, there ? w.len - asked * Few::kKeys : 0, ring + (asked % R::kStages) * (2 * R::kTile), lane);
      ++asked;
      cp_async_commit_group();
      return there;
    }
    cp_async_commit_group();
    return true;
  };
  uint32_t here = 0;      // of the tiles under way: whether their pages are there, a bit per stage
#pragma unroll
  for (int i = 0; i < R::kStages; ++i) {
    const int stage = asked % R::kStages;
    here |= static_cast<uint32_t>(ask()) << stage;
  }
  // the queries: elements 2 t and 2 t + 1 of every eight, of row g of the columns
  uint32_t q[NT][D / 16][2];
  int seen[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = nt * 8 + g, query = query_of(A, w, row);
    const uint16_t* p = S.q + (w.token0 + query) * S.q_stride + static_cast<int64_t>(head_of(A, w, row, query)) * D + 2 * t;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      q[nt][i][0] = row < w.n_here ? __ldg(reinterpret_cast<const uint32_t*>(p + i * 16)) : 0u;
      q[nt][i][1] = row < w.n_here ? __ldg(reinterpret_cast<const uint32_t*>(p + i * 16 + 8)) : 0u;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) seen[nt][e] = seen_by(A, w, query_of(A, w, nt * 8 + 2 * t + e));
  }
  float acc[NT][D / 16][4], ref[NT][2], sum[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    ref[nt][0] = ref[nt][1] = -INFINITY, sum[nt][0] = sum[nt][1] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[nt][i][0] = acc[nt][i][1] = acc[nt][i][2] = acc[nt][i][3] = 0.f;
  }
  // where this lane's rows of the ldmatrix patterns are
  const uint32_t k_row = (lane & 15) * (D * 2), k_turn = lane & 7, k_half = lane >> 4;
  const uint32_t v_row = ((lane & 7) + (lane >> 4) * 8) * (D * 2), v_half = lane >> 3 & 1;

  for (int tile = w.first; tile < stop; ++tile) {
    const int stage = tile % R::kStages;
    const uint32_t keys = ring + stage * (2 * R::kTile), values = keys + R::kTile;
    cp_async_wait_group<R::kStages - 1>();
    __syncwarp();
    float c[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      uint32_t a[4];
      ldmatrix_x4(a, keys + k_row + (((2 * i + k_half) ^ k_turn) << 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(c[nt], a, q[nt][i]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j) c[nt][j] *= A.scale_log2;
    const bool there = here >> stage & 1u;
    if (!there || (tile + 1) * Few::kKeys > w.all_see) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!there || tile * Few::kKeys + g + (j >> 1) * 8 >= seen[nt][j & 1]) c[nt][j] = -INFINITY;
    }
    // scores far above their reference, or a row's first ones
    bool more = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float h = fmaxf(c[nt][e], c[nt][e + 2]);
        more |= h > ref[nt][e] + kRescale;      // (minus infinity so far: any score is)
      }
    if (__any_sync(0xffffffffu, more)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float h = fmaxf(c[nt][e], c[nt][e + 2]);
          h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 4));
          h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 8));
          h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, 16));
          if (h > ref[nt][e] + kRescale) {
            const float f = ex2_approx(ref[nt][e] - h);      // 0 on the first keys
            ref[nt][e] = h;
            sum[nt][e] *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) acc[nt][i][e] *= f, acc[nt][i][e + 2] *= f;
          }
        }
    }
    uint32_t b[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float r = ref[nt][j & 1];
        p[j] = ex2_approx(c[nt][j] - (r == -INFINITY ? 0.f : r));
        sum[nt][j & 1] += p[j];
      }
      b[nt][0] = movmatrix_trans(pack_bf16x2(p[0], p[1]));
      b[nt][1] = movmatrix_trans(pack_bf16x2(p[2], p[3]));
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      uint32_t a[4];
      ldmatrix_x4_trans(a, values + v_row + (((2 * i + v_half) ^ k_turn) << 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(acc[nt][i], a, b[nt]);
    }
    __syncwarp();      // (the tile has been read)
    here &= ~(1u << stage);
    here |= static_cast<uint32_t>(ask()) << stage;
  }
  cp_async_wait_all();
  __syncwarp();

  // the rows' sums, to their queries' places or as a piece: a lane has elements g and g + 8 of every 16
  const size_t piece = static_cast<size_t>(max(0, w.place)) * kFew;
  uint32_t strange = 0;      // rows with a sum that is no finite number although their weights are numbers
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = sum[nt][e];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      const int row = nt * 8 + 2 * t + e;
      if (row >= w.n_here) continue;
      const size_t at = place_of(A, w, row);
      float* const to = (w.place < 0 ? A.rows + at * D : A.few_pieces + (piece + row) * D) + g;
      float none = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        to[16 * i] = acc[nt][i][e], to[16 * i + 8] = acc[nt][i][e + 2];
        none = fmaf(acc[nt][i][e], 0.f, fmaf(acc[nt][i][e + 2], 0.f, none));      // (0 times what is no finite number is no number)
      }
      if (g == 0) *(w.place < 0 ? A.row_ml + at : A.few_piece_ml + piece + row) = make_float2(ref[nt][e], l);
      if (none != 0.f && isfinite(l)) strange |= 1u << row;
    }
  __syncwarp();
  for (uint32_t rows = __reduce_or_sync(0xffffffffu, strange); rows; rows &= rows - 1) {      // rare: by hand
    const int row = __ffs(rows) - 1;
    const size_t at = place_of(A, w, row);
    sweep<D>(A, w, row, w.first * Few::kKeys, stop * Few::kKeys, w.place < 0 ? A.rows + at * D : A.few_pieces + (piece + row) * D,
             w.place < 0 ? A.row_ml + at : A.few_piece_ml + piece + row, nullptr, lane);
  }
}

// A warp's range.
template <int D>
__device__ __forceinline__ void take_few(const Args& A, Walk<Few>& walk, uint32_t ring, int lane) {
  const auto look = [&](Ahead& x) {
    x.has = walk.find(A, x.w, lane);
    if (!x.has) return;
    x.batch = x.w.first * Few::kKeys >> A.page_shift;
    x.ids = ask_ids(A, x.w, x.batch, lane), x.next_ids = ask_ids(A, x.w, x.batch + 32, lane);
  };
  // (a unit is looked for in one place: what runs once is bound by the way of its instructions)
  for (Ahead now{}, then{};;) {
    look(then);      // its page ids are on their way while the unit before it is taken
    if (now.has) {
      if (now.w.n_here <= 8) take_unit<D, 1>(A, now, ring, lane);
      else take_unit<D, 2>(A, now, ring, lane);
    }
    if (!then.has) break;
    now = then;
  }
}

}  // namespace paged
}  // namespace qc
