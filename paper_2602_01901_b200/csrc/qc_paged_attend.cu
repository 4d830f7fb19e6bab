// Attention of a step's queries over bf16 pages, where adjacent sequences of a batch share a prefix.
//
//   out = softmax(scale [q_shared K_prefix ; q_own K_own]) [V_prefix ; V_own]
//
// A prefix's keys are scored by all query rows of its group at once (its tokens times the query heads of a KV head), a sequence's
// own by its own rows.  The plan stands in qc_paged_attend.cuh, what a warp does with a unit of few rows in qc_paged_few.cuh; here are the
// units of up to 128 rows, one at a time for a block, two blocks an SM.
//
// Per tile of 64 keys: S[128 x 64] = Q K^T and O[128 x D] += P V by tcgen05.mma, Q, K and V in shared memory (K and V by tensor-map
// copies of pages), S, P and O in tensor memory.  Four warps hold a row per thread, one issues products, one fetches.  Weights are rounded to bf16
// for the second product (2^-8 of themselves at most, the operand type; their sum is not), everything else is fp32.  That leaves outputs 1.7e-3 to
// 2.2e-3 of their norm from 64 bits, where their own rounding to bf16 is 1.4e-3 to 1.7e-3.  With the weights in two bf16 parts, as the decode launches of
// one layer have them (qc_rows.cu), and twice the products, it is the latter alone, here and for few rows; the video's questions take 192 us
// instead of 158, a prefix of 64-wide heads 103 instead of 85.3, 128 queries a sequence 138 instead of 123.  One part is taken for what it costs.
//
// 64 keys and 256 columns of tensor memory let two blocks share an SM, whose phases fill each other's gaps: 1 792 rows on each of 4
// heads of 32 768 keys take 128 us with pages of 64 tokens, 938 TFLOP/s of 1 681 measured (147 with pages of 16: four times
// the copies for the one warp that asks for them).  No pipe is full there: tensor 47 %, exponentials 48 %, issue slots 40 %; without any
// exponentials the time is the same.  A block's tile takes 1 750 cycles, its rows' dependent instructions most of them (two such warps a scheduler, 168
// registers a thread), and a seventh of the whole is start and end.

#include "qc_paged_few.cuh"
#include "qc_quant.h"
#include "qc_umma.cuh"

#include <algorithm>
#include <atomic>

namespace qc {
namespace {

using namespace paged;

constexpr int kRows = Many::kRows, kKeys = Many::kKeys;
static_assert(kBlock == kRows + 64);
constexpr int kUnits = 4;        // units that are known to the block at a time
constexpr int kMeta = 8;         // tiles whose places are
constexpr uint32_t kScoresAt = 0, kOutAt = 128, kColumns = 256;   // tensor memory: two score buffers of 64 columns, D of the sums

struct Meta {
  int32_t y[4];                  // of a tile's pages: the first row in the pool, -1: the page is not there
  int32_t on, shared;            // blocks of 16 keys that are there
};

template <int D>
struct Shape {
  static constexpr int kRing = D == 128 ? 2 : 4;      // tiles of K, and of V, under way
  static constexpr uint32_t kTile = kKeys * D * 2, kHalf = kKeys * 128, kQ = kRows * D * 2, kQHalf = kRows * 128;
  static constexpr uint32_t kLarge = kQ + 2 * kRing * kTile, kSmall = kBlock / 32 * Ring<D>::kBytes, kTiles = kLarge > kSmall ? kLarge : kSmall;
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
__global__ void __launch_bounds__(kBlock, 2) paged_attend_kernel(const __grid_constant__ Args A) {
  using Z = Shape<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sQ = smem_u32(smem), sK = sQ + Z::kQ, sV = sK + Z::kRing * Z::kTile;
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
  }
  pdl_wait();
  // (not ahead of the wait: a kernel before this one may still want tensor memory for blocks that are to come; by all blocks, since those of few
  // rows ran 4 us longer without)
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&C.tmem)), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }

  // the plan, in the tiles' place until they come
  Found& found = *reinterpret_cast<Found*>(smem);
  static_assert(sizeof(Found) <= Z::kTiles, "the plan takes the tiles' place");
  const Plan plan = plan_of(A, found, C.sums);
  if (blockIdx.x == 0) {
    if (plan.fine) write_down(A, plan, found);
    else if (threadIdx.x == 0) A.plan->fine = 0;
  }
  const Line line = plan.line[0];
  const bool works = plan.fine && blockIdx.x < line.workers;
  if (blockIdx.x >= plan.many) {      // a block for units of few rows
    const Line few = plan.line[1];
    const uint32_t block = blockIdx.x - plan.many, blocks = gridDim.x - plan.many;
    // workers side by side on an SM where all warps have work, else spread over the blocks
    const uint32_t worker = few.workers < blocks * (kBlock / 32) ? warp * blocks + block : block * (kBlock / 32) + warp;
    const bool has = plan.fine && worker < few.workers;
    Walk<Few> walk;
    if (has) walk.start(A, few, worker, found, lane);
    __syncthreads();      // (the plan has been read)
    if (has) take_few<D>(A, walk, sQ + warp * Ring<D>::kBytes, lane);
  }
  tc5_fence_before();
  __syncthreads();
  tc5_fence_after();
  const uint32_t tmem = C.tmem;

  if (works && warp == 5) {
    // ------------------------------------------------------------------ units and tiles
    Walk<Many> walk;
    walk.start(A, line, blockIdx.x, found, lane);
    __syncwarp();
    fence_proxy_async();      // (the plan has been read before copies take its place)
    const int per_tile = kKeys >> A.page_shift;
    // a unit, whether there is one, and page ids, one per lane: from page `batch` of its row on, and the 32 behind them
    struct Ahead {
      Unit w;
      bool has;
      int32_t batch, ids, next_ids;
    };
    const auto look = [&](Ahead& x) {
      x.has = walk.find(A, x.w, lane);
      if (!x.has) return;
      x.batch = x.w.first * per_tile;
      x.ids = ask_ids(A, x.w, x.batch, lane), x.next_ids = ask_ids(A, x.w, x.batch + 32, lane);
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
          if (page0 - now.batch >= 32) now.batch += 32, now.ids = now.next_ids, now.next_ids = ask_ids(A, w, now.batch + 32, lane);
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
    const int row = threadIdx.x;
    // a unit as this thread sees it
    struct Mine {
      int n_here, tiles, first, len, all_see, shared, seen;
      bool real;
    };
    const auto take = [&](uint32_t n, Mine& x) {
      const Unit& u = C.units[n % kUnits];
      x.n_here = u.n_here, x.tiles = u.tiles, x.first = u.first, x.len = u.len, x.all_see = u.all_see, x.shared = u.shared;
      x.real = row < x.n_here;
      x.seen = seen_by(A, u, query_of(A, u, row));
    };
    // the unit's queries, from their places straight into shared memory; rows that are none keep what was there
    const auto ask_query = [&](uint32_t n) {
      const Unit& u = C.units[n % kUnits];
      const int query = query_of(A, u, row);
      const Stream& S = A.stream[u.shared];
      const uint16_t* p = S.q + (u.token0 + query) * S.q_stride + static_cast<int64_t>(head_of(A, u, row, query)) * D;
      if (row < u.n_here) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(sQ + (i >> 3) * Z::kQHalf + threadIdx.x * 128 + (((i & 7) ^ (threadIdx.x & 7)) << 4)), "l"(p + i * 8) : "memory");
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
      const bool idle = warp * 32 >= x.n_here;      // a warp without rows
      const auto weigh = [&](int t, uint32_t gt, uint32_t on, bool masked) {
        const uint32_t at = t_row + kScoresAt + (gt & 1u) * kKeys;
        float p[kKeys];
        {
          uint32_t r0[32], r1[32];
          tmem_ld32_nowait(at, r0);
          tmem_ld32_nowait(at + 32, r1);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 32; ++j) p[j] = __uint_as_float(r0[j]), p[32 + j] = __uint_as_float(r1[j]);
        }
        if (masked) {
          const int left = x.seen - t * kKeys;
#pragma unroll
          for (int j = 0; j < kKeys; ++j)
            if (j >= left || !(on >> (j / 16) & 1u)) p[j] = -INFINITY;
        }
        float mx[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
        for (int j = 4; j < kKeys; j += 2) mx[(j >> 1) & 3] = max3(mx[(j >> 1) & 3], p[j], p[j + 1]);
        const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * A.scale_log2;   // (the scale is positive)
        float corr = 1.f;
        if ((top > ref + kRescale || ref == -INFINITY) && top != -INFINITY) {
          corr = exp2f(ref - top);      // 0 on the first keys
          ref = top;
        }
        const float less = ref == -INFINITY ? 0.f : -ref;
        // A score times the scale, exactly, less a reference that is rounded: off by half a step of the reference, the same for all keys.  From
        // 2^24 on that may be a doubling (and no number from 2^31 on): rare, the products are rounded as it was.
        float by = A.scale_log2;
        if (__any_sync(0xffffffffu, x.real && fabsf(less) >= 16777216.f)) {
#pragma unroll
          for (int j = 0; j < kKeys; ++j) p[j] *= A.scale_log2;
          by = 1.f;
        }
        float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int j = 0; j < kKeys; j += 2) {
          const float2 y = fma2(make_float2(p[j], p[j + 1]), make_float2(by, by), make_float2(less, less));
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
        for (int j = 0; j < 32; ++j) w[j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
        tmem_st32(at, w);
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
        if (!idle) weigh(t, gt, on, on != 15u || (t + 1) * kKeys > x.all_see);
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
      const size_t piece = static_cast<size_t>(max(0, u.place)) * kRows;
      const auto sums_of = [&](int row) -> float* { return u.place < 0 ? A.rows + place_of(A, u, row) * D : A.pieces + (piece + row) * D; };
      const auto ml_of = [&](int row) -> float2* { return u.place < 0 ? A.row_ml + place_of(A, u, row) : A.piece_ml + piece + row; };
      bool strange = false;      // a sum that is no finite number although its row's weights are numbers
      if (!idle) {
        bool found = false;
        float* const to = sums_of(x.real ? row : 0);
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
        if (x.real) *ml_of(row) = make_float2(ref, sum);
        if (found && x.real && isfinite(sum)) atomicOr(&C.redo[row >> 5], 1u << (row & 31)), strange = true;
      }
      if (rows_any(strange)) {      // rare: rows whose sums a value behind a weight of 0 may have spoiled, by hand
        for (int row = warp; row < x.n_here; row += 4) {
          if (!(C.redo[row >> 5] >> (row & 31) & 1u)) continue;
          sweep<D>(A, u, row, x.first * kKeys, (x.first + x.tiles) * kKeys, sums_of(row), ml_of(row), &C.beat, lane);
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

// The parts of a row in one of its items: its whole unit's sums, or a piece of each worker that has some of the unit's tiles.
struct Parts {
  const float* sums;       // of the first worker; those of the others follow
  const float2* ml;
  int64_t sums_step, ml_step;
  uint32_t n;
};
template <int D>
__device__ __forceinline__ Parts parts_of(const Args& A, const Plan& plan, const Record& u, int kind, int64_t token, int head, int kvh) {
  Parts x{};
  if (u.tiles == 0) return x;
  const bool few = is_few(A, u.queries);
  Line line = plan.line[0];
  if (few) line = plan.line[1];
  const int64_t flat = (token - u.token0) * A.group + head - kvh * A.group;
  uint32_t first, last;
  int row = static_cast<int>(flat);
  if (few) {
    workers_of(line, u.base + kvh * unit_cost<Few>(u.tiles) + Few::kUnitCost, u.tiles, first, last);
  } else {
    const uint32_t per_head = static_cast<uint32_t>((static_cast<int64_t>(u.queries) * A.group + kRows - 1) / kRows);
    workers_of(line, u.base + (kvh * per_head + static_cast<uint32_t>(flat / kRows)) * unit_cost<Many>(u.tiles) + Many::kUnitCost, u.tiles, first, last);
    row = static_cast<int>(flat % kRows);
  }
  x.n = last - first + 1;
  if (first == last) {
    const size_t at = (static_cast<size_t>(kind) * A.n_tokens + token) * A.hq + head;
    x.sums = A.rows + at * D, x.ml = A.row_ml + at;
    return x;
  }
  const int rows = few ? kFew : kRows;
  const int64_t at = static_cast<int64_t>(first) * 2 * rows + row;      // the first worker's is its second piece, the others' their first
  x.sums = (few ? A.few_pieces : A.pieces) + at * D;
  x.ml = (few ? A.few_piece_ml : A.piece_ml) + at;
  x.sums_step = 2 * rows * D, x.ml_step = 2 * rows;
  return x;
}

// Puts the parts of each row together: kLanes lanes of kWarps warps a row, a part's reference and sum per lane.  A block's rows have their parts
// found first, a thread each.  Grid: (sequences, parts of their rows).  Bound by its start and a chain of reads, each of which says
// where the next one is (plan and records; references and sums): 4.6 us for one sequence's 32 rows, 7.9 for 7 168 with two parts each.  (Joined in the
// first kernel, by the worker that finds all parts of a row up, it would need flags that bear a number of the launch, as those of the 4-bit cache's
// attention do: not built.  Started before the first kernel's end it takes that kernel's place.)
template <int D, int kLanes, int kWarps>
__global__ void __launch_bounds__(256, kLanes == 32 ? 3 : 4) paged_join_kernel(const __grid_constant__ Args A) {
  constexpr int kAtOnce = 8 / kWarps * (32 / kLanes), kOwn = D / kLanes, kVec = kOwn < 4 ? kOwn : 4;      // rows of a block; elements of a lane
  __shared__ Parts parts[2][kAtOnce];
  __shared__ float met[kWarps > 1 ? 8 : 1][D + 2];
  pdl_wait();
  // (asked for together: what one after the other costs here is the way to memory)
  const Plan plan = *A.plan;
  const Record own = A.records[2 * blockIdx.x], prefix = A.records[2 * blockIdx.x + 1];
  if (!plan.fine) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % kWarps, j = lane % kLanes, mine = warp / kWarps * (32 / kLanes) + lane / kLanes;
  const int n_rows = own.queries * A.hq;
  for (int r0 = blockIdx.y * kAtOnce; r0 < n_rows; r0 += gridDim.y * kAtOnce) {
    if (threadIdx.x < 2 * kAtOnce) {
      const int kind = threadIdx.x / kAtOnce, r = r0 + threadIdx.x % kAtOnce, query = r / A.hq, head = r - query * A.hq;
      Parts x{};
      if (r < n_rows) x = parts_of<D>(A, plan, kind ? prefix : own, kind, own.token0 + query, head, head / A.group);
      parts[kind][threadIdx.x % kAtOnce] = x;
    }
    __syncthreads();
    const uint32_t n_first = parts[1][mine].n, n = n_first + parts[0][mine].n, most = kLanes == 32 ? n : __reduce_max_sync(0xffffffffu, n);
    float m = -INFINITY, l = 0.f, o[kOwn] = {};
    for (uint32_t i0 = sub; i0 < most; i0 += kLanes * kWarps) {
      const uint32_t i = i0 + j * kWarps;
      const Parts& x = parts[i < n_first ? 1 : 0][mine];
      const uint32_t at = i < n_first ? i : i - n_first;
      float2 ml = make_float2(-INFINITY, 0.f);
      const float* from = A.rows;      // (of parts that are none: anything, it weighs nothing)
      if (i < n) {      // (the first worker's piece is its second)
        ml = __ldcg(x.ml + at * x.ml_step + (x.n > 1 && at == 0 ? x.ml_step / 2 : 0));
        from = x.sums + at * x.sums_step + (x.n > 1 && at == 0 ? x.sums_step / 2 : 0);
      }
      const int here = static_cast<int>(min(static_cast<uint32_t>(kLanes), (most - i0 + kWarps - 1) / kWarps));
      // So many parts under way at a time: where a warp has a row there are many of them (32 questions about one image: 25.0 us one after the
      // other, 18.9 by eight), else mostly one or two (256 questions about a video: 166 us by four, 158 by two).  The first ones are
      // asked for with their references.
      constexpr int kUnder = kLanes == 32 ? 8 : 2;
      float v[kUnder][kOwn];
      const auto fetch = [&](int k0) {
#pragma unroll
        for (int k = 0; k < kUnder; ++k) {
          if (k0 + k >= here) break;
          const float* p = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(from), k0 + k, kLanes));
#pragma unroll
          for (int c = 0; c < kOwn / kVec; ++c) {
            if constexpr (kVec == 4) {
              const float4 y = __ldcg(reinterpret_cast<const float4*>(p) + c * kLanes + j);
              v[k][4 * c] = y.x, v[k][4 * c + 1] = y.y, v[k][4 * c + 2] = y.z, v[k][4 * c + 3] = y.w;
            } else {
              const float2 y = __ldcg(reinterpret_cast<const float2*>(p) + c * kLanes + j);
              v[k][2 * c] = y.x, v[k][2 * c + 1] = y.y;
            }
          }
        }
      };
      fetch(0);
      float top = ml.x;
#pragma unroll
      for (int k = kLanes / 2; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
      top = fmaxf(top, m);
      const float f = weight_of(ml, top), old = weight_of(make_float2(m, l), top);
      float sum = ml.y * f;
#pragma unroll
      for (int k = kLanes / 2; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
      l = l * old + sum, m = top;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) o[k] = old == 0.f ? 0.f : o[k] * old;
#pragma unroll 1
      for (int k0 = 0; k0 < here; k0 += kUnder) {
        if (k0) fetch(k0);
#pragma unroll
        for (int k = 0; k < kUnder; ++k) {
          if (k0 + k >= here) break;
          const float fk = __shfl_sync(0xffffffffu, f, k0 + k, kLanes);
#pragma unroll
          for (int e = 0; e < kOwn; ++e) o[e] += fk == 0.f ? 0.f : v[k][e] * fk;
        }
      }
    }
    if constexpr (kWarps > 1) {      // the warps of a row
#pragma unroll
      for (int e = 0; e < kOwn; ++e) met[warp][lane * kOwn + e] = o[e];
      if (lane == 0) met[warp][D] = m, met[warp][D + 1] = l;
      __syncthreads();
      if (sub == 0) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) top = fmaxf(top, met[warp + k][D]);
        m = top, l = 0.f;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) o[e] = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float* y = met[warp + k];
          const float f = weight_of(make_float2(y[D], y[D + 1]), top);
          l += y[D + 1] * f;
#pragma unroll
          for (int e = 0; e < kOwn; ++e) o[e] += f == 0.f ? 0.f : y[lane * kOwn + e] * f;
        }
      }
    }
    const int r = r0 + mine, query = r / A.hq;
    if (sub == 0 && r < n_rows) {
      const size_t at = static_cast<size_t>(own.token0 + query) * A.hq + r - query * A.hq;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int c = 0; c < kOwn / kVec; ++c) {
        if constexpr (kVec == 4) {
          reinterpret_cast<uint2*>(A.out + at * D)[c * kLanes + j] = make_uint2(pack_bf16x2(o[4 * c] * inv, o[4 * c + 1] * inv), pack_bf16x2(o[4 * c + 2] * inv, o[4 * c + 3] * inv));
        } else {
          reinterpret_cast<uint32_t*>(A.out + at * D)[c * kLanes + j] = pack_bf16x2(o[2 * c] * inv, o[2 * c + 1] * inv);
        }
      }
      if (A.lse && j == 0) A.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
    }
    __syncthreads();      // (the parts and the sums have been read)
  }
}

bool off(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

int32_t check_stream(const qc_paged_stream* s, const qc_paged_attend_args* a, Stream& d) {
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

// The workspace: plan and records, references, then the sums of whole units' rows and of pieces, each part at a multiple of 256 bytes.
constexpr int kMostWorkers = 296;
struct Layout {
  size_t records, row_ml, piece_ml, few_piece_ml, rows, few_pieces, pieces, bytes;
};
Layout layout_of(const qc_paged_attend_args* a) {
  const auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
  const size_t heads = static_cast<size_t>(a->n_tokens) * a->n_q_heads * (a->n_groups ? 2 : 1);
  Layout w{};
  const int64_t most_rows = static_cast<int64_t>(a->n_groups ? a->n_tokens : std::min(a->starts_dev ? a->max_queries : 1, a->n_tokens)) * (a->n_q_heads / a->n_kv_heads);
  const size_t pieces = most_rows > kFew ? static_cast<size_t>(kMostWorkers) * 2 * kRows : 0;      // (no units of many rows: none of theirs)
  const size_t few_pieces = static_cast<size_t>(kMostWorkers) * (kBlock / 32) * 2 * kFew, row = a->head_dim * 4;
  w.records = 256;
  w.row_ml = w.records + up(static_cast<size_t>(a->n_seqs) * 2 * sizeof(Record));
  w.piece_ml = w.row_ml + up(heads * 8);
  w.few_piece_ml = w.piece_ml + up(pieces * 8);
  w.rows = w.few_piece_ml + up(few_pieces * 8);
  w.few_pieces = w.rows + up(heads * row);
  w.pieces = w.few_pieces + up(few_pieces * row);
  w.bytes = w.pieces + pieces * row;
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

template <int D, int kLanes, int kWarps>
cudaError_t launch_join(const Args& A, cudaStream_t stream) {
  constexpr int kAtOnce = 8 / kWarps * (32 / kLanes);
  const int64_t rows = static_cast<int64_t>(A.starts ? A.max_queries : 1) * A.hq;
  return launch_pdl(paged_join_kernel<D, kLanes, kWarps>, dim3(A.n_seqs, static_cast<unsigned>(std::min<int64_t>((rows + kAtOnce - 1) / kAtOnce, 65535))), dim3(256), 0, stream, A);
}

// Rows an SM up to which a block, or a warp, has one row: few rows have many parts each.  One sequence's 32 rows: 12.5 us a call by blocks, 13.8 by warps;
// 896 rows of 32 questions: 18.9 by warps, 23.2 by blocks, 24.1 by eight lanes; 7 168 rows of a video's questions: 158 by eight lanes, 163 by warps.
// At the borders: 576 rows of 300 keys 29.2 by blocks, 26.5 by warps, 640 rows 31.5 and 28.5; 3 360 rows of 100 keys 43.2 by warps and 43.3 by eight lanes
// (of groups of seven with a prefix of 2 048 keys 30.0 and 28.7), 3 840 rows 51.7 and 49.7.  So both borders could lie somewhat lower.
constexpr int kJoinBlock = 4, kJoinWarp = 24;
template <int D>
cudaError_t launch(const Args& A, int device, cudaStream_t stream) {
  constexpr int kBytes = Shape<D>::kTiles + sizeof(Control);
  cudaError_t e;
  int sms = 0;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return e;
  static std::atomic<bool> configured[64] = {};     // per device: the kernel may take that much
  if (device >= 64 || !configured[device].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(paged_attend_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    if (device < 64) configured[device].store(true, std::memory_order_relaxed);
  }
  if ((e = launch_pdl(paged_attend_kernel<D>, dim3(std::min(2 * sms, kMostWorkers)), dim3(kBlock), kBytes, stream, A)) != cudaSuccess) return e;
  const int64_t rows = static_cast<int64_t>(A.n_tokens) * A.hq;
  return rows <= kJoinBlock * sms ? launch_join<D, 32, 8>(A, stream) : rows <= kJoinWarp * sms ? launch_join<D, 32, 1>(A, stream) : launch_join<D, 8, 1>(A, stream);
}

// Whether `bytes` at `p`, which the call writes, lie over anything that it reads.
bool over_inputs(const qc_paged_attend_args* a, const void* p, uint64_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p), row = static_cast<uint64_t>(a->n_q_heads) * a->head_dim * 2, n = a->n_tokens;
  const auto over = [&](const void* x, uint64_t size) {
    const uint64_t y = reinterpret_cast<uint64_t>(x);
    return y && y < at + bytes && at < y + size;
  };
  for (const qc_paged_stream* s : {&a->own, &a->shared}) {
    const uint64_t pool = static_cast<uint64_t>(s->n_pages) * a->page_size * a->n_kv_heads * a->head_dim * 2, rows = s->rows;
    if (over(s->q_dev, static_cast<uint64_t>(s->q_stride) * 2 * (n - 1) + row) || over(s->k_pool_dev, pool) || over(s->v_pool_dev, pool) ||
        over(s->pages_dev, rows * s->max_pages * 4) || over(s->lens_dev, rows * 4))
      return true;
  }
  const uint64_t seqs = a->n_seqs, groups = a->n_groups;
  return over(a->seq_ids_dev, seqs * 4) || over(a->starts_dev, seqs * 4 + 4) || over(a->groups_dev, groups * 4 + 4) || over(a->shared_ids_dev, groups * 4) ||
         over(a->status_dev, 4);
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
  Args A{};
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
  const uint64_t rows = static_cast<uint64_t>(args->n_tokens) * args->n_q_heads, out_bytes = rows * args->head_dim * 2;
  if (over_inputs(args, args->out_dev, out_bytes)) return QC_ERR_INVALID_ARG;
  if (args->lse_out_dev) {
    const uint64_t out = reinterpret_cast<uint64_t>(args->out_dev), lse = reinterpret_cast<uint64_t>(args->lse_out_dev);
    if (over_inputs(args, args->lse_out_dev, rows * 4) || (out < lse + rows * 4 && lse < out + out_bytes)) return QC_ERR_INVALID_ARG;
  }
  A.ids = args->seq_ids_dev, A.starts = args->starts_dev, A.groups = args->groups_dev, A.shared_ids = args->shared_ids_dev;
  A.out = static_cast<uint16_t*>(args->out_dev), A.lse = args->lse_out_dev, A.status = args->status_dev;
  uint8_t* const work = static_cast<uint8_t*>(args->workspace_dev);
  const Layout w = layout_of(args);
  A.plan = reinterpret_cast<Plan*>(work), A.records = reinterpret_cast<Record*>(work + w.records), A.rows = reinterpret_cast<float*>(work + w.rows);
  A.row_ml = reinterpret_cast<float2*>(work + w.row_ml), A.pieces = reinterpret_cast<float*>(work + w.pieces);
  A.few_pieces = reinterpret_cast<float*>(work + w.few_pieces);
  A.piece_ml = reinterpret_cast<float2*>(work + w.piece_ml), A.few_piece_ml = reinterpret_cast<float2*>(work + w.few_piece_ml);
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
