// Rows of K and V in 4 bits: quantising append at slots, and rows read back.
//
// A row x[0..D) (one token, one head) is held as lo = min x (bf16), r = bf16(15 / (max x - lo)) and
// codes c = rint((x - lo) * r), and stands for lo + c / r.  With the reciprocal of the step stored,
// quantising is a subtraction and a product per element, both of few bits, so that the nearest code is
// found without a division; a reader divides once per row.  (15 * r's rounding of 2^-9 moves the
// largest element by at most 0.03 steps, so codes end at 15 by themselves.)
//
// Both kernels are bound by their bytes: 2 D in and D / 2 + 4 out per row, or the other way.  Eight
// lanes take a row, so a warp holds four rows of a head: a row's smallest and largest come from
// packed bf16 operations and three exchanges, the largest together with the negated smallest.
// The layout inside a page (see qc.h) is what the matrix products of the attention read: a K row's
// codes are four runs of 16 bytes, while a word of V holds two elements of four adjacent tokens.  A
// warp therefore takes four tokens that fill such words and exchanges their bytes first (stored
// byte by byte, each word costs four partial writes).

#include "../../include/qc.h"
#include "qc_device.cuh"
#include "qc_quant.cuh"
#include "qc_quant.h"

namespace qc {
namespace {

constexpr int kRowWarps = 8;       // warps of a block, one head each
constexpr float kLeastSpan = 7.8886090522101181e-31f;   // 2^-100

struct RowArgs {
  const int32_t* slots;
  const uint16_t* k;       // append: rows in; read: null
  const uint16_t* v;
  int64_t k_stride, v_stride;   // elements from a token's rows to the next one's
  uint8_t* k_pool;
  uint8_t* v_pool;
  uint16_t* k_out;         // read: rows out
  uint16_t* v_out;
  int32_t n_tokens, hkv, page, n_pages, window;
};

__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t min_nan2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// E / 2 words of bf16 pairs of this lane's part of a row -> its codes, 8 in a word, and the row's parameters.
// Every lane of a row's eight gets the same parameters.
template <int E>
__device__ __forceinline__ void quantise_row(const uint32_t (&x)[E / 2], uint32_t (&codes)[E / 8], uint32_t& params) {
  uint32_t big = x[0], small = x[0];
#pragma unroll
  for (int i = 1; i < E / 2; ++i) big = max_nan2(big, x[i]), small = min_nan2(small, x[i]);
  big = max_nan2(big, big >> 16 | big << 16);
  small = min_nan2(small, small >> 16 | small << 16);
  // low half: the largest; high half: the smallest, negated, so that one maximum serves both
  uint32_t both = (big & 0xffffu) | ((small & 0xffff0000u) ^ 0x80000000u);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) both = max_nan2(both, __shfl_xor_sync(0xffffffffu, both, o));
  const float hi = __uint_as_float(both << 16), lo = __uint_as_float((both & 0xffff0000u) ^ 0x80000000u);
  const float span = hi - lo;
  const bool fine = span < INFINITY;   // false for NaN as well: the row stands for NaN
  const uint32_t r_bits = fine && span >= kLeastSpan ? f32_to_bf16_rne(__fdiv_rn(15.f, span)) : 0u;
  const float r = __uint_as_float(r_bits << 16);
  params = (r_bits << 16) | (fine ? __float_as_uint(lo) >> 16 : 0x7fc0u);
  // rint by adding 1.5 * 2^23: the sum's low bits are the code.  Eight sums are put together as
  // acc * 16 + sum; what the constant leaves there modulo 2^32 is taken off at the end.
  constexpr float kMagic = 12582912.f;
  constexpr uint32_t kRest = 0x4B400000u + 0xB4000000u + 0x40000000u;
#pragma unroll
  for (int w = 0; w < E / 8; ++w) {
    uint32_t acc = 0;
#pragma unroll
    for (int j = 7; j >= 0; --j) {
      const uint32_t pair = x[w * 4 + j / 2];
      const float f = __uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16);
      acc = acc * 16u + __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(f, lo), r), kMagic));
    }
    codes[w] = fine ? acc - kRest : 0u;
  }
}

// The bytes of four lanes eight apart, exchanged: lane j (of lane / 8) gets byte j of each, in order.
__device__ __forceinline__ uint32_t exchange_bytes(uint32_t x, int j) {
  const uint32_t p = __shfl_xor_sync(0xffffffffu, x, 8);
  const uint32_t r = __byte_perm(x, p, j & 1 ? 0x3715 : 0x6240);
  const uint32_t q = __shfl_xor_sync(0xffffffffu, r, 16);
  return __byte_perm(r, q, j & 2 ? 0x3276 : 0x5410);
}

template <int D>
__device__ __forceinline__ void load_part(const uint16_t* row, int part, bool on, uint32_t (&x)[D / 16]) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint4 a = on ? __ldg(reinterpret_cast<const uint4*>(row + part * (D / 8)) + i) : make_uint4(0, 0, 0, 0);
    x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = a.z, x[4 * i + 3] = a.w;
  }
}

// Grid: (windows of T.window tokens, groups of kRowWarps heads).  A warp takes the tokens of its window that
// begin a group: up to four tokens with adjacent slots that share words of V.
template <int D>
__global__ void __launch_bounds__(kRowWarps * 32) quant_append_kernel(const RowArgs T) {
  constexpr int E = D / 8;    // elements of a row per lane
  const int lane = threadIdx.x & 31, part = lane & 7, mine = lane >> 3;
  const int head = blockIdx.y * kRowWarps + (threadIdx.x >> 5);
  if (head >= T.hkv) return;
  const int32_t n_slots = T.n_pages * T.page;
  const int begin = blockIdx.x * T.window;
  // lane l looks at token begin - 4 + l: three before the window say whether its first tokens belong to a group begun there
  const int tok = begin - 4 + lane;
  const int32_t slot = tok >= 0 && tok < T.n_tokens ? T.slots[tok] : -1;
  const bool good = slot >= 0 && slot < n_slots;
  const int32_t left = __shfl_up_sync(0xffffffffu, slot, 1);
  // follows: shares its words with the token before it
  const bool follows = good && lane > 0 && (slot & 3) != 0 && left == slot - 1;
  const uint32_t heads_of_groups = __ballot_sync(0xffffffffu, good && !follows);
  const uint32_t followers = __ballot_sync(0xffffffffu, follows);
  uint32_t todo = heads_of_groups & (((1u << T.window) - 1u) << 4);
  const int64_t page_bytes = quant_page_bytes(T.hkv, D, T.page);
  while (todo) {
    const int at = __ffs(todo) - 1;                       // lane that looks at the group's first token
    todo &= todo - 1;
    const int count = __ffs(~(followers >> (at + 1)));    // 1 + the followers behind it (at most 3: a fourth has slot % 4 == 0)
    const int32_t slot0 = __shfl_sync(0xffffffffu, slot, at);
    const int32_t first = begin - 4 + at, s = slot0 + mine;
    const bool on = mine < count;
    const int32_t in_page = s % T.page;
    const size_t base = static_cast<size_t>(s / T.page) * page_bytes;
    const size_t block = base + (static_cast<size_t>(head) * T.page + (in_page & ~15)) * (D / 2);
    const size_t words = base + static_cast<size_t>(T.hkv) * T.page * (D / 2) + (static_cast<size_t>(head) * T.page + in_page) * 4;
    uint32_t xk[D / 16], xv[D / 16], ck[E / 8], cv[E / 8], pk = 0, pv = 0;
    const size_t token = static_cast<size_t>(first + mine);
    if (T.k) load_part<D>(T.k + token * T.k_stride + static_cast<size_t>(head) * D, part, on, xk);
    if (T.v) load_part<D>(T.v + token * T.v_stride + static_cast<size_t>(head) * D, part, on, xv);
    if (T.k) {
      quantise_row<E>(xk, ck, pk);
      if (on) {
        uint8_t* dst = T.k_pool + block + k_code_offset<D>(in_page & 15, part * E);
        if constexpr (D == 128) *reinterpret_cast<uint2*>(dst) = make_uint2(ck[0], ck[1]);
        else *reinterpret_cast<uint32_t*>(dst) = ck[0];
        if (part == 0) *reinterpret_cast<uint32_t*>(T.k_pool + words) = pk;
      }
    }
    if (T.v) {
      quantise_row<E>(xv, cv, pv);
      const int32_t tg = (in_page & 15) >> 2;             // the same for the whole group
      if (count == 4) {
#pragma unroll
        for (int i = 0; i < E / 8; ++i) {
          const uint32_t word = exchange_bytes(cv[i], mine);
          *reinterpret_cast<uint32_t*>(T.v_pool + block + i * 512 + (part * 4 + tg) * 16 + mine * 4) = word;
        }
      } else if (on) {
#pragma unroll
        for (int i = 0; i < E / 8; ++i)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            T.v_pool[block + i * 512 + (part * 4 + tg) * 16 + b * 4 + (in_page & 3)] = static_cast<uint8_t>(cv[i] >> (8 * b));
      }
      if (on && part == 0) *reinterpret_cast<uint32_t*>(T.v_pool + words) = pv;
    }
  }
}

// codes of 8 elements and a row's parameters -> 8 bf16 values
__device__ __forceinline__ uint4 values_of(uint32_t codes, uint32_t params) {
  const float lo = __uint_as_float(params << 16), step = quant_step(params);
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = fmaf(static_cast<float>((codes >> (4 * j)) & 15u), step, lo);
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// Grid: (groups of four tokens in the call's order, groups of kRowWarps heads).
template <int D>
__global__ void __launch_bounds__(kRowWarps * 32) quant_read_kernel(const RowArgs T) {
  constexpr int E = D / 8;
  const int lane = threadIdx.x & 31, part = lane & 7;
  const int head = blockIdx.y * kRowWarps + (threadIdx.x >> 5);
  const int token = blockIdx.x * 4 + (lane >> 3);
  if (head >= T.hkv || token >= T.n_tokens) return;
  const int32_t s = T.slots[token];
  if (s < 0 || s >= T.n_pages * T.page) return;          // its rows stay as they are
  const int32_t in_page = s % T.page, i16 = in_page & 15;
  const size_t base = static_cast<size_t>(s / T.page) * quant_page_bytes(T.hkv, D, T.page);
  const size_t block = base + (static_cast<size_t>(head) * T.page + (in_page & ~15)) * (D / 2);
  const size_t words = base + static_cast<size_t>(T.hkv) * T.page * (D / 2) + (static_cast<size_t>(head) * T.page + in_page) * 4;
  const size_t out = (static_cast<size_t>(token) * T.hkv + head) * D + part * E;
  if (T.k_out) {
    const uint8_t* src = T.k_pool + block + k_code_offset<D>(i16, part * E);
    const uint32_t params = *reinterpret_cast<const uint32_t*>(T.k_pool + words);
#pragma unroll
    for (int i = 0; i < E / 8; ++i)
      reinterpret_cast<uint4*>(T.k_out + out)[i] = values_of(reinterpret_cast<const uint32_t*>(src)[i], params);
  }
  if (T.v_out) {
    const uint32_t params = *reinterpret_cast<const uint32_t*>(T.v_pool + words);
    const uint32_t pick = (i16 & 3) | ((i16 & 3) + 4) << 4;   // this token's byte of two words
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(T.v_pool + block + i * 512 + (part * 4 + (i16 >> 2)) * 16);
      const uint32_t codes = __byte_perm(__byte_perm(w.x, w.y, pick), __byte_perm(w.z, w.w, pick), 0x5410);
      reinterpret_cast<uint4*>(T.v_out + out)[i] = values_of(codes, params);
    }
  }
}

int32_t check_shape(const qc_quant_shape* s) {
  if (!s) return QC_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (s->page_size != 16 && s->page_size != 32 && s->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (s->n_kv_heads < 1 || s->n_pages < 1) return QC_ERR_INVALID_ARG;
  if (s->n_kv_heads > QC_QUANT_MAX_HEADS || static_cast<int64_t>(s->n_pages) * s->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  return QC_OK;
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

}  // namespace
}  // namespace qc

using namespace qc;

extern "C" int32_t qc_quant_pool_bytes(const qc_quant_shape* shape, size_t* bytes) {
  if (!bytes) return QC_ERR_INVALID_ARG;
  if (const int32_t bad = check_shape(shape)) return bad;
  *bytes = static_cast<size_t>(shape->n_pages) * quant_page_bytes(shape->n_kv_heads, shape->head_dim, shape->page_size);
  return QC_OK;
}

extern "C" int32_t qc_quant_append(int32_t device, void* cuda_stream, const qc_quant_shape* shape, int32_t n_tokens, const int32_t* slots_dev,
                                   const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride, void* k_pool_dev,
                                   void* v_pool_dev) {
  if (const int32_t bad = check_shape(shape)) return bad;
  if (n_tokens < 0 || (!k_dev) != (!k_pool_dev) || (!v_dev) != (!v_pool_dev) || (!k_dev && !v_dev)) return QC_ERR_INVALID_ARG;
  if (n_tokens == 0) return QC_OK;
  if (!slots_dev || (reinterpret_cast<uintptr_t>(slots_dev) & 3)) return QC_ERR_INVALID_ARG;
  if (off16(k_dev) || off16(v_dev) || off16(k_pool_dev) || off16(v_pool_dev)) return QC_ERR_INVALID_ARG;
  if ((k_dev && (k_stride < 0 || k_stride % 8)) || (v_dev && (v_stride < 0 || v_stride % 8))) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  RowArgs a{};
  a.slots = slots_dev;
  a.k = static_cast<const uint16_t*>(k_dev), a.v = static_cast<const uint16_t*>(v_dev);
  a.k_stride = k_stride, a.v_stride = v_stride;
  a.k_pool = static_cast<uint8_t*>(k_pool_dev), a.v_pool = static_cast<uint8_t*>(v_pool_dev);
  a.n_tokens = n_tokens, a.hkv = shape->n_kv_heads, a.page = shape->page_size, a.n_pages = shape->n_pages;
  const int y = (a.hkv + kRowWarps - 1) / kRowWarps;
  // a batch's single tokens lie in pages of their own: one token per warp, so that none waits for another
  a.window = n_tokens <= 512 ? 1 : 4;
  const dim3 grid((n_tokens + a.window - 1) / a.window, y);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (shape->head_dim == 128) quant_append_kernel<128><<<grid, kRowWarps * 32, 0, stream>>>(a);
  else quant_append_kernel<64><<<grid, kRowWarps * 32, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? QC_OK : QC_ERR_CUDA;
}

extern "C" int32_t qc_quant_read(int32_t device, void* cuda_stream, const qc_quant_shape* shape, int32_t n_tokens, const int32_t* slots_dev,
                                 const void* k_pool_dev, const void* v_pool_dev, void* k_out_dev, void* v_out_dev) {
  if (const int32_t bad = check_shape(shape)) return bad;
  if (n_tokens < 0 || (!k_out_dev) != (!k_pool_dev) || (!v_out_dev) != (!v_pool_dev) || (!k_out_dev && !v_out_dev)) return QC_ERR_INVALID_ARG;
  if (n_tokens == 0) return QC_OK;
  if (!slots_dev || (reinterpret_cast<uintptr_t>(slots_dev) & 3)) return QC_ERR_INVALID_ARG;
  if (off16(k_pool_dev) || off16(v_pool_dev) || off16(k_out_dev) || off16(v_out_dev)) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  RowArgs a{};
  a.slots = slots_dev;
  a.k_pool = static_cast<uint8_t*>(const_cast<void*>(k_pool_dev)), a.v_pool = static_cast<uint8_t*>(const_cast<void*>(v_pool_dev));
  a.k_out = static_cast<uint16_t*>(k_out_dev), a.v_out = static_cast<uint16_t*>(v_out_dev);
  a.n_tokens = n_tokens, a.hkv = shape->n_kv_heads, a.page = shape->page_size, a.n_pages = shape->n_pages;
  const dim3 grid((n_tokens + 3) / 4, (a.hkv + kRowWarps - 1) / kRowWarps);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (shape->head_dim == 128) quant_read_kernel<128><<<grid, kRowWarps * 32, 0, stream>>>(a);
  else quant_read_kernel<64><<<grid, kRowWarps * 32, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? QC_OK : QC_ERR_CUDA;
}
