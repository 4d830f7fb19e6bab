// Rows of K and V in 4 bits: quantising append at slots, and rows read back.
//
// A row x[0..D) (one token, one head) is held as lo = min x (bf16), r = bf16(15 / (max x - lo)) and
// codes c = rint((x - lo) * r), and stands for lo + c / r.  With the reciprocal of the step stored,
// quantising is a subtraction and a product per element, both of few bits, so that the nearest code is
// found without a division; a reader divides once per row.  (15 * r's rounding of 2^-9 moves the
// largest element by at most 0.03 steps, so codes end at 15 by themselves.)
//
// Both kernels are bound by their bytes (2 D in and D / 2 + 4 out per row, or the other way) only while they spend few
// instructions on an element.  A warp takes a group: up to 16 tokens of one head whose slots follow one another inside a
// block of the page.  Its lanes hold what the attention's lanes read (see qc_quant.cuh), K a quarter of two
// tokens' rows and V an eighth of four tokens', so codes go to and from a page as whole vectors in lane order, and
// V's words, which hold four tokens, are put together in registers.  (With four tokens a warp and the exchanges that takes,
// 10 813 tokens of 32 heads took 111 us to store and read back; 76.7 so, of which 61 are their bytes at the copy rate and 7
// the codes' second trip.  A step of 32 tokens is two launches' time, 3.6 us.)

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
  int64_t page_bytes, code_bytes;
  int32_t n_tokens, hkv, page_shift, n_pages, window;
  bool has_k;              // blocks of z = 0 take K (and those of z = 1 V), else all take V
  bool wide;               // read: rows out begin at multiples of 32 bytes
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

// The tokens that a warp takes together: `count` tokens from `token` on, in the block of slots that begins at slot `block`, from its
// place `from` on.
struct Group {
  int32_t token, block, from, count;
};

// Calls fn for each group that begins in the warp's window of tokens.
template <typename Fn>
__device__ __forceinline__ void for_groups(const RowArgs& T, int lane, Fn fn) {
  pdl_wait();
  const int32_t n_slots = T.n_pages << T.page_shift;
  const int begin = blockIdx.x * T.window;
  // lanes look at the tokens from begin - 1 on, then at the 16 behind those
  const int tok = begin - 1 + lane;
  const auto slot_at = [&](int i) {
    const int32_t s = i >= 0 && i < T.n_tokens ? T.slots[i] : -1;
    return s < n_slots ? s : -1;
  };
  const int32_t slot = slot_at(tok);
  const int32_t left = __shfl_up_sync(0xffffffffu, slot, 1);
  const bool begins = slot >= 0 && (lane == 0 || (slot & 15) == 0 || left != slot - 1);
  const bool follows = slot >= 0 && !begins;
  uint32_t todo = __ballot_sync(0xffffffffu, begins);
  const uint32_t followers = __ballot_sync(0xffffffffu, follows);
  todo &= ((1u << T.window) - 1u) << 1;
  while (todo) {
    const int at = __ffs(todo) - 1;
    todo &= todo - 1;
    Group G;
    const int32_t slot0 = __shfl_sync(0xffffffffu, slot, at);
    G.token = begin - 1 + at, G.from = slot0 & 15, G.block = slot0 - G.from;
    G.count = __ffs(~(followers >> at >> 1));     // 1 and those that follow: 15 at most, and 17 lanes of a window and 15 more are looked at
    fn(G);
  }
}

// E bf16 elements (in pairs) -> the row's largest, and its smallest negated, over the lanes that differ in kLanes.
template <int E, int kFirst, int kLast>
__device__ __forceinline__ uint32_t ends_of(const uint32_t (&x)[E / 2]) {
  uint32_t big = x[0], small = x[0];
#pragma unroll
  for (int i = 1; i < E / 2; ++i) big = max_nan2(big, x[i]), small = min_nan2(small, x[i]);
  big = max_nan2(big, __byte_perm(big, 0, 0x1032));
  small = min_nan2(small, __byte_perm(small, 0, 0x1032));
  uint32_t both = __byte_perm(big, small ^ 0x80008000u, 0x7610);
#pragma unroll
  for (int o = kFirst; o <= kLast; o <<= 1) both = max_nan2(both, __shfl_xor_sync(0xffffffffu, both, o));
  return both;
}

struct Scale {
  float lo, r;
  uint32_t params;
  bool fine;      // false: the row stands for NaN
};
__device__ __forceinline__ Scale scale_of(uint32_t ends) {
  Scale s;
  const float hi = __uint_as_float(ends << 16);
  s.lo = __uint_as_float((ends & 0xffff0000u) ^ 0x80000000u);
  const float span = hi - s.lo;
  s.fine = span < INFINITY;
  const uint32_t r_bits = s.fine && span >= kLeastSpan ? pack_bf16x2(__fdiv_rn(15.f, span), 0.f) & 0xffffu : 0u;
  s.r = __uint_as_float(r_bits << 16);
  s.params = (r_bits << 16) | (s.fine ? __float_as_uint(s.lo) >> 16 : 0x7fc0u);
  return s;
}

// 8 elements -> 8 codes.  rint by adding 1.5 * 2^23: the sum's low bits are the code.  The sums are put together as
// acc * 16 + sum; what the constant leaves there modulo 2^32 is taken off at the end.
__device__ __forceinline__ uint32_t codes_of(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, const Scale& s) {
  constexpr float kMagic = 12582912.f;
  constexpr uint32_t kRest = 0x4B400000u + 0xB4000000u + 0x40000000u;
  const uint32_t x[4] = {x0, x1, x2, x3};
  const float2 less = make_float2(-s.lo, -s.lo), r = make_float2(s.r, s.r), magic = make_float2(kMagic, kMagic);
  uint32_t acc = 0;
#pragma unroll
  for (int j = 3; j >= 0; --j) {
    const float2 f = fma2(add2(bf16x2_to_f32(x[j]), less), r, magic);
    acc = (acc * 16u + __float_as_uint(f.y)) * 16u + __float_as_uint(f.x);
  }
  return s.fine ? acc - kRest : 0u;
}

template <int N>
__device__ __forceinline__ void load_words(const uint16_t* p, bool on, uint32_t (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint4 a = on ? __ldg(reinterpret_cast<const uint4*>(p) + i) : make_uint4(0, 0, 0, 0);
    x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = a.z, x[4 * i + 3] = a.w;
  }
}

// Four words of four bytes each, the other way round.
__device__ __forceinline__ uint4 turn(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab0 = __byte_perm(a, b, 0x5140), ab1 = __byte_perm(a, b, 0x7362), cd0 = __byte_perm(c, d, 0x5140), cd1 = __byte_perm(c, d, 0x7362);
  return make_uint4(__byte_perm(ab0, cd0, 0x5410), __byte_perm(ab0, cd0, 0x7632), __byte_perm(ab1, cd1, 0x5410), __byte_perm(ab1, cd1, 0x7632));
}

// Where a block's codes of a head, and its parameters, begin in a pool.
template <int D>
__device__ __forceinline__ void places_of(const RowArgs& T, int32_t block, int head, size_t& codes, size_t& words) {
  const int32_t page = block >> T.page_shift, in_page = block & ((1 << T.page_shift) - 1);
  const size_t base = static_cast<size_t>(page) * T.page_bytes;
  codes = base + (static_cast<size_t>(head) * (1 << T.page_shift) + in_page) * (D / 2);
  words = base + T.code_bytes + (static_cast<size_t>(head) * (1 << T.page_shift) + in_page) * 4;
}

// Grid: (windows of T.window tokens, groups of kRowWarps heads, K and V: tensors in blocks of their own, or one warp would hold
// both's rows in registers and too few would be on their way).  Four blocks an SM here and six in the read: 76.7 us for those
// 10 813 tokens, 80.8 with the registers that the compiler takes by itself.
template <int D>
__global__ void __launch_bounds__(kRowWarps * 32, 4) quant_append_kernel(const __grid_constant__ RowArgs T) {
  constexpr int kK = D / 4, kV = D / 8;      // elements of a row per lane
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int head = blockIdx.y * kRowWarps + (threadIdx.x >> 5);
  const bool is_k = blockIdx.z == 0 && T.has_k;
  if (head >= T.hkv) return;
  for_groups(T, lane, [&](const Group& G) {
    size_t codes, words;
    places_of<D>(T, G.block, head, codes, words);
    const auto has = [&](int i) { return i >= G.from && i < G.from + G.count; };
    const auto token = [&](int i) { return static_cast<int64_t>(G.token + i - G.from); };
    if (is_k) {
      uint32_t xk[2][kK / 2];
#pragma unroll
      for (int i = 0; i < 2; ++i) load_words(T.k + token(2 * g + i) * T.k_stride + head * D + t * kK, has(2 * g + i), xk[i]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const Scale s = scale_of(ends_of<kK, 1, 2>(xk[i]));
        uint32_t c[kK / 8];
#pragma unroll
        for (int w = 0; w < kK / 8; ++w) c[w] = codes_of(xk[i][4 * w], xk[i][4 * w + 1], xk[i][4 * w + 2], xk[i][4 * w + 3], s);
        if (!has(2 * g + i)) continue;
        uint8_t* dst = T.k_pool + codes + lane * 16;
        if constexpr (D == 128) *reinterpret_cast<uint4*>(dst + i * 512) = make_uint4(c[0], c[1], c[2], c[3]);
        else *reinterpret_cast<uint2*>(dst + i * 8) = make_uint2(c[0], c[1]);
        if (t == 0) *reinterpret_cast<uint32_t*>(T.k_pool + words + (2 * g + i) * 4) = s.params;
      }
    }
    if (!is_k) {
      uint32_t xv[4][kV / 2], c[kV / 8][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) load_words(T.v + token(4 * t + i) * T.v_stride + head * D + g * kV, has(4 * t + i), xv[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Scale s = scale_of(ends_of<kV, 4, 16>(xv[i]));
#pragma unroll
        for (int w = 0; w < kV / 8; ++w) c[w][i] = codes_of(xv[i][4 * w], xv[i][4 * w + 1], xv[i][4 * w + 2], xv[i][4 * w + 3], s);
        if (g == 0 && has(4 * t + i)) *reinterpret_cast<uint32_t*>(T.v_pool + words + (4 * t + i) * 4) = s.params;
      }
      uint8_t* dst = T.v_pool + codes + lane * 16;
      if (has(4 * t) && has(4 * t + 3)) {
#pragma unroll
        for (int w = 0; w < kV / 8; ++w) *reinterpret_cast<uint4*>(dst + w * 512) = turn(c[w][0], c[w][1], c[w][2], c[w][3]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (has(4 * t + i))
#pragma unroll
            for (int w = 0; w < kV / 8; ++w)
#pragma unroll
              for (int b = 0; b < 4; ++b) dst[w * 512 + b * 4 + i] = static_cast<uint8_t>(c[w][i] >> (8 * b));
      }
    }
  });
}

// 8 codes of a row -> 8 bf16 values.
__device__ __forceinline__ uint4 values_of(uint32_t codes, float lo, float step) {
  const float2 l = make_float2(lo, lo), s = make_float2(step, step), less = make_float2(-8388608.f, -8388608.f);
  uint32_t out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 c = make_float2(__uint_as_float((codes >> (8 * j) & 15u) | 0x4b000000u), __uint_as_float((codes >> (8 * j + 4) & 15u) | 0x4b000000u));
    const float2 f = fma2(add2(c, less), s, l);
    out[j] = pack_bf16x2(f.x, f.y);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// 32 bytes of a row: in one store where the rows begin at multiples of 32 (two stores of half a sector each cost twice the writes).
__device__ __forceinline__ void store_32(uint16_t* p, const uint4& a, const uint4& b, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = a;
    reinterpret_cast<uint4*>(p)[1] = b;
  }
}

// Grid as above.
template <int D>
__global__ void __launch_bounds__(kRowWarps * 32, 6) quant_read_kernel(const __grid_constant__ RowArgs T) {
  constexpr int kK = D / 4, kV = D / 8;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int head = blockIdx.y * kRowWarps + (threadIdx.x >> 5);
  const bool is_k = blockIdx.z == 0 && T.has_k;
  if (head >= T.hkv) return;
  for_groups(T, lane, [&](const Group& G) {
    size_t codes, words;
    places_of<D>(T, G.block, head, codes, words);
    const auto has = [&](int i) { return i >= G.from && i < G.from + G.count; };
    const auto row = [&](int i) { return (static_cast<int64_t>(G.token + i - G.from) * T.hkv + head) * D; };
    if (is_k) {
      uint32_t c[2][kK / 8];
      if constexpr (D == 128) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 w = __ldg(reinterpret_cast<const uint4*>(T.k_pool + codes + i * 512) + lane);
          c[i][0] = w.x, c[i][1] = w.y, c[i][2] = w.z, c[i][3] = w.w;
        }
      } else {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(T.k_pool + codes) + lane);
        c[0][0] = w.x, c[0][1] = w.y, c[1][0] = w.z, c[1][1] = w.w;
      }
      const uint2 p = __ldg(reinterpret_cast<const uint2*>(T.k_pool + words) + g);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!has(2 * g + i)) continue;
        const uint32_t params = i ? p.y : p.x;
        const float lo = __uint_as_float(params << 16), step = quant_step(params);
        uint16_t* dst = T.k_out + row(2 * g + i) + t * kK;
#pragma unroll
        for (int w = 0; w < kK / 8; w += 2) store_32(dst + w * 8, values_of(c[i][w], lo, step), values_of(c[i][w + 1], lo, step), T.wide);
      }
    }
    if (!is_k) {
      uint4 w[kV / 8];
#pragma unroll
      for (int i = 0; i < kV / 8; ++i) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(T.v_pool + codes + i * 512) + lane);
        w[i] = turn(x.x, x.y, x.z, x.w);      // a token's codes in each
      }
      const uint4 p = __ldg(reinterpret_cast<const uint4*>(T.v_pool + words) + t);
      const uint32_t params[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!has(4 * t + i)) continue;
        const float lo = __uint_as_float(params[i] << 16), step = quant_step(params[i]);
        const auto code = [&](const uint4& x) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; };
        uint16_t* dst = T.v_out + row(4 * t + i) + g * kV;
        if constexpr (D == 128) store_32(dst, values_of(code(w[0]), lo, step), values_of(code(w[1]), lo, step), T.wide);
        else *reinterpret_cast<uint4*>(dst) = values_of(code(w[0]), lo, step);
      }
    }
  });
}

int32_t check_shape(const qc_quant_shape* s) {
  if (!s) return QC_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return QC_ERR_UNSUPPORTED;
  if (s->page_size != 16 && s->page_size != 32 && s->page_size != 64) return QC_ERR_UNSUPPORTED;
  if (s->n_kv_heads < 1 || s->n_pages < 1) return QC_ERR_INVALID_ARG;
  if (s->n_kv_heads > QC_QUANT_MAX_HEADS || static_cast<int64_t>(s->n_pages) * s->page_size > INT32_MAX) return QC_ERR_UNSUPPORTED;
  return QC_OK;
}

void place(RowArgs& a, const qc_quant_shape* s, int32_t n_tokens) {
  a.n_tokens = n_tokens, a.hkv = s->n_kv_heads, a.n_pages = s->n_pages;
  a.page_shift = s->page_size == 16 ? 4 : s->page_size == 32 ? 5 : 6;
  a.page_bytes = quant_page_bytes(a.hkv, s->head_dim, s->page_size), a.code_bytes = static_cast<int64_t>(a.hkv) * s->page_size * (s->head_dim / 2);
  // a batch's single tokens lie in blocks of their own: one token per warp, so that none waits for another (32 tokens: 3.6 us
  // against 8.0)
  a.window = n_tokens <= 512 ? 1 : 16;
}

dim3 grid_of(const RowArgs& a, bool both) { return dim3((a.n_tokens + a.window - 1) / a.window, (a.hkv + kRowWarps - 1) / kRowWarps, both ? 2 : 1); }

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
  if (n_tokens > QC_QUANT_MAX_TOKENS) return QC_ERR_UNSUPPORTED;
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
  place(a, shape, n_tokens);
  a.has_k = k_dev != nullptr;
  const dim3 grid = grid_of(a, k_dev && v_dev);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = launch_pdl(shape->head_dim == 128 ? quant_append_kernel<128> : quant_append_kernel<64>, grid, dim3(kRowWarps * 32), 0, stream, a);
  return status_of(e);
}

extern "C" int32_t qc_quant_read(int32_t device, void* cuda_stream, const qc_quant_shape* shape, int32_t n_tokens, const int32_t* slots_dev,
                                 const void* k_pool_dev, const void* v_pool_dev, void* k_out_dev, void* v_out_dev) {
  if (const int32_t bad = check_shape(shape)) return bad;
  if (n_tokens < 0 || (!k_out_dev) != (!k_pool_dev) || (!v_out_dev) != (!v_pool_dev) || (!k_out_dev && !v_out_dev)) return QC_ERR_INVALID_ARG;
  if (n_tokens > QC_QUANT_MAX_TOKENS) return QC_ERR_UNSUPPORTED;
  if (n_tokens == 0) return QC_OK;
  if (!slots_dev || (reinterpret_cast<uintptr_t>(slots_dev) & 3)) return QC_ERR_INVALID_ARG;
  if (off16(k_pool_dev) || off16(v_pool_dev) || off16(k_out_dev) || off16(v_out_dev)) return QC_ERR_INVALID_ARG;
  DeviceGuard guard(device);
  if (!guard.ok()) return QC_ERR_CUDA;
  RowArgs a{};
  a.slots = slots_dev;
  a.k_pool = static_cast<uint8_t*>(const_cast<void*>(k_pool_dev)), a.v_pool = static_cast<uint8_t*>(const_cast<void*>(v_pool_dev));
  a.k_out = static_cast<uint16_t*>(k_out_dev), a.v_out = static_cast<uint16_t*>(v_out_dev);
  place(a, shape, n_tokens);
  a.wide = ((reinterpret_cast<uintptr_t>(k_out_dev) | reinterpret_cast<uintptr_t>(v_out_dev)) & 31) == 0;
  a.has_k = k_out_dev != nullptr;
  const dim3 grid = grid_of(a, k_out_dev && v_out_dev);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = launch_pdl(shape->head_dim == 128 ? quant_read_kernel<128> : quant_read_kernel<64>, grid, dim3(kRowWarps * 32), 0, stream, a);
  return status_of(e);
}
