// af1_kv.cu — rotary positions, and the paged cache of keys and values as it
// is written and read back.
//
// All kernels here move data once and compute little, so device memory (or,
// for a few tokens, the launch) bounds them: every thread holds 8 entries of
// one head, 16 bytes of FP16, and neighbouring threads hold neighbouring
// entries.
//
// The rotation of a pair is (a c - b s, b c + a s). Its products and sums are
// rounded one by one (no fused multiply-add), as are the steps of the
// quantiser, so that what a cache holds is a function of the inputs to the
// bit, whichever launch wrote it. (Paired operations are used where no product
// meets a sum: the assembler may fuse a paired product and sum.)
#include <cudaTypedefs.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace af1 {
namespace {

constexpr int kThreads = 256;
// Added to |x| < 2^22, it rounds x to a whole number (to nearest even), which
// then stands in the low bits: a conversion at the rate of an addition.
constexpr float kRound = 12582912.f;  // 1.5 * 2^23
constexpr float kTiny = 7.52316385e-37f;  // 2^-120: smaller scales are stored as 0

// NaN if either is.
__device__ __forceinline__ float min_nan(float a, float b) {
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f32(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f32(__half& y, float x) { y = __float2half_rn(x); }

// N entries at p: in 16-byte (or, for 4 FP16, 8-byte) accesses if VEC, else one by one.
template <bool VEC, int N, typename T>
__device__ __forceinline__ void load(float (&x)[N], const T* p) {
  if constexpr (VEC) {
    constexpr int B = N * (int)sizeof(T) >= 16 ? 16 : 8;
    constexpr int E = B / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < N / E; ++i) {
      alignas(16) T t[E];
      if constexpr (B == 16)
        *reinterpret_cast<uint4*>(t) = reinterpret_cast<const uint4*>(p)[i];
      else
        *reinterpret_cast<uint2*>(t) = reinterpret_cast<const uint2*>(p)[i];
#pragma unroll
      for (int j = 0; j < E; ++j) x[i * E + j] = to_f32(t[j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32(p[i]);
  }
}
template <bool VEC, int N, typename T>
__device__ __forceinline__ void store(T* p, const float (&x)[N]) {
  if constexpr (VEC) {
    constexpr int B = N * (int)sizeof(T) >= 16 ? 16 : 8;
    constexpr int E = B / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < N / E; ++i) {
      alignas(16) T t[E];
#pragma unroll
      for (int j = 0; j < E; ++j) from_f32(t[j], x[i * E + j]);
      if constexpr (B == 16)
        reinterpret_cast<uint4*>(p)[i] = *reinterpret_cast<const uint4*>(t);
      else
        reinterpret_cast<uint2*>(p)[i] = *reinterpret_cast<const uint2*>(t);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) from_f32(p[i], x[i]);
  }
}

// cos and sin of N consecutive pairs of a table row (NaN outside the table).
template <bool VEC, int N>
__device__ __forceinline__ void load_turn(float (&c)[N], float (&s)[N], const float* table, int64_t length, int half,
                                          int pos, int pair) {
  if (pos < 0 || pos >= length) {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = s[i] = __int_as_float(0x7fffffff);
    return;
  }
  const float* p = table + ((int64_t)pos * half + pair) * 2;
  if constexpr (VEC) {
    float t[2 * N];
    load<true>(t, p);
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = t[2 * i], s[i] = t[2 * i + 1];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 t = reinterpret_cast<const float2*>(p)[i];
      c[i] = t.x, s[i] = t.y;
    }
  }
}

// ---- rope --------------------------------------------------------------------

struct RopeProblem {
  const void* x;
  void* y;
  const int32_t* positions;
  const int32_t* slot;  // append: a negative slot zeroes the token's rows (nullptr: no padding)
  const float* table;   // nullptr: copy
  int64_t length, x_token, x_head, y_token, y_head;
  int heads, half, units, pairs_units;  // units of a head: pairs_units of VP pairs, then copies of 2 VP entries
  int groups;                           // of heads that a thread takes together
  int64_t total;                        // tokens * groups * units
  bool back;
};

// One unit of TAKE heads of a token, which share its turns and whose entries
// are on their way together: VP pairs of each, or 2 VP entries that are only
// copied. A thread owns both entries of its pairs, so that y may be x. Beside
// the keys and values of an append, which leave an SM 1024 threads, four heads
// to a thread take 39 us where one takes 61 (8192 tokens, 32 heads of q, 8 of k
// and v); alone, with twice the threads, one takes 13 us and four 15 (2048 tokens
// x 32 x 128 FP32).
constexpr int kAppendTake = 4;
template <typename TI, typename TO, int VP, bool IL, int TAKE>
__device__ __forceinline__ void rope_unit(const RopeProblem& p, int64_t id) {
  const int64_t row = id / p.units;
  const int u = (int)(id - row * p.units);
  const int64_t token = row / p.groups;
  const int head = (int)(row - token * p.groups) * TAKE, heads = min(TAKE, p.heads - head);
  const TI* x = static_cast<const TI*>(p.x) + token * p.x_token + head * p.x_head;
  TO* y = static_cast<TO*>(p.y) + token * p.y_token + head * p.y_head;
  constexpr bool VEC = VP > 1;
  const bool pad = p.slot != nullptr && p.slot[token] < 0;
  const bool turns = u < p.pairs_units;
  // The unit's entries, in two halves of VP.
  const int at = turns ? (IL ? u * 2 * VP : u * VP) : 2 * p.half + (u - p.pairs_units) * 2 * VP;
  const int second = turns && !IL ? p.half : VP;
  // As they stand: a conversion would wait for them before the turns are read.
  struct alignas(VP * sizeof(TI)) Raw {
    TI at[VP];
  } first_raw[TAKE], second_raw[TAKE];
#pragma unroll
  for (int h = 0; h < TAKE; ++h) {
    if (h >= heads) continue;
    first_raw[h] = *reinterpret_cast<const Raw*>(x + h * p.x_head + at);
    second_raw[h] = *reinterpret_cast<const Raw*>(x + h * p.x_head + at + second);
  }
  float a[TAKE][VP], b[TAKE][VP], c[VP], s[VP];
  if (turns) load_turn<VEC>(c, s, p.table, p.length, p.half, pad ? 0 : p.positions[token], u * VP);
#pragma unroll
  for (int h = 0; h < TAKE; ++h)
#pragma unroll
    for (int i = 0; i < VP; ++i) a[h][i] = to_f32(first_raw[h].at[i]), b[h][i] = to_f32(second_raw[h].at[i]);
  if (turns) {
    if (p.back) {
#pragma unroll
      for (int i = 0; i < VP; ++i) s[i] = -s[i];
    }
#pragma unroll
    for (int h = 0; h < TAKE; ++h) {
      auto turn = [](float& first, float& other, float c, float s) {
        const float f = first, o = other;
        first = __fsub_rn(__fmul_rn(f, c), __fmul_rn(o, s));
        other = __fadd_rn(__fmul_rn(o, c), __fmul_rn(f, s));
      };
      if constexpr (!IL) {
#pragma unroll
        for (int i = 0; i < VP; ++i) turn(a[h][i], b[h][i], c[i], s[i]);
      } else if constexpr (VP == 1) {
        turn(a[h][0], b[h][0], c[0], s[0]);
      } else {
#pragma unroll
        for (int i = 0; i < VP; i += 2) {
          turn(a[h][i], a[h][i + 1], c[i / 2], s[i / 2]);
          turn(b[h][i], b[h][i + 1], c[(VP + i) / 2], s[(VP + i) / 2]);
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < TAKE; ++h) {
    if (h >= heads) continue;
    if (pad) {
#pragma unroll
      for (int i = 0; i < VP; ++i) a[h][i] = b[h][i] = 0.f;
    }
    store<VEC>(y + h * p.y_head + at, a[h]);
    store<VEC>(y + h * p.y_head + at + second, b[h]);
  }
}

template <typename T, int VP, bool IL>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeProblem p) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id < p.total) rope_unit<T, T, VP, IL, 1>(p, id);
}

// Units of a head, and whether 4 pairs to a thread fit the sizes, strides and
// pointers (else one pair: any even rope_dim, any stride).
bool plan_rope(RopeProblem& p, int take, int64_t tokens, int dim, int rope_dim, size_t xs, size_t ys, bool il,
               bool may = true) {
  const int per = il ? 8 : 4;  // entries of one vector access
  auto fits = [&](const void* q, int64_t a, int64_t b, size_t size) {
    return (uintptr_t)q % std::min<size_t>(16, per * size) == 0 && a % 8 == 0 && b % 8 == 0;
  };
  const bool vec = may && dim % 8 == 0 && rope_dim % 8 == 0 && fits(p.x, p.x_token, p.x_head, xs) &&
                   fits(p.y, p.y_token, p.y_head, ys) && (uintptr_t)p.x % 16 == 0 && (uintptr_t)p.y % 16 == 0 &&
                   (uintptr_t)p.table % 16 == 0;
  const int vp = vec ? 4 : 1;
  p.half = rope_dim / 2;
  p.pairs_units = p.half / vp;
  p.units = p.pairs_units + (dim - rope_dim) / (2 * vp);
  p.groups = (p.heads + take - 1) / take;
  p.total = tokens * p.groups * p.units;
  return vec;
}

// ---- the table -----------------------------------------------------------------

struct RopeFreq {
  double f[128];
  double attention;
  int64_t length;
  int half;
};

__global__ void __launch_bounds__(kThreads) rope_table_kernel(const __grid_constant__ RopeFreq p, float2* table) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id >= p.length * p.half) return;
  const int64_t pos = id / p.half;
  double s, c;
  sincos((double)pos * p.f[id - pos * p.half], &s, &c);
  table[id] = make_float2((float)(c * p.attention), (float)(s * p.attention));
}

// ---- quantisers ------------------------------------------------------------------

// 8 entries of a vector that LANES neighbouring threads hold: their codes
// (or FP16 values) to `row`, the vector's scale to `scale`, and the values
// that the codes stand for to x.
template <int KIND, int LANES>
__device__ __forceinline__ void quantise(float (&x)[8], int lane, uint8_t* row, void* scale, bool keep) {
  if constexpr (KIND == AF1_KV_F16) {
    alignas(16) __half h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = __float2half_rn(x[i]), x[i] = __half2float(h[i]);
    if (keep) reinterpret_cast<uint4*>(row)[lane] = *reinterpret_cast<uint4*>(h);
  } else if constexpr (KIND == AF1_KV_INT4) {
    // Infinities and NaN show in the extremes.
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) lo = min_nan(lo, x[i]), hi = max_nan(hi, x[i]);
#pragma unroll
    for (int m = 1; m < 4; m <<= 1) {  // a group of 32 entries: 4 threads
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, m));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, m));
    }
    __half hs = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), (float)(1.0 / 15.0)));
    __half hl = __float2half_rn(lo);
    const bool good = fabsf(__half2float(hs)) <= 65504.f && fabsf(__half2float(hl)) <= 65504.f;
    if (!good) hs = hl = __ushort_as_half(0x7fff);
    const float s = __half2float(hs), l = __half2float(hl);
    const float inv = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
    // A NaN scale makes every code 0: the maximum of NaN and 0 is 0.
    float2 part[4];  // codes of entries 2 i and 2 i + 1
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 q = mul2(add2(make_float2(x[2 * i], x[2 * i + 1]), make_float2(-l, -l)), make_float2(inv, inv));
      const float2 r = add2(make_float2(fminf(fmaxf(q.x, 0.f), 15.f), fminf(fmaxf(q.y, 0.f), 15.f)),
                            make_float2(kRound, kRound));
      part[i] = add2(r, make_float2(-kRound, -kRound));
      const float2 y = fma2(part[i], make_float2(s, s), make_float2(l, l));
      x[2 * i] = y.x, x[2 * i + 1] = y.y;
    }
    // Four codes as one whole number, below 2^16.
    auto four = [](const float2& a, const float2& b) {
      return __float_as_uint(fmaf(b.y, 4096.f, fmaf(b.x, 256.f, fmaf(a.y, 16.f, a.x))) + kRound);
    };
    const uint32_t codes = __byte_perm(four(part[0], part[1]), four(part[2], part[3]), 0x5410);
    if (keep) {
      reinterpret_cast<uint32_t*>(row)[lane] = codes;
      if (lane % 4 == 0) static_cast<__half2*>(scale)[lane / 4] = __halves2half2(hs, hl);
    }
  } else {
    float top = 0.f;  // infinities and NaN show in it
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_nan(top, fabsf(x[i]));
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, m));
    const bool bad = !(top < __int_as_float(0x7f800000));
    float s = __fmul_rn(top, (float)(1.0 / (KIND == AF1_KV_INT8 ? 127.0 : 448.0)));
    if (s < kTiny) s = 0.f;
    const float inv = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
    if (bad) s = __int_as_float(0x7fffffff);
    alignas(8) uint8_t codes[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 q = bad ? make_float2(0.f, 0.f) : make_float2(__fmul_rn(x[i], inv), __fmul_rn(x[i + 1], inv));
      if constexpr (KIND == AF1_KV_INT8) {
        // |q| <= 127 (1 + 2^-22), which rounds to 127: no clamp.
        const float2 r = add2(q, make_float2(kRound, kRound));
        codes[i] = (uint8_t)__float_as_uint(r.x), codes[i + 1] = (uint8_t)__float_as_uint(r.y);
        const float2 y = mul2(add2(r, make_float2(-kRound, -kRound)), make_float2(s, s));
        x[i] = y.x, x[i + 1] = y.y;
      } else {
        const __nv_fp8x2_storage_t c = __nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, __NV_E4M3);
        *reinterpret_cast<__nv_fp8x2_storage_t*>(codes + i) = c;
        const float2 y = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(c, __NV_E4M3)));
        const float2 z = mul2(y, make_float2(s, s));
        x[i] = z.x, x[i + 1] = z.y;
      }
    }
    if (keep) {
      reinterpret_cast<uint2*>(row)[lane] = *reinterpret_cast<uint2*>(codes);
      if (lane == 0) *static_cast<float*>(scale) = s;
    }
  }
}

// 8 entries read back.
template <int KIND>
__device__ __forceinline__ void dequantise(float (&x)[8], int lane, const uint8_t* row, const void* scale) {
  if constexpr (KIND == AF1_KV_F16) {
    load<true>(x, reinterpret_cast<const __half*>(row) + 8 * lane);
  } else if constexpr (KIND == AF1_KV_INT4) {
    const uint32_t codes = reinterpret_cast<const uint32_t*>(row)[lane];
    const float2 s = __half22float2(static_cast<const __half2*>(scale)[lane / 4]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __fmaf_rn((float)(codes >> (4 * i) & 15), s.x, s.y);
  } else {
    alignas(8) uint8_t c[8];
    *reinterpret_cast<uint2*>(c) = reinterpret_cast<const uint2*>(row)[lane];
    const float s = *static_cast<const float*>(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = __fmul_rn(KIND == AF1_KV_INT8 ? (float)(int8_t)c[i]
                                           : __half2float(__half(__nv_cvt_fp8_to_halfraw(c[i], __NV_E4M3))),
                       s);
  }
}

// ---- append ------------------------------------------------------------------------

struct AppendProblem {
  KvView cache;
  PageTable pages;
  const void *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  const int32_t *seq, *slot, *positions;
  const float* table;
  int64_t length;
  __half *k_out, *v_out;
  int half;
  int64_t tokens;
  int parts;          // threads of a token's lane: each takes every parts-th head
  int k_blocks, kv_blocks;  // blocks below store keys, or values, and the others rotate q
  RopeProblem q;
};

// Blocks of the cache part: DIM / 8 threads hold one vector, 8 entries each,
// and each takes `parts`-th heads of its token, with the token's turns in
// registers. The entries that a key's own are paired with lie in another
// thread's part (or, interleaved, in its own) and are read beside them: the
// second read hits L1, and no exchange between threads depends on rope_dim.
// Issue slots and bytes in flight bound it: 8192 tokens of 8 x 128 to INT4, with
// the values back, take 20.9 us, 3.9 TB/s (without reading ahead 6 us more; ahead
// by two rounds, with the pairs by shuffles, 3 more).
template <int KIND, int DIM, typename T, bool VEC, bool IL>
__global__ void __launch_bounds__(kThreads, 4) append_kernel(const __grid_constant__ AppendProblem p) {
  if ((int)blockIdx.x >= p.kv_blocks) {
    const int64_t id = (int64_t)(blockIdx.x - p.kv_blocks) * kThreads + threadIdx.x;
    if (id < p.q.total) rope_unit<T, __half, VEC ? 4 : 1, IL, kAppendTake>(p.q, id);
    return;
  }
  constexpr int LANES = DIM / 8;
  const bool is_v = (int)blockIdx.x >= p.k_blocks;
  int64_t id = (int64_t)(blockIdx.x - (is_v ? p.k_blocks : 0)) * (kThreads / LANES) + threadIdx.x / LANES;
  const bool real = id < p.tokens * p.parts;
  if (!real) id = 0;  // keeps every lane of the shuffles below
  const int lane = threadIdx.x % LANES;
  const int heads = p.cache.heads;
  const int64_t token = id / p.parts;
  const int part = (int)(id - token * p.parts);
  const int slot = p.slot[token], seq = p.seq[token];
  const int at = 8 * lane, half = p.half;
  const bool turns = !is_v && at < 2 * half;
  const int pos = p.positions != nullptr ? p.positions[token] : slot;
  const bool first = at < half;  // VEC, not interleaved: half is a multiple of 8, the 8 entries lie in one half
  float c[8], s[8];
  if (turns) {
    if constexpr (VEC && IL) {
      float c4[4], s4[4];
      load_turn<true>(c4, s4, p.table, p.length, half, pos, at / 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = c4[i], s[i] = s4[i];
    } else if constexpr (VEC) {
      load_turn<true>(c, s, p.table, p.length, half, pos, first ? at : at - half);
      if (first) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = -s[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < (IL ? 4 : 8); ++i) {
        const int e = IL ? at / 2 + i : at + i;  // pair, or entry
        float ci[1] = {1.f}, si[1] = {0.f};
        if (IL ? e < half : e < 2 * half)
          load_turn<false>(ci, si, p.table, p.length, half, pos, IL || e < half ? e : e - half);
        c[i] = ci[0], s[i] = si[0];
      }
    }
  }
  const int64_t row0 = kv_row(p.cache, p.pages, seq, slot, 0);
  const bool keep = real && row0 >= 0;
  uint8_t* codes = is_v ? p.cache.v : p.cache.k;
  uint8_t* scales = static_cast<uint8_t*>(is_v ? p.cache.vs : p.cache.ks);
  __half* out = is_v ? p.v_out : p.k_out;
  const T* token_src = is_v ? static_cast<const T*>(p.v) + token * p.v_token : static_cast<const T*>(p.k) + token * p.k_token;
  const int64_t head_step = is_v ? p.v_head : p.k_head;
  // Every thread of a block runs the same number of rounds: the shuffles need
  // all lanes. A thread without a head in the last one writes the last head's
  // values again. The next round's entries are read ahead, as they stand.
  constexpr int RAW = VEC ? 8 * (int)sizeof(T) / 16 : 1;
  uint4 x_raw[RAW], y_raw[RAW];
  const int pair_at = first ? at + half : at - half;
  auto head_of = [&](int round) { return min(round * p.parts + part, heads - 1); };
  auto fetch = [&](int head) {
    const T* src = token_src + head * head_step;
#pragma unroll
    for (int i = 0; i < RAW; ++i) {
      x_raw[i] = reinterpret_cast<const uint4*>(src + at)[i];
      if (!IL && turns) y_raw[i] = reinterpret_cast<const uint4*>(src + pair_at)[i];
    }
  };
  if constexpr (VEC) fetch(head_of(0));
  for (int round = 0; round * p.parts < heads; ++round) {
    const int head = head_of(round);
    float x[8], y[8];
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = to_f32(reinterpret_cast<const T*>(x_raw)[i]);
        if constexpr (!IL) y[i] = to_f32(reinterpret_cast<const T*>(y_raw)[i]);
      }
      if ((round + 1) * p.parts < heads) fetch(head_of(round + 1));
    } else {
      const T* src = token_src + head * head_step;
      load<false>(x, src + at);
      if constexpr (!IL) {
        if (turns) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = at + i;
            y[i] = e < 2 * half ? to_f32(src[e < half ? e + half : e - half]) : 0.f;
          }
        }
      }
    }
    if (turns) {
      if constexpr (IL) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!VEC && at + 2 * i >= 2 * half) break;
          const float a = x[2 * i], b = x[2 * i + 1];
          x[2 * i] = __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i]));
          x[2 * i + 1] = __fadd_rn(__fmul_rn(b, c[i]), __fmul_rn(a, s[i]));
        }
      } else if constexpr (VEC) {  // s has the sign of its part
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(y[i], s[i]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (at + i >= 2 * half) break;
          const bool low = at + i < half;
          x[i] = low ? __fsub_rn(__fmul_rn(x[i], c[i]), __fmul_rn(y[i], s[i]))
                     : __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(y[i], s[i]));
        }
      }
    }
    const int64_t row = row0 < 0 ? 0 : row0 + ((int64_t)head << p.cache.shift);
    quantise<KIND, LANES>(x, lane, codes + row * kv_row_bytes(KIND, DIM), scales + row * kv_scale_bytes(KIND, DIM), keep);
    if (real && out != nullptr) {
      if (slot < 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
      }
      store<true>(out + (token * heads + head) * DIM + at, x);
    }
  }
}

// ---- read ---------------------------------------------------------------------------

struct ReadProblem {
  KvView cache;
  PageTable pages;
  const int32_t* lens;
  int64_t first, count;
  void *k_out, *v_out;
};

// A block reads kThreads / (DIM / 8) neighbouring slots, all heads of them one
// after another, so that it reads runs of a page's rows and writes one stretch
// of the output. (Blocks of one head each wrote 128-byte pieces a slot apart:
// 103 us where this takes 54, 16 sequences of up to 8190 INT4 tokens of 8 x 64.)
constexpr int kReadRows = 4;  // heads in flight

template <int KIND, int DIM, typename TO>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadProblem p, int64_t tiles) {
  constexpr int LANES = DIM / 8, ROWS = kThreads / LANES;
  const int64_t tile = blockIdx.x % tiles;
  const int seq = (int)(blockIdx.x / tiles);
  const int heads = p.cache.heads;
  const bool is_v = blockIdx.y != 0;
  const int lane = threadIdx.x % LANES;
  const int64_t at = tile * ROWS + threadIdx.x / LANES, slot = p.first + at;
  if (at >= p.count) return;
  const int64_t row0 = slot < p.lens[seq] ? kv_row(p.cache, p.pages, seq, (int)slot, 0) : -1;
  const uint8_t* codes = is_v ? p.cache.v : p.cache.k;
  const uint8_t* scales = static_cast<const uint8_t*>(is_v ? p.cache.vs : p.cache.ks);
  TO* out = static_cast<TO*>(is_v ? p.v_out : p.k_out) + (seq * p.count + at) * heads * DIM + 8 * lane;
  const int64_t step_codes = (int64_t)kv_row_bytes(KIND, DIM) << p.cache.shift;
  const int64_t step_scales = (int64_t)kv_scale_bytes(KIND, DIM) << p.cache.shift;
  codes += (row0 < 0 ? 0 : row0) * kv_row_bytes(KIND, DIM);
  scales += (row0 < 0 ? 0 : row0) * kv_scale_bytes(KIND, DIM);
  int head = 0;
  for (; head + kReadRows <= heads; head += kReadRows) {
    float x[kReadRows][8];
    if (row0 >= 0) {
#pragma unroll
      for (int i = 0; i < kReadRows; ++i)
        dequantise<KIND>(x[i], lane, codes + (head + i) * step_codes, scales + (head + i) * step_scales);
    } else {
#pragma unroll
      for (int i = 0; i < kReadRows; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) store<true>(out + (head + i) * DIM, x[i]);
  }
  for (; head < heads; ++head) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (row0 >= 0) dequantise<KIND>(x, lane, codes + head * step_codes, scales + head * step_scales);
    store<true>(out + head * DIM, x);
  }
}

// ---- tree masks -----------------------------------------------------------------------

__global__ void __launch_bounds__(kThreads) tree_mask_kernel(const int32_t* parents, int64_t total, int nodes,
                                                             uint32_t* mask) {
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (id >= total) return;
  const int64_t seq = id / nodes;
  int node = (int)(id - seq * nodes);
  uint64_t bits = 0;
  for (int step = 0; step < nodes && node >= 0 && node < nodes; ++step) {
    bits |= 1ull << node;
    node = parents[seq * nodes + node];
  }
  const int words = (nodes + 31) / 32;
  for (int w = 0; w < words; ++w) mask[id * words + w] = (uint32_t)(bits >> (32 * w));
}

// ---- host ------------------------------------------------------------------------------

int fail(int code, const char* who, const std::string& msg) { return set_error(code, std::string(who) + ": " + msg); }

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess)
    return fail(AF1_ERR_CUDA, who, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}

int current_device(const char* who, int* dev) {
  const cudaError_t e = cudaGetDevice(dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, who, cudaGetErrorString(e));
  return AF1_OK;
}

int check_table(const char* who, const float* table, int64_t length, int64_t rope_dim, int64_t dim, int dev) {
  if (rope_dim < 2 || rope_dim % 2 != 0 || rope_dim > dim)
    return fail(AF1_ERR_INVALID_ARG, who, "rope_dim must be even, at least 2 and at most the head's size");
  if (length < 1 || length > (1 << 24)) return fail(AF1_ERR_INVALID_ARG, who, "length must be 1..2^24");
  int rc = check_pointer(table, "table", dev);
  if (rc == AF1_OK) rc = check_align(table, 8, "table");
  return rc;
}

// Entries between the first and the last that a tensor's strides reach, as a bound for the 2^62 of its offsets.
bool span_ok(int64_t n, int64_t stride) { return stride >= 0 && (n <= 1 || stride <= ((int64_t)1 << 60) / n); }

// Tensor map of `rows` rows of row_bytes bytes: boxes of `box` rows by up to
// 128 bytes, swizzled by the box's width.
bool make_row_map(CUtensorMap* map, void* base, int64_t rows, int row_bytes, int box) {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    return static_cast<PFN_cuTensorMapEncodeTiled_v12000>(nullptr);
  }();
  if (fn == nullptr) return false;
  const int span = std::min(row_bytes, 128);
  const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)row_bytes};
  const cuuint32_t boxes[2] = {(cuuint32_t)span, (cuuint32_t)box}, steps[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            span == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
            : span == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                         : CU_TENSOR_MAP_SWIZZLE_32B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename F>
int with_kind(int kind, F&& f) {
  switch (kind) {
    case AF1_KV_F16: return f(std::integral_constant<int, AF1_KV_F16>());
    case AF1_KV_INT8: return f(std::integral_constant<int, AF1_KV_INT8>());
    case AF1_KV_E4M3: return f(std::integral_constant<int, AF1_KV_E4M3>());
    default: return f(std::integral_constant<int, AF1_KV_INT4>());
  }
}
template <typename F>
int with_bool(bool b, F&& f) {
  return b ? f(std::true_type()) : f(std::false_type());
}

}  // namespace

int check_pointer(const void* p, const char* name, int device) {
  if (p == nullptr) return set_error(AF1_ERR_INVALID_ARG, std::string(name) + " is NULL");
  cudaPointerAttributes at;
  const cudaError_t e = cudaPointerGetAttributes(&at, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return set_error(AF1_ERR_BAD_POINTER, std::string(name) + " is not a CUDA pointer");
  }
  if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged)
    return set_error(AF1_ERR_BAD_POINTER, std::string(name) + " is not device memory");
  if (at.type == cudaMemoryTypeDevice && at.device != device)
    return set_error(AF1_ERR_BAD_POINTER, std::string(name) + " lives on another device");
  return AF1_OK;
}

int check_align(const void* p, int bytes, const char* name) {
  if ((uintptr_t)p % bytes != 0)
    return set_error(AF1_ERR_MISALIGNED, std::string(name) + " must be " + std::to_string(bytes) + "-byte aligned");
  return AF1_OK;
}

KvView view_of(const af1_kv_desc& d) {
  int shift = 0;
  while ((1 << shift) < d.page_size) ++shift;
  return {static_cast<uint8_t*>(d.k), static_cast<uint8_t*>(d.v), d.k_scale, d.v_scale, (int)d.pages, d.kv_heads, shift};
}

}  // namespace af1

using namespace af1;

int af1_rope_frequencies(const af1_rope_params* p, double* freq, double* attention) {
  const char* who = "af1_rope_frequencies";
  if (p == nullptr || freq == nullptr || attention == nullptr)
    return fail(AF1_ERR_INVALID_ARG, who, "params, freq or attention is NULL");
  if (p->length < 1 || p->length > (1 << 24)) return fail(AF1_ERR_INVALID_ARG, who, "length must be 1..2^24");
  if (p->dim < 2 || p->dim > 256 || p->dim % 2 != 0)
    return fail(AF1_ERR_INVALID_ARG, who, "dim must be even and 2..256");
  if (p->scaling < AF1_ROPE_PLAIN || p->scaling > AF1_ROPE_RAMP) return fail(AF1_ERR_INVALID_ARG, who, "unknown scaling");
  if (!(p->base > 1.0) || !std::isfinite(p->base)) return fail(AF1_ERR_INVALID_ARG, who, "base must be above 1");
  const bool scaled = p->scaling != AF1_ROPE_PLAIN;
  if (scaled && (!(p->factor >= 1.0) || !std::isfinite(p->factor)))
    return fail(AF1_ERR_INVALID_ARG, who, "factor must be at least 1");
  if (!(p->attention >= 0.0) || !std::isfinite(p->attention))
    return fail(AF1_ERR_INVALID_ARG, who, "attention must be 0 or above");
  if (p->scaling == AF1_ROPE_BANDS || p->scaling == AF1_ROPE_RAMP) {
    if (!(p->original > 0.0) || !std::isfinite(p->original))
      return fail(AF1_ERR_INVALID_ARG, who, "original must be positive");
    if (!(p->low > 0.0) || !(p->high > p->low) || !std::isfinite(p->high))
      return fail(AF1_ERR_INVALID_ARG, who, "need 0 < low < high");
  }
  if (p->scaling == AF1_ROPE_BASE && p->dim == 2)
    return fail(AF1_ERR_INVALID_ARG, who, "AF1_ROPE_BASE needs dim above 2");
  const double kPi = 3.14159265358979323846;
  const int half = p->dim / 2;
  double base = p->base;
  if (p->scaling == AF1_ROPE_BASE) base *= std::pow(p->factor, (double)p->dim / (p->dim - 2));
  double i0 = 0.0, i1 = 0.0;
  if (p->scaling == AF1_ROPE_RAMP) {
    auto e = [&](double beta) { return p->dim * std::log(p->original / (2.0 * kPi * beta)) / (2.0 * std::log(base)); };
    i0 = std::fmax(0.0, std::floor(e(p->high)));
    i1 = std::fmin(p->dim - 1.0, std::ceil(e(p->low)));
  }
  for (int i = 0; i < half; ++i) {
    double f = std::pow(base, -2.0 * i / p->dim);
    if (p->scaling == AF1_ROPE_LINEAR) {
      f /= p->factor;
    } else if (p->scaling == AF1_ROPE_BANDS) {
      const double w = 2.0 * kPi / f;
      if (w > p->original / p->low) {
        f /= p->factor;
      } else if (w >= p->original / p->high) {
        const double g = (p->original / w - p->low) / (p->high - p->low);
        f = (1.0 - g) * f / p->factor + g * f;
      }
    } else if (p->scaling == AF1_ROPE_RAMP) {
      const double span = i1 > i0 ? i1 - i0 : 1e-3;
      const double g = std::fmin(1.0, std::fmax(0.0, (i - i0) / span));
      f = (1.0 - g) * f + g * f / p->factor;
    }
    freq[i] = f;
  }
  *attention = p->attention > 0.0 ? p->attention : p->scaling == AF1_ROPE_RAMP ? 0.1 * std::log(p->factor) + 1.0 : 1.0;
  set_error(AF1_OK, "");
  return AF1_OK;
}

int af1_rope_table(const af1_rope_params* params, float* table, void* stream) {
  RopeFreq f = {};
  int rc = af1_rope_frequencies(params, f.f, &f.attention);
  if (rc != AF1_OK) return rc;
  int dev;
  if ((rc = current_device("af1_rope_table", &dev)) != AF1_OK) return rc;
  if ((rc = check_pointer(table, "table", dev)) != AF1_OK || (rc = check_align(table, 8, "table")) != AF1_OK) return rc;
  f.length = params->length;
  f.half = params->dim / 2;
  const int64_t blocks = (f.length * f.half + kThreads - 1) / kThreads;
  rope_table_kernel<<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      f, reinterpret_cast<float2*>(table));
  return launched("af1_rope_table");
}

int af1_rope(const af1_rope_args* a, void* stream) {
  const char* who = "af1_rope";
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "args is NULL");
  if (a->tokens < 0 || a->heads < 1 || a->dim < 2 || a->dim > 1024 || a->dim % 2 != 0 || a->heads > 65536 ||
      a->tokens > (1ll << 31))
    return fail(AF1_ERR_INVALID_ARG, who, "need tokens 0..2^31, heads 1..65536, dim even and 2..1024");
  if (a->dtype != AF1_F16 && a->dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, who, "dtype must be AF1_F16 or AF1_F32");
  if ((a->flags & ~(AF1_ROPE_INTERLEAVED | AF1_ROPE_BACKWARD)) != 0) return fail(AF1_ERR_INVALID_ARG, who, "unknown flags");
  if (!span_ok(a->tokens, a->x_token) || !span_ok(a->heads, a->x_head) || !span_ok(a->tokens, a->y_token) ||
      !span_ok(a->heads, a->y_head))
    return fail(AF1_ERR_INVALID_ARG, who, "strides must not be negative");
  if (a->x == a->y && (a->x_token != a->y_token || a->x_head != a->y_head))
    return fail(AF1_ERR_INVALID_ARG, who, "in place, the strides of x and y must be equal");
  if (a->tokens == 0) return AF1_OK;
  int dev, rc;
  if ((rc = current_device(who, &dev)) != AF1_OK) return rc;
  if ((rc = check_table(who, a->table, a->length, a->rope_dim, a->dim, dev)) != AF1_OK) return rc;
  if ((rc = check_pointer(a->x, "x", dev)) != AF1_OK || (rc = check_pointer(a->y, "y", dev)) != AF1_OK ||
      (rc = check_pointer(a->positions, "positions", dev)) != AF1_OK)
    return rc;
  const size_t es = a->dtype == AF1_F16 ? 2 : 4;
  if ((rc = check_align(a->x, (int)es, "x")) != AF1_OK || (rc = check_align(a->y, (int)es, "y")) != AF1_OK ||
      (rc = check_align(a->positions, 4, "positions")) != AF1_OK)
    return rc;
  const bool il = (a->flags & AF1_ROPE_INTERLEAVED) != 0;
  RopeProblem p = {a->x, a->y, a->positions, nullptr, a->table, a->length, a->x_token, a->x_head, a->y_token, a->y_head};
  p.heads = (int)a->heads;
  p.back = (a->flags & AF1_ROPE_BACKWARD) != 0;
  const bool vec = plan_rope(p, 1, a->tokens, (int)a->dim, (int)a->rope_dim, es, es, il);
  const int64_t blocks = (p.total + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "too many entries for one call");
  return with_bool(vec, [&](auto v) {
    return with_bool(il, [&](auto i) {
      return with_bool(a->dtype == AF1_F16, [&](auto h) {
        using T = std::conditional_t<decltype(h)::value, __half, float>;
        rope_kernel<T, decltype(v)::value ? 4 : 1, decltype(i)::value>
            <<<(unsigned)blocks, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
        return launched(who);
      });
    });
  });
}

int af1_kv_create(const af1_kv_desc* d, af1_kv_cache** out) {
  const char* who = "af1_kv_create";
  if (out == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "out is NULL");
  *out = nullptr;
  if (d == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "desc is NULL");
  if (d->kind < AF1_KV_F16 || d->kind > AF1_KV_INT4) return fail(AF1_ERR_INVALID_ARG, who, "unknown kind");
  if (d->pages < 1 || d->pages > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "pages must be 1..2^31 - 1");
  if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1)) != 0)
    return fail(AF1_ERR_INVALID_ARG, who, "page_size must be 16, 32, 64, 128 or 256");
  if (d->kv_heads < 1 || d->kv_heads > 1024) return fail(AF1_ERR_INVALID_ARG, who, "kv_heads must be 1..1024");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(AF1_ERR_INVALID_ARG, who, "head_dim must be 64 or 128");
  const bool scaled = d->kind != AF1_KV_F16;
  if (scaled != (d->k_scale != nullptr) || scaled != (d->v_scale != nullptr))
    return fail(AF1_ERR_INVALID_ARG, who, "k_scale and v_scale go with INT8, E4M3 and INT4, and only with these");
  int dev, rc;
  if ((rc = current_device(who, &dev)) != AF1_OK) return rc;
  const void* ptrs[4] = {d->k, d->v, d->k_scale, d->v_scale};
  const char* names[4] = {"k", "v", "k_scale", "v_scale"};
  for (int i = 0; i < (scaled ? 4 : 2); ++i)
    if ((rc = check_pointer(ptrs[i], names[i], dev)) != AF1_OK || (rc = check_align(ptrs[i], 16, names[i])) != AF1_OK)
      return rc;
  const int64_t rows = d->pages * d->kv_heads * d->page_size;
  if (rows > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "pages * kv_heads * page_size must be below 2^31");
  int sms = 0;
  cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, who, cudaGetErrorString(e));
  af1_kv_cache* c = new (std::nothrow) af1_kv_cache();
  if (c == nullptr) return fail(AF1_ERR_CUDA, who, "host allocation failed");
  c->d = *d;
  c->device = dev;
  c->num_sms = sms;
  const int row_bytes = kv_row_bytes(d->kind, d->head_dim);
  // Boxes of a warp's step (16 rows for rows of 256 bytes), and of a tile.
  const int step = std::min(d->page_size, row_bytes >= 256 ? 16 : 32), tile = std::min(d->page_size, 128);
  bool ok = make_row_map(&c->k_step, d->k, rows, row_bytes, step) && make_row_map(&c->v_step, d->v, rows, row_bytes, step);
  c->k_tile = c->k_step, c->v_tile = c->v_step;
  if (tile != step)
    ok = ok && make_row_map(&c->k_tile, d->k, rows, row_bytes, tile) && make_row_map(&c->v_tile, d->v, rows, row_bytes, tile);
  if (!ok) {
    delete c;
    return fail(AF1_ERR_CUDA, who, "cuTensorMapEncodeTiled failed");
  }
  *out = c;
  set_error(AF1_OK, "");
  return AF1_OK;
}

void af1_kv_free(af1_kv_cache* cache) { delete cache; }

namespace {

int check_pages(const char* who, const af1_kv_cache* c, const int32_t* pages, int64_t sequences, int64_t columns,
                int64_t ld, int dev) {
  if (sequences > 65536 || columns < 1 || ld < columns || columns > ((int64_t)1 << 31) / c->d.page_size - 1 ||
      !span_ok(sequences, ld))
    return fail(AF1_ERR_INVALID_ARG, who,
                "need at most 65536 sequences, page columns of fewer than 2^31 slots in all, pages_ld >= page_columns");
  int rc = check_pointer(pages, "pages", dev);
  if (rc == AF1_OK) rc = check_align(pages, 4, "pages");
  return rc;
}

int check_cache(const char* who, const af1_kv_cache* c, int* dev) {
  if (c == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "cache is NULL");
  int rc = current_device(who, dev);
  if (rc != AF1_OK) return rc;
  if (*dev != c->device) return fail(AF1_ERR_BAD_POINTER, who, "the current device is not the cache's device");
  return AF1_OK;
}

}  // namespace

int af1_kv_append(const af1_kv_cache* c, const af1_kv_append_args* a, void* stream) {
  const char* who = "af1_kv_append";
  int dev, rc;
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "args is NULL");
  if ((rc = check_cache(who, c, &dev)) != AF1_OK) return rc;
  if (a->tokens < 0 || a->tokens > ((int64_t)1 << 31) || a->sequences < 0)
    return fail(AF1_ERR_INVALID_ARG, who, "need tokens 0..2^31 and sequences >= 0");
  if (a->dtype != AF1_F16 && a->dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, who, "dtype must be AF1_F16 or AF1_F32");
  if ((a->flags & ~AF1_ROPE_INTERLEAVED) != 0) return fail(AF1_ERR_INVALID_ARG, who, "unknown flags");
  const int heads = c->d.kv_heads, dim = c->d.head_dim;
  if (!span_ok(a->tokens, a->k_token) || !span_ok(heads, a->k_head) || !span_ok(a->tokens, a->v_token) ||
      !span_ok(heads, a->v_head))
    return fail(AF1_ERR_INVALID_ARG, who, "strides must not be negative");
  if ((a->q == nullptr) != (a->q_out == nullptr)) return fail(AF1_ERR_INVALID_ARG, who, "q and q_out go together");
  const bool has_q = a->q != nullptr;
  if (has_q && (a->q_heads < 1 || a->q_heads > 65536 || !span_ok(a->tokens, a->q_token) ||
                !span_ok(a->q_heads, a->q_head) || !span_ok(a->tokens, a->qo_token) || !span_ok(a->q_heads, a->qo_head)))
    return fail(AF1_ERR_INVALID_ARG, who, "q_heads must be 1..65536 and strides not negative");
  if (has_q && a->q == a->q_out &&
      (a->dtype != AF1_F16 || a->q_token != a->qo_token || a->q_head != a->qo_head))
    return fail(AF1_ERR_INVALID_ARG, who, "in place, q must be FP16 and the strides of q and q_out equal");
  if (a->tokens == 0) return AF1_OK;
  const bool rope = a->table != nullptr;
  if (rope && (rc = check_table(who, a->table, a->length, a->rope_dim, dim, dev)) != AF1_OK) return rc;
  if ((rc = check_pages(who, c, a->pages, a->sequences, a->page_columns, a->pages_ld, dev)) != AF1_OK) return rc;
  const int es = a->dtype == AF1_F16 ? 2 : 4;
  struct {
    const void* p;
    const char* name;
    int align;
    bool need;
  } ptrs[] = {{a->k, "k", es, true},          {a->v, "v", es, true},
              {a->seq, "seq", 4, true},       {a->slot, "slot", 4, true},
              {a->positions, "positions", 4, false}, {a->q, "q", es, false},
              {a->q_out, "q_out", 2, false},  {a->k_out, "k_out", 16, false},
              {a->v_out, "v_out", 16, false}};
  for (const auto& t : ptrs) {
    if (t.p == nullptr && !t.need) continue;
    if ((rc = check_pointer(t.p, t.name, dev)) != AF1_OK || (rc = check_align(t.p, t.align, t.name)) != AF1_OK) return rc;
  }
  const bool il = (a->flags & AF1_ROPE_INTERLEAVED) != 0;
  AppendProblem p = {};
  p.cache = view_of(c->d);
  p.pages = {a->pages, a->pages_ld, (int)a->sequences, (int)a->page_columns};
  p.k = a->k, p.v = a->v;
  p.k_token = a->k_token, p.k_head = a->k_head, p.v_token = a->v_token, p.v_head = a->v_head;
  p.seq = a->seq, p.slot = a->slot, p.positions = a->positions;
  p.table = a->table, p.length = a->length;
  p.k_out = static_cast<__half*>(a->k_out), p.v_out = static_cast<__half*>(a->v_out);
  p.half = rope ? (int)a->rope_dim / 2 : 0;
  p.tokens = a->tokens;
  // A thread takes several heads of its token (one turn for all of them) where
  // there are tokens enough to give every SM 1024 threads all the same: 8192
  // tokens of 8 x 128 as INT4 with their values take 35 us with one head to a
  // thread, 26 with two, 22.5 with four and 20.9 with eight.
  const int64_t threads = 2 * a->tokens * (dim / 8) * heads;
  const int take = (int)std::max<int64_t>(1, std::min<int64_t>(8, threads / (1024 * (int64_t)c->num_sms)));
  p.parts = (heads + take - 1) / take;
  const int per_block = kThreads / (dim / 8);
  const int64_t kv_blocks = 2 * ((a->tokens * p.parts + per_block - 1) / per_block);
  int64_t q_blocks = 0;
  // 16-byte reads of k and v, and of their pairs and turns, where sizes and
  // addresses allow them (for q too, as one variant serves both).
  auto fits = [&](const void* q, int64_t s, int64_t t) {
    return (uintptr_t)q % 16 == 0 && s * es % 16 == 0 && t * es % 16 == 0;
  };
  bool vec = fits(a->k, a->k_token, a->k_head) && fits(a->v, a->v_token, a->v_head) &&
             (!rope || ((uintptr_t)a->table % 16 == 0 && a->rope_dim % 16 == 0));
  if (has_q) {
    p.q.x = a->q, p.q.y = a->q_out;
    p.q.positions = a->positions != nullptr ? a->positions : a->slot;
    p.q.slot = a->slot;
    p.q.table = a->table, p.q.length = a->length;
    p.q.x_token = a->q_token, p.q.x_head = a->q_head, p.q.y_token = a->qo_token, p.q.y_head = a->qo_head;
    p.q.heads = (int)a->q_heads;
    vec = plan_rope(p.q, kAppendTake, a->tokens, dim, 2 * p.half, es, 2, il, vec);
    q_blocks = (p.q.total + kThreads - 1) / kThreads;
  }
  if (kv_blocks + q_blocks > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "too many entries for one call");
  p.k_blocks = (int)(kv_blocks / 2), p.kv_blocks = (int)kv_blocks;
  return with_kind(c->d.kind, [&](auto kind) {
    return with_bool(dim == 128, [&](auto wide) {
      return with_bool(a->dtype == AF1_F16, [&](auto h) {
        return with_bool(vec, [&](auto v) {
          return with_bool(il, [&](auto i) {
            using T = std::conditional_t<decltype(h)::value, __half, float>;
            append_kernel<decltype(kind)::value, decltype(wide)::value ? 128 : 64, T, decltype(v)::value,
                          decltype(i)::value>
                <<<(unsigned)(kv_blocks + q_blocks), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
            return launched(who);
          });
        });
      });
    });
  });
}

int af1_kv_read(const af1_kv_cache* c, const int32_t* pages, int64_t sequences, int64_t page_columns, int64_t pages_ld,
                const int32_t* lens, int64_t first, int64_t count, void* k_out, void* v_out, int dtype, void* stream) {
  const char* who = "af1_kv_read";
  int dev, rc;
  if ((rc = check_cache(who, c, &dev)) != AF1_OK) return rc;
  if (sequences < 0 || first < 0 || count < 0 || first > 0x7fffffff || count > 0x7fffffff)
    return fail(AF1_ERR_INVALID_ARG, who, "need sequences, first and count from 0 to 2^31 - 1");
  if (dtype != AF1_F16 && dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, who, "dtype must be AF1_F16 or AF1_F32");
  if (sequences == 0 || count == 0) return AF1_OK;
  if ((rc = check_pages(who, c, pages, sequences, page_columns, pages_ld, dev)) != AF1_OK) return rc;
  if ((rc = check_pointer(lens, "lens", dev)) != AF1_OK || (rc = check_align(lens, 4, "lens")) != AF1_OK ||
      (rc = check_pointer(k_out, "k_out", dev)) != AF1_OK || (rc = check_align(k_out, 16, "k_out")) != AF1_OK ||
      (rc = check_pointer(v_out, "v_out", dev)) != AF1_OK || (rc = check_align(v_out, 16, "v_out")) != AF1_OK)
    return rc;
  const int dim = c->d.head_dim;
  const int64_t tile = (int64_t)kThreads / (dim / 8);
  const int64_t tiles = (count + tile - 1) / tile;
  if (tiles * sequences > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "too many slots for one call");
  ReadProblem p = {view_of(c->d), {pages, pages_ld, (int)sequences, (int)page_columns}, lens, first, count, k_out, v_out};
  const dim3 grid((unsigned)(tiles * sequences), 2);
  return with_kind(c->d.kind, [&](auto kind) {
    return with_bool(dim == 128, [&](auto wide) {
      return with_bool(dtype == AF1_F16, [&](auto h) {
        using T = std::conditional_t<decltype(h)::value, __half, float>;
        read_kernel<decltype(kind)::value, decltype(wide)::value ? 128 : 64, T>
            <<<grid, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p, tiles);
        return launched(who);
      });
    });
  });
}

int af1_tree_mask(const int32_t* parents, int64_t sequences, int64_t nodes, uint32_t* mask, void* stream) {
  const char* who = "af1_tree_mask";
  if (nodes < 1 || nodes > 64 || sequences < 0 || sequences > 65536)
    return fail(AF1_ERR_INVALID_ARG, who, "need 1..64 nodes and 0..65536 sequences");
  if (sequences == 0) return AF1_OK;
  int dev, rc;
  if ((rc = current_device(who, &dev)) != AF1_OK || (rc = check_pointer(parents, "parents", dev)) != AF1_OK ||
      (rc = check_align(parents, 4, "parents")) != AF1_OK || (rc = check_pointer(mask, "mask", dev)) != AF1_OK ||
      (rc = check_align(mask, 4, "mask")) != AF1_OK)
    return rc;
  const int64_t total = sequences * nodes;
  tree_mask_kernel<<<(unsigned)((total + kThreads - 1) / kThreads), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      parents, total, (int)nodes, mask);
  return launched(who);
}
