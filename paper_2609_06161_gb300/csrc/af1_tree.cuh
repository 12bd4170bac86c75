// af1_tree.cuh — what the two kernels of af1_tree_attention share: the
// problem, FP16 operands from the cache's codes, and the division of all
// sequences' keys into units of work.
#pragma once

#include <cuda.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace af1 {

constexpr int kMaxCtas = 1024;  // counters of the workspace
static_assert(4 * kMaxCtas <= kCounterBytes, "the counters lie in the region of counters");
// Weights are at most 2^(kShift + kSlack) = 2^15 (half of FP16's range), and
// keep 11 bits down to 2^(-14 - kShift - kSlack) of the largest.
constexpr float kShift = 7.f, kSlack = 8.f;
constexpr float kInf = __builtin_huge_valf();

// Cycles that copies in flight are given to land after a wait has given up,
// however short the waits are: 10 ms.
constexpr long long kLanding = 20000000;

struct TreeProblem {
  CUtensorMap k_map, v_map;
  const __half* q;
  int64_t q_seq, q_node, q_head;
  void* out;
  int64_t o_seq, o_node, o_head;
  float* lse;
  KvView cache;
  PageTable pages;
  const int32_t *lens, *counts;
  const uint32_t* mask;
  int64_t mask_seq;
  int nodes, group, words;  // words of a mask row
  int row_tiles;
  float scale_log2;         // scale * log2(e)
  bool out_f32;
  unsigned* status;
  unsigned* counters;
  float* parts;
  long long wait_cycles;
};

static __device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) { return __byte_perm(a, b, s); }
static __device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
static __device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
static __device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
static __device__ __forceinline__ uint32_t e4m3x2(uint32_t low16) {
  uint32_t d;
  asm("{\n .reg .b16 l;\n cvt.u16.u32 l, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(d) : "r"(low16));
  return d;
}
static __device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
static __device__ __forceinline__ float low_float(uint32_t h2) { return __half2float(__ushort_as_half((unsigned short)h2)); }
static __device__ __forceinline__ float high_float(uint32_t h2) {
  return __half2float(__ushort_as_half((unsigned short)(h2 >> 16)));
}
static __device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
static __device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}
static __device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// Budgets below this many cycles are waited for without suspending the thread,
// which may take longer.
constexpr long long kSuspend = 65536;
static __device__ __forceinline__ bool mbar_test_wait(uint64_t* bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return done != 0;
}
// Bounded wait for a phase of a barrier: false where it gave up.
static __device__ __forceinline__ bool wait_phase(uint64_t* bar, uint32_t parity, long long budget) {
  if (mbar_test_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!(budget < kSuspend ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)))
    if (clock64() - t0 > budget) return false;
  return true;
}
static __device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int x, int row, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(row), "r"(smem_u32(bar))
      : "memory");
}

// What the kernel knows of a kind of cache at compile time. Shared memory
// holds the rows of a step as TMA writes them: slices of up to 128 bytes of a
// row, each slice's rows in order, 16-byte chunks swizzled so that eight
// neighbouring rows' chunks at one place lie in different banks.
template <int KIND, int DIM>
struct Kv {
  static constexpr int RB = kv_row_bytes(KIND, DIM);    // bytes of a row
  static constexpr int SB = kv_scale_bytes(KIND, DIM);  // bytes of its scales
  static constexpr int SPAN = RB < 128 ? RB : 128;      // bytes of a row in one slice
  static constexpr int SLICES = RB / SPAN;
  static constexpr int KS = DIM / 16;                   // products along a key
  static constexpr int MT = DIM / 16;                   // 16-entry blocks of a value
  static constexpr int GROUPS = KIND == AF1_KV_INT4 ? DIM / 32 : 1;
  static constexpr bool SCALED8 = KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3;
  // Byte offset of a chunk of a row in a step's k or v of KW rows.
  template <int KW>
  static __device__ __forceinline__ int at(int row, int chunk) {
    if constexpr (SPAN == 128)
      return (chunk >> 3) * (KW * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
    else if constexpr (SPAN == 64)
      return row * 64 + ((chunk ^ (row >> 1 & 3)) << 4);
    else
      return row * 32 + ((chunk ^ (row >> 2 & 1)) << 4);
  }
  // Entry of a key at place e (0, 1: the low k indices of the lanes with
  // lane % 4 == t, 2, 3: the high ones) of product ks.
  static __device__ __forceinline__ int entry(int t, int ks, int e) {
    if constexpr (KIND == AF1_KV_F16) return 64 * (ks >> 2) + 8 * (2 * t + (ks >> 1 & 1)) + 4 * (ks & 1) + e;
    else if constexpr (KIND == AF1_KV_INT4) return 32 * (ks >> 1) + 8 * t + (ks & 1) + 2 * (e >> 1) + 4 * (e & 1);
    else if constexpr (DIM == 128) return 16 * (2 * t + (ks >> 2)) + 4 * (ks & 3) + e;
    else return 16 * t + 4 * ks + e;
  }
  // Entry of a value in row g (hi: g + 8) of its block m.
  static __device__ __forceinline__ int row_entry(int m, int g, int hi) {
    if constexpr (KIND == AF1_KV_F16) return 16 * m + g + 8 * hi;
    else if constexpr (KIND == AF1_KV_INT4) return 32 * (m >> 1) + 4 * g + (m & 1) + 2 * hi;
    else return 16 * m + 2 * g + hi;
  }
};

// The a operand of product ks, from the words of keys g and g + 8.
template <int KIND, int N>
static __device__ __forceinline__ void key_operand(uint32_t (&a)[4], const uint32_t (&w)[2][N], int ks) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (KIND == AF1_KV_F16) {
      a[h] = w[h][2 * ks], a[2 + h] = w[h][2 * ks + 1];
    } else if constexpr (KIND == AF1_KV_INT8) {
      const uint32_t u = w[h][ks] ^ 0x80808080u;
      a[h] = prmt(u, 0, 0x4140), a[2 + h] = prmt(u, 0, 0x4342);
    } else if constexpr (KIND == AF1_KV_E4M3) {
      a[h] = e4m3x2(w[h][ks]), a[2 + h] = e4m3x2(w[h][ks] >> 16);
    } else {
      const uint32_t u = w[h][ks >> 1];
      const int b = 4 * (ks & 1);
      a[h] = u >> b & 0x000f000fu, a[2 + h] = u >> (8 + b) & 0x000f000fu;
    }
  }
}

// The words of one key that a lane holds.
template <typename C, int KIND, int KW, int N>
static __device__ __forceinline__ void load_key(uint32_t (&w)[N], const uint8_t* k, int row, int t) {
  if constexpr (KIND == AF1_KV_INT4) {
#pragma unroll
    for (int c = 0; c < N; ++c) w[c] = *reinterpret_cast<const uint32_t*>(k + C::template at<KW>(row, c) + 4 * t);
  } else {
    constexpr int J = C::SPAN / 64;  // chunks of a slice that a lane holds
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *reinterpret_cast<uint4*>(&w[4 * i]) =
          *reinterpret_cast<const uint4*>(k + C::template at<KW>(row, 8 * (i / J) + J * t + i % J));
  }
}

// One entry of a value in a step's buffers (scaled for INT4, the code alone
// for INT8 and E4M3).
template <int KIND, int DIM, int KW>
static __device__ __forceinline__ float value_entry(const uint8_t* v, const uint8_t* vs, int row, int e) {
  using C = Kv<KIND, DIM>;
  if constexpr (KIND == AF1_KV_F16) {
    return __half2float(*reinterpret_cast<const __half*>(v + C::template at<KW>(row, e / 8) + 2 * (e % 8)));
  } else if constexpr (KIND == AF1_KV_INT4) {
    const uint8_t byte = v[C::template at<KW>(row, e / 32) + (e % 32) / 2];
    const uint32_t s = reinterpret_cast<const uint32_t*>(vs)[row * (DIM / 32) + e / 32];
    return fmaf((float)(e % 2 ? byte >> 4 : byte & 15), low_float(s), high_float(s));
  } else {
    const uint8_t byte = v[C::template at<KW>(row, e / 16) + e % 16];
    if constexpr (KIND == AF1_KV_INT8) return (float)(int8_t)byte;
    else return __half2float(__half(__nv_cvt_fp8_to_halfraw(byte, __NV_E4M3)));
  }
}

// Whether part `part` of `parts` of a value's row holds an infinity or a NaN
// (its 8-bit scale apart).
template <int KIND, int DIM, int KW>
static __device__ __forceinline__ bool value_bad(const uint8_t* v, const uint8_t* vs, int row, int part, int parts) {
  using C = Kv<KIND, DIM>;
  bool bad = false;
  if constexpr (KIND == AF1_KV_INT4) {
    for (int i = part; i < DIM / 32; i += parts) {
      const uint32_t s = reinterpret_cast<const uint32_t*>(vs)[row * (DIM / 32) + i];
      bad |= !(15.f * fabsf(low_float(s)) + fabsf(high_float(s)) <= 65504.f);
    }
  } else if constexpr (KIND != AF1_KV_INT8) {
    for (int i = part; i < C::RB / 16; i += parts) {
      const uint4 c = *reinterpret_cast<const uint4*>(v + C::template at<KW>(row, i));
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (KIND == AF1_KV_F16)
          bad |= (w[j] & 0x7c00u) == 0x7c00u || (w[j] & 0x7c000000u) == 0x7c000000u;
        else
          bad |= __vcmpeq4(w[j] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
      }
    }
  }
  return bad;
}

// Nodes of a sequence's tree.
static __device__ __forceinline__ int node_count(const TreeProblem& p, int seq) {
  return p.counts == nullptr ? p.nodes : min(max(p.counts[seq], 0), p.nodes);
}

// 32 sequences at a time, one to a lane: their lengths, and their units (of
// one cached head and row block) summed up, SETUP of them before the first key
// of an item: what a run of its keys costs whatever its length, in a CTA.
template <int UNIT, int SETUP>
struct Sequences {
  int first;      // of the 32
  int64_t before; // units of the sequences before them
  int len, keys, units, sum;

  __device__ __forceinline__ void load(const TreeProblem& p, int at, int64_t units_before) {
    const int lane = threadIdx.x % 32, i = at + lane;
    first = at;
    before = units_before;
    len = keys = units = 0;
    if (i < p.pages.seqs) {
      len = max(p.lens[i], 0);
      keys = (int)min((int64_t)len + node_count(p, i), (int64_t)p.pages.columns << p.cache.shift);
      units = SETUP + (keys + UNIT - 1) / UNIT;
    }
    sum = units;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += other;
    }
  }
  __device__ __forceinline__ int64_t after() const { return before + __shfl_sync(0xffffffffu, sum, 31); }

  // The first 32 sequences, and the units of all.
  __device__ __forceinline__ int64_t begin(const TreeProblem& p) {
    load(p, 0, 0);
    int64_t total = after();
    for (int at = 32; at < p.pages.seqs; at += 32) {
      load(p, at, total);
      total = after();
    }
    if (p.pages.seqs > 32) load(p, 0, 0);
    return total;
  }
};

// The tensor-core kernel for more than 16 rows to a cached head
// (af1_tree_wide.cu): its workspace bytes, and its launch.
int64_t tree_wide_part_bytes(const af1_kv_cache& c);
cudaError_t launch_tree_wide(TreeProblem& p, const af1_kv_cache& c, int rows, cudaStream_t st);

}  // namespace af1
