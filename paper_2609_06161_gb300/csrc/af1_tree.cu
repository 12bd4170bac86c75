// af1_tree.cu — attention of a few new tokens (a tree of drafted tokens, or
// one token) over a paged cache of keys and values.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i k_j - m_i)
//
// over the keys j that node i sees. The q_heads / kv_heads query heads of all
// nodes that share a cached head are the rows of one product, so that the
// cache is read once for all of them.
//
// Split. An item is one sequence, one cached head and one block of 16 MT
// rows; its keys are cut into units, and every CTA takes an equal run of the
// units of all items (ragged lengths balance by themselves). Inside a CTA
// each warp takes every eighth step of KW keys of a run, with a ring of its
// own in shared memory, its own running maximum m and sum l, and an
// accumulator in registers; warps meet once a run, to join (m, l, o). Where
// an item spans CTAs, each leaves its part in the workspace and the last one
// to arrive joins them in order, so that results do not depend on timing.
//
// Codes become exact FP16 values in registers and go to m16n8k16 products
// (FP32 accumulators). A contraction may run in any order, so the entries of
// a key go to the product's k index in the order in which one lane's 16-byte
// reads give them, and q is laid out to match. The scale of an 8-bit key
// multiplies the scores, that of an 8-bit value the weights p (relative to
// the largest one so far, kept apart); 4-bit codes become scale * code + low,
// rounded once to FP16. p is rounded to FP16 (2^14 times its value, so that
// weights down to 2^-28 keep 11 bits); m, l, scores and outputs are FP32.
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace af1 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCtas = 1024;                    // counters of the workspace
constexpr int64_t kCounterOffset = 256;           // behind the status word's line
constexpr int64_t kPartOffset = kCounterOffset + 4 * kMaxCtas;
constexpr float kShift = 14.f;                    // weights are stored times 2^14
constexpr float kInf = __builtin_huge_valf();

struct TreeProblem {
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
  unsigned* counters;
  float* parts;
};

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) { return __byte_perm(a, b, s); }
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t e4m3x2(uint32_t low16) {
  uint32_t d;
  asm("{\n .reg .b16 l;\n cvt.u16.u32 l, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(d) : "r"(low16));
  return d;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// 16 bytes of global memory to shared memory, the last 16 - bytes of them zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// What the kernel knows of a kind of cache at compile time.
template <int KIND, int DIM>
struct Kv {
  static constexpr int RB = kv_row_bytes(KIND, DIM);    // bytes of a row
  static constexpr int SB = kv_scale_bytes(KIND, DIM);  // bytes of its scales
  static constexpr int CH = RB / 16;                    // 16-byte chunks of a row
  static constexpr int KW = KIND == AF1_KV_F16 ? 16 : 32;  // keys of a warp's step
  static constexpr int KS = DIM / 16;                   // products along a key
  static constexpr int WORDS = RB / 16;                 // 32-bit words of a key that one lane holds
  static constexpr int STAGE = 2 * KW * (RB + SB);      // bytes of a step: k, v, k scales, v scales
  // Byte offset of a chunk of a row in a step's k or v: the chunks of eight
  // neighbouring rows at one place lie in different banks, and so do those
  // that eight neighbouring lanes read of a key.
  static __device__ __forceinline__ int at(int row, int chunk) {
    if constexpr (CH >= 8) return row * RB + ((chunk ^ ((row & 1) << 2 | (row >> 1 & 3))) << 4);
    else if constexpr (CH == 4) return row * RB + ((chunk ^ (row >> 1 & 3)) << 4);
    else return row * RB + ((chunk ^ (row >> 2 & 1)) << 4);
  }
  // Entry of a key that stands at k index pair (e >> 1), place (e & 1), of
  // product ks in the lanes with lane % 4 == t.
  static __device__ __forceinline__ int entry(int t, int ks, int e) {
    if constexpr (KIND == AF1_KV_F16) {
      const int w = 2 * ks + (e >> 1);
      return 8 * (4 * (w / 4) + t) + 2 * (w % 4) + (e & 1);
    } else if constexpr (KIND == AF1_KV_INT4) {
      return (DIM / 4) * t + 8 * (ks >> 1) + 2 * (ks & 1) + (e >> 1) + 4 * (e & 1);
    } else {
      return 16 * (4 * (ks / 4) + t) + 4 * (ks % 4) + e;
    }
  }
  // Entry of a value that stands in column 2 t + i of output block n.
  static __device__ __forceinline__ int column(int t, int n, int i) {
    if constexpr (KIND == AF1_KV_F16) return 8 * n + 2 * t + i;
    else if constexpr (KIND == AF1_KV_INT4) return 32 * (n / 4) + 8 * t + 4 * i + n % 4;
    else return 16 * (n / 2) + 4 * t + 2 * i + n % 2;
  }
};

// The words of one key that a lane holds.
template <typename C>
__device__ __forceinline__ void load_key(uint32_t (&w)[C::WORDS], const uint8_t* k, int row, int t) {
  if constexpr (C::CH >= 4) {
#pragma unroll
    for (int j = 0; j < C::CH / 4; ++j)
      *reinterpret_cast<uint4*>(&w[4 * j]) = *reinterpret_cast<const uint4*>(k + C::at(row, 4 * j + t));
  } else {
    *reinterpret_cast<uint2*>(&w[0]) = *reinterpret_cast<const uint2*>(k + C::at(row, t / 2) + 8 * (t % 2));
  }
}

// b operand of product ks from a lane's words; s2, m2: scale and low of an
// INT4 group, twice.
template <int KIND, int N>
__device__ __forceinline__ void key_operand(uint32_t& b0, uint32_t& b1, const uint32_t (&w)[N], int ks, uint32_t s2,
                                            uint32_t m2) {
  if constexpr (KIND == AF1_KV_F16) {
    b0 = w[2 * ks], b1 = w[2 * ks + 1];
  } else if constexpr (KIND == AF1_KV_INT8) {
    const uint32_t u = w[ks] ^ 0x80808080u;
    b0 = hsub2(prmt(u, 0x64646464u, 0x4140), 0x64806480u);
    b1 = hsub2(prmt(u, 0x64646464u, 0x4342), 0x64806480u);
  } else if constexpr (KIND == AF1_KV_E4M3) {
    b0 = e4m3x2(w[ks]);
    b1 = e4m3x2(w[ks] >> 16);
  } else {
    const uint32_t u = w[ks >> 1] >> (8 * (ks & 1));
    b0 = hfma2(hsub2((u & 0x000f000fu) | 0x64006400u, 0x64006400u), s2, m2);
    b1 = hfma2(hsub2((u >> 4 & 0x000f000fu) | 0x64006400u, 0x64006400u), s2, m2);
  }
}

// b operand of output block i of a chunk, from a transposed 16-bit word of
// two keys; s2, m2: scale and low of the two keys (INT4).
template <int KIND>
__device__ __forceinline__ uint32_t value_operand(uint32_t r, int i, uint32_t s2, uint32_t m2) {
  if constexpr (KIND == AF1_KV_F16) {
    return r;
  } else if constexpr (KIND == AF1_KV_INT8) {
    return hsub2(prmt(r ^ 0x80808080u, 0x64646464u, i == 0 ? 0x4240 : 0x4341), 0x64806480u);
  } else if constexpr (KIND == AF1_KV_E4M3) {
    return e4m3x2(prmt(r, r, i == 0 ? 0x0020 : 0x0031));
  } else {
    return hfma2(hsub2((r >> (4 * i) & 0x000f000fu) | 0x64006400u, 0x64006400u), s2, m2);
  }
}

// One entry of a value in a step's buffers (scaled by its own scale for
// INT4, as the code alone for INT8 and E4M3).
template <int KIND, int DIM>
__device__ __forceinline__ float value_entry(const uint8_t* v, const uint8_t* vs, int row, int e) {
  using C = Kv<KIND, DIM>;
  if constexpr (KIND == AF1_KV_F16) {
    return __half2float(*reinterpret_cast<const __half*>(v + C::at(row, e / 8) + 2 * (e % 8)));
  } else if constexpr (KIND == AF1_KV_INT4) {
    const uint8_t byte = v[C::at(row, e / 32) + (e % 32) / 2];
    const __half2 s = reinterpret_cast<const __half2*>(vs)[row * (DIM / 32) + e / 32];
    return __half2float(__hfma(__int2half_rn(e % 2 ? byte >> 4 : byte & 15), __low2half(s), __high2half(s)));
  } else {
    const uint8_t byte = v[C::at(row, e / 16) + e % 16];
    if constexpr (KIND == AF1_KV_INT8) return (float)(int8_t)byte;
    else return __half2float(__half(__nv_cvt_fp8_to_halfraw(byte, __NV_E4M3)));
  }
}

// Whether part `part` of `parts` of a value's row holds an infinity or a NaN
// (its 8-bit scale apart).
template <int KIND, int DIM>
__device__ __forceinline__ bool value_bad(const uint8_t* v, const uint8_t* vs, int row, int part, int parts) {
  using C = Kv<KIND, DIM>;
  bool bad = false;
  if constexpr (KIND == AF1_KV_INT4) {
    for (int i = part; i < DIM / 32; i += parts) {
      const uint32_t s = reinterpret_cast<const uint32_t*>(vs)[row * (DIM / 32) + i];
      bad |= (s & 0x7c00u) == 0x7c00u || (s & 0x7c000000u) == 0x7c000000u;
    }
  } else if constexpr (KIND != AF1_KV_INT8) {
    for (int i = part; i < C::CH; i += parts) {
      const uint4 c = *reinterpret_cast<const uint4*>(v + C::at(row, i));
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

struct Run {  // a CTA's run of units within one item
  int seq, head, tile;
  int u0, u1, units;  // units u0 .. u1 - 1 of the item's `units`
  int len, keys;      // cached tokens, and keys with the nodes'
  int64_t first;      // the item's first unit in the order of all items
};

__device__ __forceinline__ int node_count(const TreeProblem& p, int seq) {
  return p.counts == nullptr ? p.nodes : min(max(p.counts[seq], 0), p.nodes);
}

// Prefix sums over sequences of units (of one cached head and row tile), by
// the whole CTA. An item without keys has one unit, that writes its zeros.
__device__ __forceinline__ int64_t scan_units(const TreeProblem& p, int unit, int64_t* prefix, int64_t* scratch) {
  const int per = (p.pages.seqs + kThreads - 1) / kThreads;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int first = threadIdx.x * per;
  const int cap = p.pages.columns << p.cache.shift;
  int64_t sum = 0;
  for (int i = first; i < min(first + per, p.pages.seqs); ++i) {
    const int keys = (int)min((int64_t)max(p.lens[i], 0) + node_count(p, i), (int64_t)cap);
    sum += max(1, (keys + unit - 1) / unit);
    prefix[i + 1] = sum;
  }
  int64_t up = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t other = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += other;
  }
  if (lane == 31) scratch[warp] = up;
  __syncthreads();
  int64_t before = up - sum, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  for (int i = first; i < min(first + per, p.pages.seqs); ++i) prefix[i + 1] += before;
  if (threadIdx.x == 0) prefix[0] = 0;
  __syncthreads();
  return total;
}

template <int KIND, int DIM, int MT, int STAGES>
__global__ void __launch_bounds__(kThreads, 1) tree_kernel(const __grid_constant__ TreeProblem p) {
  using C = Kv<KIND, DIM>;
  constexpr int KW = C::KW, NB = KW / 8, KS = C::KS, ON = DIM / 8, ROWS = 16 * MT;
  constexpr int PART = ROWS * (DIM + 2);  // floats of a part: o, m, l
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t scratch[kWarps];
  __shared__ uint8_t bad_pages[kWarps][STAGES];
  __shared__ float join_m[kWarps][ROWS], join_l[kWarps][ROWS];
  __shared__ bool last_shared;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int g = lane / 4, t = lane % 4;
  uint8_t* ring = smem + warp * (STAGES * C::STAGE);
  const uint32_t ring_u32 = smem_u32(ring);
  uint32_t* qs = reinterpret_cast<uint32_t*>(smem + kWarps * STAGES * C::STAGE);  // MT > 1: q's operands
  int64_t* prefix = reinterpret_cast<int64_t*>(smem + kWarps * STAGES * C::STAGE + (MT > 1 ? MT * KS * 512 : 0));
  float* join = reinterpret_cast<float*>(smem);  // after a run: the warps' o

  // Units of 8 steps, or fewer where that would leave CTAs without work.
  int unit = KW * kWarps;
  const int64_t lanes = (int64_t)p.cache.heads * p.row_tiles;
  int64_t per_head = scan_units(p, unit, prefix, scratch);
  while (per_head * lanes < gridDim.x && unit > 2 * KW) {
    unit /= 2;
    per_head = scan_units(p, unit, prefix, scratch);
  }
  const int64_t total = per_head * lanes;
  const int64_t ctas = min((int64_t)gridDim.x, total);  // each has a unit at least
  if (blockIdx.x >= ctas) return;
  const int64_t begin = total * blockIdx.x / ctas, end = total * (blockIdx.x + 1) / ctas;

  int64_t pos = begin;
  int seq = 0;
  {
    int hi = p.pages.seqs;  // the last sequence whose first unit is not after pos
    while (hi - seq > 1) {
      const int mid = (seq + hi) / 2;
      if (prefix[mid] * lanes <= pos) seq = mid;
      else hi = mid;
    }
  }
  while (pos < end) {
    while (prefix[seq + 1] * lanes <= pos) ++seq;
    Run r;
    r.seq = seq;
    r.units = (int)(prefix[seq + 1] - prefix[seq]);
    const int64_t local = pos - prefix[seq] * lanes;
    const int item = (int)(local / r.units);
    r.u0 = (int)(local - (int64_t)item * r.units);
    r.u1 = (int)min((int64_t)r.units, r.u0 + (end - pos));
    r.first = pos - r.u0;
    r.head = item / p.row_tiles;
    r.tile = item - r.head * p.row_tiles;
    r.len = max(p.lens[seq], 0);
    const int count = node_count(p, seq);
    r.keys = (int)min((int64_t)r.len + count, (int64_t)p.pages.columns << p.cache.shift);
    const int rows = min(ROWS, p.nodes * p.group - r.tile * ROWS);
    const int k_begin = r.u0 * unit, k_end = min(r.u1 * unit, r.keys);

    // -- copies -------------------------------------------------------------
    const int32_t* page_row = p.pages.pages + seq * p.pages.ld;
    int next_page[KW / 16];
    auto fetch_pages = [&](int key) {
#pragma unroll
      for (int i = 0; i < KW / 16; ++i) {
        const int k = key + 16 * i;
        next_page[i] = k < k_end ? page_row[k >> p.cache.shift] : -1;
      }
    };
    auto issue = [&](int key, int slot) {  // the step of KW keys at `key`, whose pages were fetched
      const uint32_t dst = ring_u32 + slot * C::STAGE;
      int64_t base[KW / 16];
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < KW / 16; ++i) {
        const int k = key + 16 * i;
        const bool ok = next_page[i] >= 0 && next_page[i] < p.cache.pages;
        if (!ok && k < k_end) bad |= 1u << i;
        base[i] = ok ? (((int64_t)next_page[i] * p.cache.heads + r.head) << p.cache.shift) +
                           (k & ((1 << p.cache.shift) - 1))
                     : -1;
      }
#pragma unroll
      for (int i = 0; i < KW * C::CH / 32; ++i) {
        const int row = (i * 32 + lane) / C::CH, ch = lane % C::CH;
        const int64_t b = base[(i * 32) / C::CH / 16];  // 32 lanes stay within 16 rows
        const bool ok = b >= 0 && key + row < k_end;
        const int64_t off = ok ? (b + row % 16) * C::RB + ch * 16 : 0;
        copy16(dst + C::at(row, ch), p.cache.k + off, ok ? 16 : 0);
        copy16(dst + KW * C::RB + C::at(row, ch), p.cache.v + off, ok ? 16 : 0);
      }
      if constexpr (C::SB > 0) {
        constexpr int KEYS = 16 / C::SB;  // keys of a 16-byte piece of scales
        constexpr int PIECES = KW / KEYS;
#pragma unroll
        for (int i = 0; i < 2 * PIECES; i += 32) {
          const int id = i + lane;
          if (id < 2 * PIECES) {
            const bool is_v = id >= PIECES;
            const int row = (id - (is_v ? PIECES : 0)) * KEYS;
            const int64_t b = KW == 16 || row < 16 ? base[0] : base[KW / 16 - 1];
            const int have = b >= 0 ? min(max(k_end - key - row, 0), KEYS) * C::SB : 0;
            const uint8_t* src = static_cast<const uint8_t*>(is_v ? p.cache.vs : p.cache.ks);
            copy16(dst + 2 * KW * C::RB + (is_v ? KW * C::SB : 0) + row * C::SB,
                   src + (have > 0 ? (b + row % 16) * C::SB : 0), have);
          }
        }
      }
      if (lane == 0) bad_pages[warp][slot] = (uint8_t)bad;
    };

    const int key0 = k_begin + warp * KW;  // this warp's steps: key0, key0 + kWarps KW, ...
    constexpr int STRIDE = kWarps * KW;
    fetch_pages(key0);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
      if (key0 + s * STRIDE < k_end) {
        issue(key0 + s * STRIDE, s);
        fetch_pages(key0 + (s + 1) * STRIDE);
      }
      copy_commit();
    }

    // -- q, laid out for the products ------------------------------------------
    auto q_operand = [&](int mt, int ks, uint32_t (&a)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int lr = mt * 16 + g + 8 * (i & 1);
        uint32_t v = 0;
        if (lr < rows) {
          const int gr = r.tile * ROWS + lr, node = gr / p.group;
          const __half* row = p.q + seq * p.q_seq + node * p.q_node + (int64_t)(r.head * p.group + gr % p.group) * p.q_head;
          const int e0 = C::entry(t, ks, 2 * (i >> 1));
          if constexpr (KIND == AF1_KV_INT4)
            v = (uint32_t)__half_as_ushort(row[e0]) | (uint32_t)__half_as_ushort(row[e0 + 4]) << 16;
          else
            v = *reinterpret_cast<const uint32_t*>(row + e0);
        }
        a[i] = v;
      }
    };
    uint32_t qf[MT == 1 ? KS : 1][4];
    if constexpr (MT == 1) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q_operand(0, ks, qf[ks]);
    } else {
      for (int i = warp; i < MT * KS; i += kWarps) {
        uint32_t a[4];
        q_operand(i / KS, i % KS, a);
        reinterpret_cast<uint4*>(qs)[i * 32 + lane] = make_uint4(a[0], a[1], a[2], a[3]);
      }
      __syncthreads();
    }

    float o[MT][ON][4], m[MT][2], l[MT][2], vref = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int n = 0; n < ON; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
      m[mt][0] = m[mt][1] = -kInf, l[mt][0] = l[mt][1] = 0.f;
    }

    // -- steps ---------------------------------------------------------------------
    int slot = 0;
    for (int key = key0; key < k_end; key += STRIDE) {
      copy_wait<STAGES - 2>();
      __syncwarp();
      {
        const int ahead = key + (STAGES - 1) * STRIDE;
        int to = slot + STAGES - 1;
        if (to >= STAGES) to -= STAGES;
        if (ahead < k_end) {
          issue(ahead, to);
          fetch_pages(ahead + STRIDE);
        }
        copy_commit();
      }
      const uint8_t* kb = ring + slot * C::STAGE;
      const uint8_t* vb = kb + KW * C::RB;
      const uint8_t* ksb = kb + 2 * KW * C::RB;
      const uint8_t* vsb = ksb + KW * C::SB;
      const uint32_t bad = bad_pages[warp][slot];

      float s[MT][NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        uint32_t w[C::WORDS];
        load_key<C>(w, kb, nb * 8 + g, t);
        uint32_t s2 = 0, m2 = 0;
        if constexpr (KIND == AF1_KV_INT4) {
          const uint32_t sm = reinterpret_cast<const uint32_t*>(ksb)[(nb * 8 + g) * (DIM / 32) + t * (DIM / 32) / 4];
          s2 = prmt(sm, sm, 0x1010), m2 = prmt(sm, sm, 0x3232);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) s[mt][nb][0] = s[mt][nb][1] = s[mt][nb][2] = s[mt][nb][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t b0, b1;
          key_operand<KIND>(b0, b1, w, ks, s2, m2);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            if constexpr (MT == 1) {
              mma(s[mt][nb], qf[ks], b0, b1);
            } else {
              uint4 a = reinterpret_cast<const uint4*>(qs)[(mt * KS + ks) * 32 + lane];
              const uint32_t aa[4] = {a.x, a.y, a.z, a.w};
              mma(s[mt][nb], aa, b0, b1);
            }
          }
        }
        float c0 = p.scale_log2, c1 = p.scale_log2;
        if constexpr (KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3) {
          const float2 sc = *reinterpret_cast<const float2*>(ksb + (nb * 8 + 2 * t) * 4);
          c0 *= sc.x, c1 *= sc.y;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          s[mt][nb][0] *= c0, s[mt][nb][1] *= c1;
          s[mt][nb][2] *= c0, s[mt][nb][3] *= c1;
        }
      }

      // Steps with nodes, with keys past the end or with missing pages.
      const bool masked = key + KW > min(r.len, k_end) || bad != 0;
      if (masked) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int lr = mt * 16 + g + 8 * hf;
            uint64_t bits = 0;
            if (lr < rows) {
              const int node = (r.tile * ROWS + lr) / p.group;
              if (p.mask == nullptr) {
                bits = (2ull << node) - 1;
              } else {
                const uint32_t* w = p.mask + seq * p.mask_seq + node * p.words;
                bits = w[0] | (p.words > 1 ? (uint64_t)w[1] << 32 : 0);
              }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int at = nb * 8 + 2 * t + i, k = key + at;
                const bool sees = k < k_end && !(bad >> (at / 16) & 1) && (k < r.len || (bits >> (k - r.len) & 1));
                if (!sees) s[mt][nb][2 * hf + i] = -kInf;
              }
          }
      }

      // Running maximum; o and l follow it.
      float alpha[MT][2], ref[MT][2];
      bool moved = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float top = fmaxf(s[mt][0][2 * hf], s[mt][0][2 * hf + 1]);
#pragma unroll
          for (int nb = 1; nb < NB; ++nb) top = fmaxf(top, fmaxf(s[mt][nb][2 * hf], s[mt][nb][2 * hf + 1]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float now = fmaxf(m[mt][hf], top);
          moved |= now > m[mt][hf];
          const float zero = now == -kInf ? 0.f : now;
          alpha[mt][hf] = ex2(m[mt][hf] - zero);
          m[mt][hf] = now;
          ref[mt][hf] = zero - kShift;
        }
      float vinv = 0.f;
      if constexpr (KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3) {
        const float vs = reinterpret_cast<const float*>(vsb)[lane];
        // Non-negative floats order as their bits.
        const uint32_t top = __reduce_max_sync(0xffffffffu, fabsf(vs) < kInf ? __float_as_uint(fabsf(vs)) : 0u);
        const float now = fmaxf(vref, __uint_as_float(top));
        if (now > vref) {
          const float f = vref / now;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < ON; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[mt][n][i] *= f;
          vref = now;
        }
        vinv = vref > 0.f ? 1.f / vref : 0.f;
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) l[mt][hf] *= alpha[mt][hf];
#pragma unroll
          for (int n = 0; n < ON; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[mt][n][i] *= alpha[mt][i / 2];
        }
      }

      // Weights.
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float2 vsc = make_float2(1.f, 1.f);
        if constexpr (KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3) {
          vsc = *reinterpret_cast<const float2*>(vsb + (nb * 8 + 2 * t) * 4);
          vsc.x *= vinv, vsc.y *= vinv;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = ex2(s[mt][nb][i] - ref[mt][i / 2]);
            l[mt][i / 2] += w;
            if constexpr (KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3)
              s[mt][nb][i] = masked && !(w > 0.f) ? 0.f : w * (i % 2 ? vsc.y : vsc.x);
            else
              s[mt][nb][i] = w;
          }
      }

      // A node's infinite or NaN value must not reach the rows that do not
      // see it, as 0 times it would: such steps sum entry by entry.
      bool slow = false;
      if (masked) {
        constexpr int PARTS = 32 / KW;
        slow = __any_sync(0xffffffffu, value_bad<KIND, DIM>(vb, vsb, lane % KW, lane / KW, PARTS));
      }
      if (slow) {
        for (int j = 0; j < KW; ++j) {
          const int from = (lane & ~3) | (j % 8) / 2;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            float w[2];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              float mine = 0.f;
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (nb == j / 8 && i == j % 2) mine = s[mt][nb][2 * hf + i];
              w[hf] = __shfl_sync(0xffffffffu, mine, from);
            }
#pragma unroll
            for (int n = 0; n < ON; ++n)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float v = value_entry<KIND, DIM>(vb, vsb, j, C::column(t, n, i));
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                  if (w[hf] != 0.f) o[mt][n][2 * hf + i] += w[hf] * v;
              }
          }
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < KW / 16; ++kk) {
          uint32_t a[MT][4];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            a[mt][0] = pack_half2(s[mt][2 * kk][0], s[mt][2 * kk][1]);
            a[mt][1] = pack_half2(s[mt][2 * kk][2], s[mt][2 * kk][3]);
            a[mt][2] = pack_half2(s[mt][2 * kk + 1][0], s[mt][2 * kk + 1][1]);
            a[mt][3] = pack_half2(s[mt][2 * kk + 1][2], s[mt][2 * kk + 1][3]);
          }
          const int row = kk * 16 + (lane & 15);
#pragma unroll
          for (int c = 0; c < C::CH; c += 2) {
            uint32_t v[4];
            ldmatrix_x4_trans(v, smem_u32(vb) + C::at(row, c + (lane >> 4)));
#pragma unroll
            for (int cc = 0; cc < 2; ++cc) {
              uint32_t s2[2] = {0, 0}, m2[2] = {0, 0};
              if constexpr (KIND == AF1_KV_INT4) {
                const uint32_t* sm = reinterpret_cast<const uint32_t*>(vsb) + (kk * 16 + 2 * t) * (DIM / 32) + c + cc;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                  const uint32_t x = sm[hf * 8 * (DIM / 32)], y = sm[(hf * 8 + 1) * (DIM / 32)];
                  s2[hf] = prmt(x, y, 0x5410), m2[hf] = prmt(x, y, 0x7632);
                }
              }
              constexpr int BLOCKS = ON / C::CH;  // output blocks of a chunk
#pragma unroll
              for (int i = 0; i < BLOCKS; ++i) {
                const uint32_t b0 = value_operand<KIND>(v[2 * cc], i, s2[0], m2[0]);
                const uint32_t b1 = value_operand<KIND>(v[2 * cc + 1], i, s2[1], m2[1]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma(o[mt][(c + cc) * BLOCKS + i], a[mt], b0, b1);
              }
            }
          }
        }
      }
      if (++slot == STAGES) slot = 0;
      __syncwarp();
    }
    copy_wait<0>();
    __syncthreads();  // every warp is done with its ring

    // -- join the warps' parts -------------------------------------------------------
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float sum = l[mt][hf];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const int lr = mt * 16 + g + 8 * hf;
        if (t == 0) join_m[warp][lr] = m[mt][hf], join_l[warp][lr] = sum;
        if (lr < rows) {
          float* to = join + (warp * ROWS + lr) * DIM;
          const float f = KIND == AF1_KV_INT8 || KIND == AF1_KV_E4M3 ? vref : 1.f;
#pragma unroll
          for (int n = 0; n < ON; ++n) {
            to[C::column(t, n, 0)] = o[mt][n][2 * hf] * f;
            to[C::column(t, n, 1)] = o[mt][n][2 * hf + 1] * f;
          }
        }
      }
    __syncthreads();
    const bool whole = r.u0 == 0 && r.u1 == r.units;
    // This run's place in the workspace: a CTA has at most two runs of parts,
    // its first and its last.
    auto part_of = [&](int cta) {
      const int64_t from = total * cta / ctas;
      return p.parts + (int64_t)(2 * cta + (from >= r.first ? 0 : 1)) * PART;
    };
    float* part = whole ? nullptr : part_of(blockIdx.x);
    auto finish = [&](int lr, int e, float mx, float sum, float acc) {
      const int gr = r.tile * ROWS + lr, node = gr / p.group, h = r.head * p.group + gr % p.group;
      const bool live = node < count && sum != 0.f;
      const float y = live ? acc / sum : 0.f;
      const int64_t at = seq * p.o_seq + node * p.o_node + h * p.o_head + e;
      if (p.out_f32) static_cast<float*>(p.out)[at] = y;
      else static_cast<__half*>(p.out)[at] = __float2half_rn(y);
      if (e == 0 && p.lse != nullptr)
        p.lse[((int64_t)seq * p.nodes + node) * p.cache.heads * p.group + h] =
            live ? (mx - kShift + log2f(sum)) * 0.69314718056f : -kInf;
    };
    for (int i = threadIdx.x; i < rows * DIM; i += kThreads) {
      const int lr = i / DIM, e = i % DIM;
      float mx = -kInf;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, join_m[w][lr]);
      const float zero = mx == -kInf ? 0.f : mx;
      float sum = 0.f, acc = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ex2(join_m[w][lr] - zero);
        sum += f * join_l[w][lr];
        acc += f * join[(w * ROWS + lr) * DIM + e];
      }
      if (whole) {
        finish(lr, e, mx, sum, acc);
      } else {
        part[lr * DIM + e] = acc;
        if (e == 0) part[ROWS * DIM + lr] = mx, part[ROWS * DIM + ROWS + lr] = sum;
      }
    }
    if (!whole) {
      // CTAs first .. last hold the item's units; the last to arrive joins.
      const int64_t item_end = r.first + r.units;
      auto holder = [&](int64_t u) {
        int64_t c = u * ctas / total;
        while (total * (c + 1) / ctas <= u) ++c;
        return (int)c;
      };
      const int c0 = holder(r.first), c1 = holder(item_end - 1);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        const unsigned arrived = atom_add_acq_rel_gpu(&p.counters[c0], 1u);
        last_shared = arrived == (unsigned)(c1 - c0);
        if (last_shared) p.counters[c0] = 0;  // as the next call finds it
      }
      __syncthreads();
      if (last_shared) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * DIM; i += kThreads) {
          const int lr = i / DIM, e = i % DIM;
          float mx = -kInf, sum = 0.f, acc = 0.f;
          for (int c = c0; c <= c1; ++c) {
            const float* from = part_of(c);
            const float pm = __ldcg(from + ROWS * DIM + lr);
            const float now = fmaxf(mx, pm);
            const float zero = now == -kInf ? 0.f : now;
            const float fa = ex2(mx - zero), fb = ex2(pm - zero);
            sum = sum * fa + __ldcg(from + ROWS * DIM + ROWS + lr) * fb;
            acc = acc * fa + __ldcg(from + lr * DIM + e) * fb;
            mx = now;
          }
          finish(lr, e, mx, sum, acc);
        }
      }
    }
    __syncthreads();  // join, join_m and qs are free again
    pos += r.u1 - r.u0;
  }
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_tree_attention: " + msg); }

// Rows (of every query head and node that share a cached head) of a CTA.
int row_blocks(int64_t rows) { return rows <= 16 ? 1 : 2; }

int64_t workspace_bytes(const af1_kv_cache& c, int64_t rows) {
  const int64_t ctas = std::min(c.num_sms, kMaxCtas);
  return kPartOffset + 2 * ctas * (16 * row_blocks(rows)) * (c.d.head_dim + 2) * 4;
}

template <int KIND, int DIM, int MT>
int launch(const TreeProblem& p, int ctas, int max_smem, cudaStream_t st) {
  using C = Kv<KIND, DIM>;
  constexpr int STAGES = C::STAGE * kWarps * 4 <= 200 * 1024 ? 4 : 3;
  static_assert(STAGES * C::STAGE >= 16 * MT * DIM * 4, "the warps' outputs are joined in their rings");
  const int smem = kWarps * STAGES * C::STAGE + (MT > 1 ? MT * C::KS * 512 : 0) + 8 * (p.pages.seqs + 1);
  auto kernel = tree_kernel<KIND, DIM, MT, STAGES>;
  cudaError_t e = smem <= max_smem ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)
                                   : cudaErrorInvalidValue;
  if (e == cudaSuccess) {
    kernel<<<ctas, kThreads, smem, st>>>(p);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}

template <int KIND>
int launch_kind(const TreeProblem& p, int dim, int mt, int ctas, int max_smem, cudaStream_t st) {
  if (dim == 128) return mt == 1 ? launch<KIND, 128, 1>(p, ctas, max_smem, st) : launch<KIND, 128, 2>(p, ctas, max_smem, st);
  return mt == 1 ? launch<KIND, 64, 1>(p, ctas, max_smem, st) : launch<KIND, 64, 2>(p, ctas, max_smem, st);
}

bool sizes_ok(const af1_kv_cache* c, int64_t sequences, int64_t nodes, int64_t q_heads) {
  return sequences >= 0 && sequences <= 1024 && nodes >= 1 && nodes <= 64 && q_heads >= 1 && q_heads <= 65536 &&
         q_heads % c->d.kv_heads == 0;
}
const char kSizes[] = "need 0..1024 sequences, 1..64 nodes and q_heads a multiple of the cache's kv_heads";

}  // namespace
}  // namespace af1

using namespace af1;

int64_t af1_tree_workspace_bytes(const af1_kv_cache* c, int64_t sequences, int64_t nodes, int64_t q_heads) {
  if (c == nullptr) return fail(AF1_ERR_INVALID_ARG, "cache is NULL");
  if (!sizes_ok(c, sequences, nodes, q_heads)) return fail(AF1_ERR_INVALID_ARG, kSizes);
  return workspace_bytes(*c, nodes * (q_heads / c->d.kv_heads));
}

int af1_tree_attention(const af1_kv_cache* c, const af1_tree_args* a, void* workspace, int64_t bytes, void* stream) {
  if (c == nullptr || a == nullptr) return fail(AF1_ERR_INVALID_ARG, "cache or args is NULL");
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return fail(AF1_ERR_CUDA, cudaGetErrorString(e));
  if (dev != c->device) return fail(AF1_ERR_BAD_POINTER, "the current device is not the cache's device");
  if (!sizes_ok(c, a->sequences, a->nodes, a->q_heads)) return fail(AF1_ERR_INVALID_ARG, kSizes);
  if (a->out_dtype != AF1_F16 && a->out_dtype != AF1_F32)
    return fail(AF1_ERR_INVALID_ARG, "out_dtype must be AF1_F16 or AF1_F32");
  if (!(std::abs(a->scale) <= 3e38f)) return fail(AF1_ERR_INVALID_ARG, "scale must be finite");
  if (a->page_columns < 1 || a->pages_ld < a->page_columns || a->pages_ld > ((int64_t)1 << 40) ||
      a->page_columns > ((int64_t)1 << 30) / c->d.page_size)
    return fail(AF1_ERR_INVALID_ARG, "need page columns of at most 2^30 slots in all and pages_ld >= page_columns");
  const int64_t most = (int64_t)1 << 40;
  const int64_t strides[7] = {a->q_seq, a->q_node, a->q_head, a->o_seq, a->o_node, a->o_head, a->mask_seq};
  for (int i = 0; i < 7; ++i)
    if (strides[i] < 0 || strides[i] > most) return fail(AF1_ERR_INVALID_ARG, "strides must be 0..2^40");
  if (a->sequences == 0) return AF1_OK;
  const int o_unit = a->out_dtype == AF1_F16 ? 8 : 4;
  for (int i = 0; i < 6; ++i)
    if (strides[i] % (i < 3 ? 8 : o_unit) != 0)
      return fail(AF1_ERR_MISALIGNED, "strides of q must be multiples of 8, of out of 8 (FP16) or 4 (FP32)");
  struct {
    const void* p;
    const char* name;
    int align;
    bool need;
  } ptrs[] = {{a->q, "q", 16, true},        {a->out, "out", 16, true},        {a->pages, "pages", 4, true},
              {a->lens, "lens", 4, true},   {a->counts, "counts", 4, false}, {a->mask, "mask", 4, false},
              {a->lse, "lse", 4, false}};
  int rc;
  for (const auto& t : ptrs) {
    if (t.p == nullptr && !t.need) continue;
    if ((rc = check_pointer(t.p, t.name, dev)) != AF1_OK || (rc = check_align(t.p, t.align, t.name)) != AF1_OK) return rc;
  }
  const int group = (int)(a->q_heads / c->d.kv_heads);
  const int64_t rows = a->nodes * group;
  if (workspace == nullptr || (uintptr_t)workspace % 256 != 0 || bytes < workspace_bytes(*c, rows))
    return fail(AF1_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                       std::to_string(workspace_bytes(*c, rows)) + " bytes");
  if (check_pointer(workspace, "workspace", dev) != AF1_OK) return fail(AF1_ERR_WORKSPACE, "workspace is not device memory");
  const int mt = row_blocks(rows);
  TreeProblem p = {};
  p.q = static_cast<const __half*>(a->q);
  p.q_seq = a->q_seq, p.q_node = a->q_node, p.q_head = a->q_head;
  p.out = a->out;
  p.o_seq = a->o_seq, p.o_node = a->o_node, p.o_head = a->o_head;
  p.lse = a->lse;
  p.cache = view_of(c->d);
  p.pages = {a->pages, a->pages_ld, (int)a->sequences, (int)a->page_columns};
  p.lens = a->lens, p.counts = a->counts, p.mask = a->mask, p.mask_seq = a->mask_seq;
  p.nodes = (int)a->nodes, p.group = group, p.words = (int)(a->nodes + 31) / 32;
  p.row_tiles = (int)((rows + 16 * mt - 1) / (16 * mt));
  p.scale_log2 = a->scale * 1.4426950408889634f;
  p.out_f32 = a->out_dtype == AF1_F32;
  p.counters = reinterpret_cast<unsigned*>(static_cast<uint8_t*>(workspace) + kCounterOffset);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kPartOffset);
  const int ctas = std::min(c->num_sms, kMaxCtas);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (c->d.kind) {
    case AF1_KV_F16: return launch_kind<AF1_KV_F16>(p, c->d.head_dim, mt, ctas, c->max_smem, st);
    case AF1_KV_INT8: return launch_kind<AF1_KV_INT8>(p, c->d.head_dim, mt, ctas, c->max_smem, st);
    case AF1_KV_E4M3: return launch_kind<AF1_KV_E4M3>(p, c->d.head_dim, mt, ctas, c->max_smem, st);
    default: return launch_kind<AF1_KV_INT4>(p, c->d.head_dim, mt, ctas, c->max_smem, st);
  }
}
