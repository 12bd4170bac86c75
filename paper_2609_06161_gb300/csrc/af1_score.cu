// af1_score.cu — log-probabilities of given tokens, entropy and the largest
// alternatives of rows of logits, in one pass over the logits.
//
// With c = log2(e) / temperature, a thread keeps a reference r (the largest x
// so far), S = sum 2^d and T = sum 2^d d over its entries, d = (x - r) c, and
// follows a new maximum by S' = f S, T' = f (T + S delta). Then
//   log p = (d - log2 S) ln 2,   entropy = (log2 S - T / S) ln 2.
// The difference comes before the factor at every temperature and for both
// types: d of the largest entry is then 0, where x c less a rounded r c would
// leave it half a unit in the last place of r c, which low temperatures raise
// past every exponent; and x c itself may overflow where d does not.
//
// The largest entries. Passing over the logits, a warp only keeps its lanes'
// maxima of every batch (of 16 or 32 entries to a lane). Every kSegment batches
// it looks back: if ceil(top / warps) lanes of every warp, or `top` lanes of
// this one, have a maximum of at least some bound, `top` entries of the row
// have, so only batches of lanes whose maximum is not below it are read again
// (about 8 to a warp, for the 20 largest of 128001 in random order), and their entries
// that are not below it are merged into the warp's list of its 32 largest, one
// to a lane, in order. Keys of 64 bits (the value as an ordered integer, then
// the index, inverted) make the order total, so that equal values go by index
// and the result does not depend on which thread saw what first. (With entries
// compared with the list as they came by, warps waited on their lists: 512 rows
// of 128001 FP16 logits took 45 us with the 20 largest where 25 without.)
//
// A cluster of CTAs takes a row (one CTA where there are rows enough to fill
// the GPU), and its first CTA joins their statistics and lists through
// distributed shared memory. Logits come by asynchronous copies, three batches of a
// warp in flight. Large calls are bound by device memory and the look back:
// those 512 rows take 33.4 us (3.9 TB/s), 27 without the largest; the pass
// itself costs one exponent and about five instructions an entry (pairs of
// entries share FP32 additions, products and multiply-adds). Small launches are bound
// by the latency of lists and joins: 5 rows of 32000 FP32 logits take 7.5 us on the
// GPU (a call from Python, which allocates four outputs, 20).
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCluster = 8;
constexpr int kSegment = 32;  // batches
constexpr float kInf = __builtin_huge_valf();

struct ScoreProblem {
  const void* logits;
  int64_t vocab, ld;
  const int32_t* tokens;
  int given;
  float *logprobs, *entropy, *top_logprobs;
  int32_t* top_ids;
  int top;
  float c;      // log2(e) / temperature
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ __half max_nan(__half a, __half b) { return __hmax_nan(a, b); }
constexpr float kLeast = -1e4f;  // 2^d is 0 from far above on; d itself may be -infinity

// r is -infinity where nothing is summed (or NaN alone).
struct Stats {
  float r = -kInf, s = 0.f, t = 0.f;
};
// The two sets of entries together.
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float c) {
  Stats o;
  o.r = fmaxf(a.r, b.r);
  if (o.r == -kInf) {
    o.s = a.s + b.s, o.t = 0.f;  // nothing, or NaN
    return o;
  }
  const float da = fmaxf((a.r - o.r) * c, kLeast), db = fmaxf((b.r - o.r) * c, kLeast);
  const float fa = ex2(da), fb = ex2(db);
  o.s = a.s * fa + b.s * fb;
  o.t = fa * (a.t + a.s * da) + fb * (b.t + b.s * db);
  return o;
}

// Larger for larger values (NaN largest, -0 as 0), then for smaller indices; never 0.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t index) {
  const int32_t b = __float_as_int(x + 0.f);
  const uint32_t k = x != x ? 0xffffffffu : (uint32_t)(b ^ ((b >> 31) | (int32_t)0x80000000));
  return (uint64_t)k << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t k = (uint32_t)(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// Entries below it cannot come before the key (-infinity for NaN or no key: none is).
__device__ __forceinline__ float key_bound(uint64_t key) {
  const float v = key_value(key);
  return key == 0 || v != v ? -kInf : v;
}
__device__ __forceinline__ float sort_descending(float x, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int d = size / 2; d > 0; d >>= 1) {
      const float other = __shfl_xor_sync(0xffffffffu, x, d);
      const bool down = size == 32 || (lane & size) == 0;
      x = ((lane & d) == 0) == down ? fmaxf(x, other) : fminf(x, other);
    }
  return x;
}

// One key to a lane: descending.
__device__ __forceinline__ uint64_t merge_step(uint64_t k, int lane, int d, bool down) {
  const uint64_t other = __shfl_xor_sync(0xffffffffu, k, d);
  const bool want_max = ((lane & d) == 0) == down;
  return want_max == (other > k) ? other : k;
}
__device__ __forceinline__ uint64_t warp_sort(uint64_t k, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int d = size / 2; d > 0; d >>= 1) k = merge_step(k, lane, d, size == 32 || (lane & size) == 0);
  return k;
}
// The 32 largest of two descending lists.
__device__ __forceinline__ uint64_t merge_lists(uint64_t a, uint64_t b, int lane) {
  const uint64_t r = __shfl_sync(0xffffffffu, b, 31 - lane);
  uint64_t k = a > r ? a : r;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) k = merge_step(k, lane, d, true);
  return k;
}

// 16 bytes to shared memory, as part of the thread's next group of copies.
__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads, 5) score_kernel(const __grid_constant__ ScoreProblem p) {
  constexpr int E = 16 / (int)sizeof(T);  // entries of a 16-byte access
  constexpr int U = 4;                    // accesses of a batch: 16 or 32 entries to a lane
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int STAGES = TOP && !HALF ? 3 : 4;  // batches of a warp's ring: 24 or 32 KB for the CTA's
  __shared__ uint4 ring[kWarps][STAGES][U][32];  // each lane reads what it has copied itself
  __shared__ Stats stats[kWarps];
  __shared__ uint64_t lists[kWarps][32];
  __shared__ T tops[TOP ? kWarps : 1][kSegment][32];  // the lanes' maxima of a segment's batches
  __shared__ uint64_t found[TOP ? kWarps : 1][64];    // keys on their way to the list
  __shared__ volatile float share[kWarps];  // ceil(top / kWarps) entries of each warp are as large
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t row = blockIdx.x / cs;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  const float c = p.c;

  // 16-byte accesses from the first boundary on; what lies before and after
  // goes to one warp, an entry to a lane.
  const int head = (int)min((int64_t)((16 - (uintptr_t)x % 16) % 16 / sizeof(T)), p.vocab);
  const int64_t nvec = (p.vocab - head) / E;
  const uint4* body = reinterpret_cast<const uint4*>(x + head);
  auto load = [&](int64_t batch, int slot) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = batch * (32 * U) + u * 32 + lane;
      if (i < nvec) copy16(&ring[warp][slot][u][lane], body + i);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const int64_t batches = (nvec + 32 * U - 1) / (32 * U);
  const int64_t first = rank * kWarps + warp, step = (int64_t)cs * kWarps;
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) load(first + i * step, i);
  int slot = 0;
  // The first given tokens' logits, for the end.
  float given = -kInf;
  if (rank == 0 && warp == 0 && lane < p.given) {
    const int id = p.tokens[row * p.given + lane];
    if (id >= 0 && id < p.vocab) given = (float)x[id];
  }

  Stats st;
  uint64_t mine = 0;    // this lane's entry of the warp's list
  uint64_t kth = 0;     // its `top`-th
  float bound = -kInf;  // entries below it cannot be among the `top`
  auto merge = [&](uint64_t key) {  // one to a lane, 0: none
    mine = merge_lists(mine, warp_sort(key, lane), lane);
    kth = __shfl_sync(0xffffffffu, mine, p.top - 1);
    bound = fmaxf(bound, key_bound(kth));
  };

  auto pass = [&](int64_t b) {  // the lane's maximum
    uint4 w[U];
    const int64_t left = nvec - b * (32 * U) - lane;  // accesses of this lane: those u with 32 u < left
    // Into the slot that the batch before was read from.
    load(b + (STAGES - 1) * step, slot == 0 ? STAGES - 1 : slot - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = ring[warp][slot][u][lane];
    if (++slot == STAGES) slot = 0;
    if ((b + 1) * (32 * U) > nvec) {  // the last, in part: -infinity changes nothing
      const uint32_t none = HALF ? 0xfc00fc00u : 0xff800000u;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (32 * u >= left) w[u] = make_uint4(none, none, none, none);
    }
    // NaN if there is one: the reference then stays, and the sums become NaN.
    T lane_top;
    if constexpr (HALF) {
      __half2 most = __half2half2(__ushort_as_half(0xfc00));
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __hmax2_nan(most, reinterpret_cast<const __half2*>(&w[u])[i]);
      lane_top = __hmax_nan(__low2half(most), __high2half(most));
    } else {
      lane_top = -kInf;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) lane_top = max_nan(lane_top, reinterpret_cast<const float*>(&w[u])[i]);
    }
    const float top = (float)lane_top;
    if (top > st.r) {
      const float d = fmaxf((st.r - top) * c, kLeast), f = ex2(d);
      st.t = f * (st.t + st.s * d);
      st.s *= f;
      st.r = top;
    }
    const float minus = st.r == -kInf ? 0.f : -st.r;
    float2 s2 = make_float2(st.s, 0.f), t2 = make_float2(st.t, 0.f);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const float2 v = HALF ? __half22float2(reinterpret_cast<const __half2*>(&w[u])[i])
                              : reinterpret_cast<const float2*>(&w[u])[i];
        const float2 d = mul2(add2(v, make_float2(minus, minus)), make_float2(c, c));
        const float2 e = make_float2(ex2(d.x), ex2(d.y));
        s2 = add2(s2, e);
        t2 = fma2(e, make_float2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast)), t2);
      }
    st.s = s2.x + s2.y;
    st.t = t2.x + t2.y;
    return lane_top;
  };
  // Batches first + k step, k0 <= k < k0 + n, whose lanes' maxima are kept; the
  // largest of them, seg_top, to a lane.
  auto look_back = [&](int64_t k0, int n, float seg_top) {
    const int part = (p.top + kWarps - 1) / kWarps - 1;
    const float sorted = sort_descending(seg_top != seg_top ? kInf : seg_top, lane);
    bound = fmaxf(bound, __shfl_sync(0xffffffffu, sorted, p.top - 1));
    const float listed = key_bound(__shfl_sync(0xffffffffu, mine, part));
    if (lane == part) share[warp] = fmaxf(sorted, listed);
    __syncthreads();
    float least = share[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) least = fminf(least, share[i]);
    bound = fmaxf(bound, least);
    uint32_t mask = 0;  // of the lane's batches
    for (int k = 0; k < n; ++k) mask |= (float)tops[warp][k][lane] < bound ? 0u : 1u << k;
    auto next_one = [&] {  // a batch of a lane: 32 k + lane, or -1
      const unsigned have = __ballot_sync(0xffffffffu, mask != 0);
      if (have == 0) return -1;
      const int from = __ffs(have) - 1, k = __shfl_sync(0xffffffffu, __ffs(mask) - 1, from);
      if (lane == from) mask &= mask - 1;
      return 32 * k + from;
    };
    constexpr int N = E * U, AT_ONCE = HALF ? 8 : 4;  // entries of such a batch, and batches (FP32: pairs of them) in flight
    int count = 0;
    while (__any_sync(0xffffffffu, mask != 0)) {
      float v[AT_ONCE];
      uint32_t index[AT_ONCE];  // below 2^31
#pragma unroll
      for (int s = 0; s < AT_ONCE; ++s) {
        int one = next_one();
        if constexpr (N < 32) {
          const int second = next_one();
          if (lane >= N) one = second;
        }
        const int64_t access = (first + (k0 + (one >> 5)) * step) * (32 * U) + lane % N / E * 32 + (one & 31);
        index[s] = one >= 0 && access < nvec ? (uint32_t)(head + access * E + lane % E) : ~0u;
        v[s] = index[s] != ~0u ? (float)x[index[s]] : -kInf;
      }
#pragma unroll
      for (int s = 0; s < AT_ONCE; ++s) {
        const uint64_t key = index[s] == ~0u || v[s] < bound ? 0 : order_key(v[s], index[s]);
        const unsigned want = __ballot_sync(0xffffffffu, key > kth);
        if (key > kth) found[warp][count + __popc(want & ((1u << lane) - 1))] = key;
        count += __popc(want);
        if (count >= 32) {
          __syncwarp();
          const uint64_t now = found[warp][lane], rest = found[warp][32 + lane];
          __syncwarp();
          found[warp][lane] = rest;
          count -= 32;
          merge(now);
        }
      }
    }
    __syncwarp();
    if (count > 0) merge(lane < count ? found[warp][lane] : 0);
    __syncwarp();
  };
  const int64_t rounds = (batches - rank * kWarps + step - 1) / step;  // of the CTA's first warp: the most
  for (int64_t k0 = 0; k0 < rounds; k0 += kSegment) {
    const int n = (int)min((int64_t)kSegment, (batches - first + step - 1) / step - k0);  // may be 0, or less
    T most = (T)-kInf;
    for (int k = 0; k < n; ++k) {
      const T one = pass(first + (k0 + k) * step);
      if constexpr (TOP) tops[warp][k][lane] = one, most = max_nan(most, one);
    }
    if constexpr (TOP) look_back(k0, n, (float)most);
  }
  if (rank == 0 && warp == 0) {  // the ends: fewer than 2 E entries
    const int64_t tail = p.vocab - head - nvec * E;
    const int64_t i = lane < head ? lane : head + nvec * E + (lane - head);
    const bool real = lane < head + tail;
    const float v = real ? (float)x[i] : -kInf;
    Stats one;
    if (real) one.r = v, one.s = v == -kInf ? 0.f : ex2(v - v);
    st = join(st, one, c);
    if constexpr (TOP) {
      const uint64_t key = real && !(v < bound) ? order_key(v, (uint32_t)i) : 0;
      if (__any_sync(0xffffffffu, key > kth)) merge(key);
    }
  }

  // -- join: lanes, warps, the cluster's CTAs ---------------------------------
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    Stats other;
    other.r = __shfl_xor_sync(0xffffffffu, st.r, d);
    other.s = __shfl_xor_sync(0xffffffffu, st.s, d);
    other.t = __shfl_xor_sync(0xffffffffu, st.t, d);
    st = join(st, other, c);
  }
  if (lane == 0) stats[warp] = st;
  if constexpr (TOP) lists[warp][lane] = mine;
  __syncthreads();
  if constexpr (TOP) {
#pragma unroll
    for (int n = kWarps / 2; n > 0; n >>= 1) {
      if (warp < n) {
        mine = merge_lists(mine, lists[warp + n][lane], lane);
        if (n > 1) lists[warp][lane] = mine;
      }
      if (n > 1) __syncthreads();
    }
  }
  if (warp == 0) {
    st = stats[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) st = join(st, stats[w], c);
    if (cs > 1) {
      __syncwarp();
      if (lane == 0) stats[0] = st;
      if constexpr (TOP) lists[0][lane] = mine;
    }
  }
  if (cs > 1) {
    cluster.sync();
    if (rank == 0 && warp == 0) {
      Stats far[kMaxCluster - 1];
      uint64_t far_list[kMaxCluster - 1];
#pragma unroll
      for (int i = 0; i < kMaxCluster - 1; ++i) {
        if (i + 1 >= cs) break;
        far[i] = *cluster.map_shared_rank(&stats[0], i + 1);
        if constexpr (TOP) far_list[i] = cluster.map_shared_rank(&lists[0][0], i + 1)[lane];
      }
#pragma unroll
      for (int i = 0; i < kMaxCluster - 1; ++i) {
        if (i + 1 >= cs) break;
        st = join(st, far[i], c);
        if constexpr (TOP) mine = merge_lists(mine, far_list[i], lane);
      }
    }
    cluster.sync();  // the other CTAs' shared memory is read until here
  }
  if (rank != 0 || warp != 0) return;
  const float ln2 = 0.6931471805599453f;
  const float log_s = st.s > 0.f || st.s != st.s ? log2f(st.s) : -kInf;
  const float none = -kInf;
  auto logprob = [&](float v) {
    if (v == none && st.s == st.s) return none;
    // The difference over the temperature, which does not overflow where its multiple by log2(e) would.
    return fmaf(v - st.r, c * ln2, -log_s * ln2);
  };
  if (lane == 0 && p.entropy != nullptr)
    p.entropy[row] = st.r == -kInf && st.s == st.s ? 0.f : (log_s - st.t / st.s) * ln2;
  for (int i = lane; i < p.given; i += 32) {
    float v = given;
    if (i >= 32) {
      const int id = p.tokens[row * p.given + i];
      v = id >= 0 && id < p.vocab ? (float)x[id] : -kInf;
    }
    p.logprobs[row * p.given + i] = logprob(v);
  }
  if constexpr (TOP) {
    if (lane < p.top) {
      p.top_logprobs[row * p.top + lane] = logprob(key_value(mine));
      p.top_ids[row * p.top + lane] = (int32_t)~(uint32_t)mine;
    }
  }
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_token_logprobs: " + msg); }

template <typename T, bool TOP>
cudaError_t launch(const ScoreProblem& p, int64_t rows, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, score_kernel<T, TOP>, p);
}

}  // namespace
}  // namespace af1

using namespace af1;

int af1_token_logprobs(const af1_logprob_args* a, void* stream) {
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, "args is NULL");
  if (a->rows < 0 || a->rows > (1 << 24) || a->vocab < 1 || a->vocab > 0x7fffffff || a->ld < a->vocab ||
      a->ld > ((int64_t)1 << 36))
    return fail(AF1_ERR_INVALID_ARG, "need rows 0..2^24, vocab 1..2^31 - 1, vocab <= ld <= 2^36");
  if (a->dtype != AF1_F16 && a->dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, "dtype must be AF1_F16 or AF1_F32");
  if (a->reserved != 0) return fail(AF1_ERR_INVALID_ARG, "reserved must be 0");
  if (!(a->temperature >= 1e-30f) || !(a->temperature <= 1e30f))
    return fail(AF1_ERR_INVALID_ARG, "temperature must be 1e-30..1e30");
  if (a->rows == 0) return AF1_OK;
  if (a->given < 0 || a->given > 1024 || (a->given > 0) != (a->logprobs != nullptr) ||
      (a->given > 0) != (a->tokens != nullptr))
    return fail(AF1_ERR_INVALID_ARG, "given must be 0..1024, with tokens and logprobs where it is not 0");
  if (a->top < 0 || a->top > 32 || a->top > a->vocab || (a->top > 0) != (a->top_logprobs != nullptr) ||
      (a->top > 0) != (a->top_ids != nullptr))
    return fail(AF1_ERR_INVALID_ARG, "top must be 0..32 and at most vocab, with top_logprobs and top_ids where it is not 0");
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, cudaGetErrorString(e));
  struct {
    const void* p;
    const char* name;
    int align;
  } ptrs[] = {{a->logits, "logits", a->dtype == AF1_F16 ? 2 : 4}, {a->tokens, "tokens", 4},
              {a->logprobs, "logprobs", 4},                       {a->entropy, "entropy", 4},
              {a->top_logprobs, "top_logprobs", 4},               {a->top_ids, "top_ids", 4}};
  int rc;
  for (int i = 0; i < 6; ++i) {
    if (i > 0 && ptrs[i].p == nullptr) continue;
    if ((rc = check_pointer(ptrs[i].p, ptrs[i].name, dev)) != AF1_OK ||
        (rc = check_align(ptrs[i].p, ptrs[i].align, ptrs[i].name)) != AF1_OK)
      return rc;
  }
  ScoreProblem p = {a->logits,  a->vocab,   a->ld,           a->tokens,  (int)a->given, a->logprobs,
                    a->entropy, a->top_logprobs, a->top_ids, a->top,     1.4426950408889634f / a->temperature};
  // CTAs of a row: as many as five to an SM allow, while each of their warps
  // has a batch.
  const int64_t batches = a->vocab / (kThreads * (a->dtype == AF1_F16 ? 32 : 16)) + 1;
  int cluster = 1;
  while (cluster < kMaxCluster && a->rows * cluster * 2 <= 5 * sms && 2 * cluster <= batches) cluster *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == AF1_F16)
    e = a->top > 0 ? launch<__half, true>(p, a->rows, cluster, st) : launch<__half, false>(p, a->rows, cluster, st);
  else
    e = a->top > 0 ? launch<float, true>(p, a->rows, cluster, st) : launch<float, false>(p, a->rows, cluster, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
