// af1_score.cu — log-probabilities of given tokens, entropy and the largest
// alternatives of rows of logits, in one pass over the logits.
//
// With y = x / temperature, a thread keeps m = max x, S = sum 2^d and
// T = sum 2^d d over its entries, d = (x - m) log2(e) / temperature, and
// follows a new maximum by S' = f S, T' = f (T + S delta). Then
//   log p = (d - log2 S) ln 2,   entropy = (log2 S - T / S) ln 2.
//
// The largest entries: each warp keeps its 32 largest so far, one to a lane,
// in order. Keys of 64 bits (the value as an ordered integer, then the index,
// inverted) make the order total, so that equal values go by index and the
// result does not depend on which thread saw what first. An entry is looked
// at again only where it may be among the `top`: not below the `top`-th of
// any warp of its CTA, which the warps share.
//
// A cluster of CTAs takes a row (one where there are rows enough to fill the
// GPU), and its first CTA joins their statistics and lists through
// distributed shared memory. Device memory bounds large calls: one exponent
// and about eight instructions an entry.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCluster = 8;
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
  float inv_t;  // 1 / temperature
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Stats {
  float m = -kInf, s = 0.f, t = 0.f;
};

// The two sets of entries together.
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float c) {
  Stats r;
  r.m = fmaxf(a.m, b.m);
  if (r.m == -kInf) {
    r.s = a.s + b.s, r.t = 0.f;  // nothing, or NaN
    return r;
  }
  const float da = fmaxf((a.m - r.m) * c, -1e4f), db = fmaxf((b.m - r.m) * c, -1e4f);
  const float fa = ex2(da), fb = ex2(db);
  r.s = a.s * fa + b.s * fb;
  r.t = fa * (a.t + a.s * da) + fb * (b.t + b.s * db);
  return r;
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
__device__ __forceinline__ float key_bound(uint64_t key) {  // entries below it cannot matter
  return key == 0 ? -kInf : key_value(key);
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

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) score_kernel(const __grid_constant__ ScoreProblem p) {
  constexpr int E = 16 / (int)sizeof(T);  // entries of a 16-byte access
  constexpr int U = 16 / E;               // accesses of a batch: 16 entries to a lane
  __shared__ Stats stats[kWarps];
  __shared__ uint64_t lists[kWarps][32];
  __shared__ int bound_shared;  // largest `top`-th entry of a warp, as an ordered integer
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

  if (threadIdx.x == 0) bound_shared = (int)0x80000000;
  __syncthreads();

  Stats st;
  uint64_t mine = 0;             // this lane's entry of the warp's list
  uint64_t kth = 0;              // its `top`-th
  float bound = -kInf;           // entries below it cannot be among the `top`
  auto consider = [&](float v, bool real, uint32_t index) {
    const bool maybe = real && !(v < bound);
    const uint64_t key = maybe ? order_key(v, index) : 0;
    unsigned want = __ballot_sync(0xffffffffu, key > kth);
    if (want == 0) return;
    if (__popc(want) > 6) {
      mine = merge_lists(mine, warp_sort(key, lane), lane);
    } else {
      while (want != 0) {
        const int from = __ffs(want) - 1;
        want &= want - 1;
        const uint64_t k = __shfl_sync(0xffffffffu, key, from);
        const int at = __popc(__ballot_sync(0xffffffffu, mine > k));
        const uint64_t up = __shfl_up_sync(0xffffffffu, mine, 1);
        mine = lane < at ? mine : lane == at ? k : up;
      }
    }
    kth = __shfl_sync(0xffffffffu, mine, p.top - 1);
    bound = fmaxf(bound, key_bound(kth));
  };

  auto load = [&](uint4 (&w)[U], int64_t batch) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = batch * (32 * U) + u * 32 + lane;
      if (i < nvec) w[u] = __ldcs(body + i);
    }
  };
  const int64_t batches = (nvec + 32 * U - 1) / (32 * U);
  const int64_t first = rank * kWarps + warp, step = (int64_t)cs * kWarps;
  uint4 next[U];
  load(next, first);
  for (int64_t b = first; b < batches; b += step) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
    if (b + step < batches) load(next, b + step);
    float v[16];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* e = reinterpret_cast<const T*>(&w[u]);
      const bool real = b * (32 * U) + u * 32 + lane < nvec;
#pragma unroll
      for (int i = 0; i < E; ++i) v[u * E + i] = real ? (float)e[i] : -kInf;
    }
    float top = v[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, v[i]);
    if (top > st.m) {
      const float d = fmaxf((st.m - top) * c, -1e4f), f = ex2(d);
      st.t = f * (st.t + st.s * d);
      st.s *= f;
      st.m = top;
    }
    const float mx = st.m == -kInf ? 0.f : st.m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // The difference first: the products alone may overflow.
      const float d = (v[i] - mx) * c, e = ex2(d);
      st.s += e;
      st.t = fmaf(e, fmaxf(d, -1e4f), st.t);
    }
    if constexpr (TOP) {
      const int shared = *static_cast<volatile int*>(&bound_shared);
      bound = fmaxf(bound, __int_as_float(shared < 0 ? shared ^ 0x7fffffff : shared));
      bool any = false;  // also where a NaN hides the maximum
#pragma unroll
      for (int i = 0; i < 16; ++i) any |= !(v[i] < bound);
      if (__any_sync(0xffffffffu, any)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int64_t vec = b * (32 * U) + (i / E) * 32 + lane;
          consider(v[i], vec < nvec, (uint32_t)(head + vec * E + i % E));
        }
        if (lane == 0) {
          const int o = __float_as_int(bound);
          atomicMax(&bound_shared, o < 0 ? o ^ 0x7fffffff : o);
        }
      }
    }
  }
  if (rank == 0 && warp == 0) {  // the ends: fewer than 2 E entries
    const int64_t tail = p.vocab - head - nvec * E;
    const int64_t i = lane < head ? lane : head + nvec * E + (lane - head);
    const bool real = lane < head + tail;
    const float v = real ? (float)x[i] : -kInf;
    Stats one;
    if (real) one.m = v, one.s = v == -kInf ? 0.f : ex2((v - v) * c);
    st = join(st, one, c);
    if constexpr (TOP) consider(v, real, (uint32_t)i);
  }

  // -- join: lanes, warps, the cluster's CTAs ---------------------------------
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    Stats other;
    other.m = __shfl_xor_sync(0xffffffffu, st.m, d);
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
      for (int r = 1; r < cs; ++r) {
        st = join(st, *cluster.map_shared_rank(&stats[0], r), c);
        if constexpr (TOP) mine = merge_lists(mine, cluster.map_shared_rank(&lists[0][0], r)[lane], lane);
      }
    }
    cluster.sync();  // the other CTAs' shared memory is read until here
  }
  if (rank != 0 || warp != 0) return;
  const float ln2 = 0.6931471805599453f;
  const float log_s = st.s > 0.f || st.s != st.s ? log2f(st.s) : -kInf;
  auto logprob = [&](float v) { return v == -kInf && st.s == st.s ? -kInf : fmaf(v - st.m, p.inv_t, -log_s * ln2); };
  if (lane == 0 && p.entropy != nullptr)
    p.entropy[row] = st.m == -kInf && st.s == st.s ? 0.f : (log_s - st.t / st.s) * ln2;
  for (int i = lane; i < p.given; i += 32) {
    const int id = p.tokens[row * p.given + i];
    const float v = id >= 0 && id < p.vocab ? (float)x[id] : -kInf;
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
  if (!(a->temperature > 0.f) || !(a->temperature < kInf) || !(1.f / a->temperature < kInf))
    return fail(AF1_ERR_INVALID_ARG, "temperature must be positive and finite");
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
                    a->entropy, a->top_logprobs, a->top_ids, a->top,     1.4426950408889634f / a->temperature,
                    1.f / a->temperature};
  // CTAs of a row: enough to give every SM four, while a CTA keeps a batch for
  // each warp.
  const int64_t batches = a->vocab / (kThreads * 16) + 1;
  int cluster = 1;
  while (cluster < kMaxCluster && a->rows * cluster < 4 * sms && 2 * cluster <= batches) cluster *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == AF1_F16)
    e = a->top > 0 ? launch<__half, true>(p, a->rows, cluster, st) : launch<__half, false>(p, a->rows, cluster, st);
  else
    e = a->top > 0 ? launch<float, true>(p, a->rows, cluster, st) : launch<float, false>(p, a->rows, cluster, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
