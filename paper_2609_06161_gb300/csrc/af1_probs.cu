// af1_probs.cu — probabilities of rows of logits after temperature and cuts.
//
// With c = log2(e) / T and M the largest entry, p_i = 2^((x_i - M) c) / S over
// the entries that are kept: those of at least M + T ln(min_p) among the k
// largest. Both cuts come to one bound: x > low, or x = low and the index at
// most `last`.
//
// A cluster of CTAs takes a row, each CTA a stretch of it, which it reads once
// into shared memory. The k-th largest is found there by four counts of 8 bits
// each of the entries' keys (their bits as ordered integers), which the CTAs
// add up through distributed shared memory; ties at the bound go by index. So
// a row is read once and written once, and device memory bounds large calls.
#include <cooperative_groups.h>

#include <algorithm>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMost = 100 * 1024 / 16;  // 16-byte accesses of a CTA's stretch in shared memory
constexpr float kInf = __builtin_huge_valf();

struct ProbsProblem {
  const void* logits;
  int64_t ld;
  float* probs;
  int64_t probs_ld;
  int vocab;
  const float* temperature;
  const int32_t* top_k;
  const float* min_p;
  float all_temperature, all_min_p;
  int all_top_k;
  int held;  // accesses that a CTA keeps in shared memory; 0: its stretch is read again for every pass
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
// Larger for larger values, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  const int32_t b = __float_as_int(x + 0.f);
  return (uint32_t)(b ^ ((b >> 31) | (int32_t)0x80000000));
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

struct Settings {
  float temperature, min_p;
  int top_k;
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) probs_kernel(const __grid_constant__ ProbsProblem p) {
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ uint4 stretch[];
  // Read by the cluster's other CTAs, each written once for a purpose.
  __shared__ Settings settings;
  __shared__ float cta_top, cta_sum;
  __shared__ int cta_first, cta_count, cta_equal, cta_last;
  __shared__ int hist[4][256];
  __shared__ float warp_f[kWarps];
  __shared__ int warp_i[kWarps], counts[256], found[2];
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t row = blockIdx.x / cs;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  float* out = p.probs + row * p.probs_ld;

  // Entry v of the row is entry v + skew of 16-byte accesses from the boundary before the row on.
  const int skew = (int)((uintptr_t)x / sizeof(T) % E);
  const int64_t all = ((int64_t)p.vocab + skew + E - 1) / E;
  const int begin = (int)(all * rank / cs), end = (int)(all * (rank + 1) / cs);
  auto fetch = [&](int i) -> uint4 {  // entries outside the row are -infinity, which changes nothing
    const int64_t v = (int64_t)i * E - skew;
    if (v >= 0 && v + E <= p.vocab) return __ldg(reinterpret_cast<const uint4*>(x + v));
    alignas(16) T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = v + e >= 0 && v + e < p.vocab ? x[v + e] : (T)-kInf;
    return *reinterpret_cast<const uint4*>(t);
  };
  const bool held = p.held > 0;
  auto entries = [&](int i, float (&f)[E]) {
    const uint4 w = held ? stretch[i - begin] : fetch(i);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = (float)reinterpret_cast<const T*>(&w)[e];
  };

  // -- the largest entry, and the row's settings
  if (tid == 0) {
    settings.temperature = p.temperature == nullptr ? p.all_temperature : p.temperature[row];
    settings.min_p = p.min_p == nullptr ? p.all_min_p : p.min_p[row];
    settings.top_k = p.top_k == nullptr ? p.all_top_k : p.top_k[row];
  }
  float top = -kInf;
  constexpr int U = 4;
  for (int i0 = begin + tid; i0 < end; i0 += U * kThreads) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * kThreads < end) w[u] = fetch(i0 + u * kThreads);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * kThreads >= end) break;
      if (held) stretch[i0 + u * kThreads - begin] = w[u];
#pragma unroll
      for (int e = 0; e < E; ++e) top = max_nan(top, (float)reinterpret_cast<const T*>(&w[u])[e]);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (lane == 0) warp_f[warp] = top;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) top = max_nan(top, warp_f[w]);
    cta_top = top;
  }
  cluster.sync();
  for (int i = 0; i < cs; ++i) top = max_nan(i == 0 ? -kInf : top, *cluster.map_shared_rank(&cta_top, i));
  const Settings set = *cluster.map_shared_rank(&settings, 0);

  auto write = [&](auto&& f) {  // f(entry, index)
    for (int i = begin + tid; i < end; i += kThreads) {
      const int64_t v = (int64_t)i * E - skew;
      float y[E];
      entries(i, y);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = f(y[e], (int)(v + e));
      if (v >= 0 && v + E <= p.vocab && (uintptr_t)(out + v) % 16 == 0) {
#pragma unroll
        for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(out + v + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (v + e >= 0 && v + e < p.vocab) out[v + e] = y[e];
      }
    }
  };
  auto block_sum = [&](int n) {  // for all threads
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    __syncthreads();
    if (lane == 0) warp_i[warp] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kWarps; ++w) n += warp_i[w];
    return n;
  };

  if (!(top < kInf) || top == -kInf) {
    const float y = top == -kInf ? 0.f : __int_as_float(0x7fffffff);
    write([&](float, int) { return y; });
    cluster.sync();  // the CTAs' memory was read
    return;
  }
  if (!(set.temperature >= 1e-30f)) {  // greedy: the first of the largest
    int first = 0x7fffffff;
    for (int i = begin + tid; i < end && first == 0x7fffffff; i += kThreads) {
      float f[E];
      entries(i, f);
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (f[e] == top) first = (int)((int64_t)i * E - skew + e);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) first = min(first, __shfl_xor_sync(0xffffffffu, first, d));
    if (lane == 0) warp_i[warp] = first;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) first = min(first, warp_i[w]);
      cta_first = first;
    }
    cluster.sync();
    for (int i = 0; i < cs; ++i) first = min(i == 0 ? 0x7fffffff : first, *cluster.map_shared_rank(&cta_first, i));
    write([&](float, int v) { return v == first ? 1.f : 0.f; });
    cluster.sync();
    return;
  }

  // -- what is kept: above `low`, or equal to it up to the index `last`
  const float t = fminf(set.temperature, 1e30f), c = 1.4426950408889634f / t;
  const float share = fminf(fmaxf(set.min_p, 0.f), 1.f);
  // Entries are compared with the FP64 bound: the least FP32 that is not below it does the same.
  float low = share > 0.f ? __double2float_ru((double)top + (double)t * log((double)share)) : -kInf;
  int last = 0x7fffffff;
  if (set.top_k >= 1 && set.top_k < p.vocab) {
    int n = 0;
    for (int i = begin + tid; i < end; i += kThreads) {
      float f[E];
      entries(i, f);
#pragma unroll
      for (int e = 0; e < E; ++e) n += f[e] >= low ? 1 : 0;
    }
    n = block_sum(n);
    if (tid == 0) cta_count = n;
    cluster.sync();
    int64_t kept = 0;
    for (int i = 0; i < cs; ++i) kept += *cluster.map_shared_rank(&cta_count, i);
    if (kept > set.top_k) {
      // The k-th largest key, 8 bits at a time.
      uint32_t prefix = 0;
      int k = set.top_k, equal = 0;
#pragma unroll
      for (int level = 0; level < 4; ++level) {
        const int shift = 24 - 8 * level;
        if (tid < 256) hist[level][tid] = 0;
        if (tid < 2) found[tid] = 0;
        __syncthreads();
        for (int i = begin + tid; i < end; i += kThreads) {
          float f[E];
          entries(i, f);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t key = order_key(f[e]);
            if (f[e] >= low && (level == 0 || key >> (shift + 8) == prefix)) atomicAdd(&hist[level][key >> shift & 255], 1);
          }
        }
        cluster.sync();
        if (tid < 256) {
          int sum = 0;
          for (int i = 0; i < cs; ++i) sum += *cluster.map_shared_rank(&hist[level][tid], i);
          counts[tid] = sum;
        }
        __syncthreads();
        if (warp == 0) {  // 8 bins to a lane, the largest first
          int sum = 0;
          for (int b = 0; b < 8; ++b) sum += counts[255 - (lane * 8 + b)];
          int upto = sum;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const int other = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += other;
          }
          const int from = __ffs(__ballot_sync(0xffffffffu, upto >= k)) - 1;
          if (lane == from) {
            int left = k - (upto - sum), b = 255 - lane * 8;
            while (b > 0 && left > counts[b]) left -= counts[b], --b;
            found[0] = b, found[1] = left;
          }
        }
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)found[0];
        k = found[1];  // of the entries with this prefix
        equal = counts[found[0]];
        __syncthreads();
      }
      low = key_value(prefix);
      if (k < equal) {  // the first k of the equal ones: their counts by stretches of warps
        const int per = (end - begin + kWarps - 1) / kWarps;
        const int from = begin + warp * per, to = min(end, from + per);
        int mine = 0;
        for (int i = from + lane; i < to; i += 32) {
          float f[E];
          entries(i, f);
#pragma unroll
          for (int e = 0; e < E; ++e) mine += f[e] == low ? 1 : 0;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) warp_i[warp] = mine;
        if (tid == 0) cta_last = -1;
        __syncthreads();
        if (tid == 0) {
          int sum = 0;
          for (int w = 0; w < kWarps; ++w) sum += warp_i[w];
          cta_equal = sum;
        }
        cluster.sync();
        for (int i = 0; i < rank; ++i) k -= *cluster.map_shared_rank(&cta_equal, i);
        for (int w = 0; w < warp; ++w) k -= warp_i[w];
        if (k >= 1 && k <= mine) {  // the k-th of this warp's
          for (int i0 = from; i0 < to && k > 0; i0 += 32) {
            const int i = i0 + lane;
            float f[E];
            unsigned same = 0;
            if (i < to) {
              entries(i, f);
#pragma unroll
              for (int e = 0; e < E; ++e) same |= f[e] == low ? 1u << e : 0u;
            }
            const int sum = __popc(same);
            int upto = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
              const int other = __shfl_up_sync(0xffffffffu, upto, d);
              if (lane >= d) upto += other;
            }
            if (upto - sum < k && k <= upto) {
              for (int left = k - (upto - sum); left > 1; --left) same &= same - 1;
              cta_last = (int)((int64_t)i * E - skew) + __ffs(same) - 1;
            }
            k -= __shfl_sync(0xffffffffu, upto, 31);
          }
        }
        cluster.sync();
        last = -1;
        for (int i = 0; i < cs; ++i) last = max(last, *cluster.map_shared_rank(&cta_last, i));
      }
    }
  }

  // -- the sum, and the row
  auto weight = [&](float v, int index) {
    const bool kept = v > low || (v == low && index <= last);
    return kept ? ex2((v - top) * c) : 0.f;
  };
  float sum = 0.f;
  for (int i = begin + tid; i < end; i += kThreads) {
    float f[E];
    entries(i, f);
#pragma unroll
    for (int e = 0; e < E; ++e) sum += weight(f[e], (int)((int64_t)i * E - skew + e));
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) warp_f[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    sum = 0.f;
    for (int w = 0; w < kWarps; ++w) sum += warp_f[w];
    cta_sum = sum;
  }
  cluster.sync();
  sum = 0.f;
  for (int i = 0; i < cs; ++i) sum += *cluster.map_shared_rank(&cta_sum, i);
  const float inverse = 1.f / sum;  // sum is at least 1
  write([&](float v, int index) { return weight(v, index) * inverse; });
  cluster.sync();  // the CTAs' memory was read
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_token_probs: " + msg); }

template <typename T>
cudaError_t launch(const ProbsProblem& p, int64_t rows, int cluster, cudaStream_t st) {
  const int smem = p.held * 16;
  // Always the most, so that calls of several threads do not lower each other's.
  cudaError_t e = cudaFuncSetAttribute(probs_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost * 16);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, probs_kernel<T>, p);
}

}  // namespace
}  // namespace af1

using namespace af1;

int af1_token_probs(const af1_probs_args* a, void* stream) {
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, "args is NULL");
  if (a->rows < 0 || a->rows > (1 << 24) || a->vocab < 1 || a->vocab > 0x7fffffff || a->ld < a->vocab ||
      a->ld > ((int64_t)1 << 36) || a->probs_ld < a->vocab || a->probs_ld > ((int64_t)1 << 36))
    return fail(AF1_ERR_INVALID_ARG, "need rows 0..2^24, vocab 1..2^31 - 1, vocab <= ld, probs_ld <= 2^36");
  if (a->dtype != AF1_F16 && a->dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, "dtype must be AF1_F16 or AF1_F32");
  if (a->rows == 0) return AF1_OK;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, cudaGetErrorString(e));
  const int es = a->dtype == AF1_F16 ? 2 : 4;
  struct {
    const void* p;
    const char* name;
    int align;
    bool need;
  } ptrs[] = {{a->logits, "logits", es, true},
              {a->probs, "probs", 4, true},
              {a->temperature, "temperature", 4, false},
              {a->top_k, "top_k", 4, false},
              {a->min_p, "min_p", 4, false}};
  for (const auto& t : ptrs) {
    if (t.p == nullptr && !t.need) continue;
    int rc;
    if ((rc = check_pointer(t.p, t.name, dev)) != AF1_OK || (rc = check_align(t.p, t.align, t.name)) != AF1_OK) return rc;
  }
  ProbsProblem p = {a->logits, a->ld,    a->probs,           a->probs_ld,  (int)a->vocab,  a->temperature,
                    a->top_k,  a->min_p, a->all_temperature, a->all_min_p, a->all_top_k, 0};
  // CTAs of a row: as many as give each a batch of accesses, while two of them
  // to an SM hold all rows, or until a stretch fits in the 100 KB that leave two CTAs to an SM.
  const int64_t accesses = (a->vocab * es + 15) / 16 + 1;
  int cluster = 1;
  while (cluster < kMaxCluster &&
         ((a->rows * cluster * 2 <= 2 * sms && accesses >= 2 * cluster * kThreads) || accesses > kMost * cluster))
    cluster *= 2;
  const int64_t stretch = (accesses + cluster - 1) / cluster;
  p.held = stretch <= kMost ? (int)stretch : 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  e = a->dtype == AF1_F16 ? launch<__half>(p, a->rows, cluster, st) : launch<float>(p, a->rows, cluster, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
