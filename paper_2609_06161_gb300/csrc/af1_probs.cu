// af1_probs.cu — probabilities of rows of logits after temperature and cuts.
//
// With c = log2(e) / T and M the largest entry, p_i = 2^((x_i - M) c) / S over
// the entries that are kept: those of at least M + T ln(min_p) among the k
// largest. Both cuts come to one bound: x > low, or x = low and the index at
// most `last`.
//
// A cluster of CTAs takes a row, each CTA a stretch of it, which it reads once
// into shared memory (up to 100 KB; longer ones are read again for every pass). A row is
// written once, so device memory bounds large calls; small ones are bound by the
// chain of one pass and exchange after another.
//   - Nothing cut: every CTA sums its weights relative to its own largest entry;
//     one exchange, then the row is written.
//   - Cut: the k-th largest lane's maximum bounds the k-th largest entry from below. The
//     entries that reach the bound and the least share (300 of 128001 for k = 200)
//     are listed as keys of 64 bits (the value as an ordered integer, then the
//     index, inverted), so that ties go by index; every CTA gets all keys, finds the k-th
//     and sums the kept weights. The row's zeros are on their way by then, so that
//     only the kept entries are left to write.
//   - Where more entries reach the bound than the lists hold (1024 of a row, each CTA its share
//     of them; large k, and ordinary k where likely tokens lie close together): the
//     k-th's bin, of 2048 of equal width, by a count of all entries, and then its entries
//     listed; where these are too many, too (ties), the k-th key by counts of its digits.
//     A CTA adds up its share of all CTAs' counts (every CTA adding up all of them: 2.3 ms
//     for 200 rows of 128001 FP32, k = 900, that took 0.15 so). 200 such rows with k = 300 take 66 us
//     where likely tokens are spread evenly, 135 where the mean falls by half a unit an octave of ids.
// FP64 is slow enough here that the cut's logarithm, computed by every thread, took a
// CTA 8 us: one thread computes it while the first entries are on their way.
//
// Measured (GPU, from a CUDA graph): 512 rows of 128001 FP16 logits with cuts
// of their own 88 us (4.5 TB/s of logits and probabilities; of measured 6.8), uncut 81; 128 rows of 128000 FP32
// uncut 29 (4.5 TB/s); 5 of 32000 FP32 with k = 50 7.0. Waits bound large calls: a warp that is issued has waited 7 cycles
// at barriers. The 512 rows have 64 KB stretches with cuts, three CTAs or 24 warps to an SM, and 32 KB without, five
// CTAs; with cuts 32 KB take as long (88.5).
// Earlier steps with cuts had 32 KB: there a CTA's life under load was 17 us, of which its copies landed after 5, the first
// exchange took 2, listing 2.5, the second exchange 3. Persistent clusters with the next row on its way, three to
// an SM, took 170 us for 99 then, stretches of 16 KB 170, 512 threads 131, and a row read again instead of held 110.
#include <cooperative_groups.h>

#include <algorithm>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kLogThreads = 8, kThreads = 1 << kLogThreads;
// CTAs to an SM; of rows that are not held four, whose 64 registers each spare spills (20 rows of 1000003 FP32, uncut: 84.3
// us, with five 86.4).
constexpr int kBlocks = 5, kLongBlocks = 4;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kLogListed = 10, kListed = 1 << kLogListed;  // keys of a row that its CTAs list
constexpr int kFew = 768;            // a top_k that the lists mostly have room for
constexpr int kBins = 2048;
constexpr int kMost = 100 * 1024 / 16;  // 16-byte pieces of a CTA's stretch in shared memory
constexpr int kPart = 32;  // pieces whose weights a thread adds up one after another
constexpr float kInf = __builtin_huge_valf();
constexpr float kLeast = -1e4f;  // 2^d is 0 from far above on

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
  int log_cluster;
  int held;  // pieces that a CTA keeps in shared memory; 0: its stretch is read again for every pass
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
// Not by way of the read-only cache: the row is written later.
__device__ __forceinline__ uint4 load_plain(const uint4* at) {
  uint4 w;
  asm("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(at));
  return w;
}
// Larger for larger values, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  const int32_t b = __float_as_int(x + 0.f);
  return (uint32_t)(b ^ ((b >> 31) | (int32_t)0x80000000));
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
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

struct Settings {
  float temperature, min_p;
  int top_k;
};

// 16 bytes of entries as they lie.
template <typename T>
struct Piece {
  uint4 w;
  __device__ __forceinline__ T at(int e) const { return reinterpret_cast<const T*>(&w)[e]; }
  __device__ __forceinline__ float most() const {  // NaN if there is one
    if constexpr (sizeof(T) == 2) {
      const __half2* h = reinterpret_cast<const __half2*>(&w);
      const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
      return __half2float(__hmax_nan(__low2half(m), __high2half(m)));
    } else {
      const float* f = reinterpret_cast<const float*>(&w);
      return max_nan(max_nan(f[0], f[1]), max_nan(f[2], f[3]));
    }
  }
};

// All threads of the cluster meet; what those that `wrote` wrote to the others' memory is seen there. (A release by every
// thread costs them all a wait for their stores.)
__device__ __forceinline__ void meet(bool wrote) {
  if (wrote) asm volatile("fence.acq_rel.cluster;" ::: "memory");
  __syncwarp();
  cluster_arrive_relaxed();
  cluster_wait();
}

// A sum of parts that carries what its roundings lose. One FP32 sum of all of a thread's weights was off by 2^-13 for a row of
// 2^26 nearly equal entries, whose roundings go one way, and would be by more for longer ones.
struct LongSum {
  float sum = 0.f, over = 0.f;
  __device__ __forceinline__ void add(float part) {
    const float y = part - over, t = sum + y;
    over = (t - sum) - y;
    sum = t;
  }
};

// What a CTA says of its stretch to the others.
struct Said {
  float top, bound, sum;
};

// IN_PLACE: probs is logits. HELD: a CTA keeps its stretch in shared memory; otherwise it reads it again for every pass, and
// the thread that read a piece last writes it. Kernels of their own: with both ways of a choice in one, registers did not
// suffice (sums in parts beside short ones: 128 rows of 128000 FP32, uncut, 34.8 us for 30.4 before and 28.7 so).
template <typename T, bool IN_PLACE, bool HELD>
__global__ void __launch_bounds__(kThreads, HELD ? kBlocks : kLongBlocks) probs_kernel(const __grid_constant__ ProbsProblem p) {
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ uint4 stretch[];
  __shared__ alignas(16) uint4 zeros[64];
  // Written by the cluster's CTAs, each once for a purpose.
  __shared__ Settings settings, here_settings;
  __shared__ double cut;
  __shared__ Said said[kMaxCluster];
  __shared__ float all_sums[kMaxCluster];
  __shared__ int all_first[kMaxCluster], all_listed[kMaxCluster], all_equal[kMaxCluster], all_last[kMaxCluster];
  __shared__ alignas(16) uint64_t lists[kListed];  // of every CTA a part; later the keys near the k-th, or counts of digits
  // The CTA's own.
  __shared__ float warp_f[kWarps], tried[2 * kWarps];
  __shared__ int warp_i[kWarps], found[3], here_listed, here_last;
  __shared__ int reached[kWarps][2 * kWarps];
  static_assert(2 * kWarps <= 32, "");
  __shared__ uint64_t kth_key;
  __shared__ int parts[kThreads], here_few;
  uint64_t* const few = lists;
  __shared__ double here_cut;
  __shared__ float here_low;
  __shared__ long long warp_mass[kWarps];
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = 1 << p.log_cluster, rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t row = blockIdx.x >> p.log_cluster;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld;
  float* out = p.probs + row * p.probs_ld;

  // Entry v of the row is entry v + skew of 16-byte pieces from the boundary before the row on; this CTA has the pieces
  // `begin` .. begin + n - 1, numbered from 0, of which those from j0 up to j1 lie in the row as a whole.
  const int skew = (int)((uintptr_t)x / sizeof(T) % E);
  const int64_t all = ((int64_t)p.vocab + skew + E - 1) / E;
  const int begin = (int)(all * rank >> p.log_cluster), n = (int)(all * (rank + 1) >> p.log_cluster) - begin;
  const int64_t first_entry = (int64_t)begin * E - skew;
  const int j0 = first_entry < 0 ? 1 : 0, j1 = first_entry + (int64_t)n * E > p.vocab ? n - 1 : n;
  const uint4* source = reinterpret_cast<const uint4*>(x + first_entry);
  auto index_of = [&](int j) { return (int)(first_entry + (int64_t)j * E); };
  auto fetch = [&](int j) {  // entries outside the row are -infinity, which changes nothing
    Piece<T> y;
    if (j >= j0 && j < j1) {
      y.w = IN_PLACE ? load_plain(source + j) : __ldg(source + j);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int64_t v = first_entry + (int64_t)j * E + e;
        reinterpret_cast<T*>(&y.w)[e] = v >= 0 && v < p.vocab ? x[v] : (T)-kInf;
      }
    }
    return y;
  };
  auto piece = [&](int j) {
    if constexpr (!HELD) return fetch(j);
    Piece<T> y;
    y.w = stretch[j];
    return y;
  };
  float* const target = out + first_entry;
  const bool wide = (uintptr_t)target % 16 == 0;
  auto write_some = [&](int from, int step, auto&& f) {  // f(piece's number, results)
#pragma unroll 2
    for (int j = from; j < n; j += step) {
      float y[E];
      f(j, y);
      if (wide && j >= j0 && j < j1) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<float4*>(target + (int64_t)j * E + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int64_t v = first_entry + (int64_t)j * E + e;
          if (v >= 0 && v < p.vocab) out[v] = y[e];
        }
      }
    }
  };

  auto write = [&](auto&& f) { write_some(tid, kThreads, f); };

  // -- the stretch: its largest entry; its sum, where nothing is cut; a bound that top_k entries of the row reach
  cluster_arrive_relaxed();  // the others' memory is written to when they have begun
  Settings set = {};
  auto uncut = [&] { return (set.top_k < 1 || set.top_k >= p.vocab) && !(set.min_p > 0.f); };
  auto few_kept = [&] {
    return !IN_PLACE && (!(set.temperature >= 1e-30f) || set.min_p > 0.f || (!uncut() && set.top_k <= kFew));
  };
  // While the first entries are on their way: the settings; the cut in FP64, which is slow, by one thread; zeros, where few
  // entries will be kept, which are then all that is left to write (not in place: they would overtake the entries).
  bool zeroed = false;
  auto zeros_are_there = [&] {  // before anything else is written to their places, or the CTA ends
    if (warp == 1) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (zeroed) __syncthreads();
  };
  auto meanwhile = [&] {
    set.temperature = p.temperature == nullptr ? p.all_temperature : __ldg(p.temperature + row);
    set.min_p = p.min_p == nullptr ? p.all_min_p : __ldg(p.min_p + row);
    set.top_k = p.top_k == nullptr ? p.all_top_k : __ldg(p.top_k + row);
    zeroed = few_kept();
    if (zeroed && wide) {
      // One warp has 1 KB of zeros copied to all of them; the ends are written one by one.
      if (warp == 1) {
        zeros[lane] = zeros[32 + lane] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        const int bytes = max(0, j1 - j0) * E * 4;
        for (int at = lane * (int)sizeof(zeros); at < bytes; at += 32 * (int)sizeof(zeros))
          asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(
                           reinterpret_cast<uint8_t*>(target + (int64_t)j0 * E) + at),
                       "r"(smem_u32(zeros)), "r"(min((int)sizeof(zeros), bytes - at))
                       : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      } else if (warp == 2 && lane < 2 * E) {
        const int j = lane < E ? 0 : n - 1;
        const int64_t v = first_entry + (int64_t)j * E + lane % E;
        if (!(j >= j0 && j < j1) && v >= 0 && v < p.vocab) out[v] = 0.f;
      }
    } else if (zeroed && warp != 0) {  // not by the warp whose stores the others wait for
      write_some(tid - 32, kThreads - 32, [&](int, float (&y)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = 0.f;
      });
    }
    if (tid == 0) {
      here_settings = set, here_listed = 0, here_last = -1;
      if (set.min_p > 0.f) here_cut = (double)fminf(set.temperature, 1e30f) * log((double)fminf(set.min_p, 1.f));
    }
  };
  float top = -kInf;
  if constexpr (HELD) {
    for (int j = tid; j < n; j += kThreads) {  // each thread's own pieces
      if (j >= j0 && j < j1)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&stretch[j])), "l"(source + j) : "memory");
      else
        stretch[j] = fetch(j).w;
    }
    meanwhile();
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 4
    for (int j = tid; j < n; j += kThreads) top = max_nan(top, piece(j).most());
  } else {
    constexpr int U = 4;
    meanwhile();
    for (int at = tid; at < n; at += U * kThreads) {
      Piece<T> w[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * kThreads < n) w[u] = fetch(at + u * kThreads);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * kThreads < n) top = max_nan(top, w[u].most());
    }
  }
  float most = top;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
  if (lane == 0) warp_f[warp] = most;
  __syncthreads();
  set = here_settings;  // every thread the first one's
  zeroed = few_kept();
  // Where `need` lanes of every CTA have an entry of at least some bound, top_k entries of the row have. Each warp puts
  // its lanes' largest in order and gives two from about as far down as the bound lies; the largest of these that enough
  // lanes reach is the CTA's, and the least of the CTAs' the row's.
  const int whole = min((int)(all >> p.log_cluster), kThreads) / 32;  // warps whose lanes all have entries, in every CTA
  const int need = (int)(((int64_t)max(set.top_k, 0) + cs - 1) >> p.log_cluster);
  const int part = whole == 0 || need > 32 * kWarps ? 33 : (need + whole - 1) / whole;  // lanes of each
  const bool bounded = set.top_k >= 1 && part <= 32;
  if (bounded) {
    const float sorted = sort_descending(top, lane);  // a row with a NaN has no use for it
    const float near = __shfl_sync(0xffffffffu, sorted, lane == 0 ? part - 1 : max(part - 2, 0));
    if (lane < 2) tried[warp * 2 + lane] = warp < whole ? near : kInf;
    __syncthreads();
    int reach = 0;
#pragma unroll
    for (int l = 0; l < 2 * kWarps; ++l) {
      const int count = __popc(__ballot_sync(0xffffffffu, sorted >= tried[l]));
      if (lane == l) reach = count;
    }
    if (lane < 2 * kWarps) reached[warp][lane] = reach;
  }
  top = warp_f[lane % kWarps];
#pragma unroll
  for (int d = kWarps / 2; d > 0; d >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));

  float c = 1.4426950408889634f / fminf(set.temperature, 1e30f);
  auto weights = [&](const Piece<T>& w, float2 (&y)[E / 2], float over) {  // without cuts
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      float2 v;
      if constexpr (sizeof(T) == 2)
        v = __half22float2(reinterpret_cast<const __half2*>(&w.w)[e]);
      else
        v = reinterpret_cast<const float2*>(&w.w)[e];
      const float2 d = mul2(add2(v, make_float2(-over, -over)), make_float2(c, c));
      y[e] = make_float2(ex2(d.x), ex2(d.y));
    }
  };
  auto block_sum = [&](float sum) {  // for all threads
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    __syncthreads();
    if (lane == 0) warp_f[warp] = sum;
    __syncthreads();
    sum = warp_f[lane % kWarps];
#pragma unroll
    for (int d = kWarps / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum;
  };
  // part(from, to): the sum of the thread's weights among these pieces.
  auto sum_parts = [&](auto&& part) {
    if constexpr (HELD) return part(0, n);  // at most 25 pieces of a thread
    LongSum sums;
    for (int from = 0; from < n; from += kPart * kThreads) sums.add(part(from, min(n, from + kPart * kThreads)));
    return sums.sum;
  };
  float sum = 0.f;
  if (uncut() && set.temperature >= 1e-30f && top > -kInf && top < kInf) {
    sum = block_sum(sum_parts([&](int from, int to) {
      float2 sums = make_float2(0.f, 0.f);
      for (int j = from + tid; j < to; j += kThreads) {
        float2 y[E / 2];
        weights(piece(j), y, top);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) sums = add2(sums, y[e]);
      }
      return sums.x + sums.y;
    }));
  }
  __syncthreads();
  cluster_wait();
  if (warp == 0) {
    float bound = set.top_k < 1 ? kInf : -kInf;
    if (bounded) {
      if (lane < 2 * whole) {
        int lanes = 0;
        for (int w = 0; w < kWarps; ++w) lanes += reached[w][lane];
        if (lanes >= need) bound = tried[lane];
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) bound = fmaxf(bound, __shfl_xor_sync(0xffffffffu, bound, d));
    }
    if (lane < cs) {
      *cluster.map_shared_rank(&said[rank], lane) = {top, bound, sum};
      // Everyone takes the first CTA's settings, and so the same way.
      if (rank == 0) {
        *cluster.map_shared_rank(&settings, lane) = set;
        *cluster.map_shared_rank(&cut, lane) = here_cut;
      }
    }
  }
  meet(tid < cs);
  set = settings;
  Said one = said[lane % kMaxCluster < cs ? lane % kMaxCluster : 0];
  top = one.top;
  float bound = one.bound;
#pragma unroll
  for (int d = kMaxCluster / 2; d > 0; d >>= 1) {
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
    bound = fminf(bound, __shfl_xor_sync(0xffffffffu, bound, d));
  }

  if (!(top < kInf) || top == -kInf) {
    zeros_are_there();
    const float fill = top == -kInf ? 0.f : __int_as_float(0x7fffffff);
    write([&](int, float (&y)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fill;
    });
    return;
  }
  if (!(set.temperature >= 1e-30f)) {  // greedy: the first of the largest
    int first = 0x7fffffff;
    for (int j = tid; j < n && first == 0x7fffffff; j += kThreads) {
      const Piece<T> w = piece(j);
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if ((float)w.at(e) == top) first = index_of(j) + e;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) first = min(first, __shfl_xor_sync(0xffffffffu, first, d));
    if (lane == 0) warp_i[warp] = first;
    __syncthreads();
    if (tid < cs) {
      for (int w = 0; w < kWarps; ++w) first = min(first, warp_i[w]);
      *cluster.map_shared_rank(&all_first[rank], tid) = first;
    }
    meet(tid < cs);
    first = all_first[0];
    for (int i = 1; i < cs; ++i) first = min(first, all_first[i]);
    zeros_are_there();
    if (zeroed) {
      if (tid == 0 && first >= first_entry && first < first_entry + (int64_t)n * E) out[first] = 1.f;
      return;
    }
    write([&](int j, float (&y)[E]) {
      const int v = index_of(j);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = v + e == first ? 1.f : 0.f;
    });
    return;
  }
  const float t = fminf(set.temperature, 1e30f);
  c = 1.4426950408889634f / t;
  if (uncut()) {
    zeros_are_there();
    const float mine = lane < cs ? one.sum * ex2(fmaxf((one.top - top) * c, kLeast)) : 0.f;
    sum = one.top > -kInf ? mine : 0.f;  // a stretch of -infinity alone has no sum
#pragma unroll
    for (int d = kMaxCluster / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    sum = __shfl_sync(0xffffffffu, sum, 0);
    const float inverse = 1.f / sum;  // sum is at least about 1
    write([&](int j, float (&y)[E]) {
      float2 z[E / 2];
      weights(piece(j), z, top);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        z[e] = mul2(z[e], make_float2(inverse, inverse));
        y[2 * e] = z[e].x, y[2 * e + 1] = z[e].y;
      }
    });
    return;
  }

  // -- what is kept: above `low`, or equal to it up to the index `last`
  float low = -kInf;
  if (set.min_p > 0.f) {
    // Entries are compared with the FP64 bound: the least FP32 that is not below it does the same.
    if (tid == 0) here_low = __double2float_ru((double)top + cut);
    __syncthreads();
    low = here_low;
  }
  int last = 0x7fffffff;
  const int top_k = set.top_k < 1 || set.top_k >= p.vocab ? 0x7fffffff : set.top_k;
  // The entries from `least_value` on that `is_one` takes, as keys that put them in order; everyone gets everyone's.
  // Whether the lists hold them all; `listed` of them.
  const int room = kListed >> p.log_cluster;
  int listed = 0;
  auto list_entries = [&](float least_value, bool some, auto&& is_one) {
    for (int j = tid; some && j < n; j += kThreads) {
      const Piece<T> w = piece(j);
      if (w.most() < least_value) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = (float)w.at(e);
        const int index = index_of(j) + e;
        if (v >= least_value && index >= 0 && index < p.vocab && is_one(v)) {
          const int at = atomicAdd(&here_listed, 1);
          if (at < room) lists[rank * room + at] = (uint64_t)order_key(v) << 32 | (uint32_t)~index;
        }
      }
    }
    __syncthreads();
    const int mine = some ? here_listed : room + 1;
    if (tid < cs) *cluster.map_shared_rank(&all_listed[rank], tid) = mine;
    if (mine <= room)
      for (int i = tid; i < mine << p.log_cluster; i += kThreads) {  // key i / cs to CTA i % cs
        uint64_t* key = &lists[rank * room + (i >> p.log_cluster)];
        if ((i & (cs - 1)) != rank) *cluster.map_shared_rank(key, i & (cs - 1)) = *key;
      }
    meet(tid < max(cs, min(mine, room + 1) << p.log_cluster));
    bool fits = true;
    listed = 0;
    for (int i = 0; i < cs; ++i) fits = fits && all_listed[i] <= room, listed += min(all_listed[i], room);
    return fits;
  };
  // All listed keys, a few to a thread (0: none).
  constexpr int kOwn = kListed / kThreads;
  uint64_t key[kOwn];
  auto take_keys = [&] {
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int slot = tid + i * kThreads, of = slot >> (kLogListed - p.log_cluster);
      key[i] = of < cs && slot - of * room < all_listed[of] ? lists[slot] : 0;
    }
  };
  auto value_of = [&](uint64_t k) { return key_value((uint32_t)(k >> 32)); };
  // The key that k - 1 others are above: first the part of the range, one of kThreads equal ones, that it lies in, then its
  // place among the keys of that part, which are few but for ties. `lowest`: -infinity if it is not known.
  auto kth_of_keys = [&](int k, float lowest) {
    __syncthreads();
    parts[tid] = 0;
    if (tid == 0) here_few = 0;
    if (lowest == -kInf) {
      lowest = kInf;
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (key[i] != 0 && value_of(key[i]) > -kInf) lowest = fminf(lowest, value_of(key[i]));
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) lowest = fminf(lowest, __shfl_xor_sync(0xffffffffu, lowest, d));
      if (lane == 0) warp_f[warp] = lowest;
      __syncthreads();
      for (int w = 0; w < kWarps; ++w) lowest = fminf(lowest, warp_f[w]);
    }
    // (Differences, products and minima keep the order of values, however they are rounded.)
    const float scale = top > lowest ? (float)kThreads / (top - lowest) : 0.f;
    auto part_of = [&](uint64_t one) { return (int)fminf((top - value_of(one)) * scale, (float)(kThreads - 1)); };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (key[i] != 0) atomicAdd(&parts[part_of(key[i])], 1);
    __syncthreads();
    const int have = parts[tid];
    int upto = have;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += other;
    }
    if (lane == 31) warp_i[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += warp_i[w];
    if (upto - have < k && k <= upto) found[0] = tid, found[1] = k - (upto - have);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (key[i] != 0 && part_of(key[i]) == found[0]) few[atomicAdd(&here_few, 1)] = key[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (key[i] != 0 && part_of(key[i]) == found[0]) {
        int above = 0;
        for (int j = 0; j < here_few; ++j) above += few[j] > key[i] ? 1 : 0;
        if (above == found[1] - 1) kth_key = key[i];
      }
    __syncthreads();
    return kth_key;
  };
  const float from = top_k < p.vocab ? fmaxf(low, bound) : low;
  const bool fits = list_entries(from, from > -kInf || p.vocab <= room, [](float) { return true; });
  float inverse;
  if (fits) {
    take_keys();
    uint64_t least = 0;
    if (listed > top_k) {
      least = kth_of_keys(top_k, from);
      low = value_of(least), last = (int)~(uint32_t)least;
    } else {
      low = from;  // these are all: at `low` or above, or as many as the k
    }
    // Lists are in no order, so that their weights are added up as whole multiples of 2^-40.
    long long mass = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      if (key[i] != 0 && key[i] >= least) mass += __float2ll_rn(ex2((value_of(key[i]) - top) * c) * 1099511627776.f);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, d);
    if (lane == 0) warp_mass[warp] = mass;
    __syncthreads();
    mass = warp_mass[lane % kWarps];
#pragma unroll
    for (int d = kWarps / 2; d > 0; d >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, d);
    inverse = 1.f / ((float)mass * 9.094947017729282e-13f);
    zeros_are_there();
    if (zeroed) {  // this CTA's entries to their places
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (key[i] != 0 && key[i] >= least && (tid + i * kThreads) >> (kLogListed - p.log_cluster) == rank)
          out[(int)~(uint32_t)key[i]] = ex2((value_of(key[i]) - top) * c) * inverse;
      return;
    }
  } else {
    if (top_k < p.vocab) {
      // Counts of all entries in bins, the largest entries in the first, where the lists lay. A CTA adds up its share of
      // the bins and gives the sums to all.
      int* const counts = reinterpret_cast<int*>(lists);
      static_assert(sizeof(lists) >= kBins * sizeof(int), "");
      auto count_bins = [&](int bins, auto&& bin_of) {  // bin_of(value): below 0 for none
        cluster.sync();  // what lies there was read
        for (int i = tid; i < bins; i += kThreads) counts[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kThreads) {
          const Piece<T> w = piece(j);
          if (w.most() < from) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float v = (float)w.at(e);
            const int bin = v >= from ? bin_of(v) : -1;
            if (bin >= 0) atomicAdd(&counts[bin], 1);
          }
        }
        cluster.sync();
        const int share = bins >> p.log_cluster;
        for (int i = rank * share + tid; i < (rank + 1) * share; i += kThreads) {
          int sum_of = 0;
          for (int r = 0; r < cs; ++r) sum_of += *cluster.map_shared_rank(&counts[i], r);
          for (int r = 0; r < cs; ++r) *cluster.map_shared_rank(&counts[i], r) = sum_of;
        }
        cluster.sync();
      };
      // The bin of the k-th entry, its place there and how many are there, in `found`; the number of all.
      auto find_bin = [&](int bins, int k) {
        const int per = bins / kThreads;
        int some[kBins / kThreads], here = 0;
#pragma unroll
        for (int j = 0; j < kBins / kThreads; ++j) here += some[j] = j < per ? counts[tid * per + j] : 0;
        int upto = here;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int other = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += other;
        }
        if (lane == 31) warp_i[warp] = upto;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < kWarps; ++w) {
          if (w < warp) upto += warp_i[w];
          total += warp_i[w];
        }
        if (upto - here < k && k <= upto) {
          int left = k - (upto - here);
#pragma unroll
          for (int j = 0; j < kBins / kThreads; ++j) {
            if (j < per && left > 0 && left <= some[j]) found[0] = tid * per + j, found[1] = left, found[2] = some[j];
            left -= some[j];
          }
        }
        __syncthreads();
        return total;
      };
      // Bins of equal width first: what is in the k-th's bin mostly fits the lists.
      float lowest = from;
      if (from == -kInf) {
        lowest = kInf;
        for (int j = tid; j < n; j += kThreads) {
          const Piece<T> w = piece(j);
#pragma unroll
          for (int e = 0; e < E; ++e)
            if ((float)w.at(e) > -kInf) lowest = fminf(lowest, (float)w.at(e));
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) lowest = fminf(lowest, __shfl_xor_sync(0xffffffffu, lowest, d));
        __syncthreads();
        if (lane == 0) warp_f[warp] = lowest;
        __syncthreads();
        if (tid < cs) {
          for (int w = 0; w < kWarps; ++w) lowest = fminf(lowest, warp_f[w]);
          *cluster.map_shared_rank(&all_sums[rank], tid) = lowest;
        }
        meet(tid < cs);
        lowest = all_sums[0];
        for (int i = 1; i < cs; ++i) lowest = fminf(lowest, all_sums[i]);
      }
      const float scale = top > lowest ? (float)kBins / (top - lowest) : 0.f;
      auto wide_bin = [&](float v) { return (int)fminf((top - v) * scale, (float)(kBins - 1)); };
      count_bins(kBins, wide_bin);
      bool cut = find_bin(kBins, top_k) > top_k;
      if (!cut) {
        low = from;  // all that reach it
      } else {
        const int bin = found[0], place = found[1];
        const bool try_lists = found[2] <= kListed;
        if (tid == 0) here_listed = 0;
        cluster.sync();  // counts were read
        if (list_entries(from, try_lists, [&](float v) { return wide_bin(v) == bin; })) {
          take_keys();
          const uint64_t least = kth_of_keys(place, -kInf);
          low = value_of(least), last = (int)~(uint32_t)least;
          cut = false;
        }
      }
      // Many of nearly the same value: by digits of their keys, 11, 11 and 10 bits (FP16 has 22).
      uint32_t prefix = 0;
      int k = top_k, equal = 0;
      constexpr int kLevels = sizeof(T) == 2 ? 2 : 3;
      for (int level = 0; cut && level < kLevels; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level < 2 ? 11 : 10, bins = 1 << bits;
        count_bins(bins, [&](float v) {
          const uint32_t one = order_key(v);
          return level == 0 || one >> (shift + bits) == prefix ? bins - 1 - (int)(one >> shift & (bins - 1)) : -1;
        });
        find_bin(bins, k);
        prefix = prefix << bits | (uint32_t)(bins - 1 - found[0]);
        k = found[1];  // of the entries with this prefix
        equal = found[2];
      }
      if (cut) {
        // The bits that FP16 does not have are 0, and 1 in the keys of negative values.
        low = key_value(sizeof(T) == 4 ? prefix : prefix << 10 | (prefix >> 21 & 1 ? 0u : 1023u));
        if (k < equal) {  // the first k of the equal ones: their counts by stretches of warps
          const int per = (n + kWarps - 1) / kWarps;
          const int from_here = warp * per, to = min(n, from_here + per);
          int same_here = 0;
          for (int i = from_here + lane; i < to; i += 32) {
            const Piece<T> w = piece(i);
#pragma unroll
            for (int e = 0; e < E; ++e) same_here += (float)w.at(e) == low ? 1 : 0;
          }
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) same_here += __shfl_xor_sync(0xffffffffu, same_here, d);
          if (lane == 0) warp_i[warp] = same_here;
          __syncthreads();
          if (tid < cs) {
            int sum_here = 0;
            for (int w = 0; w < kWarps; ++w) sum_here += warp_i[w];
            *cluster.map_shared_rank(&all_equal[rank], tid) = sum_here;
          }
          cluster.sync();
          for (int i = 0; i < rank; ++i) k -= all_equal[i];
          for (int w = 0; w < warp; ++w) k -= warp_i[w];
          if (k >= 1 && k <= same_here) {  // the k-th of this warp's
            for (int i0 = from_here; i0 < to && k > 0; i0 += 32) {
              const int i = i0 + lane;
              unsigned same = 0;
              if (i < to) {
                const Piece<T> w = piece(i);
#pragma unroll
                for (int e = 0; e < E; ++e) same |= (float)w.at(e) == low ? 1u << e : 0u;
              }
              const int have = __popc(same);
              int upto = have;
#pragma unroll
              for (int d = 1; d < 32; d <<= 1) {
                const int other = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += other;
              }
              if (upto - have < k && k <= upto) {
                for (int left = k - (upto - have); left > 1; --left) same &= same - 1;
                here_last = index_of(i) + __ffs(same) - 1;
              }
              k -= __shfl_sync(0xffffffffu, upto, 31);
            }
          }
          __syncthreads();
          if (tid < cs) *cluster.map_shared_rank(&all_last[rank], tid) = here_last;
          cluster.sync();
          last = -1;
          for (int i = 0; i < cs; ++i) last = max(last, all_last[i]);
        }
      }
    }
    sum = block_sum(sum_parts([&](int start, int to) {
      float some = 0.f;
      for (int j = start + tid; j < to; j += kThreads) {
        const Piece<T> w = piece(j);
        if (w.most() < low) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float v = (float)w.at(e);
          if (v > low || (v == low && index_of(j) + e <= last)) some += ex2((v - top) * c);
        }
      }
      return some;
    }));
    if (tid < cs) *cluster.map_shared_rank(&all_sums[rank], tid) = sum;
    cluster.sync();  // counts were read, too
    sum = 0.f;
    for (int i = 0; i < cs; ++i) sum += all_sums[i];
    inverse = 1.f / sum;
    zeros_are_there();
  }
  write([&](int j, float (&y)[E]) {
    const Piece<T> w = piece(j);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.f;
    if (w.most() >= low) {
      const int index = index_of(j);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = (float)w.at(e);
        if (v > low || (v == low && index + e <= last)) y[e] = ex2((v - top) * c) * inverse;
      }
    }
  });
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_token_probs: " + msg); }

// Whether a row of one matrix overlaps a row of another; bytes, and strides of at least a row.
bool rows_overlap(const void* x, int64_t width, int64_t ld, const void* y, int64_t y_width, int64_t y_ld, int64_t rows) {
  const int64_t a = (int64_t)(uintptr_t)x, b = (int64_t)(uintptr_t)y;
  if (a + (rows - 1) * ld + width <= b || b + (rows - 1) * y_ld + y_width <= a) return false;
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {  // the one that ends first overlaps no later row
    if (a + i * ld + width <= b + j * y_ld)
      ++i;
    else if (b + j * y_ld + y_width <= a + i * ld)
      ++j;
    else
      return true;
  }
  return false;
}

template <typename T, bool IN_PLACE, bool HELD>
cudaError_t launch(const ProbsProblem& p, int64_t rows, cudaStream_t st) {
  const int cluster = 1 << p.log_cluster;
  const int smem = p.held * 16;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [] {
    const cudaError_t first =
        cudaFuncSetAttribute(probs_kernel<T, IN_PLACE, HELD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost * 16);
    if (first != cudaSuccess) return first;
    return cudaFuncSetAttribute(probs_kernel<T, IN_PLACE, HELD>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
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
  return cudaLaunchKernelEx(&cfg, probs_kernel<T, IN_PLACE, HELD>, p);
}

}  // namespace
}  // namespace af1

using namespace af1;

int af1_token_probs(const af1_probs_args* a, void* stream) {
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, "args is NULL");
  if (a->rows < 0 || a->rows > (1 << 24) || a->vocab < 1 || a->vocab > (1 << 30) || a->ld < a->vocab ||
      a->ld > ((int64_t)1 << 36) || a->probs_ld < a->vocab || a->probs_ld > ((int64_t)1 << 36))
    return fail(AF1_ERR_INVALID_ARG, "need rows 0..2^24, vocab 1..2^30, vocab <= ld, probs_ld <= 2^36");
  if (a->dtype != AF1_F16 && a->dtype != AF1_F32) return fail(AF1_ERR_INVALID_ARG, "dtype must be AF1_F16 or AF1_F32");
  if (a->rows == 0) return AF1_OK;
  const int es = a->dtype == AF1_F16 ? 2 : 4;
  const bool in_place = a->logits == a->probs && es == 4 && (a->rows == 1 || a->ld == a->probs_ld);
  if (!in_place && rows_overlap(a->logits, a->vocab * es, a->ld * es, a->probs, a->vocab * 4, a->probs_ld * 4, a->rows))
    return fail(AF1_ERR_INVALID_ARG, "rows of probs overlap rows of logits (in place: FP32, with one stride)");
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, cudaGetErrorString(e));
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
                    a->top_k,  a->min_p, a->all_temperature, a->all_min_p, a->all_top_k, 0, 0};
  // CTAs of a row: until all rows have one to an SM, while each thread has two pieces (5 rows of 32000 FP32: 8 CTAs to a row
  // 7.0 us, two 9.5); and until a stretch is at most 64 KB where entries are cut, and 40 KB where not. Cuts cost a CTA as
  // much as 30 KB, whatever its stretch, and write little at its end (200 rows of 128001 FP32, k = 300: 67 us in 8 CTAs, 81
  // in 16; FP16 takes as long in 4 as in 8); without them more CTAs to an SM, in different passes, are faster (200 rows of
  // 128001 FP16: 37 us in 8, 40 in 4; 512 in 16, of 16 KB: 106 for 81).
  const bool cuts = a->top_k != nullptr || a->min_p != nullptr || a->all_top_k > 0 || a->all_min_p > 0.f;
  const int64_t most = cuts ? 4096 : 2560, pieces = (a->vocab * es + 15) / 16 + 1;
  auto more = [&](int64_t ctas) {
    return pieces > most * ctas || (a->rows * ctas <= sms && pieces >= 4 * kThreads * ctas);
  };
  while ((1 << p.log_cluster) < kMaxCluster && more(1 << p.log_cluster)) ++p.log_cluster;
  const int64_t part = (pieces + (1 << p.log_cluster) - 1) >> p.log_cluster;
  p.held = part <= kMost ? (int)part : 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.held > 0)
    e = a->dtype == AF1_F16 ? launch<__half, false, true>(p, a->rows, st)
        : in_place          ? launch<float, true, true>(p, a->rows, st)
                            : launch<float, false, true>(p, a->rows, st);
  else
    e = a->dtype == AF1_F16 ? launch<__half, false, false>(p, a->rows, st)
        : in_place          ? launch<float, true, false>(p, a->rows, st)
                            : launch<float, false, false>(p, a->rows, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
