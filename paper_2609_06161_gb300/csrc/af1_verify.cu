// af1_verify.cu — drafted tokens accepted or rejected by the target's
// probabilities and given random numbers, and the token that follows.
//
// At a node with the target's row P and the draft's row Q, the children's
// tokens were drawn from Q. With c = 0, Z = Z' = 1 at first, a child x with the
// number u is accepted if u Q(x) Z < r Z', r = max(P(x) - c Q(x), 0), and the walk
// goes on there. A rejection leaves the residual R = max(P - c Q, 0) with
// c += Z / Z' (residuals of residuals are residuals with a larger c), without
// the tokens that were rejected here; Z = sum R; and where siblings are drawn
// without repetition Z' -= Q(x), what is left of Q. Where the walk ends, the
// token that follows is drawn from R. The tokens that come out have the
// target's distribution whatever Q is. Without Q the children are given guesses:
// accepted if u Z < r, and Z -= r at a rejection.
//
// Comparisons decide, so that every step is defined to the last bit: P - c Q is
// an FP32 product and difference, each rounded; masses are whole multiples of
// 2^-40 of it, so that their sums do not depend on an order; the walk's few
// numbers are FP64. A sum of whole numbers costs no wide arithmetic: the bits of
// r + 12 count multiples of 2^-20, those of the rest (exact) and a constant count
// multiples of 2^-40, and both add up as 32-bit integers.
//
// A cluster of CTAs takes a sequence. The numbers that the walk needs (four to a
// node) are fetched for all nodes at once by the first and given to all. One warp of
// every CTA walks, all alike, so that only masses are exchanged; the others wait for rows to sum. Every
// warp has a stretch of the vocabulary, so that a row is summed and then searched
// (one warp's stretch, by marks in it) where the sum of the stretches before
// passes the bound. Only rows that the walk needs are summed, and with a draft, where they may be
// summed more than once, they are kept in shared memory if all sequences' have room there at once (of 16
// sequences over 128001 tokens they have not, of 15 they have).
//
// What bounds it is latency: launch, two trips to memory for the nodes, their exchange, half a
// microsecond for every node that is looked at, and for every row its trip, an exchange and the search.
// GPU times: 8 chains of 5 over 32000 tokens 7.7 us; 64 guessed trees of 32 over 128000 13 (33 MB of rows, of which
// device memory would need 4.8); 16 trees of 16 over 128001, drawn without repetition, 25 (2.4): two to
// four sums of a row of P and Q one after another, 3 to 5 us each, at the 64 registers of two CTAs to an SM,
// which spill 44 bytes. FP64 is slow enough to count:
// with every thread walking the three took 14, 34 and 41 us; clear cases are decided in FP32 beside it.
#include <cooperative_groups.h>

#include <algorithm>

#include "af1_internal.h"
#include "af1_kv.cuh"
#include "af1_ptx.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kThreads = 512;
constexpr int kLogWarps = 4, kWarps = 1 << kLogWarps;
static_assert(kThreads == 32 * kWarps, "");
constexpr int kMaxCluster = 16;
constexpr int kMaxNodes = 64;
constexpr int kMostHeld = 208 * 1024;  // bytes of shared memory beside the kernel's own 6 KB; half where two CTAs share an SM
constexpr double kUnit = 1099511627776.0;  // 2^40

struct VerifyProblem {
  const float* probs;
  int64_t p_seq, p_node;
  const float* draft;
  int64_t q_seq, q_node;
  const int32_t *tokens, *parents, *counts;
  const float* uniforms;
  int32_t *path, *lengths, *following;
  int nodes, vocab;
  bool distinct;
  int log_cluster;
  int held;  // 16-byte pieces of a row that a warp keeps in shared memory; 0: they are read again for every pass
};

// Probabilities as they count: 0 to 1, NaN as 0.
__device__ __forceinline__ float clamped(float p) { return __saturatef(p); }
// Of such, with c at least 0: at most 1.
__device__ __forceinline__ float residual(float p, float q, float c) {
  return __saturatef(__fsub_rn(p, __fmul_rn(c, q)));
}

// Sums of masses: the bits of r + 12 and of what is left of r count multiples of 2^-20 and of 2^-40 in their low
// parts, and the others add up to a known number. For up to 2048 entries, or 64 in each lane of a warp.
struct Masses {
  uint32_t high = 0, low = 0;
  __device__ __forceinline__ void add(float x, float y) {
    const float2 r = make_float2(x, y);
    const float2 t = add2(r, make_float2(12.f, 12.f));
    const float2 l = fma2(add2(t, make_float2(-12.f, -12.f)), make_float2(-1.f, -1.f), r);  // exact
    const float2 f = add2(l, make_float2(kFine, kFine));
    high += __float_as_uint(t.x) + __float_as_uint(t.y);
    low += __float_as_uint(f.x) + __float_as_uint(f.y);
  }
  static constexpr float kFine = 1.52587890625e-05f * 0.75f;  // 1.5 * 2^-17, whose last place is 2^-40
  // Of n entries.
  __device__ __forceinline__ long long total(uint32_t n) const {
    return ((long long)(uint32_t)(high - n * 0x41400000u) << 20) + (int32_t)(low - n * 0x37400000u);
  }
  __device__ __forceinline__ long long warp_total(uint32_t n) const {  // n in all lanes
    Masses all;
    all.high = __reduce_add_sync(0xffffffffu, high), all.low = __reduce_add_sync(0xffffffffu, low);
    return all.total(n);
  }
};
__device__ __forceinline__ long long mass_of(float r) {
  Masses m;
  m.add(r, 0.f);
  return m.total(2);
}
__device__ __forceinline__ long long warp_sum(long long x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

// All threads of the cluster meet; what those that `wrote` wrote to the others' memory is seen there. (A release by every
// thread costs them all a wait for their stores.)
__device__ __forceinline__ void meet(int ctas, bool wrote) {
  if (ctas == 1) {
    __syncthreads();
    return;
  }
  if (wrote) asm volatile("fence.acq_rel.cluster;" ::: "memory");
  __syncwarp();
  cluster_arrive_relaxed();
  cluster_wait();
}

// What the CTA's warps are to do with a row.
struct Order {
  int node;       // whose row
  int draw;       // 0: the mass of R, 1: draw from it
  float c;
  uint64_t gone;  // nodes whose tokens are rejected here, no token twice
};
constexpr int kMarks = 32;       // sums of a warp's stretch that are kept for the search,
constexpr int kMarkPieces = 128;  // of so many pieces at least

template <bool DRAFT>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyProblem p) {
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t seq = blockIdx.x / cs;
  extern __shared__ float4 pieces[];
  __shared__ Order order;
  __shared__ int walked[kMaxNodes];
  __shared__ long long marks[kWarps][kMarks], warp_mass[kWarps], drawn;
  // Written by the cluster's CTAs.
  __shared__ long long cta_mass[2][kMaxCluster];
  __shared__ int nodes, parent[kMaxNodes], token[kMaxNodes];
  __shared__ float u[kMaxNodes], px[kMaxNodes], qx[kMaxNodes];
  const float* probs = p.probs + seq * p.p_seq;
  const float* draft = DRAFT ? p.draft + seq * p.q_seq : nullptr;
  cluster_arrive_relaxed();  // the others' memory is written to when they have begun

  // What the walk needs of the nodes: read by the first CTA for all, so that all walk alike.
  if (rank == 0) {
    const int n = p.counts == nullptr ? p.nodes : max(0, min(p.nodes, p.counts[seq]));
    int up = -1, x = 0;
    float w = 0.f, a = 0.f, b = 0.f;
    if (tid < n) {
      const int64_t at = seq * p.nodes + tid;
      up = p.parents[at], x = p.tokens[at], w = p.uniforms[at];
      if (!(tid > 0 && up >= 0 && up < n && x >= 0 && x < p.vocab)) up = -1;
      if (up >= 0) {
        a = __ldg(probs + up * p.p_node + x);
        if (DRAFT) b = __ldg(draft + up * p.q_node + x);
      }
    }
    cluster_wait();
    if (tid < kMaxNodes)
      for (int i = 0; i < cs; ++i) {
        *cluster.map_shared_rank(&parent[tid], i) = up;
        *cluster.map_shared_rank(&token[tid], i) = x;
        *cluster.map_shared_rank(&u[tid], i) = w;
        *cluster.map_shared_rank(&px[tid], i) = clamped(a);
        *cluster.map_shared_rank(&qx[tid], i) = clamped(b);
        if (tid == 0) *cluster.map_shared_rank(&nodes, i) = n;
      }
  } else {
    cluster_wait();
  }
  meet(cs, rank == 0 && tid < kMaxNodes);
  const int n = nodes;

  // A row's stretch of this CTA in 16-byte pieces from the boundary before the row on: entry v of the row is entry v +
  // skew of these pieces, whose first and last may lie outside in part. Each warp has a part of the stretch.
  int skew = 0, begin = 0, end = 0;
  bool together = false;  // P and Q lie alike
  const float *prow = nullptr, *qrow = nullptr;
  int row_node = -1;
  auto take_row = [&](int node) {
    if (node == row_node) return;
    row_node = node;
    prow = probs + node * p.p_node;
    qrow = DRAFT ? draft + node * p.q_node : nullptr;
    skew = (int)((uintptr_t)prow / 4 % 4);
    together = !DRAFT || (uintptr_t)qrow / 4 % 4 == skew;
    const int all = (p.vocab + skew + 3) / 4;  // at most 2^20 + 1
    const int shift = p.log_cluster + kLogWarps;  // at most 8
    begin = all * (rank * kWarps + warp) >> shift, end = all * (rank * kWarps + warp + 1) >> shift;
  };
  auto load = [&](int i, float4& a, float4& b) {  // entries outside the row are 0
    const int v = 4 * i - skew;
    const bool whole = v >= 0 && v + 4 <= p.vocab;
    if (whole) a = __ldg(reinterpret_cast<const float4*>(prow + v));
    if (DRAFT && whole && together) b = __ldg(reinterpret_cast<const float4*>(qrow + v));
    if (whole && together) return;
    float x[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool inside = v + e >= 0 && v + e < p.vocab;
      x[e] = inside ? __ldg(prow + v + e) : 0.f;
      y[e] = DRAFT && inside ? __ldg(qrow + v + e) : 0.f;
    }
    a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(y[0], y[1], y[2], y[3]);
  };
  float4* const held_p = pieces + warp * p.held;
  float4* const held_q = pieces + (kWarps + warp) * p.held;
  int kept_node = -1;
  // The warp's part to shared memory, each lane's own pieces.
  auto keep_row = [&](int node) {
    if (node == kept_node) return;
    kept_node = node;
    for (int i = begin + lane; i < end; i += 32) {
      const int v = 4 * i - skew;
      if (v >= 0 && v + 4 <= p.vocab && together) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&held_p[i - begin])), "l"(prow + v) : "memory");
        if (DRAFT)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(&held_q[i - begin])), "l"(qrow + v)
                       : "memory");
      } else {
        float4 a, b = make_float4(0.f, 0.f, 0.f, 0.f);
        load(i, a, b);
        held_p[i - begin] = a;
        if (DRAFT) held_q[i - begin] = b;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
  };
  const bool keeps = p.held > 0;
  auto fetch = [&](int i, float4& a, float4& b) {
    if (keeps) {
      a = held_p[i - begin];
      if (DRAFT) b = held_q[i - begin];
    } else {
      load(i, a, b);
    }
  };
  auto value = [&](float a, float b, float c) { return DRAFT ? residual(clamped(a), clamped(b), c) : clamped(a); };
  // What the rejected tokens among these pieces would add.
  auto gone_mass = [&](const Order& o, int from, int to) {
    long long sum = 0;
#pragma unroll
    for (int k = 0; k < kMaxNodes; k += 32) {
      const int at = (token[k + lane] + skew) / 4;
      if ((o.gone >> (k + lane) & 1) != 0 && at >= from && at < to) sum += mass_of(value(px[k + lane], qx[k + lane], o.c));
    }
    return warp_sum(sum);
  };
  // The masses of all CTAs' stretches of R, in cta_mass of this turn, and their sum. All threads of all CTAs. The warp's is
  // in warp_mass; up to every so many pieces of its stretch, with the rejected tokens, in marks.
  int turn = 0, step = 32;
  auto total_mass = [&](const Order& o) {
    turn ^= 1;
    take_row(o.node);
    if (keeps) keep_row(o.node);
    constexpr int U = DRAFT ? 2 : 4;
    static_assert(kMarkPieces % (32 * U) == 0, "");
    step = max(1, (end - begin + kMarkPieces * kMarks - 1) / (kMarkPieces * kMarks)) * kMarkPieces;  // from mark to mark
    long long upto = 0;
    for (int from = begin, mark = 0; from < end; from += step, ++mark) {
      for (int at = from; at < min(end, from + step); at += kMarkPieces) {
        Masses m;
        uint32_t entries = 0;
        for (int i = at; i < min(end, at + kMarkPieces); i += 32 * U) {
          entries += 32 * U * 4;
          float4 a[U], b[U];
          // All pieces in the stretch and, read from the row, in the row: no piece is looked at by itself.
          if (i + 32 * U <= end && (keeps || (together && 4 * i >= skew && 4 * (i + 32 * U) - skew <= p.vocab))) {
            const float4* x = keeps ? held_p + (i - begin) : reinterpret_cast<const float4*>(prow + 4 * i - skew);
            const float4* y = keeps ? held_q + (i - begin) : reinterpret_cast<const float4*>(qrow + 4 * i - skew);
#pragma unroll
            for (int k = 0; k < U; ++k) {
              a[k] = x[32 * k + lane];
              b[k] = DRAFT ? y[32 * k + lane] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
          } else {
#pragma unroll
            for (int k = 0; k < U; ++k) {
              a[k] = b[k] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (i + 32 * k + lane < end) fetch(i + 32 * k + lane, a[k], b[k]);
            }
          }
#pragma unroll
          for (int k = 0; k < U; ++k) {
            m.add(value(a[k].x, b[k].x, o.c), value(a[k].y, b[k].y, o.c));
            m.add(value(a[k].z, b[k].z, o.c), value(a[k].w, b[k].w, o.c));
          }
        }
        upto += m.warp_total(entries);
      }
      if (lane == 0) marks[warp][mark] = upto;
    }
    if (o.gone != 0) upto -= gone_mass(o, begin, end);
    if (lane == 0) warp_mass[warp] = upto;
    __syncthreads();
    if (tid < cs) {
      long long sum = 0;
      for (int w = 0; w < kWarps; ++w) sum += warp_mass[w];
      *cluster.map_shared_rank(&cta_mass[turn][rank], tid) = sum;
    }
    meet(cs, tid < cs);
    long long sum = 0;
    for (int i = 0; i < cs; ++i) sum += cta_mass[turn][i];
    return sum;
  };
  // Draws from R. The search is the warp's whose stretch the bound falls in.
  auto draw = [&](Order o) {
    long long all = total_mass(o);
    if (all <= 0) {  // nothing is left: from P
      o.c = 0.f, o.gone = 0;
      all = total_mass(o);
    }
    if (all <= 0) {
      if (rank == 0 && tid == 0) p.following[seq] = -1;
      return;
    }
    if (tid == 0) {  // FP64 is slow: one thread's
      const float u1 = fminf(fmaxf(u[0], 0.f), 0.99999994f);  // 1 - 2^-24; NaN is 0
      drawn = __double2ll_rd(__dmul_rn((double)u1, (double)all));
    }
    __syncthreads();
    long long bound = drawn;
    for (int i = 0; i < rank; ++i) bound -= cta_mass[turn][i];
    if (bound < 0 || bound >= cta_mass[turn][rank]) return;
    for (int w = 0; w < warp; ++w) bound -= warp_mass[w];
    if (bound < 0 || bound >= warp_mass[warp]) return;
    int from = begin;
    long long before = 0;
    for (int mark = 0; from + step < end; ++mark, from += step) {
      const long long upto = marks[warp][mark] - (o.gone != 0 ? gone_mass(o, begin, from + step) : 0);
      if (bound < upto) break;
      before = upto;
    }
    bound -= before;
    for (int i = from; i < end; i += 32) {
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
      const int at = i + lane;
      if (at < end) fetch(at, a, b);
      long long m[4] = {mass_of(value(a.x, b.x, o.c)), mass_of(value(a.y, b.y, o.c)), mass_of(value(a.z, b.z, o.c)),
                        mass_of(value(a.w, b.w, o.c))};
      for (uint64_t left = o.gone; left != 0; left &= left - 1) {
        const int place = token[__ffsll((long long)left) - 1] + skew - 4 * at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (place == e) m[e] = 0;
      }
      const long long sum = m[0] + m[1] + m[2] + m[3];
      long long upto = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long other = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += other;
      }
      const unsigned behind = __ballot_sync(0xffffffffu, upto > bound);
      if (behind != 0) {
        if (lane == __ffs(behind) - 1) {
          long long left = bound - (upto - sum);
          int e = 0;
          while (e < 3 && left >= m[e]) left -= m[e], ++e;
          p.following[seq] = 4 * at - skew + e;
        }
        return;
      }
      bound -= __shfl_sync(0xffffffffu, upto, 31);
    }
  };

  if (n == 0) {
    if (rank == 0) {
      for (int i = tid; i < p.nodes; i += kThreads) p.path[seq * p.nodes + i] = -1;
      if (tid == 0) p.lengths[seq] = 0, p.following[seq] = -1;
    }
    return;
  }
  // The walk is the first warp's of every CTA (FP64 is slow), whose lanes take the same steps; the others do the rows.
  if (warp != 0) {
    for (;;) {
      __syncthreads();  // the order is given
      const Order o = order;
      if (o.draw != 0) {
        draw(o);
        return;
      }
      total_mass(o);
    }
  }
  // Each lane keeps two nodes.
  const int parent0 = parent[lane], parent1 = parent[lane + 32], token0 = token[lane], token1 = token[lane + 32];
  auto nodes_with = [&](int x0, int x1, int x) {
    return (uint64_t)__ballot_sync(0xffffffffu, x1 == x) << 32 | __ballot_sync(0xffffffffu, x0 == x);
  };
  int at = 0, length = 1;
  uint64_t left = nodes_with(parent0, parent1, 0), gone = 0;
  double c = 0.0, z = 1.0, zq = 1.0;
  float near_z = 1.f, near_zq = 1.f;
  bool stale = false;  // z is of the residual before
  if (lane == 0) walked[0] = 0;
  while (left != 0) {
    const int child = __ffsll((long long)left) - 1;
    left &= left - 1;
    const bool again = (nodes_with(token0, token1, token[child]) & gone) != 0;
    if (DRAFT && (!(zq > 0.0) || (again && p.distinct))) continue;
    if (stale) {
      if (lane == 0) order = {at, 0, (float)c, gone};
      __syncthreads();
      const long long mass = total_mass(order);
      z = (double)mass * (1.0 / kUnit), near_z = (float)mass * (float)(1.0 / kUnit);
      stale = false;
    }
    // Clear cases are decided in FP32, whose errors are far below these margins, without waiting for FP64, which is slow.
    const float r = again ? 0.f : DRAFT ? residual(px[child], qx[child], (float)c) : px[child];
    const float near_reach = DRAFT ? u[child] * qx[child] * near_z : u[child] * near_z, near_r = DRAFT ? r * near_zq : r;
    const float margin = 2e-5f * (near_reach + near_r) + 1e-5f * (DRAFT ? r : u[child]) + 1e-35f;
    bool accepted = near_r - near_reach > margin;
    if (!accepted && !(near_reach - near_r > margin)) {
      if (!DRAFT) {
        z = 1.0;
        for (uint64_t some = gone; some != 0; some &= some - 1) z = __dsub_rn(z, (double)px[__ffsll((long long)some) - 1]);
      }
      const double reach = DRAFT ? __dmul_rn(__dmul_rn(u[child], qx[child]), z) : __dmul_rn(u[child], z);
      accepted = reach < (DRAFT ? __dmul_rn(r, zq) : (double)r);
    }
    if (accepted) {
      if (lane == 0) walked[length] = child;
      ++length;
      at = child, left = nodes_with(parent0, parent1, at), gone = 0;
      c = 0.0, z = zq = 1.0, near_z = near_zq = 1.f;
      continue;
    }
    if (DRAFT) {
      c = __dadd_rn(c, zq == 1.0 ? z : __ddiv_rn(z, zq));
      if (p.distinct) zq = __dsub_rn(zq, (double)qx[child]), near_zq -= qx[child];
      stale = true;
    } else {
      near_z -= r;
    }
    if (!again) gone |= 1ull << child;
  }
  if (lane == 0) order = {at, 1, (float)c, gone};
  __syncthreads();
  draw(order);
  if (rank == 0) {
    for (int i = lane; i < p.nodes; i += 32) p.path[seq * p.nodes + i] = i < length ? walked[i] : -1;
    if (lane == 0) p.lengths[seq] = length;
  }
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_verify_tree: " + msg); }

bool span_ok(int64_t n, int64_t stride) { return stride >= 0 && (n <= 1 || stride <= ((int64_t)1 << 60) / n); }

template <bool DRAFT>
cudaError_t launch(const VerifyProblem& p, int64_t sequences, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sequences * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = p.held * kWarps * 16 * (DRAFT ? 2 : 1);
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = once_per_device(done, [] {
    const cudaError_t first = cudaFuncSetAttribute(verify_kernel<DRAFT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostHeld);
    if (first != cudaSuccess) return first;
    return cudaFuncSetAttribute(verify_kernel<DRAFT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  if (e != cudaSuccess) return e;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_kernel<DRAFT>, p);
}

}  // namespace
}  // namespace af1

using namespace af1;

int af1_verify_tree(const af1_verify_args* a, void* stream) {
  if (a == nullptr) return fail(AF1_ERR_INVALID_ARG, "args is NULL");
  if (a->sequences < 0 || a->sequences > 65536 || a->nodes < 1 || a->nodes > kMaxNodes || a->vocab < 1 ||
      a->vocab > (1 << 22))
    return fail(AF1_ERR_INVALID_ARG, "need 0..65536 sequences, 1..64 nodes and 1..2^22 tokens in the vocabulary");
  const bool draft = a->draft != nullptr;
  if (!span_ok(a->sequences, a->probs_seq) || !span_ok(a->nodes, a->probs_node) ||
      (draft && (!span_ok(a->sequences, a->draft_seq) || !span_ok(a->nodes, a->draft_node))))
    return fail(AF1_ERR_INVALID_ARG, "strides must not be negative");
  if ((a->flags & ~AF1_VERIFY_DISTINCT) != 0) return fail(AF1_ERR_INVALID_ARG, "unknown flags");
  if (a->flags != 0 && !draft) return fail(AF1_ERR_INVALID_ARG, "AF1_VERIFY_DISTINCT is of drafted probabilities");
  if (a->reserved != 0) return fail(AF1_ERR_INVALID_ARG, "reserved must be 0");
  if (a->sequences == 0) return AF1_OK;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, cudaGetErrorString(e));
  struct {
    const void* p;
    const char* name;
    bool need;
  } ptrs[] = {{a->probs, "probs", true},         {a->draft, "draft", false},  {a->tokens, "tokens", true},
              {a->parents, "parents", true},     {a->counts, "counts", false}, {a->uniforms, "uniforms", true},
              {a->path, "path", true},           {a->lengths, "lengths", true}, {a->following, "following", true}};
  for (const auto& t : ptrs) {
    if (t.p == nullptr && !t.need) continue;
    int rc;
    if ((rc = check_pointer(t.p, t.name, dev)) != AF1_OK || (rc = check_align(t.p, 4, t.name)) != AF1_OK) return rc;
  }
  VerifyProblem p = {a->probs,  a->probs_seq, a->probs_node, a->draft,   a->draft_seq,  a->draft_node, a->tokens,
                     a->parents, a->counts,   a->uniforms,   a->path,    a->lengths,    a->following,  (int)a->nodes,
                     (int)a->vocab, (a->flags & AF1_VERIFY_DISTINCT) != 0, 0, 0};
  // CTAs of a sequence: as many as two to an SM allow, while each of their warps has 128 entries (one tree over 128000
  // tokens: 8 CTAs 9.9 us, 16 7.8). Clusters lie within parts of the GPU, whose SMs are no multiple of theirs: at one CTA
  // to an SM there is room for 7 clusters of 16, 15 of 8, 36 of 4 and 76 of 2 (16 trees, kept rows of 128 KB a CTA: 16
  // clusters of 8 came in two waves and took 9 us for a sum, where reading the rows again takes 5).
  const int64_t alone[] = {sms, sms / 2, sms * 36 / 152, sms * 15 / 152, sms * 7 / 152};
  int level = 0;
  while (level < 4 && a->sequences <= 2 * alone[level + 1] && a->vocab >= (128 * kWarps << (level + 1))) ++level;
  const int cluster = 1 << level;
  p.log_cluster = level;
  // A row that may be summed more than once is kept, where all CTAs have room for their parts at once.
  const int64_t part = ((a->vocab + 3 + 3) / 4 + cluster * kWarps - 1) / (cluster * kWarps) + 1;
  const int64_t room = a->sequences <= alone[level] ? kMostHeld : kMostHeld / 2;
  if (draft && part * kWarps * 32 <= room) p.held = (int)part;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  e = draft ? launch<true>(p, a->sequences, cluster, st) : launch<false>(p, a->sequences, cluster, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
