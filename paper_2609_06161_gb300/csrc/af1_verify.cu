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
// numbers are FP64. A sum of whole numbers costs no wide arithmetic: an FP32
// addition of 12 and back splits r into a multiple of 2^-20 and a rest, another
// addition rounds the rest to a multiple of 2^-40, and 16 of either add up
// exactly in FP32 before they go to 64-bit integers.
//
// A cluster of CTAs takes a sequence. The numbers that the walk needs (four to a
// node) are fetched for all nodes at once; its first CTA walks, the
// others wait for rows to sum: every CTA has a stretch of the vocabulary, so
// that a row is summed and then searched (one warp's stretch) where the sum of
// the stretches before passes the bound. Only rows that the walk needs are read.
#include <cooperative_groups.h>

#include <algorithm>

#include "af1_internal.h"
#include "af1_kv.cuh"

namespace cg = cooperative_groups;

namespace af1 {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxNodes = 64;
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
};

// Probabilities as they count: 0 to 1, NaN as 0.
__device__ __forceinline__ float clamped(float p) { return fminf(fmaxf(p, 0.f), 1.f); }
__device__ __forceinline__ float residual(float p, float q, float c) {
  return fmaxf(__fsub_rn(p, __fmul_rn(c, q)), 0.f);
}
// Sums of masses of at most 16 entries each, until they are added up.
struct Masses {
  float high = 0.f, low = 0.f;
  __device__ __forceinline__ void add(float r) {
    const float h = __fsub_rn(__fadd_rn(r, 12.f), 12.f);  // to 2^-20
    constexpr float kFine = 1.52587890625e-05f * 0.75f;    // 1.5 * 2^-17, whose last place is 2^-40
    const float l = __fsub_rn(__fadd_rn(__fsub_rn(r, h), kFine), kFine);
    high = __fadd_rn(high, h);
    low = __fadd_rn(low, l);
  }
  __device__ __forceinline__ long long total() const {
    return ((long long)__float2int_rn(high * 1048576.f) << 20) + __float2int_rn(low * 1099511627776.f);
  }
};

__device__ __forceinline__ long long mass_of(float r) {
  Masses m;
  m.add(r);
  return m.total();
}
__device__ __forceinline__ long long warp_sum(long long x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

// What the cluster's CTAs are to do with a row.
struct Order {
  int what;   // 0: nothing more, 1: the mass of R, 2: draw from it
  int node;   // whose row
  float c;
  float u;    // of the draw
  int gone;   // tokens rejected here
};
struct Gone {
  int token;
  float p, q;
};

template <bool DRAFT>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyProblem p) {
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t seq = blockIdx.x / cs;
  __shared__ Order order;
  __shared__ Gone gone[kMaxNodes];
  __shared__ long long warp_mass[kWarps], cta_mass[kMaxCluster];  // cta_mass: of all CTAs, written by each
  __shared__ long long drawn;
  __shared__ int parent[kMaxNodes], token[kMaxNodes];
  __shared__ float u[kMaxNodes], px[kMaxNodes], qx[kMaxNodes];
  const float* probs = p.probs + seq * p.p_seq;
  const float* draft = DRAFT ? p.draft + seq * p.q_seq : nullptr;

  // One row's stretch of this warp, in 16-byte accesses from the boundary before the row on: entry `v` of the row is
  // entry v + skew of these accesses, whose first and last may lie outside in part.
  int begin = 0, end = 0;  // accesses
  int skew = 0;
  bool together = false;  // P and Q lie alike
  const float *prow = nullptr, *qrow = nullptr;
  auto take_row = [&](int node) {
    prow = probs + node * p.p_node;
    qrow = DRAFT ? draft + node * p.q_node : nullptr;
    skew = (int)((uintptr_t)prow / 4 % 4);
    together = !DRAFT || (uintptr_t)qrow / 4 % 4 == skew;
    const int all = (p.vocab + skew + 3) / 4;  // at most 2^20 + 1
    const int parts = cs * kWarps, part = rank * kWarps + warp;  // at most 128
    begin = all * part / parts, end = all * (part + 1) / parts;
  };
  auto load = [&](int i, float (&a)[4], float (&b)[4]) {  // entries outside the row are 0
    const int v = 4 * i - skew;
    const bool whole = v >= 0 && v + 4 <= p.vocab;
    if (whole) {
      const float4 x = __ldg(reinterpret_cast<const float4*>(prow + v));
      a[0] = x.x, a[1] = x.y, a[2] = x.z, a[3] = x.w;
    }
    if (DRAFT && whole && together) {
      const float4 x = __ldg(reinterpret_cast<const float4*>(qrow + v));
      b[0] = x.x, b[1] = x.y, b[2] = x.z, b[3] = x.w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool inside = v + e >= 0 && v + e < p.vocab;
      if (!whole) a[e] = inside ? __ldg(prow + v + e) : 0.f;
      if (DRAFT && !(whole && together)) b[e] = inside ? __ldg(qrow + v + e) : 0.f;
    }
  };
  auto value = [&](float a, float b, float c) { return DRAFT ? residual(clamped(a), clamped(b), c) : clamped(a); };
  // The mass of this warp's stretch of R.
  auto warp_total = [&](float c, int n_gone) {
    long long sum = 0;
    constexpr int U = DRAFT ? 2 : 4;
    for (int i = begin; i < end; i += 32 * U) {
      float a[U][4], b[U][4];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int at = i + 32 * k + lane;
        if (at < end) {
          load(at, a[k], b[k]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) a[k][e] = b[k][e] = 0.f;
        }
      }
      Masses m;
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) m.add(value(a[k][e], b[k][e], c));
      sum += m.total();
    }
    for (int g = lane; g < n_gone; g += 32) {
      const int at = (gone[g].token + skew) / 4;
      if (at >= begin && at < end) sum -= mass_of(value(gone[g].p, gone[g].q, c));
    }
    return warp_sum(sum);
  };
  // The masses of all CTAs, in cta_mass; the returned one is their sum. All threads of all CTAs.
  auto total_mass = [&](const Order& o) {
    take_row(o.node);
    const long long mine = warp_total(o.c, o.gone);
    if (lane == 0) warp_mass[warp] = mine;
    __syncthreads();
    if (tid < cs) {
      long long sum = 0;
      for (int w = 0; w < kWarps; ++w) sum += warp_mass[w];
      *cluster.map_shared_rank(&cta_mass[rank], tid) = sum;
    }
    cluster.sync();
    long long sum = 0;
    for (int i = 0; i < cs; ++i) sum += cta_mass[i];
    return sum;
  };
  // Everyone gets the first CTA's order, and the tokens that it leaves out.
  auto receive = [&] {
    cluster.sync();  // it is written
    const Order o = *cluster.map_shared_rank(&order, 0);
    if (rank != 0 && tid < o.gone) gone[tid] = *cluster.map_shared_rank(&gone[tid], 0);
    __syncthreads();
    return o;
  };
  // Draws from R. The search is the CTA's whose stretch the bound falls in.
  auto draw = [&](Order o) {
    long long all = total_mass(o);
    if (all <= 0) {  // nothing is left: from P
      cluster.sync();  // cta_mass was read
      o.c = 0.f, o.gone = 0;
      all = total_mass(o);
    }
    if (all <= 0) {
      if (rank == 0 && tid == 0) p.following[seq] = -1;
      return;
    }
    if (tid == 0) {  // FP64 is slow: one thread's
      const float u1 = fminf(fmaxf(o.u, 0.f), 0.99999994f);  // 1 - 2^-24; NaN is 0
      drawn = __double2ll_rd(__dmul_rn((double)u1, (double)all));
    }
    __syncthreads();
    long long bound = drawn;
    for (int i = 0; i < rank; ++i) bound -= cta_mass[i];
    if (bound < 0 || bound >= cta_mass[rank]) return;
    for (int w = 0; w < warp; ++w) bound -= warp_mass[w];
    if (bound < 0 || bound >= warp_mass[warp]) return;
    for (int i = begin; i < end; i += 32) {
      float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
      const int at = i + lane;
      if (at < end) load(at, a, b);
      long long m[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = mass_of(value(a[e], b[e], o.c));
        for (int g = 0; g < o.gone; ++g)
          if (gone[g].token == 4 * at - skew + e) m[e] = 0;
        sum += m[e];
      }
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

  auto follow = [&] {
    for (;;) {
      const Order o = receive();
      if (o.what == 0) {
        cluster.sync();  // the first CTA's memory was read
        return;
      }
      if (o.what == 2) {
        draw(o);
        return;
      }
      total_mass(o);
    }
  };
  if (rank != 0) {
    follow();
    return;
  }

  const int n = p.counts == nullptr ? p.nodes : max(0, min(p.nodes, p.counts[seq]));
  if (tid < p.nodes) {
    const int64_t at = seq * p.nodes + tid;
    const int up = p.parents[at], x = p.tokens[at];
    const bool real = tid > 0 && tid < n && up >= 0 && up < n && x >= 0 && x < p.vocab;
    parent[tid] = real ? up : -1;
    token[tid] = x;
    u[tid] = p.uniforms[at];
    px[tid] = real ? clamped(probs[up * p.p_node + x]) : 0.f;
    qx[tid] = DRAFT && real ? clamped(draft[up * p.q_node + x]) : 0.f;
  }
  __syncthreads();
  // The walk is one warp's (FP64 is slow), whose lanes take the same steps; its first writes.
  if (warp != 0) {
    follow();
    return;
  }
  int at = 0, length = 1, n_gone = 0;
  double c = 0.0, z = 1.0, zq = 1.0;
  bool stale = false;  // z is of the residual before
  if (n > 0 && tid == 0) p.path[seq * p.nodes] = 0;
  for (int i = 1; n > 0;) {
    while (i < n && parent[i] != at) ++i;
    if (i >= n) break;
    const int child = i++;
    int seen = 0;
    while (seen < n_gone && gone[seen].token != token[child]) ++seen;
    const bool again = seen < n_gone;
    if (DRAFT && (!(zq > 0.0) || (again && p.distinct))) continue;
    if (stale) {
      if (tid == 0) order = {1, at, (float)c, 0.f, n_gone};
      const Order o = receive();
      z = (double)total_mass(o) * (1.0 / kUnit);
      stale = false;
    }
    const double r = again ? 0.f : DRAFT ? residual(px[child], qx[child], (float)c) : px[child];
    const double left = DRAFT ? __dmul_rn(__dmul_rn(u[child], qx[child]), z) : __dmul_rn(u[child], z);
    if (left < (DRAFT ? __dmul_rn(r, zq) : r)) {
      if (tid == 0) p.path[seq * p.nodes + length] = child;
      ++length;
      at = child, i = 1, n_gone = 0;
      c = 0.0, z = zq = 1.0;
      continue;
    }
    if (DRAFT) {
      c = __dadd_rn(c, __ddiv_rn(z, zq));
      if (p.distinct) zq = __dsub_rn(zq, (double)qx[child]);
      stale = true;
    } else {
      z = __dsub_rn(z, r);
    }
    __syncwarp();  // the list was read
    if (!again) {
      if (tid == 0) gone[n_gone] = {token[child], px[child], qx[child]};
      ++n_gone;
    }
    __syncwarp();
  }
  if (n == 0) length = 0;
  for (int i = length + lane; i < p.nodes; i += 32) p.path[seq * p.nodes + i] = -1;
  if (tid == 0) {
    p.lengths[seq] = length;
    order = {n > 0 ? 2 : 0, at, (float)c, u[0], n_gone};
    if (n == 0) p.following[seq] = -1;
  }
  const Order o = receive();
  if (o.what == 2)
    draw(o);
  else
    cluster.sync();
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_verify_tree: " + msg); }

bool span_ok(int64_t n, int64_t stride) { return stride >= 0 && (n <= 1 || stride <= ((int64_t)1 << 60) / n); }

template <bool DRAFT>
cudaError_t launch(const VerifyProblem& p, int64_t sequences, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sequences * cluster));
  cfg.blockDim = dim3(kThreads);
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
                     (int)a->vocab, (a->flags & AF1_VERIFY_DISTINCT) != 0};
  // CTAs of a sequence: as many as two to an SM allow, while each of their warps has 128 entries.
  int cluster = 1;
  while (cluster < kMaxCluster && a->sequences * cluster * 2 <= 2 * sms && a->vocab >= 2 * cluster * kWarps * 128) cluster *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  e = draft ? launch<true>(p, a->sequences, cluster, st) : launch<false>(p, a->sequences, cluster, st);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}
