// af1_tree.cu — attention of a few new tokens (a tree of drafted tokens, or
// one token) over a paged cache of keys and values.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i k_j - m_i)
//
// over the keys j that node i sees. The q_heads / kv_heads query heads of all
// nodes that share a cached head are the rows of one product, so that the
// cache is read once for all of them.
//
// Split. An item is one sequence and one cached head, with 8 NT rows at most;
// its keys are cut into units of kUnit, and every CTA takes an equal run of
// the units of all items (ragged lengths balance by themselves; each item
// counts some units more, for what a run costs whatever its length: without
// them the CTA that had eight short items ran 102 us where the others ran 70).
// Inside a CTA each warp takes every W-th step of KW keys of a run, with a ring
// of its own in shared memory that TMA fills, its own running maximum m and sum
// l, and an accumulator in registers; warps meet once a run, to join (m, l, o).
// Where an item spans CTAs, each leaves its part in the workspace and the
// last one to arrive joins them in order, so that results do not depend on
// timing.
//
// Products. Few rows and many keys: the keys are the 16 rows of the products
// S^T = K Q^T, the entries of a value those of O^T = V^T P^T (m16n8k16, FP32
// accumulators), and 8 rows of q a column block, so that nothing is computed
// for rows that do not exist beyond a block of 8. A contraction may run in any
// order: the entries of a key go to the product's k index in the order in
// which one lane's reads give them, and q is laid out to match.
//
// Codes become exact FP16 values in registers. Those of the keys of INT4 and
// INT8 (plus 128) go in as the fraction bits of FP16 subnormals, 2^-24 times
// the code, at one mask or byte permutation for two entries; the 128 and the
// 2^24 are taken back in the FP32 scores, where 128 sum q is a constant of the
// row. (A value's 128 would have to be taken back from a sum over all keys, in
// which it is far larger than the result, so values of INT8 are made signed.)
// Scales stay in FP32: a key's multiplies its scores (INT4: those of each
// group of 32 entries, whose lows are contracted with the sums of q over the
// groups), so that no entry of a key is rounded; a value's multiplies the
// weights p. Only INT4's values, code * scale + low, are rounded to FP16: with
// p times the scale in place of p, errors of the two terms would not cancel
// where they do.
// p is rounded to FP16, times 2^kShift, relative to a maximum that is moved
// only when a score passes it by 2^kSlack, and to the largest value scale so
// far; m, l, scores and outputs are FP32. Of INT4, whose values are rounded, too,
// what rounding adds to the largest weight of every 4 is added to the divisor as
// well, where it cancels most of what it adds to the output: 2.8e-4 of the norm for
// one token over 4000 keys where it was 2.9e-4, and at most 1.43 times what FP16
// outputs make where it was 1.62 (32 sequences of up to 8192 tokens 76 us for 74).
//
// Bound: device memory where contexts are long (32 sequences of up to 8192 INT8
// tokens, 8 heads of 128, 4 queries each: 70 us, 0.86 of the copy rate), latency
// where they are short (1000 FP16 tokens: 9 us).
#include "af1_tree.cuh"

namespace af1 {
namespace {

constexpr int kUnit = 64;                         // keys of a unit
constexpr int kMinRun = 256;                      // keys of a CTA, at least (where there are so many)
constexpr int kSetup = 10;                        // units that a run's beginning and end are worth (with 4, 4 trees
                                                  // of 4 over 8000 E4M3 tokens took 33 us instead of 31; 16: 30,
                                                  // but 32 long INT4 sequences 77 instead of 74)
constexpr float kCode = 16777216.f;               // 2^24: codes as subnormals

template <int KIND, int DIM, int NT, int W, int KW, int STAGES>
struct Shape {
  using C = Kv<KIND, DIM>;
  static constexpr int ROWS = 8 * NT;
  static constexpr int RING = W * STAGES * 2 * KW * C::RB;    // k and v of every stage of every warp
  static constexpr int SCALES = W * STAGES * 2 * KW * C::SB;
  static constexpr int JOIN = W * ROWS * DIM * 4;             // the warps' o, over the ring
  static constexpr int SMEM = RING + SCALES + 1024;
  static constexpr int PART = ROWS * (DIM + 2);               // floats of a part: o, m, l
  static_assert(JOIN <= RING, "the warps' outputs are joined over their rings");
  static_assert((KW * C::RB) % 512 == 0, "a stage keeps the swizzle's alignment");
};

template <int KIND, int DIM, int NT, int W, int KW, int STAGES, int CTAS>
__global__ void __launch_bounds__(32 * W, CTAS) tree_kernel(const __grid_constant__ TreeProblem p) {
  using C = Kv<KIND, DIM>;
  using S = Shape<KIND, DIM, NT, W, KW, STAGES>;
  constexpr int KS = C::KS, MT = C::MT, MB = KW / 16, ROWS = S::ROWS, GROUPS = C::GROUPS;
  constexpr int WORDS = C::RB / 16;        // 32-bit words of a key that one lane holds
  constexpr int STAGE = 2 * KW * C::RB;    // bytes of a step's k and v
  constexpr bool INT4 = KIND == AF1_KV_INT4;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[W][STAGES];
  __shared__ float join_m[W][ROWS], join_l[W][ROWS];
  __shared__ bool last_shared;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int g = lane / 4, t = lane % 4;
  uint8_t* ring = smem + warp * (STAGES * STAGE);
  uint8_t* ring_scales = smem + S::RING + warp * (STAGES * 2 * KW * C::SB);
  float* join = reinterpret_cast<float*>(smem);

  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) mbar_init(&bars[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();

  // This CTA's units: begin .. end - 1 of all items'.
  const int64_t lanes = p.cache.heads;
  Sequences<kUnit, kSetup> sq;
  const int64_t total = sq.begin(p) * lanes;
  int64_t ctas = min((int64_t)gridDim.x, (total * kUnit + kMinRun - 1) / kMinRun);
  ctas = min(ctas, total);  // each has a unit at least
  if (blockIdx.x >= ctas) return;
  // The first `more` CTAs have one unit more than the others.
  const int64_t per = total / ctas, more = total - per * ctas;
  const int64_t begin = per * blockIdx.x + min((int64_t)blockIdx.x, more);
  const int64_t end = begin + per + (blockIdx.x < more ? 1 : 0);

  const int rows = p.nodes * p.group;
  uint32_t phases = 0;   // of the warp's barriers
  bool alive = true;     // no wait has given up
  for (int64_t pos = begin; pos < end;) {
    while (sq.after() * lanes <= pos) sq.load(p, sq.first + 32, sq.after());
    const int which = __popc(__ballot_sync(0xffffffffu, (sq.before + sq.sum) * lanes <= pos));
    const int seq = sq.first + which;
    const int units = __shfl_sync(0xffffffffu, sq.units, which);
    const int len = __shfl_sync(0xffffffffu, sq.len, which), keys = __shfl_sync(0xffffffffu, sq.keys, which);
    const int64_t seq_first = (sq.before + __shfl_sync(0xffffffffu, sq.sum, which) - units) * lanes;
    const int head = (int)((pos - seq_first) / units);
    const int64_t first = seq_first + (int64_t)head * units;  // the item's first unit
    const int from = (int)(pos - first), to = (int)min((int64_t)units, from + (end - pos));
    const int u0 = max(from - kSetup, 0), u1 = to - kSetup;  // units of keys
    pos += to - from;
    const int k_begin = u0 * kUnit, k_end = min(u1 * kUnit, keys);

    if (keys == 0 && from == 0) {  // nothing to see: the item's first CTA writes its zeros
      for (int i = threadIdx.x; i < rows * DIM; i += 32 * W) {
        const int lr = i / DIM, e = i % DIM, node = lr / p.group, h = head * p.group + lr - node * p.group;
        const int64_t at = seq * p.o_seq + node * p.o_node + h * p.o_head + e;
        if (p.out_f32) static_cast<float*>(p.out)[at] = 0.f;
        else static_cast<__half*>(p.out)[at] = __ushort_as_half(0);
        if (e == 0 && p.lse != nullptr)
          p.lse[((int64_t)seq * p.nodes + node) * p.cache.heads * p.group + h] = -kInf;
      }
    }
    if (u1 <= 0) continue;

    // -- copies -------------------------------------------------------------
    constexpr int STRIDE = W * KW;
    const int key0 = k_begin + warp * KW;  // this warp's steps: key0, key0 + STRIDE, ...
    const int32_t* page_row = p.pages.pages + seq * p.pages.ld;
    const bool one_box = KW == 16 || p.cache.shift >= 5;  // a step lies in one page
    int next_page[MB];
    auto fetch_pages = [&](int key) {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int k = key + 16 * i;
        next_page[i] = (i == 0 || !one_box) && k < k_end ? page_row[k >> p.cache.shift] : -1;
      }
    };
    uint32_t bad_pages = 0;  // two bits a stage: 16 keys each whose page is missing
    auto issue = [&](int key, int slot) {  // the step of KW keys at `key`, whose pages were fetched
      uint32_t bad = 0;
      const int boxes = one_box ? 1 : MB;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const bool ok = next_page[i] >= 0 && next_page[i] < p.cache.pages;
        if (i < boxes && !ok && key + 16 * i < k_end) bad |= one_box ? 3u : 1u << i;
      }
      bad_pages = (bad_pages & ~(3u << (2 * slot))) | bad << (2 * slot);
      if (lane == 0) {
        uint64_t* bar = &bars[warp][slot];
        const int box = KW / boxes;
        int have = 0;
#pragma unroll
        for (int i = 0; i < MB; ++i) have += i < boxes && next_page[i] >= 0 && next_page[i] < p.cache.pages;
        mbar_expect_tx(bar, have * box * 2 * (C::RB + C::SB));
        uint8_t* to = ring + slot * STAGE;
        uint8_t* scales = ring_scales + slot * (2 * KW * C::SB);
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          if (i >= boxes || next_page[i] < 0 || next_page[i] >= p.cache.pages) continue;
          const int64_t row = (((int64_t)next_page[i] * p.cache.heads + head) << p.cache.shift) +
                              ((key + 16 * i) & ((1 << p.cache.shift) - 1));
#pragma unroll
          for (int s = 0; s < C::SLICES; ++s) {
            const int off = s * (KW * 128) + i * 16 * C::SPAN;
            tma_rows(smem_u32(to + off), &p.k_map, s * 128, (int)row, bar);
            tma_rows(smem_u32(to + KW * C::RB + off), &p.v_map, s * 128, (int)row, bar);
          }
          if constexpr (C::SB > 0) {
            bulk_g2s(scales + i * 16 * C::SB, static_cast<const uint8_t*>(p.cache.ks) + row * C::SB, box * C::SB, bar);
            bulk_g2s(scales + (KW + i * 16) * C::SB, static_cast<const uint8_t*>(p.cache.vs) + row * C::SB,
                     box * C::SB, bar);
          }
        }
      }
    };
    fetch_pages(key0);

    // -- q: the b operands, and its sums over the entries of a group -----------
    uint32_t qf[NT][KS][2];
    float q128[NT][2];           // INT8: 128 sum q of rows 2 t and 2 t + 1
    uint32_t q_sums[INT4 ? NT : 1];  // INT4: sum q / 32 over group t of row g, in two parts
    auto load_q = [&](int nt, uint32_t (&b)[KS][2]) {
      const int lr = nt * 8 + g, node = lr / p.group;
      const __half* row = p.q + seq * p.q_seq + node * p.q_node + (int64_t)(head * p.group + lr - node * p.group) * p.q_head;
      float sum[GROUPS];
#pragma unroll
      for (int c = 0; c < GROUPS; ++c) sum[c] = 0.f;
      auto add = [&](int c, uint32_t w) { sum[c] += low_float(w) + high_float(w); };
      if constexpr (INT4) {
#pragma unroll
        for (int c = 0; c < GROUPS; ++c) {
          const uint4 w = lr < rows ? *reinterpret_cast<const uint4*>(row + 32 * c + 8 * t) : make_uint4(0, 0, 0, 0);
          b[2 * c][0] = prmt(w.x, w.z, 0x5410), b[2 * c][1] = prmt(w.y, w.w, 0x5410);
          b[2 * c + 1][0] = prmt(w.x, w.z, 0x7632), b[2 * c + 1][1] = prmt(w.y, w.w, 0x7632);
          add(c, w.x), add(c, w.y), add(c, w.z), add(c, w.w);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint2 w = lr < rows ? *reinterpret_cast<const uint2*>(row + C::entry(t, ks, 0)) : make_uint2(0, 0);
          b[ks][0] = w.x, b[ks][1] = w.y;
          if constexpr (KIND == AF1_KV_INT8) add(0, w.x), add(0, w.y);
        }
      }
      if constexpr (INT4 || KIND == AF1_KV_INT8) {
#pragma unroll
        for (int c = 0; c < GROUPS; ++c) {
          sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], 1);
          sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], 2);
        }
      }
      if constexpr (KIND == AF1_KV_INT8) {
        q128[nt][0] = 128.f * __shfl_sync(0xffffffffu, sum[0], 8 * t);
        q128[nt][1] = 128.f * __shfl_sync(0xffffffffu, sum[0], 8 * t + 4);
      }
      if constexpr (INT4) {
        float mine = 0.f;
#pragma unroll
        for (int c = 0; c < GROUPS; ++c)
          if (c == t) mine = sum[c] * (1.f / 32.f);
        const float hi = __half2float(__float2half_rn(mine));
        q_sums[nt] = pack_half2(hi, mine - hi);
      }
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) load_q(nt, qf[nt]);

    int issued = 0;  // steps of this run
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
      const int key = key0 + s * STRIDE;
      if (key < k_end && alive) {
        issue(key, s);
        ++issued;
        fetch_pages(key + STRIDE);
      }
    }

    // o^T: block m, column block nt: entries row_entry(m, g, i / 2) of rows 2 t + i % 2.
    float o[MT][NT][4], m[NT][2], l[NT][2], over[NT][2], vref = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.f;
      m[nt][0] = m[nt][1] = -kInf, l[nt][0] = l[nt][1] = over[nt][0] = over[nt][1] = 0.f;
    }

    // -- steps ---------------------------------------------------------------------
    int slot = 0, waited = 0;
    for (int key = key0; key < k_end && alive; key += STRIDE) {
      {
        const int ahead = key + (STAGES - 1) * STRIDE;
        int to = slot + STAGES - 1;
        if (to >= STAGES) to -= STAGES;
        if (ahead < k_end) {
          issue(ahead, to);
          ++issued;
          fetch_pages(ahead + STRIDE);
        }
      }
      alive = __all_sync(0xffffffffu, wait_phase(&bars[warp][slot], phases >> slot & 1, p.wait_cycles));
      if (!alive) break;
      phases ^= 1u << slot;
      ++waited;
      const uint8_t* kb = ring + slot * STAGE;
      const uint8_t* vb = kb + KW * C::RB;
      const uint8_t* ksb = ring_scales + slot * (2 * KW * C::SB);
      const uint8_t* vsb = ksb + KW * C::SB;
      const uint32_t bad = bad_pages >> (2 * slot) & 3u;

      // Scores of keys mb 16 + g + 8 (i / 2), rows 2 t + i % 2.
      float s[MB][NT][4];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        uint32_t w[2][WORDS];
#pragma unroll
        for (int h = 0; h < 2; ++h) load_key<C, KIND, KW>(w[h], kb, mb * 16 + 8 * h + g, t);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[mb][nt][0] = s[mb][nt][1] = s[mb][nt][2] = s[mb][nt][3] = 0.f;
        if constexpr (INT4) {
          const uint32_t* sc = reinterpret_cast<const uint32_t*>(ksb);
          uint32_t a[4] = {0, 0, 0, 0};
          float key_scale[2][GROUPS];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = (mb * 16 + 8 * h + g) * GROUPS;
            const uint32_t low = GROUPS == 4 || t < GROUPS ? sc[at + (GROUPS == 4 ? t : t & 1)] : 0;
            a[h] = prmt(low, low, 0x3232);
#pragma unroll
            for (int c = 0; c < GROUPS; ++c) key_scale[h][c] = low_float(sc[at + c]) * (kCode / 32.f);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma(s[mb][nt], a, q_sums[nt], 0);
#pragma unroll
          for (int c = 0; c < GROUPS; ++c) {
            uint32_t a0[4], a1[4];
            key_operand<KIND>(a0, w, 2 * c);
            key_operand<KIND>(a1, w, 2 * c + 1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float acc[4] = {0.f, 0.f, 0.f, 0.f};
              mma(acc, a0, qf[nt][2 * c][0], qf[nt][2 * c][1]);
              mma(acc, a1, qf[nt][2 * c + 1][0], qf[nt][2 * c + 1][1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) s[mb][nt][i] = fmaf(acc[i], key_scale[i / 2][c], s[mb][nt][i]);
            }
          }
          const float f = 32.f * p.scale_log2;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[mb][nt][i] *= f;
        } else {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            uint32_t a[4];
            key_operand<KIND>(a, w, ks);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma(s[mb][nt], a, qf[nt][ks][0], qf[nt][ks][1]);
          }
          float f[2] = {p.scale_log2, p.scale_log2};
          if constexpr (C::SCALED8) {
            f[0] *= reinterpret_cast<const float*>(ksb)[mb * 16 + g];
            f[1] *= reinterpret_cast<const float*>(ksb)[mb * 16 + 8 + g];
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = s[mb][nt][i];
              if constexpr (KIND == AF1_KV_INT8) x = fmaf(x, kCode, -q128[nt][i % 2]);
              s[mb][nt][i] = x * f[i / 2];
            }
        }
      }

      // Steps with nodes, with keys past the end or with missing pages.
      const bool masked = key + KW > min(len, k_end) || bad != 0;
      if (masked) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int lr = nt * 8 + 2 * t + i;
            uint64_t bits = 0;
            if (lr < rows) {
              const int node = lr / p.group;
              if (p.mask == nullptr) {
                bits = (2ull << node) - 1;
              } else {
                const uint32_t* w = p.mask + seq * p.mask_seq + node * p.words;
                bits = w[0] | (p.words > 1 ? (uint64_t)w[1] << 32 : 0);
              }
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int k = key + mb * 16 + 8 * h + g;
                const bool sees = k < k_end && !(bad >> mb & 1) && (k < len || (bits >> (k - len) & 1));
                if (!sees) s[mb][nt][2 * h + i] = -kInf;
              }
          }
      }

      // The maximum moves where a score is kSlack above it.
      bool grow = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = fmaxf(s[0][nt][i], s[0][nt][2 + i]);
#pragma unroll
          for (int mb = 1; mb < MB; ++mb) x = fmaxf(x, fmaxf(s[mb][nt][i], s[mb][nt][2 + i]));
          top[nt][i] = x;
          grow |= x > m[nt][i] + kSlack;
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = top[nt][i];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            const float now = fmaxf(m[nt][i], x);
            const float alpha = ex2(m[nt][i] - (now == -kInf ? 0.f : now));
            m[nt][i] = now;
            l[nt][i] *= alpha, over[nt][i] *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][nt][i] *= alpha, o[mt][nt][2 + i] *= alpha;
          }
      }
      // So does the largest scale of a value, with room to twice what it was.
      float vinv = 0.f;
      if constexpr (C::SCALED8) {
        const int row = lane % KW;
        const bool real = !masked || (key + row < k_end && !(bad >> (row / 16) & 1));
        float x = fabsf(reinterpret_cast<const float*>(vsb)[row]);
        x = x < kInf ? x : 0.f;
        // Non-negative floats order as their bits.
        const float most = __uint_as_float(__reduce_max_sync(0xffffffffu, real ? __float_as_uint(x) : 0u));
        if (most > vref) {
          const float now = 2.f * most, f = vref / now;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[mt][nt][i] *= f;
          vref = now;
        }
        vinv = vref > 0.f ? 1.f / vref : 0.f;
      }

      // A node's infinite or NaN value (or scale of it) must reach the rows that
      // see it, however small their weight, and no other, as 0 times it would:
      // such steps sum entry by entry, with weights of at least 2^-120.
      bool slow = false;
      if (masked) {
        bool odd = value_bad<KIND, DIM, KW>(vb, vsb, lane % KW, lane / KW, 32 / KW);
        if constexpr (C::SCALED8) {  // scales past the end are never used
          const int row = lane % KW;
          odd |= key + row < k_end && !(bad >> (row / 16) & 1) && !(fabsf(reinterpret_cast<const float*>(vsb)[row]) < kInf);
        }
        slow = __any_sync(0xffffffffu, odd);
        if (__builtin_expect(slow, 0)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (s[mb][nt][i] > -kInf) s[mb][nt][i] = fmaxf(s[mb][nt][i], m[nt][i % 2] - kShift - 120.f);
        }
      }

      // Weights.
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float ref[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ref[i] = (m[nt][i] == -kInf ? 0.f : m[nt][i]) - kShift;
          if constexpr (INT4) {
            const float x = ex2(top[nt][i] - ref[i]);
            over[nt][i] += __half2float(__float2half_rn(x)) - x;
          }
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = ex2(s[mb][nt][i] - ref[i % 2]);
            l[nt][i % 2] += x;
            s[mb][nt][i] = x;
          }
      }

      if (__builtin_expect(slow, 0)) {
        for (int j = 0; j < KW; ++j) {
          const int from = (j % 8) * 4 + t;
          float vs = 1.f;
          if constexpr (C::SCALED8) vs = reinterpret_cast<const float*>(vsb)[j] * vinv;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float mine = 0.f;
#pragma unroll
              for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  if (j / 8 == 2 * mb + h) mine = s[mb][nt][2 * h + i];
              x[i] = __shfl_sync(0xffffffffu, mine, from);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float v = value_entry<KIND, DIM, KW>(vb, vsb, j, C::row_entry(mt, g, h)) * vs;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (x[i] != 0.f) o[mt][nt][2 * h + i] += x[i] * v;
              }
          }
        }
      } else {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const uint32_t v_addr = smem_u32(vb);
          const int row = mb * 16 + (lane & 15), hi = lane >> 4;
          // Weights of the 16 keys, times c of each key, as b operands.
          auto weights = [&](int nt, float c0, float c1, uint32_t (&b)[2]) {
            const float x[4] = {s[mb][nt][0] * c0, s[mb][nt][1] * c0, s[mb][nt][2] * c1, s[mb][nt][3] * c1};
            // 0 times a missing key's scale is 0.
            auto ok = [&](int i) { return masked && !(s[mb][nt][i] > 0.f) ? 0.f : x[i]; };
            b[0] = transpose8(pack_half2(ok(0), ok(1)));
            b[1] = transpose8(pack_half2(ok(2), ok(3)));
          };
          if constexpr (INT4) {
            const uint32_t* sc = reinterpret_cast<const uint32_t*>(vsb) + mb * 16 * GROUPS;
            uint32_t b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) weights(nt, 1.f, 1.f, b[nt]);
#pragma unroll
            for (int c = 0; c < GROUPS; c += 2) {
              uint32_t v[4];
              ldmatrix_x4_trans(v, v_addr + C::template at<KW>(row, c + hi));
#pragma unroll
              for (int cc = 0; cc < 2; ++cc) {
                uint32_t s2[2], low2[2];  // of keys 2 t and 2 t + 1, and of those 8 on
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const uint32_t x = sc[(2 * t + 8 * h) * GROUPS + c + cc], y = sc[(2 * t + 1 + 8 * h) * GROUPS + c + cc];
                  s2[h] = prmt(x, y, 0x5410), low2[h] = prmt(x, y, 0x7632);
                }
#pragma unroll
                for (int odd = 0; odd < 2; ++odd) {
                  uint32_t a[4];
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const uint32_t code = v[2 * cc + i / 2] >> (4 * odd + 8 * (i % 2)) & 0x000f000fu;
                    a[i] = hfma2(hsub2(code | 0x64006400u, 0x64006400u), s2[i / 2], low2[i / 2]);
                  }
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt) mma(o[2 * (c + cc) + odd][nt], a, b[nt][0], b[nt][1]);
                }
              }
            }
          } else {
            float c0 = 1.f, c1 = 1.f;
            if constexpr (C::SCALED8) {
              c0 = reinterpret_cast<const float*>(vsb)[mb * 16 + g] * vinv;
              c1 = reinterpret_cast<const float*>(vsb)[mb * 16 + 8 + g] * vinv;
            }
            uint32_t b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) weights(nt, c0, c1, b[nt]);
            constexpr int PER = KIND == AF1_KV_F16 ? 1 : 2;  // 16-entry blocks of two chunks
#pragma unroll
            for (int mt = 0; mt < MT; mt += PER) {
              uint32_t v[4];
              ldmatrix_x4_trans(v, v_addr + C::template at<KW>(row, (KIND == AF1_KV_F16 ? 2 * mt : mt) + hi));
#pragma unroll
              for (int cc = 0; cc < PER; ++cc) {
                uint32_t a[4];
                if constexpr (KIND == AF1_KV_F16) {
                  a[0] = v[0], a[1] = v[2], a[2] = v[1], a[3] = v[3];
                } else {
#pragma unroll
                  for (int h = 0; h < 2; ++h) {
                    if constexpr (KIND == AF1_KV_INT8) {
                      const uint32_t u = v[2 * cc + h] ^ 0x80808080u;
                      a[2 * h] = hsub2(prmt(u, 0x64646464u, 0x4240), 0x64806480u);
                      a[2 * h + 1] = hsub2(prmt(u, 0x64646464u, 0x4341), 0x64806480u);
                    } else {
                      const uint32_t u = prmt(v[2 * cc + h], 0, 0x3120);
                      a[2 * h] = e4m3x2(u);
                      a[2 * h + 1] = e4m3x2(u >> 16);
                    }
                  }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma(o[mt + cc][nt], a, b[nt][0], b[nt][1]);
              }
            }
          }
        }
      }
      if (++slot == STAGES) slot = 0;
      __syncwarp();  // the slot is free again
    }
    if (!alive) {
      // A wait gave up: let the copies in flight land (within a limit)
      // before shared memory changes hands, and report it.
      for (; waited < issued; ++waited) {
        if (wait_phase(&bars[warp][slot], phases >> slot & 1, max(p.wait_cycles, kLanding))) phases ^= 1u << slot;
        if (++slot == STAGES) slot = 0;
      }
      if (lane == 0) atomicOr(p.status, kStatusTimeout);
    }
    __syncthreads();  // every warp is done with its ring

    // -- join the warps' parts -------------------------------------------------------
    // Entry e of row lr is kept at e ^ 8 (lr / 2 % 4): the lanes of a store
    // then write different banks.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = l[nt][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        // What rounding adds to the largest weights of the steps, and so to the output,
        // it adds to the divisor (of the output), too.
        float even = 1.f;
        if constexpr (INT4) {
          float off = over[nt][i];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) off += __shfl_xor_sync(0xffffffffu, off, d);
          if (sum > 0.f) even = sum / (sum + off);
        }
        const int lr = nt * 8 + 2 * t + i;
        if (g == 0) join_m[warp][lr] = m[nt][i], join_l[warp][lr] = sum;
        if (lr >= rows) continue;
        float* to_row = join + (warp * ROWS + lr) * DIM;
        const float f = C::SCALED8 ? vref : 1.f;
        if constexpr (KIND == AF1_KV_F16) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            to_row[C::row_entry(mt, g, 0) ^ (8 * t)] = o[mt][nt][i];
            to_row[C::row_entry(mt, g, 1) ^ (8 * t)] = o[mt][nt][2 + i];
          }
        } else if constexpr (INT4) {
#pragma unroll
          for (int mt = 0; mt < MT; mt += 2)
            *reinterpret_cast<float4*>(to_row + (C::row_entry(mt, g, 0) ^ (8 * t))) =
                make_float4(o[mt][nt][i] * even, o[mt + 1][nt][i] * even, o[mt][nt][2 + i] * even,
                            o[mt + 1][nt][2 + i] * even);
        } else {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            *reinterpret_cast<float2*>(to_row + (C::row_entry(mt, g, 0) ^ (8 * t))) =
                make_float2(o[mt][nt][i] * f, o[mt][nt][2 + i] * f);
        }
      }
    __syncthreads();
    const bool whole = u0 == 0 && to == units;
    // Parts of an item: CTAs c0 .. c1 hold its units of keys. A CTA leaves at
    // most two, in its first run (of an item that began before) and in its
    // last one (of an item that it is the first to hold).
    auto holder = [&](int64_t u) {
      const int64_t large = more * (per + 1);
      return (int)(u < large ? u / (per + 1) : more + (u - large) / per);
    };
    int c0 = 0, c1 = 0;
    if (!whole) c0 = holder(first + kSetup), c1 = holder(first + units - 1);
    auto part_of = [&](int c) { return p.parts + (int64_t)(2 * c + (c == c0 ? 1 : 0)) * S::PART; };
    float* part = part_of(blockIdx.x);
    const int live_nodes = node_count(p, seq);
    auto finish = [&](int lr, int e, float mx, float sum, float4 acc) {
      const int node = lr / p.group, h = head * p.group + lr - node * p.group;
      const bool live = node < live_nodes && sum != 0.f;
      const float f = live ? 1.f / sum : 0.f;
      const float4 y = live ? make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f) : make_float4(0.f, 0.f, 0.f, 0.f);
      const int64_t at = seq * p.o_seq + node * p.o_node + h * p.o_head + e;
      if (p.out_f32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = y;
      else
        *reinterpret_cast<uint2*>(static_cast<__half*>(p.out) + at) =
            make_uint2(pack_half2(y.x, y.y), pack_half2(y.z, y.w));
      if (e == 0 && p.lse != nullptr)
        p.lse[((int64_t)seq * p.nodes + node) * p.cache.heads * p.group + h] =
            live ? (mx - kShift + log2f(sum)) * 0.69314718056f : -kInf;
    };
    auto add = [](float4& acc, float f, const float4& x) {
      acc.x = fmaf(f, x.x, acc.x), acc.y = fmaf(f, x.y, acc.y), acc.z = fmaf(f, x.z, acc.z), acc.w = fmaf(f, x.w, acc.w);
    };
    for (int i = threadIdx.x; i < rows * (DIM / 4); i += 32 * W) {
      const int lr = i / (DIM / 4), e = i % (DIM / 4) * 4;
      float mx = -kInf;
#pragma unroll
      for (int w = 0; w < W; ++w) mx = fmaxf(mx, join_m[w][lr]);
      const float zero = mx == -kInf ? 0.f : mx;
      float sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = ex2(join_m[w][lr] - zero);
        sum = fmaf(f, join_l[w][lr], sum);
        add(acc, f, *reinterpret_cast<const float4*>(join + (w * ROWS + lr) * DIM + (e ^ (8 * (lr / 2 % 4)))));
      }
      if (whole) {
        finish(lr, e, mx, sum, acc);
      } else {
        *reinterpret_cast<float4*>(part + lr * DIM + e) = acc;
        if (e == 0) *reinterpret_cast<float2*>(part + ROWS * DIM + 2 * lr) = make_float2(mx, sum);
      }
    }
    if (!whole) {
      __syncthreads();
      if (threadIdx.x == 0) {  // the CTA's writes above are released with it
        const unsigned arrived = atom_add_acq_rel_gpu(&p.counters[c0], 1u);
        last_shared = arrived == (unsigned)(c1 - c0);
        if (last_shared) p.counters[c0] = 0;  // as the next call finds it
      }
      __syncthreads();
      if (last_shared) {
        for (int i = threadIdx.x; i < rows * (DIM / 4); i += 32 * W) {
          const int lr = i / (DIM / 4), e = i % (DIM / 4) * 4;
          float mx = -kInf, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c = c0; c <= c1; c += 4) {  // four parts' loads in flight
            float2 ml[4];
            float4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* from = part_of(min(c + j, c1));
              ml[j] = __ldcg(reinterpret_cast<const float2*>(from + ROWS * DIM + 2 * lr));
              x[j] = __ldcg(reinterpret_cast<const float4*>(from + lr * DIM + e));
            }
            float now = mx;
#pragma unroll
            for (int j = 0; j < 4; ++j) now = fmaxf(now, ml[j].x);
            const float zero = now == -kInf ? 0.f : now;
            const float f = ex2(mx - zero);
            sum *= f, acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (c + j > c1) continue;
              const float fj = ex2(ml[j].x - zero);
              sum = fmaf(fj, ml[j].y, sum);
              add(acc, fj, x[j]);
            }
            mx = now;
          }
          finish(lr, e, mx, sum, acc);
        }
      }
    }
    // The rings, written through the generic proxy above, go back to TMA.
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
}

int fail(int code, const std::string& msg) { return set_error(code, "af1_tree_attention: " + msg); }

// Blocks of 8 rows (of every query head and node that share a cached head) that
// a CTA has; 0: the tensor-core kernel, whose products have 128 rows. Going
// over the keys again for 16 rows more did not pay: 4 sequences of up to 6001
// tokens with 20 rows of E4M3 took 32 us where 30 are taken there, 24 of INT4 32
// and 31, 32 of FP16 33 and 30, of INT8 33 and 31; 64 of E4M3 47 and 31. (It was a
// tenth faster for 32 short sequences of 32 rows of INT8.) Blocks of 32 rows, which
// leave an SM 8 warps, were no better.
int row_blocks(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 0; }

int64_t workspace_bytes(const af1_kv_cache& c, int64_t rows) {
  if (row_blocks(rows) == 0) return kScratchOffset + tree_wide_part_bytes(c);
  const int64_t ctas = std::min(3 * c.num_sms, kMaxCtas);  // at most three CTAs to an SM
  return kScratchOffset + 2 * ctas * (8 * row_blocks(rows)) * (c.d.head_dim + 2) * 4;
}

template <int KIND, int DIM, int NT, int W, int KW, int STAGES, int CTAS>
int launch(const TreeProblem& p, int sms, cudaStream_t st) {
  constexpr int smem = Shape<KIND, DIM, NT, W, KW, STAGES>::SMEM;
  auto kernel = tree_kernel<KIND, DIM, NT, W, KW, STAGES, CTAS>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) {
    kernel<<<std::min(sms * CTAS, kMaxCtas), 32 * W, smem, st>>>(p);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}

// Warps, keys of a step and stages of a kind: what fills the shared memory.
template <int KIND, int DIM, int NT>
int launch_rows(TreeProblem& p, const af1_kv_cache& c, cudaStream_t st) {
  constexpr int RB = kv_row_bytes(KIND, DIM);
  constexpr int KW = RB >= 256 ? 16 : 32;
  constexpr int W = 4;
  constexpr int CTAS = 3;
  constexpr int BYTES = 2 * KW * (RB + kv_scale_bytes(KIND, DIM)) * W;
  constexpr int FIT = (222 * 1024 / CTAS - 4096) / BYTES;
  constexpr int STAGES = FIT > 4 ? 4 : FIT;
  static_assert(STAGES >= 2, "");
  p.k_map = c.k_step, p.v_map = c.v_step;
  return launch<KIND, DIM, NT, W, KW, STAGES, CTAS>(p, c.num_sms, st);
}

template <int KIND>
int launch_kind(TreeProblem& p, const af1_kv_cache& c, int nt, cudaStream_t st) {
  if (c.d.head_dim == 128)
    return nt == 1 ? launch_rows<KIND, 128, 1>(p, c, st) : launch_rows<KIND, 128, 2>(p, c, st);
  return nt == 1 ? launch_rows<KIND, 64, 1>(p, c, st) : launch_rows<KIND, 64, 2>(p, c, st);
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
  // With log2(e), a code's 2^24 and a key's scale it has to stay finite, as 0 times it is 0.
  if (!(std::abs(a->scale) <= 1e30f)) return fail(AF1_ERR_INVALID_ARG, "scale must be -1e30..1e30");
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
  const int nt = row_blocks(rows);
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
  p.scale_log2 = a->scale * 1.4426950408889634f;
  p.out_f32 = a->out_dtype == AF1_F32;
  p.counters = reinterpret_cast<unsigned*>(static_cast<uint8_t*>(workspace) + kStatusBytes);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kScratchOffset);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  p.status = static_cast<unsigned*>(workspace);
  p.wait_cycles = wait_budget();
  if (nt == 0) {
    const cudaError_t e = launch_tree_wide(p, *c, (int)rows, st);
    if (e != cudaSuccess) return fail(AF1_ERR_CUDA, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
    set_error(AF1_OK, "");
    return AF1_OK;
  }
  switch (c->d.kind) {
    case AF1_KV_F16: return launch_kind<AF1_KV_F16>(p, *c, nt, st);
    case AF1_KV_INT8: return launch_kind<AF1_KV_INT8>(p, *c, nt, st);
    case AF1_KV_E4M3: return launch_kind<AF1_KV_E4M3>(p, *c, nt, st);
    default: return launch_kind<AF1_KV_INT4>(p, *c, nt, st);
  }
}
