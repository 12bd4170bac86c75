// af1_tree_wide.cu — attention of drafted tokens over the paged cache where
// more than 16 rows (nodes times query heads) share a cached head: the same
// operator as af1_tree.cu, with tcgen05 products of 128 rows.
//
// An item is one sequence, one cached head and a block of 128 rows; its keys
// are cut into tiles of 128, and every CTA (one to an SM) takes an equal run
// of the tiles of all items, as in af1_tree.cu. For one tile
//   S = Q K^T   (128 x 128, FP32, tensor memory)
//   P = 2^(S f - m + kShift) as FP16, tensor memory
//   O += P V    (P from tensor memory, V from shared memory)
// S and P have two buffers, so that the products of one tile run under the
// exponents of another. (Two streams of tiles, each with scores, weights and
// output of its own, waited for one another's latencies: 115 us for trees of
// 64 over 32768 INT4 tokens.)
// Roles of the 19 warps:
//   0-3, 4-7  softmax of the tile's first and second 64 keys: a thread has one
//             row. The weights are formed relative to the maximum so far, and
//             formed again (after O is scaled) only where a score of either
//             half passes it by more than kSlack binary places;
//   8-11, 12-15  decode keys, and values: thread i turns vector i of a tile
//             from codes into FP16 in the 128-byte-swizzled operand tile (keys
//             K-major, values with their entries along N). INT8 and E4M3 stay
//             codes, exact in FP16; a key's scale multiplies the scores, a
//             value's the weights (relative to a power of two that bounds the
//             scales so far, which the exponents take in). INT4 has a scale and a
//             low for each group of 32 entries: see below. FP16 tiles arrive by
//             TMA and are only looked at where a sequence ends;
//   16, 18    TMA copies of keys, and of values, one for up to 128 rows of a
//             page, into the ring of codes (one warp for both took 0.65 us for
//             each, which held up the decoders);
//   17        one lane issues the products. (A lane each for Q K^T and P V, and a
//             wait more for the softmax, took 2 % longer.)
// Keys and values each have a ring of codes and two operand tiles (but as said
// below), with barriers of their own: whoever waits on a barrier meets each of its phases in
// turn, as a test of a phase's parity needs. (The softmax skips phases of P V,
// as the scores that it waits for come after them.)
//
// INT4. Values, code * scale + low, are rounded to FP16 once. Keys are not: with
// scale = high + rest, high its first seven significant bits, (code - 7.5) high and
// (code - 7.5) rest are FP16 numbers, and two products sum both; one product more
// of 16 entries adds (low + 7.5 scale) times the sum of q over each group, that sum
// and 7.5 times it in two FP16 parts each. So a score has the precision that
// af1_tree.cu gives it; where products with the rest are subnormal, for scales
// below 2^-13, each is off by 2^-25. What is left are roundings of weights and
// values; of the largest weight of every 32 what rounding adds is added to the
// divisor, too, where it cancels most of what it adds to the output. (Rounded
// keys made the outputs' error 7.8e-4 of the norm, weights as if not rounded 3.2e-4;
// it is 3.0e-4, FP16 outputs alone 2.1e-4. All weights as rounded in the divisor:
// 3.0e-4 and a tenth slower; the same for 8 bits: 2.3e-4 for 2.9e-4, but 118 us for
// 101.) The second part costs a third of the tensor time and of shared memory, which
// for entries of 128 leaves values one operand tile and each ring of codes one
// stage: 99 us for the tree of 64 below where rounded keys took 87, 78 with entries
// of 64 for 71. (Keys in one operand tile of two parts, values in two: 132 us; its
// halves in turn: 112; halves in a ring of three: 127; halves by all eight warps:
// 120. A thread's fixed costs, waits and fences, are half of what a tile takes it.)
//
// Infinities and NaN: the values of slots past the end are zeros, a node's
// value that is not finite (or its scale) is left out of the product (0 times it
// would reach the rows that do not see it) and added to the rows that see it at
// the end.
//
// Bound: a softmax warp's chain of steps for a tile (wait, read, exponents,
// agree, arrive), which queue in shared memory behind the decoders' stores and
// the products' operands. With all 128 rows in use a tile's exponents take 1024
// cycles (16 a cycle), its products 1024, or 1600 of INT4; the chain takes 2200:
// 91 us for a tree of 64 nodes and 8 queries to a head over 32768 FP16 tokens of 8
// heads (760 TFLOP/s), 98 of E4M3, 101 of INT8, whose scales every row reads. INT4
// with entries of 128 is bound by the decoders: of keys, 2500 cycles and their waits,
// and of values, which wait for the products with those before (2700; together 99
// us, 0.58 of the issue slots, 0.48 of the tensor pipe). Where CTAs have few
// tiles, it is what a run costs once (first pages, keys and q 6 us, the first tile
// 2, join 5 to 10): 4 trees of 16 over 6001 E4M3 tokens take 31 us.
// All waits are bounded; a wait that gives up sets the status word, and what
// depends on it is skipped. Where one has, no copy is issued any more, and before
// shared or tensor memory changes hands the copies and products in flight end.
#include "af1_tree.cuh"

namespace af1 {
namespace {

constexpr int BK = 128;        // keys of a tile
constexpr int kThreads = 608;
// Tiles that a run's beginning and end are worth. (4 trees of 16 over 6001 E4M3
// tokens, 16 of them over 2000, one of 64 over 32768 INT4 tokens: 35, 38 and 107 us
// with 4 tiles, 30, 38 and 105 with 5, 31, 37 and 99 with 8.)
constexpr int kSetupTiles = 8;
constexpr int kRows = 128;
constexpr int kOutAt = 2 * BK, kWeightsAt = 3 * BK;  // columns of tensor memory, behind two tiles of scores
constexpr int kNotes = 4;      // tiles whose scales and page bits are kept: keys are decoded up to three tiles ahead
constexpr float kLeastScale = -60.f;  // of a value's scale's exponent: smaller ones count as 2^-60

template <int KIND, int DIM>
struct Wide {
  using C = Kv<KIND, DIM>;
  static constexpr bool F16 = KIND == AF1_KV_F16;
  static constexpr int OP = BK * DIM * 2;                    // bytes of an operand tile
  static constexpr int CODES = BK * C::RB;
  static constexpr int SCALES = (C::SCALED8 ? 2 : 1) * BK * C::SB;  // 8 bits: of keys and values, with the keys
  // Operand tiles: two of keys, which of INT4 have two parts, then two of values
  // (one where there is no room for two), then q.
  static constexpr bool SPLIT = KIND == AF1_KV_INT4;
  static constexpr int V_TILE = SPLIT ? 4 : 2, V_SLOTS = SPLIT && DIM == 128 ? 1 : 2;
  // Rings of codes (FP16: the operand tiles themselves). Decoders hold a stage
  // only while they read it; where the room is short there is one.
  static constexpr int K_STAGES = SPLIT && DIM == 128 ? 1 : 2, V_STAGES = !F16 && DIM == 128 ? 1 : 2;
  static constexpr int K_BYTES = CODES + SCALES, V_BYTES = CODES + (C::SCALED8 ? 0 : SCALES);
  static constexpr int RINGS = F16 ? 0 : K_STAGES * K_BYTES + V_STAGES * V_BYTES;
  // INT4: sums of q over the groups, and the groups' scales and lows.
  static constexpr int GROUP_BYTES = SPLIT ? 2 * BK * 32 : 0;
  static constexpr int SMEM =
      (V_TILE + V_SLOTS + 1) * OP + GROUP_BYTES + RINGS + (C::SCALED8 ? 2 * kNotes * BK * 4 : 0) + 1024;
  static constexpr int PART = kRows * (DIM + 2);  // floats: o, m, l, each along the rows (to a multiple of 4 of them)
  static constexpr int COPIES = 10 * DIM / 8 * 16;  // bytes of a part for 4 rows, as it is joined
  static_assert(2 * COPIES * (kRows / 4) <= SMEM - 1024, "two parts are on their way");
};

// 16 bytes to shared memory, as part of the thread's next group of copies.
__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

struct Plan {
  int64_t per, more, end;  // units of a CTA, the CTAs with one more, and where this one's end
};

struct Barriers {
  Plan plan;
  uint64_t op_ready[2][2], op_empty[2][2], code_full[2][2], code_empty[2][2];  // of keys and values
  uint64_t s_full[2], p_ready[2], pv_done[2], q_ready;  // by tile
  uint64_t groups_empty;                    // INT4: the tile of the keys' groups
  uint64_t drained;                         // products, after a wait that gave up
  uint32_t tmem;
  volatile int gave_up;
  int issued[2];                            // of keys and values: the last tile whose copies were
  uint32_t code_bad[2][2], tile_bad[kNotes];   // bits: 16 keys each whose page is missing
  uint32_t nodes_bad[4][2];                 // by run that has keys: nodes whose value is not finite (values are
                                            // decoded at most two tiles, their scales, which come with the keys,
                                            // three, so three such runs, ahead of their use)
  alignas(16) float top[2][2][kRows], sum[2][kRows];    // of the halves of a tile (by tile), and of a run
  float over[2][kRows];                     // INT4: what rounding has added to the largest weights
  float q_scale[kRows];                     // INT4: what the rows of q were divided by
  alignas(16) float value_top[kNotes][4];        // by tile and warp: power of two above the values' scales
  // Parts of items that this CTA has left: of its first and of its last run.
  struct {
    int c0, c1, seq, head, tile, rows;
  } part[2];
  int parts;
  bool last[2];
};

// The runs of this CTA, one after another, known to every warp. What stays the
// same lies in shared memory: every thread of the softmax needs its registers.
struct Runs {
  Sequences<BK, kSetupTiles> sq;
  int64_t pos, first;
  int seq, head, tile, len, keys, units, from, to, k_begin, k_end, tiles;

  __device__ __forceinline__ bool begin(const TreeProblem& p, Plan& plan) {
    const int64_t lanes = (int64_t)p.cache.heads * p.row_tiles;
    const int64_t total = sq.begin(p) * lanes;
    const int64_t ctas = min((int64_t)gridDim.x, total);
    if (blockIdx.x >= ctas) return false;
    const int64_t per = total / ctas, more = total - per * ctas;
    pos = per * blockIdx.x + min((int64_t)blockIdx.x, more);
    if (threadIdx.x == 0) plan.per = per, plan.more = more, plan.end = pos + per + (blockIdx.x < more ? 1 : 0);
    return true;
  }
  // The next run; tiles is 0 where it has no keys of its own.
  __device__ __forceinline__ bool next(const TreeProblem& p, const volatile Plan& plan) {
    const int64_t end = plan.end;
    if (pos >= end) return false;
    const int64_t lanes = (int64_t)p.cache.heads * p.row_tiles;
    while (sq.after() * lanes <= pos) sq.load(p, sq.first + 32, sq.after());
    const int which = __popc(__ballot_sync(0xffffffffu, (sq.before + sq.sum) * lanes <= pos));
    seq = sq.first + which;
    units = __shfl_sync(0xffffffffu, sq.units, which);
    len = __shfl_sync(0xffffffffu, sq.len, which);
    keys = __shfl_sync(0xffffffffu, sq.keys, which);
    const int64_t seq_first = (sq.before + __shfl_sync(0xffffffffu, sq.sum, which) - units) * lanes;
    const int item = (int)((pos - seq_first) / units);
    first = seq_first + (int64_t)item * units;
    from = (int)(pos - first);
    to = (int)min((int64_t)units, from + (end - pos));
    pos += to - from;
    head = item / p.row_tiles;
    tile = item - head * p.row_tiles;
    const int u0 = max(from - kSetupTiles, 0), u1 = to - kSetupTiles;
    k_begin = u0 * BK, k_end = min(u1 * BK, keys);
    tiles = max(u1 - u0, 0);
    return true;
  }
  __device__ __forceinline__ int rows(const TreeProblem& p) const {
    return min(kRows, p.nodes * p.group - tile * kRows);
  }
};

__device__ __forceinline__ int part_ld(int rows) { return (rows + 3) & ~3; }

// The CTA that has unit u.
__device__ __forceinline__ int holder(const volatile Plan& plan, int64_t u) {
  const int64_t per = plan.per, more = plan.more, large = more * (per + 1);
  return (int)(u < large ? u / (per + 1) : more + (u - large) / per);
}

// Suspends the thread for up to 20 us (a hint): a poll that came back at once
// would take the schedulers' slots from the warps that work.
__device__ __forceinline__ bool try_wait_long(uint64_t* bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
// Shared-memory matrices: 128-byte swizzle, 8 rows 1024 bytes apart; `lead`: bytes
// between 64-entry groups where the entries run along M or N. The upper half of
// the description is a constant.
constexpr uint32_t kMatrixHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// Rows of 32 bytes, with a 32-byte swizzle, 8 of them 256 bytes apart.
constexpr uint32_t kGroupsHigh = (256 >> 4) | 1u << 14 | 6u << 29;
__device__ __forceinline__ uint32_t matrix(uint32_t addr, int lead) {
  return ((addr >> 4) & 0x3fffu) | (uint32_t)(lead >> 4) << 16;
}
template <uint32_t HIGH = kMatrixHigh>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate ? 1u : 0u), "n"(HIGH)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate ? 1u : 0u), "n"(kMatrixHigh)
      : "memory");
}
// True in one lane of the warp.
__device__ __forceinline__ bool elect() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 32 columns of this thread's row; `meanwhile` runs before they are waited for.
template <typename F>
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&x)[32], F meanwhile) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
  meanwhile();
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&x)[32]) {
  tmem_load(addr, x, [] {});
}
template <typename F>
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&x)[16], F meanwhile) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
  meanwhile();
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Where entry pair and group places stand: INT4's decode takes 4 apart nibbles
// at once, so place 2 i + h of every 8 is entry i + 4 h. q is laid out alike,
// and the outputs are put back.
template <int KIND>
__device__ __forceinline__ constexpr int place_entry(int place) {
  return KIND == AF1_KV_INT4 ? (place & ~7) | ((place & 7) >> 1) | (place & 1) << 2 : place;
}

template <int KIND, int DIM>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const __grid_constant__ TreeProblem p) {
  using C = Kv<KIND, DIM>;
  using S = Wide<KIND, DIM>;
  constexpr bool F16 = S::F16, INT4 = KIND == AF1_KV_INT4;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Barriers bar;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* ops = smem;
  uint8_t* qt = smem + (S::V_TILE + S::V_SLOTS) * S::OP;
  uint8_t* groups_q = qt + S::OP;
  uint8_t* groups_k = groups_q + S::GROUP_BYTES / 2;
  uint8_t* codes = qt + S::OP + S::GROUP_BYTES;
  float* key_scale = reinterpret_cast<float*>(codes + S::RINGS);
  // Tile `at` of the CTA's (keys or values): its operand tile, and its codes
  // with the scales behind them.
  auto op_slot = [&](bool is_v, int at) { return S::V_SLOTS == 1 && is_v ? 0 : at & 1; };
  auto op_turn = [&](bool is_v, int at) { return S::V_SLOTS == 1 && is_v ? at : at >> 1; };
  auto op_place = [&](bool is_v, int at) { return is_v ? S::V_TILE + op_slot(true, at) : (S::SPLIT ? 2 : 1) * (at & 1); };
  auto op_tile = [&](bool is_v, int at) { return ops + op_place(is_v, at) * S::OP; };
  auto code_stage = [&](bool is_v, int at) { return is_v ? at % S::V_STAGES : at % S::K_STAGES; };
  auto code_turn = [&](bool is_v, int at) { return is_v ? at / S::V_STAGES : at / S::K_STAGES; };
  auto code_tile = [&](bool is_v, int at) {
    if constexpr (F16) return op_tile(is_v, at);
    return codes + (is_v ? S::K_STAGES * S::K_BYTES + code_stage(true, at) * S::V_BYTES
                         : code_stage(false, at) * S::K_BYTES);
  };
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;

  Runs run;
  if (!run.begin(p, bar.plan)) return;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bar.op_ready[i / 2][i % 2], 4);
      mbar_init(&bar.op_empty[i / 2][i % 2], 1);
      mbar_init(&bar.code_full[i / 2][i % 2], 1);
      mbar_init(&bar.code_empty[i / 2][i % 2], 4);
      bar.nodes_bad[i][0] = bar.nodes_bad[i][1] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar.s_full[i], 1);
      mbar_init(&bar.p_ready[i], 8);
      mbar_init(&bar.pv_done[i], 1);
    }
    mbar_init(&bar.q_ready, 8);
    mbar_init(&bar.drained, 1);
    mbar_init(&bar.groups_empty, 1);
    bar.gave_up = 0, bar.parts = 0;
    bar.issued[0] = bar.issued[1] = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = bar.tmem;
  float* value_scale = key_scale + kNotes * BK;

  // Bounded wait; once one has given up, all return at once.
  auto wait = [&](uint64_t* b, uint32_t parity) {
    if (try_wait_long(b, parity)) return true;
    const long long t0 = clock64();
    while (!try_wait_long(b, parity)) {
      if (bar.gave_up) return false;
      if (clock64() - t0 > p.wait_cycles) {
        bar.gave_up = 1;
        return false;
      }
    }
    return true;
  };

  int tiles_done = 0, runs_done = 0;  // before this run (runs: those with keys)
  if (warp == 16 || warp == 18) {
    // ---- copies ------------------------------------------------------------------
    const bool is_v = warp == 18;
    const CUtensorMap* map = is_v ? &p.v_map : &p.k_map;
    // A box is a page's rows, up to a tile's; the lanes hold the pages of `group` tiles.
    const int box_shift = min(p.cache.shift, 7), box = 1 << box_shift, boxes = BK >> box_shift;
    const int group_shift = box_shift - 2;  // 32 / boxes
    const bool leads = lane < boxes;
    while (run.next(p, bar.plan)) {
      const int32_t* page_row = p.pages.pages + run.seq * p.pages.ld;
      const int n = run.tiles;
      auto pages_of = [&](int b) {  // lane l: box l % boxes of tile (b << group_shift) + l / boxes
        const int k = run.k_begin + ((b * 32 + lane) << box_shift);
        return k < run.k_end ? page_row[k >> p.cache.shift] : -1;
      };
      int now = n > 0 ? pages_of(0) : -1, next = n > 0 ? pages_of(1) : -1;
      for (int j = 0; j < n; ++j) {
        const int in_group = j & ((1 << group_shift) - 1);
        if (j > 0 && in_group == 0) {
          now = next;
          next = pages_of((j >> group_shift) + 1);
        }
        const int page = __shfl_sync(0xffffffffu, now, (in_group * boxes + lane) & 31);
        const int at = tiles_done + j, st = code_stage(is_v, at);
        const int k = run.k_begin + j * BK + (lane << box_shift);
        const bool mine = leads && k < run.k_end;
        const bool there = mine && page >= 0 && page < p.cache.pages;
        const unsigned have = __ballot_sync(0xffffffffu, there);
        const unsigned lack = __ballot_sync(0xffffffffu, mine && !there);
        const int64_t row =
            (((int64_t)page * p.cache.heads + run.head) << p.cache.shift) + (k & ((1 << p.cache.shift) - 1));
        // Decoders free a stage whose copies they gave up on, too, but only after
        // gave_up is set: nothing is issued into it.
        const bool ok =
            wait(F16 ? &bar.op_empty[is_v][st] : &bar.code_empty[is_v][st], (code_turn(is_v, at) & 1) ^ 1) && !bar.gave_up;
        if (!__all_sync(0xffffffffu, ok)) continue;
        if (lane == 0) {
          uint32_t bad = 0;  // a bit for each 16 keys
          for (unsigned left = lack; left != 0; left &= left - 1)
            bad |= ((1u << (box / 16)) - 1) << ((__ffs(left) - 1) * (box / 16));
          bar.code_bad[is_v][st] = bad;
          const int per_key = C::RB + (C::SCALED8 ? (is_v ? 0 : 2 * C::SB) : C::SB);
          mbar_expect_tx(&bar.code_full[is_v][st], __popc(have) * box * per_key);
          bar.issued[is_v] = at;
        }
        __syncwarp();
        if (there) {
          uint8_t* to = code_tile(is_v, at) + lane * box * C::SPAN;
          uint64_t* full = &bar.code_full[is_v][st];
#pragma unroll
          for (int s = 0; s < C::SLICES; ++s)
            tma_rows(smem_u32(to + s * (BK * 128)), map, s * 128, (int)row, full);
          if constexpr (C::SB > 0) {
            uint8_t* to_scales = code_tile(is_v, at) + S::CODES + lane * box * C::SB;
            if (!C::SCALED8 || !is_v)
              bulk_g2s(to_scales, static_cast<const uint8_t*>(is_v ? p.cache.vs : p.cache.ks) + row * C::SB, box * C::SB,
                       full);
            if (C::SCALED8 && !is_v)
              bulk_g2s(to_scales + BK * C::SB, static_cast<const uint8_t*>(p.cache.vs) + row * C::SB, box * C::SB,
                       full);
          }
        }
      }
      tiles_done += n;
    }
  } else if (warp >= 8 && warp < 16) {
    // ---- decode ---------------------------------------------------------------------
    const int row = threadIdx.x % 128;
    const bool is_v = warp >= 12;
    for (; run.next(p, bar.plan); runs_done += run.tiles > 0) {
      const int n = run.tiles;
      for (int j = 0; j < n; ++j) {
        const int at = tiles_done + j, st = code_stage(is_v, at), slot = op_slot(is_v, at);
        // Copies keep to budgets below a suspension, too. (Of the other waits, which
        // are for warps of this CTA, that cost 4 us of 86.)
        bool ok = true;
        if (p.wait_cycles >= kSuspend) ok = wait(&bar.code_full[is_v][st], code_turn(is_v, at) & 1);
        else if (!wait_phase(&bar.code_full[is_v][st], code_turn(is_v, at) & 1, p.wait_cycles)) bar.gave_up = 1, ok = false;
        if (!F16 && S::V_SLOTS > 1) ok = wait(&bar.op_empty[is_v][slot], (op_turn(is_v, at) & 1) ^ 1) && ok;
        ok = __all_sync(0xffffffffu, ok);
        const bool started = ok;
        const int key = run.k_begin + j * BK + row;
        const uint32_t bad = bar.code_bad[is_v][st];
        const bool gone = key >= run.k_end || (bad >> (row / 16) & 1);
        const bool node = key >= run.len;
        uint8_t* to = op_tile(is_v, at) + row * 128;
        auto place = [&](int c) { return to + (c >> 3) * (BK * 128) + (((c & 7) ^ (row & 7)) << 4); };
        if (ok) {
          if constexpr (!F16) {
            const uint8_t* from = code_tile(is_v, at);
            const uint8_t* sc = from + S::CODES;
            if constexpr (C::SCALED8) {
              if (!is_v) {
                const int note = at % kNotes;
                float vs = reinterpret_cast<const float*>(sc)[BK + row];
                if ((gone || node) && !(fabsf(vs) < kInf)) {
                  if (!gone) atomicOr(&bar.nodes_bad[runs_done % 4][(key - run.len) / 32], 1u << ((key - run.len) % 32));
                  vs = 0.f;
                }
                key_scale[note * BK + row] = reinterpret_cast<const float*>(sc)[row] * fabsf(p.scale_log2);
                value_scale[note * BK + row] = vs;
                // Non-negative floats order as their bits.
                const uint32_t most =
                    __reduce_max_sync(0xffffffffu, !gone && fabsf(vs) < kInf ? __float_as_uint(fabsf(vs)) : 0u);
                if (lane == 0) bar.value_top[note][warp % 4] = fmaxf((float)((int)(most >> 23) - 126), kLeastScale);
              }
            }
            // Keys and values share this code: the roles of a scheduler share its
            // instruction cache. All of the row is read before the first store:
            // loads are not moved over stores.
            uint4 in[C::RB / 16];
            uint32_t group[4];
#pragma unroll
            for (int c = 0; c < C::RB / 16; ++c) in[c] = *reinterpret_cast<const uint4*>(from + C::template at<BK>(row, c));
            if constexpr (INT4) {
#pragma unroll
              for (int c = 0; c < C::GROUPS; ++c)
                group[c] = reinterpret_cast<const uint32_t*>(sc)[row * C::GROUPS + c];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.code_empty[is_v][st]);  // the stage is read
            if (S::V_SLOTS == 1)  // what it waits for, decoding does too: not before the row is read
              ok = __all_sync(0xffffffffu, wait(&bar.op_empty[is_v][slot], (op_turn(is_v, at) & 1) ^ 1));
            const uint32_t swizzle = (uint32_t)(row & 7) << 4;
            if (INT4 && !is_v) {
#pragma unroll
              for (int c = 0; c < C::GROUPS; ++c) {
                const uint32_t scale2 = prmt(group[c], group[c], 0x1010), high2 = scale2 & 0xfff0fff0u;
                const uint32_t rest2 = hsub2(scale2, high2);
                const uint32_t w[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                  uint32_t h[4], r[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    // As fraction bits of 64 + code, less 71.5.
                    const uint32_t u = e == 0 ? w[q] << 4 : w[q] >> (4 * e - 4);
                    const uint32_t code = hsub2((u & 0x00f000f0u) | 0x54005400u, 0x54785478u);
                    h[e] = hmul2(code, high2), r[e] = hmul2(code, rest2);
                  }
                  uint8_t* at16 = to + (c >> 1) * (BK * 128) + ((((4 * c + q) & 7) << 4) ^ swizzle);
                  *reinterpret_cast<uint4*>(at16) = make_uint4(h[0], h[1], h[2], h[3]);
                  *reinterpret_cast<uint4*>(at16 + S::OP) = make_uint4(r[0], r[1], r[2], r[3]);
                }
              }
              // Twice the low and twice the scale of each group; one tile of these.
              ok = __all_sync(0xffffffffu, wait(&bar.groups_empty, (at & 1) ^ 1)) && ok;
              if (ok) {
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                  uint4 of = make_uint4(0, 0, 0, 0);
                  if (c < C::GROUPS)
                    of = make_uint4(prmt(group[c], group[c], 0x3232), prmt(group[c], group[c], 0x1010),
                                    prmt(group[c + 1], group[c + 1], 0x3232), prmt(group[c + 1], group[c + 1], 0x1010));
                  reinterpret_cast<uint4*>(groups_k + row * 32)[c / 2 ^ (row >> 2 & 1)] = of;
                }
              }
            } else
#pragma unroll
            for (int c = 0; c < C::RB / 16; ++c) {
              const uint32_t w[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
              uint32_t scale2 = 0, low2 = 0;
              if constexpr (INT4) scale2 = prmt(group[c], group[c], 0x1010), low2 = prmt(group[c], group[c], 0x3232);
              constexpr int OUT = INT4 ? 4 : 2;  // 16-byte pieces of FP16
#pragma unroll
              for (int q = 0; q < OUT; ++q) {
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  if constexpr (INT4) {
                    // As fraction bits of 1024 + code, or, 4 bits up, of 64 + code.
                    const uint32_t u = e < 2 ? w[q] : w[q] >> 8;
                    h[e] = e % 2 ? hsub2((u & 0x00f000f0u) | 0x54005400u, 0x54005400u)
                                 : hsub2((u & 0x000f000fu) | 0x64006400u, 0x64006400u);
                    h[e] = hfma2(h[e], scale2, low2);
                  } else {
                    const uint32_t u = w[2 * q + e / 2];
                    if constexpr (KIND == AF1_KV_INT8)
                      h[e] = hsub2(prmt(u ^ 0x80808080u, 0x64646464u, e % 2 ? 0x4342 : 0x4140), 0x64806480u);
                    else
                      h[e] = e4m3x2(e % 2 ? u >> 16 : u);
                  }
                }
                const int piece = c * OUT + q;
                *reinterpret_cast<uint4*>(to + (piece >> 3) * (BK * 128) + (((piece & 7) << 4) ^ swizzle)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
              }
            }
          }
          bool odd_value = false;  // a value that is not finite, of a node
          if (is_v && (gone || node)) {
#pragma unroll 1
            for (int c = 0; c < DIM / 8; ++c) {
              uint4 v = *reinterpret_cast<uint4*>(place(c));
              uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7c00u) == 0x7c00u) w[e] &= 0xffff0000u, odd_value = true;
                if ((w[e] & 0x7c000000u) == 0x7c000000u) w[e] &= 0x0000ffffu, odd_value = true;
                if (gone) w[e] = 0;
              }
              *reinterpret_cast<uint4*>(place(c)) = v;
            }
          }
          if (odd_value && !gone) {
            const int bit = key - run.len;
            atomicOr(&bar.nodes_bad[runs_done % 4][bit / 32], 1u << (bit % 32));
          }
          if (!is_v && row == 0) bar.tile_bad[at % kNotes] = bad;
        }
        fence_async();
        __syncwarp();
        if (lane == 0) {
          if (!F16 && !started) mbar_arrive(&bar.code_empty[is_v][st]);
          mbar_arrive(&bar.op_ready[is_v][slot]);
        }
      }
      tiles_done += n;
    }
  } else if (warp == 17) {
    // ---- products ---------------------------------------------------------------------
    // The whole warp runs the loop and one elected lane issues: values that the
    // compiler knows to be alike in all lanes (read from lane 0) stay in the
    // registers that the instruction takes. P V of a tile comes before Q K^T of
    // the second tile after it, so that the arrival of those scores tells that
    // the weights' place is free too.
    const uint32_t base = __shfl_sync(0xffffffffu, tmem, 0);
    const uint32_t q_matrix = matrix(smem_u32(qt), 16), op_matrix = matrix(smem_u32(ops), 16);
    const uint32_t q_groups = matrix(smem_u32(groups_q), 16), k_groups = matrix(smem_u32(groups_k), 16);
    constexpr uint32_t kLead = (uint32_t)(BK * 128 - 16) >> 4 << 16;  // values: 64 entries in a group
    constexpr uint32_t kScores = 1u << 4 | (uint32_t)(BK >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
    constexpr uint32_t kOutput = 1u << 4 | 1u << 16 | (uint32_t)(DIM >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
    for (; run.next(p, bar.plan); runs_done += run.tiles > 0) {
      const int n = __shfl_sync(0xffffffffu, run.tiles, 0);
      if (n == 0) continue;
      bool ok = wait(&bar.q_ready, runs_done & 1);
      for (int j = 0; j < n + 2; ++j) {
        const int at = tiles_done + j, buf = at & 1, turn = at >> 1 & 1;  // the tile two before: the same buffers
        const bool first = j < n, second = j >= 2;
        auto output = [&] {
          if (ok) {
            const uint32_t b = op_matrix + kLead + op_place(true, at) * (S::OP >> 4);
#pragma unroll
            for (int ks = 0; ks < BK / 16; ++ks)
              mma_ts(base + kOutAt, base + kWeightsAt + buf * (BK / 2) + ks * 8, b + (ks * 2048 >> 4), kOutput,
                     j > 2 || ks > 0);
          }
          commit(&bar.pv_done[buf]);
          commit(&bar.op_empty[1][op_slot(true, at)]);
        };
        if (second) {
          ok = wait(&bar.op_ready[1][op_slot(true, at)], op_turn(true, at - 2) & 1) && ok;
          ok = wait(&bar.p_ready[buf], turn ^ 1) && ok;
        }
        if (S::V_SLOTS == 1) {  // the output's products free the one tile of values: at once
          ok = __all_sync(0xffffffffu, ok);
          fence_after();
          if (second && elect()) output();
          __syncwarp();
        }
        if (first) ok = wait(&bar.op_ready[0][buf], turn) && ok;
        ok = __all_sync(0xffffffffu, ok);
        fence_after();
        if (elect()) {
          if (S::V_SLOTS > 1 && second) output();
          if (first) {
            if constexpr (INT4) {  // first: the decoders wait for the one tile of groups
              if (ok) mma_ss<kGroupsHigh>(base + buf * BK, q_groups, k_groups, kScores, false);
              commit(&bar.groups_empty);
            }
            if (ok) {
              const uint32_t b = op_matrix + op_place(false, at) * (S::OP >> 4);
#pragma unroll
              for (int part = 0; part < (INT4 ? 2 : 1); ++part)
#pragma unroll
                for (int ks = 0; ks < DIM / 16; ++ks) {
                  const int off = ((ks / 4) * (BK * 128) + (ks % 4) * 32) >> 4;
                  mma_ss(base + buf * BK, q_matrix + off, b + part * (S::OP >> 4) + off, kScores, INT4 || ks > 0);
                }
            }
            commit(&bar.s_full[buf]);
            commit(&bar.op_empty[0][buf]);
          }
        }
        __syncwarp();
      }
      tiles_done += n;
    }
  } else if (warp < 8) {
    // ---- softmax, and the ends of the runs ------------------------------------------------
    const int half = warp / 4;  // of a tile's keys, and of the output's entries
    const int row = threadIdx.x % 128;
    const uint32_t base = tmem + ((uint32_t)(warp % 4 * 32) << 16);
    float scale = fmaxf(fabsf(p.scale_log2), 1e-30f);  // -infinity times it stays so
    const int e0 = half * (DIM / 2);
    for (; run.next(p, bar.plan); runs_done += run.tiles > 0) {
      const int n = run.tiles, rows = run.rows(p);
      const bool real = row < rows;
      // Where this row's node and query head stand (found again where they are
      // needed: between lie the steps, that need the registers).
      auto place = [&](int& node, int& head) {
        const int gr = run.tile * kRows + row;
        node = gr / p.group, head = run.head * p.group + gr - node * p.group;
      };
      if (run.keys == 0 && run.from == 0 && half == 0 && real) {  // nothing to see: the item's first CTA writes its zeros
        int node, head;
        place(node, head);
        const int64_t at = run.seq * p.o_seq + node * p.o_node + head * p.o_head;
        for (int e = 0; e < DIM; e += 8) {
          if (p.out_f32) {
            reinterpret_cast<float4*>(static_cast<float*>(p.out) + at + e)[0] = make_float4(0.f, 0.f, 0.f, 0.f);
            reinterpret_cast<float4*>(static_cast<float*>(p.out) + at + e)[1] = make_float4(0.f, 0.f, 0.f, 0.f);
          } else {
            *reinterpret_cast<uint4*>(static_cast<__half*>(p.out) + at + e) = make_uint4(0, 0, 0, 0);
          }
        }
        if (p.lse != nullptr) p.lse[((int64_t)run.seq * p.nodes + node) * p.cache.heads * p.group + head] = -kInf;
      }
      if (n == 0) continue;
      uint64_t bits = 0;
      {
        int node, head;
        place(node, head);
        if (real) {
          if (p.mask == nullptr) {
            bits = (2ull << node) - 1;
          } else {
            const uint32_t* w = p.mask + run.seq * p.mask_seq + node * p.words;
            bits = w[0] | (p.words > 1 ? (uint64_t)w[1] << 32 : 0);
          }
        }
        // q of this run (the products with the one before are done), whole rows at
        // a time; a negative scale turns its signs.
        constexpr int CHUNKS = DIM / 8, N = 16 * CHUNKS / 32;
        const uint32_t sign = p.scale_log2 < 0.f ? 0x80008000u : 0u;
        const int c = lane % CHUNKS, r0 = warp * 16 + lane / CHUNKS;
        uint4 v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = r0 + i * (32 / CHUNKS), gr = run.tile * kRows + r, of = gr / p.group;
          v[i] = make_uint4(0, 0, 0, 0);
          if (r < rows)
            v[i] = *reinterpret_cast<const uint4*>(p.q + run.seq * p.q_seq + of * p.q_node +
                                                   (int64_t)(run.head * p.group + gr - of * p.group) * p.q_head + 8 * c);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = r0 + i * (32 / CHUNKS);
          if constexpr (INT4)
            v[i] = make_uint4(prmt(v[i].x, v[i].z, 0x5410), prmt(v[i].x, v[i].z, 0x7632),
                              prmt(v[i].y, v[i].w, 0x5410), prmt(v[i].y, v[i].w, 0x7632));
          v[i].x ^= sign, v[i].y ^= sign, v[i].z ^= sign, v[i].w ^= sign;
          if constexpr (INT4) {
            // The sum over each group of 32 entries (four lanes), in two FP16 parts, and
            // 7.5 times it. Rows whose sums are too large for that are divided by 256,
            // below which their largest entry stays above 1.
            auto both = [](uint32_t h2) { return low_float(h2) + high_float(h2); };
            float sum = (both(v[i].x) + both(v[i].y)) + (both(v[i].z) + both(v[i].w));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            float most = fabsf(sum);
#pragma unroll
            for (int d = 4; d < CHUNKS; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const bool large = most > 8192.f;
            if (large) {
              const uint32_t down = 0x1c001c00u;  // 1 / 256
              v[i] = make_uint4(hmul2(v[i].x, down), hmul2(v[i].y, down), hmul2(v[i].z, down), hmul2(v[i].w, down));
              sum *= 1.f / 256.f;
            }
            if (c == 0) bar.q_scale[r] = large ? 256.f : 1.f;
            auto parts = [](float x) {
              const float hi = __half2float(__float2half_rn(x));
              return pack_half2(hi, x - hi);
            };
            const int at16 = (c / 8) ^ (r >> 2 & 1);
            if (c % 4 == 0)
              *reinterpret_cast<uint2*>(groups_q + r * 32 + at16 * 16 + c / 4 % 2 * 8) =
                  make_uint2(parts(sum), parts(7.5f * sum));
            if (C::GROUPS == 2 && c == 1)
              *reinterpret_cast<uint4*>(groups_q + r * 32 + (at16 ^ 1) * 16) = make_uint4(0, 0, 0, 0);
          }
          *reinterpret_cast<uint4*>(qt + (c >> 3) * (BK * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.q_ready);
        if constexpr (INT4) {
          named_sync(1, 256);
          scale = fmaxf(fabsf(p.scale_log2), 1e-30f) * bar.q_scale[row];
        }
      }
      const bool warp_real = (warp % 4) * 32 < rows;
      // Weights are 2^(score - m - ev + kShift), times a value's scale, which is below 2^ev.
      float m = -kInf, l = 0.f, l_over = 0.f, ev = C::SCALED8 ? kLeastScale : 0.f;
      bool ok = true;
      for (int j = 0; j < n; ++j) {
        const int key = run.k_begin + j * BK, at = tiles_done + j, buf = at & 1;
        ok = wait(&bar.s_full[buf], at >> 1 & 1) && ok;  // and the weights of the tile two before are used
        fence_after();
        ok = __all_sync(0xffffffffu, ok);
        const uint32_t scores = base + buf * BK + half * (BK / 2);
        const int c_first = half * (BK / 2);  // column of the tile
        constexpr int COLS = C::SCALED8 ? 16 : 32;  // at a time: as many as the registers hold, with their scales
        const int at_tile = at % kNotes;
        const bool work = ok && warp_real;
        const uint32_t bad = bar.tile_bad[at_tile];
        const bool masked = key + BK > min(run.len, run.k_end) || bad != 0;
        const float* ks = key_scale + at_tile * BK + c_first;
        const float* vs = value_scale + at_tile * BK + c_first;
        float top = -kInf;
        auto hide = [&](int c, float (&x)[COLS]) {  // -infinity where the row does not see
          auto low = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1; };  // n columns
          const int k0 = key + c_first + c, d = k0 - run.len;  // the first column's key, and node
          uint32_t sees = low(-d);
          if (d >= 0) sees |= d < 64 ? (uint32_t)(bits >> d) : 0u;
          else if (d > -32) sees |= (uint32_t)(bits << -d);
          sees &= low(run.k_end - k0);
          if (bad >> ((c_first + c) / 16) & 1) sees &= 0xffff0000u;
          if (bad >> ((c_first + c) / 16) & 2) sees &= 0x0000ffffu;
#pragma unroll
          for (int i = 0; i < COLS; ++i)
            if (!(sees >> i & 1)) x[i] = -kInf;
        };
        // The half's weights relative to `ref`, and its largest score.
        float2 sum;
        float over;
        auto pass = [&](float ref) {
          float most = -kInf;
          sum = make_float2(0.f, 0.f), over = 0.f;
#pragma unroll 1
          for (int c = 0; c < BK / 2; c += COLS) {
            float x[COLS];
            float4 f8[COLS / 4];
            auto fetch = [&](const float* from) {  // here, not one by one where they are used
              if constexpr (C::SCALED8) {
#pragma unroll
                for (int i = 0; i < COLS / 4; ++i) f8[i] = *reinterpret_cast<const float4*>(from + c + 4 * i);
                asm volatile("" ::: "memory");
              }
            };
            tmem_load(scores + c, x, [&] { fetch(ks); });
#pragma unroll
            for (int i = 0; i < COLS; i += 4) {  // exponents of the weights
              float4 f = make_float4(scale, scale, scale, scale);
              if constexpr (C::SCALED8) f = f8[i / 4];
              const float2 a = fma2(make_float2(x[i], x[i + 1]), make_float2(f.x, f.y), make_float2(-ref, -ref));
              const float2 b = fma2(make_float2(x[i + 2], x[i + 3]), make_float2(f.z, f.w), make_float2(-ref, -ref));
              x[i] = a.x, x[i + 1] = a.y, x[i + 2] = b.x, x[i + 3] = b.y;
            }
            fetch(vs);
            if (masked) hide(c, x);
            float t0 = x[0], t1 = x[1];
#pragma unroll
            for (int i = 2; i < COLS - 2; i += 4) t0 = max3(t0, x[i], x[i + 1]), t1 = max3(t1, x[i + 2], x[i + 3]);
            t0 = max3(t0, x[COLS - 2], x[COLS - 1]);
            most = max3(most, t0, t1);
            if constexpr (INT4) {  // the largest weight, as above
              const float w = ex2(fmaxf(t0, t1));
              over += __half2float(__float2half_rn(w)) - w;
            }
            uint32_t r[COLS / 2];
#pragma unroll
            for (int i = 0; i < COLS; i += 4) {
              float2 a = make_float2(ex2(x[i]), ex2(x[i + 1])), b = make_float2(ex2(x[i + 2]), ex2(x[i + 3]));
              sum = add2(sum, add2(a, b));
              if constexpr (C::SCALED8) {
                const float4 f = f8[i / 4];
                a = mul2(a, make_float2(f.x, f.y)), b = mul2(b, make_float2(f.z, f.w));
              }
              r[i / 2] = pack_half2(a.x, a.y), r[i / 2 + 1] = pack_half2(b.x, b.y);
            }
            tmem_store(base + kWeightsAt + buf * (BK / 2) + (c_first + c) / 2, r);
          }
          top = most + ref;
          tmem_wait_store();
        };
        // The weights relative to the maximum so far, which mostly holds; where a
        // row's has to move (both halves agree on that), they are formed again.
        auto reference = [&] { return (m == -kInf ? 0.f : m) + ev - kShift; };
        if (work) pass(reference());
        float ev_now = ev;
        if constexpr (C::SCALED8) {
          const float4 most = *reinterpret_cast<const float4*>(bar.value_top[at_tile]);
          const float tile_top = fmaxf(fmaxf(most.x, most.y), fmaxf(most.z, most.w));
          if (tile_top > ev) ev_now = tile_top + 1.f;  // with room, as moving costs as much as a tile
        }
        // The two warps that have these rows agree.
        bar.top[buf][half][row] = top;
        named_sync(2 + warp % 4, 64);
        top = fmaxf(top, bar.top[buf][half ^ 1][row]);
        if (__any_sync(0xffffffffu, work && (top > m + kSlack || ev_now > ev))) {
          if (work) {
            const float now = fmaxf(m, top);
            const float alpha = ex2(m - (now == -kInf ? 0.f : now) + (ev - ev_now));
            m = now, ev = ev_now;
            l *= alpha, l_over *= alpha;
            if (j > 0) {
              ok = wait(&bar.pv_done[buf ^ 1], (at - 1) >> 1 & 1);
              ok = __all_sync(0xffffffffu, ok);
              fence_after();
#pragma unroll 1
              for (int c = e0; c < e0 + DIM / 2; c += 32) {
                float x[32];
                tmem_load(base + kOutAt + c, x);
                uint32_t r[16];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
                  for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(x[16 * hf + i] * alpha);
                  tmem_store(base + kOutAt + c + 16 * hf, r);
                }
              }
            }
            pass(reference());
          }
        }
        if (work) l += sum.x + sum.y, l_over += over;
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.p_ready[buf]);
      }
      m += ev;  // the reference that sums and outputs share
      // -- the run's end ------------------------------------------------------------------
      {
        const int last = tiles_done + n - 1;
        bar.sum[half][row] = l;
        if constexpr (INT4) bar.over[half][row] = l_over;
        ok = wait(&bar.pv_done[last & 1], last >> 1 & 1) && ok;
        fence_after();
        ok = __all_sync(0xffffffffu, ok);
        const uint32_t* odd = bar.nodes_bad[runs_done % 4];
        const uint64_t poison = (odd[0] | (uint64_t)odd[1] << 32) & bits;
        named_sync(1, 256);
        if (threadIdx.x == 0) bar.nodes_bad[runs_done % 4][0] = bar.nodes_bad[runs_done % 4][1] = 0;
        const float sum = l + bar.sum[half ^ 1][row];
        // What rounding adds to the largest weights, and so to the output, it adds to the
        // divisor, too (of the output: lse takes the sum of what they were before).
        const float even = INT4 && sum > 0.f ? sum / (sum + (l_over + bar.over[half ^ 1][row])) : 1.f;
        const bool whole = run.from <= kSetupTiles && run.to == run.units;
        int c0 = 0, c1 = 0, node, head;
        if (!whole)
          c0 = holder(bar.plan, run.first + kSetupTiles), c1 = holder(bar.plan, run.first + run.units - 1);
        place(node, head);
        __half* out16 = static_cast<__half*>(p.out) + run.seq * p.o_seq + node * p.o_node + head * p.o_head;
        float* out32 = static_cast<float*>(p.out) + run.seq * p.o_seq + node * p.o_node + head * p.o_head;
        const int live_nodes = node_count(p, run.seq);
        auto part_of = [&](int c) { return p.parts + (int64_t)(2 * c + (c == c0 ? 1 : 0)) * S::PART; };
        float* part = part_of(blockIdx.x);
        const bool live = node < live_nodes;
        auto write = [&](int place, float inv, const float (&x)[8]) {  // 8 places of the row
          float y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) y[place_entry<KIND>(i)] = inv == 0.f ? 0.f : x[i] * inv;
          if (p.out_f32) {
            reinterpret_cast<float4*>(out32 + place)[0] = make_float4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<float4*>(out32 + place)[1] = make_float4(y[4], y[5], y[6], y[7]);
          } else {
            *reinterpret_cast<uint4*>(out16 + place) = make_uint4(pack_half2(y[0], y[1]), pack_half2(y[2], y[3]),
                                                                  pack_half2(y[4], y[5]), pack_half2(y[6], y[7]));
          }
        };
        auto inverse = [&](float total) { return live && total != 0.f ? 1.f / total : 0.f; };
        if (ok && warp_real) {
#pragma unroll 1
          for (int c = e0; c < e0 + DIM / 2; c += 32) {
            float x[32];
            tmem_load(base + kOutAt + c, x);
            if constexpr (INT4) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] *= even;
            }
            if (poison != 0) {  // infinite and NaN values of nodes that this row sees
              for (uint64_t left = poison; left != 0; left &= left - 1) {
                const int slot = run.len + __ffsll((long long)left) - 1;
                if (slot < run.k_begin || slot >= run.k_end) continue;
                const int64_t at = kv_row(p.cache, p.pages, run.seq, slot, run.head);
                if (at < 0) continue;
                const uint8_t* v = p.cache.v + at * C::RB;
                const uint8_t* vs = static_cast<const uint8_t*>(p.cache.vs) + at * C::SB;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const int e = place_entry<KIND>(c + i);
                  float y;
                  if constexpr (F16) {
                    y = __half2float(reinterpret_cast<const __half*>(v)[e]);
                  } else if constexpr (INT4) {
                    const uint32_t sc = reinterpret_cast<const uint32_t*>(vs)[e / 32];
                    y = fmaf((float)(v[e / 2] >> (e % 2 * 4) & 15), low_float(sc), high_float(sc));
                  } else {  // times a scale that is not finite, or, of a finite one, by code alone
                    const float scale = *reinterpret_cast<const float*>(vs);
                    y = KIND == AF1_KV_INT8 ? (float)(int8_t)v[e]
                                            : __half2float(__half(__nv_cvt_fp8_to_halfraw(v[e], __NV_E4M3)));
                    if (!(fabsf(scale) < kInf)) y *= scale;
                  }
                  y = __half2float(__float2half_rn(y));
                  if (!(fabsf(y) <= 65504.f)) x[i] += y;
                }
              }
            }
            if (real && whole) {
#pragma unroll
              for (int i = 0; i < 32; i += 8) {
                const float y[8] = {x[i], x[i + 1], x[i + 2], x[i + 3], x[i + 4], x[i + 5], x[i + 6], x[i + 7]};
                write(c + i, inverse(sum), y);
              }
            } else if (real) {
#pragma unroll
              for (int i = 0; i < 32; ++i) part[(c + i) * part_ld(rows) + row] = x[i];
            }
          }
          if (real && half == 0) {
            if (!whole) part[DIM * part_ld(rows) + row] = m, part[(DIM + 1) * part_ld(rows) + row] = sum;
            else if (p.lse != nullptr)
              p.lse[((int64_t)run.seq * p.nodes + node) * p.cache.heads * p.group + head] = live && sum != 0.f ? (m - kShift + log2f(sum)) * 0.69314718056f : -kInf;
          }
        }
        if (!whole && threadIdx.x == 0) bar.part[bar.parts++] = {c0, c1, run.seq, run.head, run.tile, rows};
      }
      tiles_done += n;
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (bar.gave_up) {  // by any role: no role waits any more
    // Copies and products may still be on their way. They end, within a limit,
    // before the parts are joined over the tiles and tensor memory goes.
    const long long t0 = clock64(), limit = max(p.wait_cycles, kLanding);
    if ((warp == 16 || warp == 18) && lane == 0) {
      const bool is_v = warp == 18;
      const int issued = bar.issued[is_v];
      for (int at = max(issued + 1 - (is_v ? S::V_STAGES : S::K_STAGES), 0); at <= issued; ++at)
        while (!mbar_try_wait(&bar.code_full[is_v][code_stage(is_v, at)], code_turn(is_v, at) & 1) &&
               clock64() - t0 < limit) {
        }
    }
    if (warp == 17 && elect()) {  // the lane that issued the products
      commit(&bar.drained);
      while (!mbar_try_wait(&bar.drained, 0) && clock64() - t0 < limit) {
      }
    }
    if (threadIdx.x == 0) atomicOr(p.status, kStatusTimeout);
    __syncthreads();
  }
  // ---- items that span CTAs: the last CTA to arrive joins the parts, in order.
  // A thread has 8 places of 4 rows, and copies them (and the rows' maxima and
  // sums) to slots of its own in shared memory, whose tiles are used up, two or
  // four parts ahead; the parts of this CTA's two items follow one another.
  if ((int)threadIdx.x < bar.parts) {  // the CTA's parts are released with it
    unsigned* counter = &p.counters[bar.part[threadIdx.x].c0];
    const unsigned others = bar.part[threadIdx.x].c1 - bar.part[threadIdx.x].c0;
    const bool last = atom_add_acq_rel_gpu(counter, 1u) == others;
    bar.last[threadIdx.x] = last;
    if (last) *counter = 0;  // as the next call finds it
  }
  __syncthreads();
  int steps[2] = {0, 0}, quads[2] = {1, 1};
  for (int i = 0; i < bar.parts; ++i) {
    if (bar.last[i]) steps[i] = bar.part[i].c1 - bar.part[i].c0 + 1;
    quads[i] = part_ld(bar.part[i].rows) / 4;
  }
  const int most = steps[1] > 0 ? max(quads[0], quads[1]) : quads[0], ahead = most <= kRows / 8 ? 4 : 2;
  auto slot = [&](int step, int which) {
    return smem + ((step & (ahead - 1)) * 10 + which) * (DIM / 8 * 16 * most) + threadIdx.x * 16;
  };
  auto fetch = [&](int step) {
    const int i = step >= steps[0], k = step - (i ? steps[0] : 0);
    const int q = i ? quads[1] : quads[0], row0 = threadIdx.x % q * 4, e0 = threadIdx.x / q * 8;
    if (k < (i ? steps[1] : steps[0]) && e0 < DIM) {
      const float* from = p.parts + (int64_t)(2 * (bar.part[i].c0 + k) + (k == 0 ? 1 : 0)) * S::PART + row0;
#pragma unroll
      for (int e = 0; e < 8; ++e) copy16(slot(step, e), from + (e0 + e) * (4 * q));
      copy16(slot(step, 8), from + DIM * (4 * q));
      copy16(slot(step, 9), from + (DIM + 1) * (4 * q));
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int step = 0; step < (steps[0] + steps[1] > 0 ? ahead : 0); ++step) fetch(step);
  for (int i = 0, step = 0; i < 2; ++i) {
    const int q = i ? quads[1] : quads[0], row0 = threadIdx.x % q * 4, e0 = threadIdx.x / q * 8;
    const int end = step + (i ? steps[1] : steps[0]);
    if (step == end) continue;
    float m[4], l[4], acc[8][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      m[r] = -kInf, l[r] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e][r] = 0.f;
    }
    for (; step < end; ++step) {
      if (ahead == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else asm volatile("cp.async.wait_group 1;" ::: "memory");
      if (e0 < DIM) {
        float part_m[4], part_l[4], a[4], b[4];
        *reinterpret_cast<float4*>(part_m) = *reinterpret_cast<const float4*>(slot(step, 8));
        *reinterpret_cast<float4*>(part_l) = *reinterpret_cast<const float4*>(slot(step, 9));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float now = fmaxf(m[r], part_m[r]), zero = now == -kInf ? 0.f : now;
          a[r] = ex2(m[r] - zero), b[r] = ex2(part_m[r] - zero);
          l[r] = fmaf(b[r], part_l[r], l[r] * a[r]);
          m[r] = now;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y[4];
          *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(slot(step, e));
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[e][r] = fmaf(b[r], y[r], acc[e][r] * a[r]);
        }
      }
      fetch(step + ahead);
    }
    if (e0 < DIM) {
      const int seq = bar.part[i].seq, live_nodes = node_count(p, seq);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (row0 + r >= bar.part[i].rows) break;
        const int gr = bar.part[i].tile * kRows + row0 + r, node = gr / p.group;
        const int head = bar.part[i].head * p.group + gr - node * p.group;
        const bool live = node < live_nodes && l[r] != 0.f;
        const float inv = live ? 1.f / l[r] : 0.f;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[place_entry<KIND>(e)] = live ? acc[e][r] * inv : 0.f;
        const int64_t at = seq * p.o_seq + node * p.o_node + head * p.o_head + e0;
        if (p.out_f32) {
          reinterpret_cast<float4*>(static_cast<float*>(p.out) + at)[0] = make_float4(y[0], y[1], y[2], y[3]);
          reinterpret_cast<float4*>(static_cast<float*>(p.out) + at)[1] = make_float4(y[4], y[5], y[6], y[7]);
        } else {
          *reinterpret_cast<uint4*>(static_cast<__half*>(p.out) + at) = make_uint4(
              pack_half2(y[0], y[1]), pack_half2(y[2], y[3]), pack_half2(y[4], y[5]), pack_half2(y[6], y[7]));
        }
        if (e0 == 0 && p.lse != nullptr)
          p.lse[((int64_t)seq * p.nodes + node) * p.cache.heads * p.group + head] =
              live ? (m[r] - kShift + log2f(l[r])) * 0.69314718056f : -kInf;
      }
    }
  }
  if (warp == 16)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int KIND, int DIM>
cudaError_t launch(const TreeProblem& p, int sms, cudaStream_t st) {
  constexpr int smem = Wide<KIND, DIM>::SMEM;
  auto kernel = wide_kernel<KIND, DIM>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  kernel<<<std::min(sms, kMaxCtas), kThreads, smem, st>>>(p);
  return cudaGetLastError();
}

template <int KIND>
cudaError_t launch_kind(const TreeProblem& p, const af1_kv_cache& c, cudaStream_t st) {
  return c.d.head_dim == 128 ? launch<KIND, 128>(p, c.num_sms, st) : launch<KIND, 64>(p, c.num_sms, st);
}

}  // namespace

int64_t tree_wide_part_bytes(const af1_kv_cache& c) {
  return 2 * (int64_t)std::min(c.num_sms, kMaxCtas) * kRows * (c.d.head_dim + 2) * 4;
}

cudaError_t launch_tree_wide(TreeProblem& p, const af1_kv_cache& c, int rows, cudaStream_t st) {
  p.row_tiles = (rows + kRows - 1) / kRows;
  p.k_map = c.k_tile, p.v_map = c.v_tile;
  switch (c.d.kind) {
    case AF1_KV_F16: return launch_kind<AF1_KV_F16>(p, c, st);
    case AF1_KV_INT8: return launch_kind<AF1_KV_INT8>(p, c, st);
    case AF1_KV_E4M3: return launch_kind<AF1_KV_E4M3>(p, c, st);
    default: return launch_kind<AF1_KV_INT4>(p, c, st);
  }
}

}  // namespace af1
