// af1_pages.cu — what happens to the cache's pages between two steps of
// drafted tokens: accepted slots move behind the prefix, pages are copied, and
// the table of pages is forked, reserved in and released.
//
// Nothing is computed on keys and values: rows of codes and scales move as they
// are, those of all layers in one launch (a launch for each of 32 layers would
// take longer than their rows). Device memory bounds large calls (100 INT4
// pages of 128 slots in 16 layers, 525 MB: 79 us, 6.6 TB/s; 64 paths of 7 moved
// rows in 32 FP16 layers, 117 MB in pieces of 256 bytes: 19 us, 25 from a cold
// cache), and latency the others (2 to 4 us). The table's calls decide on the device, so that the lengths
// that verification gives need not reach the host: fork, reserve and release take
// 12.7 us for 256 sequences over 131072 pages, 9.7 for 16 over 1000. Reserve's one block looks
// for free pages 4096 at a time: 6.4 us for 512 of 131072 free ones, 34 where only the last 1 percent
// are free, 215 of 1000000.
#include <algorithm>

#include "af1_internal.h"
#include "af1_kv.cuh"

namespace af1 {
namespace {

constexpr int kMaxCaches = 256;
constexpr int kLaunchCaches = 60;  // 64 bytes each in the 4 KB of a launch's arguments
constexpr int kMaxNodes = 64;
constexpr int kMaxSequences = 1024;

struct Moved {
  KvView view;
  int row_bytes, scale_bytes;
  int row_shift, scale_shift;  // 16-byte accesses of a row of codes, words of its scales: 1 << shift
};
struct Caches {
  Moved c[kLaunchCaches];
};

// ---- accepted slots ------------------------------------------------------------

struct CompactProblem {
  PageTable pages;
  const int32_t *first, *index, *counts;
  int nodes;
};
constexpr int kMoveWarps = 4;
constexpr int kInFlight = 8;  // accesses of a lane

// A warp moves the rows of one head of one sequence's keys or values. Rows that
// fit its lanes' registers (4 KB) are all read before the first is written, so
// that the slots may come in any order; longer lists too where no slot lies
// before the one that it goes to (as on the path of a tree whose nodes come
// after their parents: what a batch of rows overwrites lies before all that is
// read after it). The others pass through local memory.
template <typename T>
__device__ __forceinline__ void move_rows(void* base, int shift, const int2* moves, int n, bool ordered, int lane) {
  T* x = static_cast<T*>(base);  // rows of 1 << shift accesses; item i is access i of the moves' rows
  const int total = n << shift, mask = (1 << shift) - 1;
  auto source = [&](int item) { return ((int64_t)moves[item >> shift].x << shift) + (item & mask); };
  auto target = [&](int item) { return ((int64_t)moves[item >> shift].y << shift) + (item & mask); };
  if (total <= 32 * kInFlight || ordered) {
    for (int at = lane; at - lane < total; at += 32 * kInFlight) {
      T v[kInFlight];
#pragma unroll
      for (int i = 0; i < kInFlight; ++i)
        if (at + i * 32 < total) v[i] = x[source(at + i * 32)];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kInFlight; ++i)
        if (at + i * 32 < total) x[target(at + i * 32)] = v[i];
      __syncwarp();
    }
    return;
  }
  T v[kMaxNodes * 16 / 32];
  for (int at = lane, i = 0; at < total; at += 32, ++i) v[i] = x[source(at)];
  __syncwarp();
  for (int at = lane, i = 0; at < total; at += 32, ++i) x[target(at)] = v[i];
}

__global__ void __launch_bounds__(32 * kMoveWarps) compact_kernel(const __grid_constant__ Caches caches,
                                                                  const __grid_constant__ CompactProblem p) {
  const Moved& m = caches.c[blockIdx.y];
  const int lane = threadIdx.x % 32;
  const int64_t unit = (int64_t)blockIdx.x * kMoveWarps + threadIdx.x / 32;
  const int64_t seq = unit / (2 * m.view.heads);
  if (seq >= p.pages.seqs) return;
  const int part = (int)(unit - seq * (2 * m.view.heads)), head = part >> 1;
  const bool is_v = (part & 1) != 0;
  const int n = min(p.nodes, p.counts[seq]);
  const int64_t first = p.first[seq];
  __shared__ int2 lists[kMoveWarps][kMaxNodes];  // rows, without what stays where it is
  int2* moves = lists[threadIdx.x / 32];
  int count = 0;
  bool ordered = true;
  for (int j0 = 0; j0 < n; j0 += 32) {
    const int j = j0 + lane, at = j < n ? p.index[seq * p.nodes + j] : j;
    const int64_t s = first + at, t = first + j;
    int2 rows = make_int2(-1, -1);
    if (at != j && s >= 0 && s <= 0x7fffffff && t >= 0 && t <= 0x7fffffff)
      rows = make_int2((int)kv_row(m.view, p.pages, (int)seq, (int)s, head),
                       (int)kv_row(m.view, p.pages, (int)seq, (int)t, head));
    const bool moved = rows.x >= 0 && rows.y >= 0;
    ordered = ordered && __all_sync(0xffffffffu, !moved || at > j);
    const unsigned want = __ballot_sync(0xffffffffu, moved);
    if (moved) moves[count + __popc(want & ((1u << lane) - 1))] = rows;
    count += __popc(want);
  }
  if (count == 0) return;
  __syncwarp();
  move_rows<uint4>(is_v ? m.view.v : m.view.k, m.row_shift, moves, count, ordered, lane);
  if (m.scale_bytes > 0)
    move_rows<uint32_t>(is_v ? m.view.vs : m.view.ks, m.scale_shift, moves, count, ordered, lane);
}

// ---- copied pages ----------------------------------------------------------------

constexpr int kCopyThreads = 128;

__device__ __forceinline__ void copy_bytes(uint8_t* to, const uint8_t* from, int bytes) {
  const int n = bytes / 16;
  const uint4* x = reinterpret_cast<const uint4*>(from);
  uint4* y = reinterpret_cast<uint4*>(to);
  for (int at = threadIdx.x; at < n; at += kInFlight * kCopyThreads) {
    uint4 v[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (at + i * kCopyThreads < n) v[i] = x[at + i * kCopyThreads];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i)
      if (at + i * kCopyThreads < n) y[at + i * kCopyThreads] = v[i];
  }
  // Scales of a few rows: less than 16 bytes left, in words.
  const int words = bytes % 16 / 4;
  if ((int)threadIdx.x < words)
    reinterpret_cast<uint32_t*>(to + n * 16)[threadIdx.x] = reinterpret_cast<const uint32_t*>(from + n * 16)[threadIdx.x];
}

// A block copies the rows of one head of one page of keys or values.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ Caches caches, const int32_t* copies) {
  const Moved& m = caches.c[blockIdx.y];
  const int part = blockIdx.z;
  if (part >= 2 * m.view.heads) return;
  const int head = part >> 1;
  const bool is_v = (part & 1) != 0;
  const int32_t* entry = copies + (int64_t)blockIdx.x * 3;
  const int from = entry[0], to = entry[1], rows = min(entry[2], 1 << m.view.shift);
  if (from < 0 || from >= m.view.pages || to < 0 || to >= m.view.pages || rows < 1 || from == to) return;
  const int64_t source = ((int64_t)from * m.view.heads + head) << m.view.shift;
  const int64_t target = ((int64_t)to * m.view.heads + head) << m.view.shift;
  uint8_t* codes = is_v ? m.view.v : m.view.k;
  copy_bytes(codes + target * m.row_bytes, codes + source * m.row_bytes, rows * m.row_bytes);
  if (m.scale_bytes > 0) {
    uint8_t* scales = static_cast<uint8_t*>(is_v ? m.view.vs : m.view.ks);
    copy_bytes(scales + target * m.scale_bytes, scales + source * m.scale_bytes, rows * m.scale_bytes);
  }
}

// ---- the table -------------------------------------------------------------------

struct TableView {
  int32_t *table, *refs;
  int64_t ld;
  int seqs, columns, pages, shift;
};
__device__ __forceinline__ bool holds(const TableView& t, int page) { return page >= 0 && page < t.pages; }

// A block takes a few columns of all rows: it reads them all before it writes.
constexpr int kForkColumns = 8, kForkThreads = 1024;
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const TableView t, const int32_t* parents) {
  __shared__ int32_t old[kMaxSequences * kForkColumns];
  const int column = blockIdx.x * kForkColumns + threadIdx.x % kForkColumns;
  const bool inside = column < t.columns;
  constexpr int kRows = kForkThreads / kForkColumns;
  for (int s = threadIdx.x / kForkColumns; s < t.seqs; s += kRows)
    if (inside) old[s * kForkColumns + threadIdx.x % kForkColumns] = t.table[s * t.ld + column];
  __syncthreads();
  if (!inside) return;
  for (int s = threadIdx.x / kForkColumns; s < t.seqs; s += kRows) {
    const int parent = parents[s];
    if (parent == s) continue;
    const int was = old[s * kForkColumns + threadIdx.x % kForkColumns];
    const int now = parent >= 0 && parent < t.seqs ? old[parent * kForkColumns + threadIdx.x % kForkColumns] : -1;
    if (now == was) continue;
    if (holds(t, was)) atomicSub(&t.refs[was], 1);
    if (holds(t, now)) atomicAdd(&t.refs[now], 1);
    t.table[s * t.ld + column] = now;
  }
}

constexpr int kReleaseThreads = 256;
__global__ void __launch_bounds__(kReleaseThreads) release_kernel(const TableView t, const int32_t* lens) {
  const int s = blockIdx.y;
  const int64_t kept = ((int64_t)max(lens[s], 0) + (1 << t.shift) - 1) >> t.shift;
  const int column = blockIdx.x * kReleaseThreads + threadIdx.x;
  if (column < kept || column >= t.columns) return;
  int32_t* entry = &t.table[s * t.ld + column];
  const int page = *entry;
  if (holds(t, page)) atomicSub(&t.refs[page], 1);
  if (page != -1) *entry = -1;
}

// One block. The entries that the slots lie in are numbered in order of sequences and columns; a thread takes every
// 1024th. Up to kNear of them, what is noted of them lies in shared memory, and pages that several of them hold meet in a
// hash table there; of more, in the workspace, and pages meet in refs. (With a warp to a sequence and all notes in the
// workspace a step of 256 sequences, fork and release among it, took 34 us.)
constexpr int kReserveThreads = 1024;
constexpr int kReserveWarps = kReserveThreads / 32;
constexpr int kNear = 1024, kLogSlots = 11, kSlots = 1 << kLogSlots;
// What is noted of an entry; below 0: page -1 - note is to be replaced.
enum : int32_t { kOwn = 0, kMissing = 1, kShared = 2, kLast = 3, kKeeps = 4 };

__device__ __forceinline__ int block_exclusive(int x, int* warps, int* total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int other = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += other;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int w = warps[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += other;
    }
    warps[lane] = w;
  }
  __syncthreads();
  *total = warps[kReserveWarps - 1];
  return (warp > 0 ? warps[warp - 1] : 0) + sum - x;
}

__global__ void __launch_bounds__(kReserveThreads) reserve_kernel(const TableView t, const int32_t* first,
                                                                  const int32_t* counts, int32_t* copies,
                                                                  int32_t* lacking, int32_t* far_notes, int32_t* far_list) {
  __shared__ int begin[kMaxSequences], before[kMaxSequences + 1], warps[kReserveWarps];
  __shared__ int near_notes[kNear], near_list[kNear];
  __shared__ int slot_page[kSlots], slot_count[kSlots], slot_last[kSlots];
  const int tid = threadIdx.x;
  const int page_mask = (1 << t.shift) - 1;
  int columns = 0;
  if (tid < t.seqs) {
    const int64_t f = first[tid], n = counts[tid];
    if (f >= 0 && n >= 1)
      columns = (int)max((int64_t)0, min((int64_t)t.columns, ((f + n - 1) >> t.shift) + 1) - (f >> t.shift));
    begin[tid] = columns > 0 ? (int)(f >> t.shift) : 0;
    copies[tid * 3] = copies[tid * 3 + 1] = copies[tid * 3 + 2] = -1;
  }
  for (int i = tid; i < kSlots; i += kReserveThreads) slot_page[i] = -1, slot_count[i] = 0, slot_last[i] = -1;
  int entries;
  const int own_before = block_exclusive(columns, warps, &entries);
  if (tid < t.seqs) before[tid] = own_before;
  if (tid == 0) before[t.seqs] = entries;
  __syncthreads();
  const bool near = entries <= kNear;
  int32_t* const notes = near ? near_notes : far_notes;
  int32_t* const list = near ? near_list : far_list;
  auto sequence_of = [&](int i) {  // before[s] <= i < before[s + 1]
    int s = 0;
    for (int half = kMaxSequences / 2; half > 0; half /= 2)
      if (s + half < t.seqs && before[s + half] <= i) s += half;
    return s;
  };
  auto entry_of = [&](int i) {
    const int s = sequence_of(i);
    return &t.table[s * t.ld + begin[s] + (i - before[s])];
  };
  bool shared = false;
  int page0 = -1;  // of the thread's first entry, whose place and page are not looked up again
  int32_t* entry0 = nullptr;
  for (int i = tid; i < entries; i += kReserveThreads) {
    int32_t* entry = entry_of(i);
    const int page = *entry, count = holds(t, page) ? __ldcg(&t.refs[page]) : 0;
    if (i == tid) entry0 = entry, page0 = page;
    int note = !holds(t, page) ? kMissing : kOwn;
    if (count > 1) {
      note = kShared, shared = true;
      if (near) {  // at most half of the slots are taken
        int at = (int)((uint32_t)page * 2654435769u >> (32 - kLogSlots));
        for (;;) {
          const int found = atomicCAS(&slot_page[at], -1, page);
          if (found == -1 || found == page) break;
          at = (at + 1) % kSlots;
        }
        static_assert(kNear * 2 <= kSlots, "");
        atomicAdd(&slot_count[at], 1);
        atomicMax(&slot_last[at], i);
        note = at << 3 | kShared;
      }
    }
    notes[i] = note;
  }
  auto each = [&](auto&& f) {  // f(number, its place in the table, its page), of entries that a page is held by
    for (int i = tid; i < entries; i += kReserveThreads) {
      int32_t* entry = i == tid ? entry0 : entry_of(i);
      f(i, entry, i == tid ? page0 : *entry);
    }
  };
  if (__syncthreads_or(shared)) {
    // Of the entries of a page that are no fewer than its count, the last keeps it.
    if (near) {
      each([&](int i, int32_t*, int page) {
        if ((notes[i] & 7) != kShared) return;
        const int at = notes[i] >> 3;
        // A page that all of its holders write to has as many entries here as its count says.
        const bool keeps = slot_last[at] == i && slot_count[at] >= __ldcg(&t.refs[page]);
        notes[i] = keeps ? kKeeps : -1 - page;
      });
      __syncthreads();
      each([&](int i, int32_t*, int page) {
        if (notes[i] < 0) atomicSub(&t.refs[page], 1);
      });
      __syncthreads();
    } else {
      // By the count, which comes to 0 then, and stands for the largest number for a moment.
      each([&](int i, int32_t*, int page) {
        if (notes[i] == kShared) atomicSub(&t.refs[page], 1);
      });
      __syncthreads();
      each([&](int i, int32_t*, int page) {
        if (notes[i] == kShared) notes[i] = __ldcg(&t.refs[page]) <= 0 ? kLast : -1 - page;
      });
      __syncthreads();
      each([&](int i, int32_t*, int page) {
        if (notes[i] == kLast) atomicMin(&t.refs[page], -2 - i);
      });
      __syncthreads();
      each([&](int i, int32_t*, int page) {
        if (notes[i] == kLast) notes[i] = __ldcg(&t.refs[page]) == -2 - i ? kKeeps : -1 - page;
      });
      __syncthreads();
    }
    each([&](int i, int32_t*, int page) {
      if (notes[i] == kKeeps) __stcg(&t.refs[page], 1);
    });
    __syncthreads();
  }
  // The list of entries that need a page.
  int total = 0;
  for (int base = 0; base < entries; base += kReserveThreads) {
    const int i = base + tid, note = i < entries ? notes[i] : kOwn;
    const bool need = note < 0 || note == kMissing;
    int here;
    const int rank = block_exclusive(need ? 1 : 0, warps, &here);
    if (need) list[total + rank] = i;
    total += here;
  }
  __syncthreads();
  // Free pages, in order, to the list's entries.
  int found = 0;
  for (int64_t base = 0; base < t.pages && found < total; base += 4 * kReserveThreads) {
    int free = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t page = base + 4 * tid + i;
      if (page < t.pages && __ldcg(&t.refs[page]) == 0) free |= 1 << i;
    }
    int here;
    int rank = found + block_exclusive(__popc(free), warps, &here);
    for (; free != 0 && rank < total; free &= free - 1, ++rank) {
      const int page = (int)(base + 4 * tid + __ffs(free) - 1);
      const int i = list[rank], s = sequence_of(i), c = begin[s] + (i - before[s]);
      t.table[s * t.ld + c] = page;
      __stcg(&t.refs[page], 1);
      const int note = notes[i], f = first[s];
      if (note < 0 && c == f >> t.shift && (f & page_mask) != 0) {
        copies[s * 3] = -1 - note;
        copies[s * 3 + 1] = page;
        copies[s * 3 + 2] = f & page_mask;
      }
    }
    found += here;
  }
  if (found < total) {  // all as it was
    __syncthreads();
    for (int k = tid; k < total; k += kReserveThreads) {
      const int i = list[k], note = notes[i];
      int32_t* entry = entry_of(i);
      if (k < found) __stcg(&t.refs[*entry], 0);
      *entry = note < 0 ? -1 - note : -1;
      if (note < 0) atomicAdd(&t.refs[-1 - note], 1);
    }
    if (tid < t.seqs) copies[tid * 3] = copies[tid * 3 + 1] = copies[tid * 3 + 2] = -1;
  }
  if (tid == 0) *lacking = max(0, total - found);
}

// ---- host ------------------------------------------------------------------------

int fail(int code, const char* who, const std::string& msg) { return set_error(code, std::string(who) + ": " + msg); }

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess)
    return fail(AF1_ERR_CUDA, who, std::string(cudaGetErrorName(e)) + " (" + cudaGetErrorString(e) + ")");
  set_error(AF1_OK, "");
  return AF1_OK;
}

int current_device(const char* who, int* dev) {
  const cudaError_t e = cudaGetDevice(dev);
  if (e != cudaSuccess) return fail(AF1_ERR_CUDA, who, cudaGetErrorString(e));
  return AF1_OK;
}

int check_words(const void* p, const char* name, int dev) {
  const int rc = check_pointer(p, name, dev);
  return rc == AF1_OK ? check_align(p, 4, name) : rc;
}

int check_caches(const char* who, const af1_kv_cache* const* caches, int64_t count, int* dev) {
  if (caches == nullptr || count < 1 || count > kMaxCaches)
    return fail(AF1_ERR_INVALID_ARG, who, "need 1..256 caches");
  const int rc = current_device(who, dev);
  if (rc != AF1_OK) return rc;
  for (int64_t i = 0; i < count; ++i) {
    if (caches[i] == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "a cache is NULL");
    if (caches[i]->device != *dev) return fail(AF1_ERR_BAD_POINTER, who, "the current device is not the caches' device");
    if (caches[i]->d.page_size != caches[0]->d.page_size)
      return fail(AF1_ERR_INVALID_ARG, who, "the caches must have one page size");
    for (int64_t j = 0; j < i; ++j)
      if (caches[i]->d.k == caches[j]->d.k || caches[i]->d.v == caches[j]->d.v)
        return fail(AF1_ERR_INVALID_ARG, who, "a buffer is given twice");
  }
  return AF1_OK;
}

// launch(caches, how many, the most heads) for up to kLaunchCaches at a time.
template <typename F>
int in_parts(const char* who, const af1_kv_cache* const* caches, int64_t count, F&& launch) {
  for (int64_t at = 0; at < count; at += kLaunchCaches) {
    Caches some;
    const int n = (int)std::min<int64_t>(kLaunchCaches, count - at);
    int heads = 1;
    for (int i = 0; i < n; ++i) {
      const af1_kv_desc& d = caches[at + i]->d;
      Moved& m = some.c[i];
      m = {view_of(d), kv_row_bytes(d.kind, d.head_dim), kv_scale_bytes(d.kind, d.head_dim), 0, 0};
      while (16 << m.row_shift < m.row_bytes) ++m.row_shift;
      while (4 << m.scale_shift < m.scale_bytes) ++m.scale_shift;
      heads = std::max(heads, d.kv_heads);
    }
    launch(some, n, heads);
    const int rc = launched(who);
    if (rc != AF1_OK) return rc;
  }
  return AF1_OK;
}

int check_table(const char* who, const af1_page_table* t, TableView* view) {
  if (t == nullptr) return fail(AF1_ERR_INVALID_ARG, who, "table is NULL");
  if (t->page_size < 16 || t->page_size > 256 || (t->page_size & (t->page_size - 1)) != 0)
    return fail(AF1_ERR_INVALID_ARG, who, "page_size must be 16, 32, 64, 128 or 256");
  if (t->reserved != 0) return fail(AF1_ERR_INVALID_ARG, who, "reserved must be 0");
  if (t->sequences < 0 || t->sequences > kMaxSequences || t->columns < 1 || t->columns > (1 << 20) ||
      t->columns > ((int64_t)1 << 31) / t->page_size - 1 || t->ld < t->columns || t->ld > ((int64_t)1 << 36))
    return fail(AF1_ERR_INVALID_ARG, who,
                "need at most 1024 sequences, 1..2^20 columns of fewer than 2^31 slots in all, columns <= ld <= 2^36");
  if (t->pages < 1 || t->pages > 0x7fffffff) return fail(AF1_ERR_INVALID_ARG, who, "pages must be 1..2^31 - 1");
  int shift = 0;
  while ((1 << shift) < t->page_size) ++shift;
  *view = {t->table, t->refs, t->ld, (int)t->sequences, (int)t->columns, (int)t->pages, shift};
  return AF1_OK;
}

int check_table_pointers(const char* who, const TableView& t, int* dev) {
  int rc = current_device(who, dev);
  if (rc == AF1_OK) rc = check_words(t.table, "table", *dev);
  if (rc == AF1_OK) rc = check_words(t.refs, "refs", *dev);
  return rc;
}

int64_t reserve_bytes(const TableView& t) { return std::max<int64_t>(256, 8 * (int64_t)t.seqs * t.columns); }

}  // namespace
}  // namespace af1

using namespace af1;

int af1_kv_compact(const af1_kv_cache* const* caches, int64_t count, const int32_t* pages, int64_t sequences,
                   int64_t page_columns, int64_t pages_ld, const int32_t* first, const int32_t* index, int64_t nodes,
                   const int32_t* counts, void* stream) {
  const char* who = "af1_kv_compact";
  int dev, rc;
  if (nodes < 1 || nodes > kMaxNodes || sequences < 0 || sequences > 65536)
    return fail(AF1_ERR_INVALID_ARG, who, "need 1..64 nodes and 0..65536 sequences");
  if ((rc = check_caches(who, caches, count, &dev)) != AF1_OK) return rc;
  if (sequences == 0) return AF1_OK;
  if (page_columns < 1 || page_columns > ((int64_t)1 << 31) / caches[0]->d.page_size - 1 || pages_ld < page_columns ||
      pages_ld > ((int64_t)1 << 60) / sequences)
    return fail(AF1_ERR_INVALID_ARG, who, "need page columns of fewer than 2^31 slots in all, pages_ld >= page_columns");
  if ((rc = check_words(pages, "pages", dev)) != AF1_OK || (rc = check_words(first, "first", dev)) != AF1_OK ||
      (rc = check_words(index, "index", dev)) != AF1_OK || (rc = check_words(counts, "counts", dev)) != AF1_OK)
    return rc;
  const CompactProblem p = {{pages, pages_ld, (int)sequences, (int)page_columns}, first, index, counts, (int)nodes};
  return in_parts(who, caches, count, [&](const Caches& some, int n, int heads) {
    const int64_t units = 2 * sequences * heads;  // at most 2^27
    compact_kernel<<<dim3((unsigned)((units + kMoveWarps - 1) / kMoveWarps), n), 32 * kMoveWarps, 0,
                     static_cast<cudaStream_t>(stream)>>>(some, p);
  });
}

int af1_kv_copy(const af1_kv_cache* const* caches, int64_t count, const int32_t* copies, int64_t entries, void* stream) {
  const char* who = "af1_kv_copy";
  int dev, rc;
  if (entries < 0 || entries > (1 << 20)) return fail(AF1_ERR_INVALID_ARG, who, "need 0..2^20 entries");
  if ((rc = check_caches(who, caches, count, &dev)) != AF1_OK) return rc;
  if (entries == 0) return AF1_OK;
  if ((rc = check_words(copies, "copies", dev)) != AF1_OK) return rc;
  return in_parts(who, caches, count, [&](const Caches& some, int n, int heads) {
    copy_kernel<<<dim3((unsigned)entries, n, 2 * heads), kCopyThreads, 0, static_cast<cudaStream_t>(stream)>>>(some, copies);
  });
}

int af1_pages_fork(const af1_page_table* table, const int32_t* parents, void* stream) {
  const char* who = "af1_pages_fork";
  TableView t;
  int dev, rc;
  if ((rc = check_table(who, table, &t)) != AF1_OK) return rc;
  if (t.seqs == 0) return AF1_OK;
  if ((rc = check_table_pointers(who, t, &dev)) != AF1_OK || (rc = check_words(parents, "parents", dev)) != AF1_OK) return rc;
  fork_kernel<<<(t.columns + kForkColumns - 1) / kForkColumns, kForkThreads, 0, static_cast<cudaStream_t>(stream)>>>(t, parents);
  return launched(who);
}

int64_t af1_pages_workspace_bytes(const af1_page_table* table) {
  TableView t;
  const int rc = check_table("af1_pages_workspace_bytes", table, &t);
  if (rc != AF1_OK) return rc;
  set_error(AF1_OK, "");
  return reserve_bytes(t);
}

int af1_pages_reserve(const af1_page_table* table, const int32_t* first, const int32_t* counts, int32_t* copies,
                      int32_t* lacking, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "af1_pages_reserve";
  TableView t;
  int dev, rc;
  if ((rc = check_table(who, table, &t)) != AF1_OK) return rc;
  if (t.seqs > 0 && (workspace == nullptr || (uintptr_t)workspace % 256 != 0 || workspace_bytes < reserve_bytes(t)))
    return fail(AF1_ERR_WORKSPACE, who, "need a 256-byte aligned workspace of af1_pages_workspace_bytes bytes");
  if ((rc = current_device(who, &dev)) != AF1_OK || (rc = check_words(lacking, "lacking", dev)) != AF1_OK) return rc;
  if (t.seqs > 0 &&
      ((rc = check_table_pointers(who, t, &dev)) != AF1_OK || (rc = check_words(first, "first", dev)) != AF1_OK ||
       (rc = check_words(counts, "counts", dev)) != AF1_OK || (rc = check_words(copies, "copies", dev)) != AF1_OK ||
       (rc = check_pointer(workspace, "workspace", dev)) != AF1_OK))
    return rc;
  int32_t* notes = static_cast<int32_t*>(workspace);
  reserve_kernel<<<1, kReserveThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      t, first, counts, copies, lacking, notes, notes + (int64_t)t.seqs * t.columns);
  return launched(who);
}

int af1_pages_release(const af1_page_table* table, const int32_t* lens, void* stream) {
  const char* who = "af1_pages_release";
  TableView t;
  int dev, rc;
  if ((rc = check_table(who, table, &t)) != AF1_OK) return rc;
  if (t.seqs == 0) return AF1_OK;
  if ((rc = check_table_pointers(who, t, &dev)) != AF1_OK || (rc = check_words(lens, "lens", dev)) != AF1_OK) return rc;
  release_kernel<<<dim3((t.columns + kReleaseThreads - 1) / kReleaseThreads, t.seqs), kReleaseThreads, 0,
                   static_cast<cudaStream_t>(stream)>>>(t, lens);
  return launched(who);
}
