// af1_kv.cuh — the paged cache as the kernels see it, and the checks that
// the entry points of the step around the linears share.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <string>

#include "af1.h"

struct af1_kv_cache {
  af1_kv_desc d;
  int device = 0;
  int num_sms = 0;
  // Tensor maps of k and v as rows of codes, in boxes of a page's rows up to
  // those of a warp's step (af1_tree.cu), and of a tile (af1_tree_wide.cu).
  CUtensorMap k_step, v_step, k_tile, v_tile;
};

namespace af1 {

// Rows (one vector of one head in one slot) are numbered
// (page * kv_heads + head) * page_size + slot % page_size.
struct KvView {
  uint8_t *k, *v;
  void *ks, *vs;
  int pages, heads, shift;  // page_size = 1 << shift
};
struct PageTable {
  const int32_t* pages;
  int64_t ld;
  int seqs, columns;
};

// Bytes of a row of codes, and of its scales.
static __host__ __device__ constexpr int kv_row_bytes(int kind, int dim) {
  return kind == AF1_KV_F16 ? 2 * dim : kind == AF1_KV_INT4 ? dim / 2 : dim;
}
static __host__ __device__ constexpr int kv_scale_bytes(int kind, int dim) {
  return kind == AF1_KV_F16 ? 0 : kind == AF1_KV_INT4 ? dim / 8 : 4;
}

// The first row of `head` in the page of `slot`, plus slot % page_size; -1
// where the slot is not in the table or its page not in the cache.
static __device__ __forceinline__ int64_t kv_row(const KvView& c, const PageTable& t, int seq, int slot, int head) {
  const int col = slot >> c.shift;
  if (slot < 0 || col >= t.columns || seq < 0 || seq >= t.seqs) return -1;
  const int page = t.pages[seq * t.ld + col];
  if (page < 0 || page >= c.pages) return -1;
  return (((int64_t)page * c.heads + head) << c.shift) + (slot & ((1 << c.shift) - 1));
}

// Host: a device pointer of the current device; AF1_OK or an error that is
// set. nullptr is INVALID_ARG.
int check_pointer(const void* p, const char* name, int device);
int check_align(const void* p, int bytes, const char* name);
KvView view_of(const af1_kv_desc& d);
// Sets a kernel's attributes once for each device (setting them takes longer than a launch): `done` has a bit for each
// of the first 64, set by the first call that succeeds. They are the same for every call, so that threads may race.
template <typename F>
cudaError_t once_per_device(std::atomic<uint64_t>& done, F&& set) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (e != cudaSuccess || (done.load(std::memory_order_acquire) & bit) != 0) return e;
  e = set();
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

}  // namespace af1
