// What every part of the library's host side shares: the handle, its errors and its device memory, pinned blocks for
// numbers that kernels leave for the host.
#pragma once
#include "../../include/spgemm.h"

#include <hip/hip_runtime.h>

#include <cstring>
#include <mutex>
#include <string>
#include <vector>

#include "common.hpp"

struct TimedLaunch {
  int cls;
  hipEvent_t start, stop;
};

struct spgemm_context {
  hipStream_t stream = nullptr;
  spgemm_allocator alloc{};
  bool has_alloc = false;
  int timing = 0;
  int force = 0;
  int direct_min = spg::kDirectMinDefault;
  int64_t col_list = 1;   // 0 off, 1 automatic size, larger: byte limit
  int block_table = 1;    // 0: never build the block-offset table of B (pieces are bisected)
  int64_t merge_limit = 0xffffffffLL;   // components of the outer product's all array and a batch together: fewer
  int search_ratio = 4;   // searched tiles for rows with at most this many products per entry (0: never)
  int row_block = 0;      // 1: A is a block of rows of a larger matrix (row pointer values are that matrix's positions)
  double whole_ip = 0;    // ... and the products of all its rows
  std::string err = "";
  bool device_ready = false;
  bool big_lds_ready = false;
  int num_cus = 0;
  std::vector<TimedLaunch> timed;        // launches of the phase in flight
  std::vector<hipEvent_t> event_pool;
  hipStream_t second = nullptr;   // of spgemm_pipelined, and the device it is on: made when first wanted, released with the handle
  int second_device = -1;
  void* work = nullptr;           // scratch memory of the attention and cache calls, of the largest one so far
  size_t work_bytes = 0;
  bool work_captured = false;     // a graph has it in its nodes
  std::vector<void*> outgrown;    // blocks that graphs still have, after a larger call: released with the handle
};

namespace spg {

// Pinned host memory where kernels leave numbers for the host (the symbolic ones the control block).  Allocating and releasing it costs 50 to
// 300 us, so a few blocks wait for the next calls; a call holds its own from before its first kernel until its stream has been
// waited for, whatever handle, stream or thread it comes from: the lease itself waits where the call returns before it has (an
// allocation that is refused while kernels are on their way).
class PinnedBlocks {
 public:
  Control* take() {
    {
      std::lock_guard<std::mutex> lock(mutex_);
      if (n_ > 0) return free_[--n_];
    }
    void* p = nullptr;
    if (hipHostMalloc(&p, sizeof(Control), hipHostMallocPortable) == hipSuccess) return static_cast<Control*>(p);
    (void)hipGetLastError();
    return nullptr;
  }
  void give(Control* p) {
    {
      std::lock_guard<std::mutex> lock(mutex_);
      if (n_ < kKeep) { free_[n_++] = p; return; }
    }
    (void)hipHostFree(p);
  }

 private:
  static constexpr int kKeep = 16;
  std::mutex mutex_;
  Control* free_[kKeep] = {};
  int n_ = 0;
};
inline PinnedBlocks g_pinned;

struct PinnedLease {
  Control* p;
  explicit PinnedLease(hipStream_t stream) : p(g_pinned.take()), stream_(stream) {}
  ~PinnedLease() {
    if (!p) return;
    if (written_) (void)hipStreamSynchronize(stream_);
    g_pinned.give(p);
  }
  void written() { written_ = true; }   // kernels that write to the block are about to be launched
  void waited() { written_ = false; }   // and all of them are done
  PinnedLease(const PinnedLease&) = delete;
  PinnedLease& operator=(const PinnedLease&) = delete;

 private:
  hipStream_t stream_;
  bool written_ = false;
};

inline int fail(spgemm_context* h, int code, const std::string& msg) {
  if (h) h->err = msg;
  return code;
}

#define HIP_TRY(h, expr)                                                                 \
  do {                                                                                   \
    hipError_t e_ = (expr);                                                              \
    if (e_ != hipSuccess)                                                                \
      return fail((h), SPGEMM_HIP_ERROR, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

inline void* dev_alloc(spgemm_context* h, size_t bytes) {
  if (bytes == 0) bytes = 256;
  if (h->has_alloc) return h->alloc.alloc(h->alloc.ctx, bytes);
  void* p = nullptr;
  if (hipMalloc(&p, bytes) == hipSuccess) return p;
  (void)hipGetLastError();   // (the thread's last error stays until it is asked for: a call that goes on without would find it behind its kernels)
  return nullptr;
}

inline void dev_free(spgemm_context* h, void* p) {
  if (!p) return;
  if (h->has_alloc) h->alloc.free(h->alloc.ctx, p);
  else (void)hipFree(p);
}

template <typename K>
int allow_lds(spgemm_context* h, K kernel, size_t bytes) {
  HIP_TRY(h, hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  return SPGEMM_OK;
}

inline int ensure_device(spgemm_context* h) {
  if (h->device_ready) return SPGEMM_OK;
  int dev = 0;
  HIP_TRY(h, hipGetDevice(&dev));
  hipDeviceProp_t prop;
  HIP_TRY(h, hipGetDeviceProperties(&prop, dev));
  if (prop.warpSize != kWave) return fail(h, SPGEMM_UNSUPPORTED, "device is not wave64");
  h->num_cus = prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
  h->device_ready = true;
  return SPGEMM_OK;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace spg
