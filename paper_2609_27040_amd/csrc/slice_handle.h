// The handle behind ema_slice_t and what every file of entry points needs of it.
#pragma once

#include "ema_slice.h"

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <vector>

#include "kernels.h"
#include "slice_book.h"

// Readers of the slab lists that may be under way without waiting for each other.
constexpr uint32_t kSlabUses = 8;

struct ema_slice {
  ema_kv_shape shape{};
  int64_t bb = 0;
  bool host_only = false;
  bool checked = false;
  int device = -1;
  ema::SliceBook book;
  char* local = nullptr;
  char* slice = nullptr;
  int32_t* d_err = nullptr;
  int32_t* d_work = nullptr;
  size_t work_cap = 0;          // ints
  int32_t* h_work = nullptr;    // pinned
  size_t h_work_cap = 0;        // ints
  hipEvent_t h_work_ev = nullptr;   // after the last upload from h_work
  bool h_work_pending = false;
  hipEvent_t d_work_ev = nullptr;   // after the last kernel that read d_work
  bool d_work_pending = false;
  float* d_part = nullptr;          // stream-K partial slots (fixed size)
  size_t part_cap = 0;              // floats
  int32_t* d_info = nullptr;        // stream-K: two ints per workgroup
  size_t info_cap = 0;              // ints
  float* d_gpart = nullptr;         // grid form: split-K partials (grows)
  size_t gpart_cap = 0;             // floats
  bool attn_grid = false;           // EMA_CREATE_ATTN_GRID: always the grid form
  void* noalloc_ws = nullptr;       // this device's fixed workspace (not owned)
  // slab mode: every layer group's swap sources (staging order), on the device
  int32_t* d_slab = nullptr;
  int32_t* h_slab = nullptr;        // pinned
  size_t slab_cap = 0;              // ints
  int64_t slab_built = -1;          // slab version the device lists were built for
  hipEvent_t slab_up_ev = nullptr;  // after the last upload of the lists
  bool slab_up_pending = false;     // not yet waited for on the host
  bool slab_up_recorded = false;    // the event stands for the lists' upload
  hipEvent_t slab_use_ev[kSlabUses] = {};   // after the last kernels that read them
  uint32_t slab_uses = 0;           // how many have been launched
};

namespace ema {

// Records the message behind an error code for ema_last_error.
int set_error(int code, const std::string& msg);

// Called from the catch handler of every entry point: no C++ exception
// crosses the C ABI; host allocation failures become EMA_ERR_NOMEM.
int internal_error();

int hip_error(hipError_t e, const char* what);

#define HIP_TRY(call, what)                    \
  do {                                         \
    hipError_t e_ = (call);                    \
    if (e_ != hipSuccess) return ema::hip_error(e_, what); \
  } while (0)

PoolView pool_view(const ema_slice* h);

// Makes the handle's device current for the rest of an entry point and puts
// the caller's device back when the entry point returns.
class DeviceScope {
 public:
  DeviceScope() = default;
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  ~DeviceScope() {
    if (prev_ >= 0) (void)hipSetDevice(prev_);
  }
  int enter(const ema_slice* h) {
    int cur = -1;
    HIP_TRY(hipGetDevice(&cur), "hipGetDevice");
    if (cur != h->device) {
      HIP_TRY(hipSetDevice(h->device), "hipSetDevice");
      prev_ = cur;
    }
    return EMA_OK;
  }

 private:
  int prev_ = -1;
};

// Reads n ints of a device array to the host (checked mode).
int fetch_ints(const int32_t* dev, int64_t n, hipStream_t st, std::vector<int32_t>* out);

int is_capturing(hipStream_t st, bool* yes);

}  // namespace ema
