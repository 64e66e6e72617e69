// What the entry points of the operators share: argument checks on the host.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "slice_handle.h"

namespace ema {

inline int inval(const char* what, const char* why) {
  return set_error(EMA_ERR_INVAL, std::string(what) + ": " + why);
}

inline int32_t log2_of(int32_t x) {   // of a power of two
  int32_t s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The host's view of a device array in checked mode, or the caller's own array on
// a host-only handle.
class HostInts {
 public:
  int get(const ema_slice* h, const int32_t* p, int64_t n, hipStream_t st) {
    if (h->host_only) {
      data_ = p;
      return EMA_OK;
    }
    const int rc = fetch_ints(p, n, st, &copy_);
    data_ = copy_.data();
    return rc;
  }
  int32_t operator[](int64_t i) const { return data_[i]; }

 private:
  const int32_t* data_ = nullptr;
  std::vector<int32_t> copy_;
};

// Whether the call's arrays are to be validated on the host; a stream that
// captures cannot be read back from.
inline int must_check(const ema_slice* h, hipStream_t st, const char* what, bool* yes) {
  *yes = h->host_only || h->checked;
  if (h->host_only || !h->checked) return EMA_OK;
  bool capturing = false;
  if (int rc = is_capturing(st, &capturing)) return rc;
  return capturing ? inval(what, "a checked handle cannot read its arrays back during stream "
                                 "capture")
                   : EMA_OK;
}

}  // namespace ema
