// Host side shared by the layers' entry points (dense.hip, norm.hip, dropout.hip): argument
// checks, workspaces.
#pragma once

#include <vector>

#include "common.h"

namespace ot {

inline int check_rows(const void* p, int64_t ld, int64_t rows, int64_t len, int elem, const char* what,
                      const char* name) {
  OT_REQUIRE(p != nullptr, "%s: NULL %s", what, name);
  OT_REQUIRE(reinterpret_cast<uintptr_t>(p) % 16 == 0, "%s: %s is not 16-byte aligned", what, name);
  OT_REQUIRE(rows <= 1 || (ld >= len && ld % (16 / elem) == 0),
             "%s: leading dimension %lld of %s is not a multiple of %d of at least %lld", what, (long long)ld, name,
             16 / elem, (long long)len);
  return OT_OK;
}

inline int check_values(const void* p, int align, const char* what, const char* name) {
  OT_REQUIRE(reinterpret_cast<uintptr_t>(p) % align == 0, "%s: %s is not aligned to its elements", what, name);
  return OT_OK;
}

inline int check_device(int device, const char* what) {
  int now = -1;
  OT_HIP(hipGetDevice(&now));
  if (now != device)
    return set_error(OT_E_STATE, "%s: device %d is current, the object lives on %d", what, now, device);
  return OT_OK;
}

// Device memory of an object for calls of up to `rows` rows (or samples).
struct Workspace {
  unsigned char* p = nullptr;
  int64_t rows = 0, size = 0;               // size: bytes at p
  bool captured = false;                    // a captured call may name p
  std::vector<unsigned char*> kept;         // replaced after such a call

  int allocate(int64_t n, int64_t bytes, const char* what) {
    unsigned char* q = nullptr;
    if (bytes > 0) {
      const hipError_t e = hipMalloc(reinterpret_cast<void**>(&q), (size_t)bytes);
      if (e != hipSuccess) {
        (void)hipGetLastError();
        return set_error(OT_E_NOMEM, "%s: hipMalloc of %lld bytes failed: %s", what, (long long)bytes,
                         hipGetErrorString(e));
      }
    }
    if (p) {
      if (captured) {
        kept.push_back(p);                  // (reserved before: cannot throw)
        captured = false;
      } else {
        (void)hipFree(p);                   // waits for the device
      }
    }
    p = q;
    rows = n;
    size = bytes;
    return OT_OK;
  }
  // Before a call of n rows that uses the workspace: bytes(n), what calls of up to n rows need, is allocated where
  // there is less, unless the stream is under capture.
  template <class Bytes>
  int begin(int64_t n, hipStream_t st, const char* what, Bytes bytes) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    OT_HIP(hipStreamIsCapturing(st, &cap));
    if (n > rows) {
      const int64_t need = bytes(n);
      if (need <= size) {
        rows = n;
      } else {
        if (cap != hipStreamCaptureStatusNone)
          return set_error(OT_E_STATE, "%s: a call of %lld under capture, workspaces hold %lld", what, (long long)n,
                           (long long)rows);
        kept.reserve(kept.size() + 1);
        const int rc = allocate(n, need, what);
        if (rc) return rc;
      }
    }
    if (cap != hipStreamCaptureStatusNone) captured = true;
    return OT_OK;
  }
  void release() {
    if (p) (void)hipFree(p);                // waits for the device
    for (unsigned char* q : kept) (void)hipFree(q);
  }
};

}  // namespace ot
