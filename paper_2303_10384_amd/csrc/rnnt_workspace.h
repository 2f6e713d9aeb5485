// A call's workspace: the caller's, or one taken for the call, stream-ordered.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "rnnt_mi355x.h"

namespace rnnt {

// None is taken on a stream under capture: a graph of several calls, each with an allocation and a free of its
// own, has faulted when it was replayed, and the cause is not known, so a captured call brings its workspace.
struct Workspace {
  char* ptr = nullptr;

  Workspace() = default;
  Workspace(const Workspace&) = delete;
  Workspace& operator=(const Workspace&) = delete;
  ~Workspace() {
    if (owned_) (void)hipFreeAsync(owned_, stream_);
  }
  rnnt_status_t take(void* given, size_t given_bytes, size_t need, hipStream_t stream) {
    if (given && given_bytes < need) return RNNT_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(given) % 256 != 0) return RNNT_ERR_ALIGNMENT;
    ptr = static_cast<char*>(given);
    if (ptr || need == 0) return RNNT_OK;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &capture) != hipSuccess) return failed();
    if (capture != hipStreamCaptureStatusNone) return RNNT_ERR_WORKSPACE;
    if (hipMallocAsync(&owned_, need, stream) != hipSuccess) {
      owned_ = nullptr;
      return failed();
    }
    stream_ = stream;
    ptr = static_cast<char*>(owned_);
    return RNNT_OK;
  }

 private:
  // the error is this call's status: it is not left for the check behind the next launch to find
  static rnnt_status_t failed() {
    (void)hipGetLastError();
    return RNNT_ERR_HIP;
  }

  void* owned_ = nullptr;
  hipStream_t stream_ = nullptr;
};

}  // namespace rnnt
