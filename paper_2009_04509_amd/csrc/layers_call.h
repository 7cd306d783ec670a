// What the entry points over matrices share: their handle, argument checks, scratch and
// launches with their timer.
#pragma once

#include <cstring>
#include <exception>
#include <new>
#include <string>

#include "call.h"
#include "internal.h"

struct pointid_layers_s {
  int device;
  int cus;
  pointid::ScratchPool scratch;
};

namespace pointid {

constexpr int64_t kMaxRows = int64_t(1) << 28;         // m (a launch has fewer than 2^32 threads)

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int size_of(int dtype) { return dtype == POINTID_FP32 ? 4 : 2; }

// No exception crosses the ABI.
template <class F>
int guarded(F&& f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return POINTID_ENOMEM;
  } catch (...) {
    return POINTID_EHIP;
  }
}

// Leaves the calling function with a status that is not OK.
#define TRY(call)                            \
  do {                                       \
    const int rc_ = (call);                  \
    if (rc_ != POINTID_OK) return rc_;       \
  } while (0)

// ---- argument checks

// A matrix of the call; `may_miss`: NULL (or NULL data) is allowed.
inline int check_matrix(const pointid_matrix* a, const char* name, int dtype, int64_t rows, int64_t cols, bool may_miss = false) {
  if (!a || !a->data) {
    if (may_miss || rows == 0) return POINTID_OK;
    return set_error(POINTID_EINVAL, std::string(name) + " is NULL");
  }
  if (reinterpret_cast<uintptr_t>(a->data) % size_of(dtype))
    return set_error(POINTID_EINVAL, std::string(name) + " is not aligned to its elements");
  if (rows > 1 && a->ld < cols)
    return set_error(POINTID_EINVAL, std::string(name) + ": row pitch below its columns");
  if (rows > 1 && a->ld > INT64_MAX / 8 / rows)
    return set_error(POINTID_EINVAL, std::string(name) + ": row pitch out of range");
  return POINTID_OK;
}

inline int check_floats(const float* p, const char* name) {
  if (p && reinterpret_cast<uintptr_t>(p) % 4)
    return set_error(POINTID_EINVAL, std::string(name) + " is not aligned to its elements");
  return POINTID_OK;
}

// The pitch of one row is never used: any value stands for its columns.
inline pointid_matrix matrix_of(const pointid_matrix* a, int64_t rows, int64_t cols) {
  pointid_matrix r = {nullptr, cols};
  if (a && a->data) r = *a;
  if (rows <= 1 || !r.data) r.ld = round_up(cols, 8);
  return r;
}

// ---- a call: scratch pieces sized before any is taken, launches with their timer

class Call {
 public:
  Call(pointid_layers l, hipStream_t stream) : ws_(&l->scratch, stream), stream_(stream) {}
  // scratch: the caller's, of `bytes`, or NULL for the handle's
  Call(pointid_layers l, hipStream_t stream, void* scratch, uint64_t bytes)
      : ws_(scratch ? Workspace(scratch, (size_t)bytes) : Workspace(&l->scratch, stream)), stream_(stream),
        own_(!scratch) {}

  // a piece of the call's scratch, taken by reserve()
  template <class T>
  void want(T** out, size_t bytes) {
    if (count_ < kMaxPieces) pieces_[count_++] = {reinterpret_cast<void**>(out), bytes};
  }
  int reserve() {
    size_t total = 0;
    for (int i = 0; i < count_; ++i) total += pad256(pieces_[i].bytes);
    if (total == 0) return POINTID_OK;
    // a graph would use the buffer again whenever it is replayed, past the cache's care
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (own_ && hipStreamIsCapturing(stream_, &capture) == hipSuccess && capture != hipStreamCaptureStatusNone)
      return set_error(POINTID_EINVAL, "the call takes scratch, which a captured stream cannot");
    hipError_t e = ws_.reserve(total);
    if (e != hipSuccess && !own_) return set_error(POINTID_EINVAL, "the call's scratch is too small");
    if (e != hipSuccess) return hip_fail(e, "scratch buffer");
    for (int i = 0; i < count_; ++i) {
      e = ws_.get(pieces_[i].bytes, pieces_[i].out);
      if (e != hipSuccess) return hip_fail(e, "workspace (layers)");
    }
    scratch_ = own_;
    return POINTID_OK;
  }
  // f: the launch; `last`: of the call (it also records the scratch's completion)
  template <class F>
  int run(const char* name, bool last, F&& f) {
    KernelTimer kt(name, stream_);
    hipError_t e;
    if (last && scratch_) {
      EndsCall end(ws_);
      e = f();
      end.launched(e);
    } else {
      e = f();
    }
    return e == hipSuccess ? POINTID_OK : hip_fail(e, name);
  }
  hipStream_t stream() const { return stream_; }

 private:
  static constexpr int kMaxPieces = 16;
  struct Piece {
    void** out;
    size_t bytes;
  };
  Workspace ws_;
  hipStream_t stream_;
  Piece pieces_[kMaxPieces];
  int count_ = 0;
  bool own_ = true;
  bool scratch_ = false;
};

}  // namespace pointid
