// What every call of the C ABI shares: error text, the device of a call, kernel
// timing, and device scratch from a cache that lives with a handle.
#pragma once

#include <atomic>
#include <map>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "internal.h"

namespace pointid {

// Error text of a failed HIP call (this thread); returns the status code for it.
int hip_fail(hipError_t e, const char* what);

// Per-handle cache of device scratch buffers, reused across calls.  A call
// takes one buffer big enough for all its scratch and records an event on its
// stream after enqueueing its work; the next user of the buffer either runs on
// the same stream (stream order protects it) or finds that event complete, and
// only when neither is possible waits for it on its own stream.  Buffers are
// allocated only when no free one fits, so steady-state calls allocate nothing.
struct ScratchPool {
  struct Entry {
    void* ptr = nullptr;
    size_t bytes = 0;
    hipEvent_t done = nullptr;     // recorded after the last user's work
    hipStream_t last = nullptr;    // stream of the last user
    bool used = false;             // `done` has been recorded
    bool busy = false;             // taken by a call being enqueued
  };
  std::mutex mu;
  std::vector<Entry> entries;
};

// Makes `dev` current for the scope of a call and restores the caller's device.
class DeviceScope {
 public:
  explicit DeviceScope(int dev) {
    if (hipGetDevice(&old_) != hipSuccess) old_ = -1;
    if (old_ != dev) err_ = hipSetDevice(dev);
  }
  ~DeviceScope() {
    if (old_ >= 0 && err_ == hipSuccess) (void)hipSetDevice(old_);
  }
  hipError_t error() const { return err_; }

 private:
  int old_ = -1;
  hipError_t err_ = hipSuccess;
};

// ---- optional per-kernel timing (pointid_timing_*)
//
// The timed kernels of one call form a chain on its stream: the first is timed
// from an event recorded on the stream just before it, and every kernel
// carries a stop event on its own dispatch (hipExtLaunchKernel); a kernel's
// time runs from the end of the one before it (or that first event) to its
// own end, the launch gap in between charged to it.  A stop event on a
// dispatch adds nothing to the stream; a recorded event leaves a gap of about
// 3.5 us (one per call), and a start event on the dispatch about 5 us and
// 10-20 us of host time.
// Events are reference counted: a record holds its two, and the chain holds
// its last stop event until the next kernel has taken it as its start.
struct TimingRec {
  const char* name;
  hipEvent_t a, b;
};
struct Timing {
  std::atomic<bool> on{false};
  std::mutex mu;
  std::vector<TimingRec> pending;
  std::map<std::string, std::pair<double, int64_t>> total;
  std::map<hipEvent_t, int> refs;
  // with mu held
  void hold(hipEvent_t e) { ++refs[e]; }
  void release(hipEvent_t e) {
    auto it = refs.find(e);
    if (it == refs.end() || --it->second > 0) return;
    refs.erase(it);
    (void)hipEventDestroy(e);
  }
};
Timing& timing();                 // the library's

// The calling thread's chain; a call's workspace opens it (nested workspaces
// share it).
struct TimingChain {
  int depth = 0;
  hipStream_t stream = nullptr;
  hipEvent_t last = nullptr;                 // held by the chain
};
TimingChain& timing_chain();
class ChainScope {
 public:
  ChainScope() { ++timing_chain().depth; }
  ~ChainScope() {
    TimingChain& c = timing_chain();
    if (--c.depth > 0 || !c.last) return;
    std::lock_guard<std::mutex> g(timing().mu);
    timing().release(c.last);
    c.last = nullptr;
  }
};

// Times the one launch in its scope while timing is enabled.
class KernelTimer {
 public:
  KernelTimer(const char* name, hipStream_t s) : name_(name), s_(s) {
    Timing& T = timing();
    if (!T.on.load(std::memory_order_relaxed)) return;
    if (hipEventCreate(&b_) != hipSuccess) return;
    TimingChain& c = timing_chain();
    std::lock_guard<std::mutex> g(T.mu);
    if (c.depth > 0 && c.last && c.stream == s) {
      a_ = c.last;                           // the previous kernel's end
    } else if (hipEventCreate(&a_) != hipSuccess) {
      (void)hipEventDestroy(b_);
      return;
    } else if (hipEventRecord(a_, s) != hipSuccess) {
      (void)hipEventDestroy(a_);
      (void)hipEventDestroy(b_);
      return;
    }
    T.hold(a_);
    T.hold(b_);
    LaunchEvents& ev = launch_events();
    ev.start = nullptr;
    ev.stop = b_;
    active_ = true;
  }
  ~KernelTimer() {
    if (!active_) return;
    LaunchEvents& ev = launch_events();
    const bool launched = ev.stop == nullptr;   // the launch took the events
    ev = LaunchEvents();
    Timing& T = timing();
    std::lock_guard<std::mutex> g(T.mu);
    if (!launched) {                         // nothing was launched (an empty call)
      T.release(a_);
      T.release(b_);
      return;
    }
    TimingChain& c = timing_chain();
    if (c.depth > 0) {
      if (c.last) T.release(c.last);
      c.last = b_;
      c.stream = s_;
      T.hold(b_);
    }
    T.pending.push_back({name_, a_, b_});
  }

 private:
  const char* name_;
  hipStream_t s_;
  hipEvent_t a_{}, b_{};
  bool active_ = false;
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr size_t kScratchAlign = 256;
constexpr size_t kMaxScratchBuffers = 512;
inline size_t pad256(size_t b) { return (b + kScratchAlign - 1) / kScratchAlign * kScratchAlign; }

// One call's scratch: a buffer of the handle's ScratchPool, handed back (with
// its event recorded on the call's stream) when the scope ends.
class Workspace {
 public:
  Workspace(ScratchPool* pool, hipStream_t s) : pool_(pool), s_(s) {}
  // A caller-provided buffer of `cap` bytes instead of the pool: reserve only
  // checks the size, and nothing is allocated or recorded.
  Workspace(void* base, size_t cap) : pool_(nullptr), s_(nullptr) {
    fixed_ = true;
    base_ = static_cast<char*>(base);
    cap_ = cap;
  }
  ~Workspace() {
    if (idx_ < 0) return;
    hipError_t e = recorded_ ? hipSuccess : hipEventRecord(done_, s_);
    // without the event, the next user could not tell when this call's work
    // is done: wait for it here (an error path only)
    if (e != hipSuccess) (void)hipStreamSynchronize(s_);
    std::lock_guard<std::mutex> g(pool_->mu);
    ScratchPool::Entry& en = pool_->entries[idx_];
    en.busy = false;
    en.last = s_;
    en.used = (e == hipSuccess);
  }

  // Takes a buffer of at least `bytes` for this call.
  hipError_t reserve(size_t bytes) {
    if (fixed_) return bytes <= cap_ ? hipSuccess : hipErrorInvalidValue;
    std::unique_lock<std::mutex> g(pool_->mu);
    std::vector<ScratchPool::Entry>& v = pool_->entries;
    int same = -1, ready = -1, any = -1;
    for (int i = 0; i < (int)v.size(); ++i) {
      const ScratchPool::Entry& en = v[i];
      if (en.busy || !en.ptr || en.bytes < bytes) continue;   // (empty slots are skipped)
      if (en.last == s_ || !en.used) {
        if (same < 0 || en.bytes < v[same].bytes) same = i;
      } else if (hipEventQuery(en.done) == hipSuccess) {
        if (ready < 0 || en.bytes < v[ready].bytes) ready = i;
      } else if (any < 0 || en.bytes < v[any].bytes) {
        any = i;
      }
    }
    int pick = same >= 0 ? same : ready;
    if (pick < 0 && (v.size() >= kMaxScratchBuffers)) pick = any;
    if (pick >= 0) {
      take(pick);
      const bool wait = v[pick].used && v[pick].last != s_ && pick != ready;
      g.unlock();
      return wait ? hipStreamWaitEvent(s_, done_, 0) : hipSuccess;
    }
    // a new buffer, sized to the next power of two (at least 4 MiB) so that
    // requests of varying size share buffers; past 1 GiB to the next 256 MiB,
    // so that a very large call does not reserve up to twice its need.  It
    // takes the slot of a buffer pointid_trim freed, if there is one.
    int slot = -1;
    for (int i = 0; i < (int)v.size() && slot < 0; ++i)
      if (!v[i].ptr && !v[i].busy) slot = i;
    if (slot < 0) {
      v.emplace_back();
      slot = (int)v.size() - 1;
    }
    v[slot] = ScratchPool::Entry();
    v[slot].busy = true;
    g.unlock();
    size_t cap = size_t(4) << 20;
    while (cap < bytes && cap < (size_t(1) << 30)) cap <<= 1;
    if (cap < bytes) cap = (bytes + (size_t(256) << 20) - 1) & ~((size_t(256) << 20) - 1);
    void* p = nullptr;
    hipEvent_t ev = nullptr;
    hipError_t e = hipEventCreateWithFlags(&ev, hipEventDisableTiming);
    if (e == hipSuccess) e = hipMalloc(&p, cap);
    g.lock();
    if (e != hipSuccess) {
      if (ev) (void)hipEventDestroy(ev);
      v[slot] = ScratchPool::Entry();            // empty, free: skipped by later calls
      return e;
    }
    v[slot].ptr = p;
    v[slot].bytes = cap;
    v[slot].done = ev;
    take(slot);
    return hipSuccess;
  }

  // Lets the calling thread's next launch record the completion event at the
  // end of its kernel (no packet of its own on the stream); false for a
  // caller's buffer, which has no event.
  bool attach_done() {
    if (fixed_ || idx_ < 0) return false;
    LaunchEvents& ev = launch_events();
    if (ev.stop) return false;
    ev.stop = done_;
    return true;
  }
  void mark_recorded() { recorded_ = true; }

  // Carves the next piece (256-byte aligned) out of the reserved buffer.
  hipError_t get(size_t bytes, void** out) {
    *out = nullptr;
    if (bytes == 0) return hipSuccess;
    if ((idx_ < 0 && !fixed_) || used_ + pad256(bytes) > cap_) return hipErrorInvalidValue;
    *out = base_ + used_;
    used_ += pad256(bytes);
    return hipSuccess;
  }

 private:
  void take(int i) {                           // with pool_->mu held
    ScratchPool::Entry& en = pool_->entries[i];
    en.busy = true;
    idx_ = i;
    base_ = static_cast<char*>(en.ptr);
    cap_ = en.bytes;
    done_ = en.done;
  }

  ChainScope chain_;                           // the call's timed kernels
  ScratchPool* pool_;
  hipStream_t s_;
  bool fixed_ = false;
  bool recorded_ = false;
  int idx_ = -1;
  char* base_ = nullptr;
  size_t cap_ = 0, used_ = 0;
  hipEvent_t done_ = nullptr;
};

// Scope of a call's last launch: the launch also records the workspace's
// completion event.
class EndsCall {
 public:
  explicit EndsCall(Workspace& ws) : ws_(ws), on_(ws.attach_done()) {}
  ~EndsCall() {
    if (on_) launch_events().stop = nullptr;
  }
  void launched(hipError_t e) {
    if (on_ && e == hipSuccess && launch_events().stop == nullptr) ws_.mark_recorded();
  }

 private:
  Workspace& ws_;
  bool on_;
};

// The buffers of a handle's cache, idle or not, freed (with the device synchronised).
void free_scratch(ScratchPool* pool);
// pointid_trim over one cache, on the current device.
int trim_scratch(ScratchPool* pool, uint64_t keep_bytes, uint64_t* cached_bytes);

}  // namespace pointid
