// Host side of a handle, shared by the library's source files: its state,
// error text, device guard, the cache of uploaded host tables, grow-on-demand
// buffers and timed launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <string>
#include <vector>

#include "shampoo.h"

namespace shp {

struct GraftBlock;

inline int cdiv(int a, int b) { return (a + b - 1) / b; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Key of a host table for the upload cache (a hit is confirmed by memcmp,
// so the hash only filters): four independent multiply-xorshift chains over
// 8-byte words (a table of a few tens of KB hashes in microseconds, where a
// byte-serial chain took tens), then the tail bytes.
inline uint64_t table_hash(const void* p, size_t n) {
  const unsigned char* c = static_cast<const unsigned char*>(p);
  uint64_t h[4] = {0x243F6A8885A308D3ull, 0x13198A2E03707344ull, 0xA4093822299F31D0ull, 0x082EFA98EC4E6C89ull};
  size_t i = 0;
  for (; i + 32 <= n; i += 32)
    for (int l = 0; l < 4; ++l) {
      uint64_t w;
      memcpy(&w, c + i + 8 * l, 8);
      h[l] = (h[l] ^ w) * 0x9E3779B97F4A7C15ull;
      h[l] ^= h[l] >> 29;
    }
  uint64_t r = h[0] ^ (h[1] << 17 | h[1] >> 47) ^ (h[2] << 31 | h[2] >> 33) ^ (h[3] << 47 | h[3] >> 17);
  for (; i < n; ++i) r = (r ^ c[i]) * 1099511628211ull;
  return r ^ (uint64_t)n;
}

struct TableEntry {
  uint64_t key = 0;
  size_t bytes = 0, cap = 0;
  void* dev = nullptr;
  void* host = nullptr;
  hipEvent_t ev = nullptr;
  uint64_t last = 0;
  bool used = false;
  bool own = false;  // dev and host are allocations of this entry (else its slab slot)
};
// Cached tables per handle, and the bytes of an entry's slot in the handle's
// slabs (larger tables are allocated).  A step over one of a few gradient
// buffers uses about six tables: 64 entries were replaced in turn by a
// program cycling 16 buffers, a copy before every launch.  Beyond about 40
// buffers in turn every table is copied again, as it was beyond 10.
constexpr int kTableEntries = 256;
constexpr size_t kTableSlot = 4096;

struct TimedLaunch {
  int cls;
  hipEvent_t a, b;
};

struct Handle {
  int device = 0;
  std::string err;
  std::vector<TableEntry> cache;
  char* slab_dev = nullptr;  // kTableEntries slots each, allocated with the first table
  char* slab_host = nullptr;
  std::vector<int> pending;  // cache entries referenced by the launches being enqueued
  uint64_t clock = 0;
  void* zbuf = nullptr;  // intermediate G Rr of two-sided preconditioning (grown on demand)
  size_t zbuf_cap = 0;
  void* partial = nullptr;
  size_t partial_cap = 0;
  void* sort_tmp = nullptr;  // rocPRIM temporary storage of the embedding row compaction
  size_t sort_tmp_cap = 0;
  int32_t* pinned = nullptr;  // kCountInts ints
  hipEvent_t poll_ev[2] = {nullptr, nullptr};
  bool timing = false;
  std::vector<TimedLaunch> timed;
  std::vector<hipEvent_t> spare_events;
  // shampoo_graft_noalloc: this device's address of `scratch`, the pinned
  // staging of its block table and the event of the last table copy
  void* noalloc_dev = nullptr;
  GraftBlock* noalloc_host = nullptr;
  hipEvent_t noalloc_ev = nullptr;
  // shampoo_precondition_graft: graft pass 2 of a chunk of blocks runs on
  // `side` while the next chunk's GEMMs run on the caller's stream (both at
  // the default priority); `handoff` orders the two
  hipStream_t side = nullptr;
  hipEvent_t handoff = nullptr;
};

struct DeviceGuard {
  int old = -1;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&old) != hipSuccess) old = -1;
    if (old != dev) (void)hipSetDevice(dev);
  }
  ~DeviceGuard() {
    int cur = -1;
    if (old >= 0 && hipGetDevice(&cur) == hipSuccess && cur != old) (void)hipSetDevice(old);
  }
};

inline shampoo_status fail(Handle* h, shampoo_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  if (h) h->err = buf;
  return code;
}

#define HIP_TRY(h, expr)                                                                   \
  do {                                                                                     \
    hipError_t e_ = (expr);                                                                \
    if (e_ != hipSuccess) return fail((h), SHAMPOO_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define STATUS_TRY(expr)               \
  do {                                 \
    shampoo_status s_ = (expr);        \
    if (s_ != SHAMPOO_OK) return s_;   \
  } while (0)

// Device copy of a host table, cached by content.  An entry is reused only
// after every launch that referenced it has completed (event per entry).
inline shampoo_status upload_table(Handle* h, const void* data, size_t bytes, hipStream_t s, const void** out) {
  const uint64_t key = table_hash(data, bytes);
  for (size_t i = 0; i < h->cache.size(); ++i) {
    TableEntry& e = h->cache[i];
    if (e.used && e.key == key && e.bytes == bytes && memcmp(e.host, data, bytes) == 0) {
      e.last = ++h->clock;
      h->pending.push_back((int)i);
      *out = e.dev;
      return SHAMPOO_OK;
    }
  }
  int slot = -1;
  if (!h->slab_dev) HIP_TRY(h, hipMalloc(reinterpret_cast<void**>(&h->slab_dev), kTableEntries * kTableSlot));
  if (!h->slab_host)
    HIP_TRY(h, hipHostMalloc(reinterpret_cast<void**>(&h->slab_host), kTableEntries * kTableSlot, hipHostMallocDefault));
  if (h->cache.size() < (size_t)kTableEntries) {
    h->cache.emplace_back();
    slot = (int)h->cache.size() - 1;
    h->cache[slot].dev = h->slab_dev + slot * kTableSlot;
    h->cache[slot].host = h->slab_host + slot * kTableSlot;
    h->cache[slot].cap = kTableSlot;
    HIP_TRY(h, hipEventCreateWithFlags(&h->cache[slot].ev, hipEventDisableTiming));
  } else {
    uint64_t best = UINT64_MAX;
    for (size_t i = 0; i < h->cache.size(); ++i)
      if (h->cache[i].last < best) { best = h->cache[i].last; slot = (int)i; }
    HIP_TRY(h, hipEventSynchronize(h->cache[slot].ev));
  }
  TableEntry& e = h->cache[slot];
  if (e.cap < bytes) {
    e.used = false;
    e.cap = 0;
    if (e.own && e.dev) HIP_TRY(h, hipFree(e.dev));
    if (e.own && e.host) HIP_TRY(h, hipHostFree(e.host));
    e.dev = e.host = nullptr;
    e.own = true;
    const size_t cap = align256(bytes);
    HIP_TRY(h, hipMalloc(&e.dev, cap));
    HIP_TRY(h, hipHostMalloc(&e.host, cap, hipHostMallocDefault));
    e.cap = cap;
  }
  memcpy(e.host, data, bytes);
  HIP_TRY(h, hipMemcpyAsync(e.dev, e.host, bytes, hipMemcpyHostToDevice, s));
  e.key = key;
  e.bytes = bytes;
  e.used = true;
  e.last = ++h->clock;
  h->pending.push_back(slot);
  *out = e.dev;
  return SHAMPOO_OK;
}

// Marks every table referenced since the last call as in use up to here.
inline shampoo_status tables_done(Handle* h, hipStream_t s) {
  for (int i : h->pending) HIP_TRY(h, hipEventRecord(h->cache[i].ev, s));
  h->pending.clear();
  return SHAMPOO_OK;
}

inline shampoo_status grow(Handle* h, void** buf, size_t* cap, size_t bytes, hipStream_t s) {
  if (*cap >= bytes) return SHAMPOO_OK;
  // The old buffer may still be read by queued work of this handle, which is
  // ordered on its stream (one handle per stream).
  HIP_TRY(h, hipStreamSynchronize(s));
  if (*buf) HIP_TRY(h, hipFree(*buf));
  *buf = nullptr;
  *cap = 0;
  const size_t c = align256(bytes + bytes / 4);
  HIP_TRY(h, hipMalloc(buf, c));
  *cap = c;
  return SHAMPOO_OK;
}

inline hipEvent_t take_event(Handle* h) {
  if (!h->spare_events.empty()) {
    hipEvent_t e = h->spare_events.back();
    h->spare_events.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  if (hipEventCreate(&e) != hipSuccess) return nullptr;
  return e;
}

template <typename F>
shampoo_status launch(Handle* h, int cls, hipStream_t s, F&& f) {
  hipEvent_t a = nullptr, b = nullptr;
  if (h->timing) {
    a = take_event(h);
    b = take_event(h);
    if (!a || !b) return fail(h, SHAMPOO_EHIP, "hipEventCreate failed");
    HIP_TRY(h, hipEventRecord(a, s));
  }
  f();
  HIP_TRY(h, hipGetLastError());
  if (h->timing) {
    HIP_TRY(h, hipEventRecord(b, s));
    h->timed.push_back({cls, a, b});
  }
  return SHAMPOO_OK;
}

}  // namespace shp
