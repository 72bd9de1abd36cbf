// Host-side helpers shared by libcas's host sources (no device code).
#pragma once

#include <hip/hip_runtime.h>

#include <functional>
#include <string>
#include <vector>

#include "../../include/cas.h"

namespace cas {

// Records msg as this thread's last error and returns s.
cas_status_t set_error(cas_status_t s, const std::string &msg);
// CAS_ERR_HIP with the HIP error's text.
cas_status_t set_hip_error(const char *what, hipError_t e);

// Byte range [lo, hi) of a tensor that a call reads or writes. Writes of one
// owner may coincide.
struct Interval {
  uintptr_t lo, hi;
  bool write;
  uintptr_t owner;
  const char *what;
};
// Whether every written interval is disjoint from all others; msg names a pair
// that is not.
bool overlap_free(std::vector<Interval> &iv, std::string &msg);

// CAS_ERR_WORKSPACE (and the size that the call needs) unless ws holds `need` bytes.
cas_status_t check_workspace(void *ws, size_t have, size_t need);

// Writes launch tables of `bytes` bytes to ws on the stream with fill().
using TableUpload = std::function<cas_status_t(size_t bytes, void *ws, hipStream_t stream, const std::function<void(char *)> &fill)>;

// cas_paged_decode_run for some of a call's tokens: rows of lse are lse_stride
// apart (q, o and lse are at the first token's place), and the tables go up by `upload`.
cas_status_t decode_run_part(const cas_decode_plan_t *plan, const void *q, const void *k_pages, const void *v_pages, void *o,
                             float *lse, int lse_stride, void *workspace, size_t ws_bytes, const TableUpload &upload,
                             hipStream_t stream);
// Key tiles and shared page runs of a plan.
void decode_plan_counts(const cas_decode_plan_t *plan, int64_t *key_tiles, int32_t *shared_runs);

// launch(), bracketed by timing events while cas_timing_enable is on.
hipError_t timed_launch(const char *name, hipStream_t s, const std::function<hipError_t()> &launch);

// Compute units and XCDs of the current device, looked up once per device.
// gfx950 has 32 CUs per XCD (256 and 8 on a whole MI355X; a partition shows
// fewer). Without a device (planning-only use) the whole MI355X is assumed.
struct Topology {
  int cus = 256, xcds = 8;
};
Topology device_topology();

// One host <-> device copy of a list; bytes == 0 entries are skipped.
struct HostCopy {
  const void *src;
  void *dst;
  size_t bytes;
};
// Enqueues the copies on stream s in list order. Runs of consecutive entries
// that continue both the previous source and the previous destination go out
// as one transfer (fewer, larger DMA transfers keep the host link busier).
hipError_t enqueue_copies(const HostCopy *c, int n, hipMemcpyKind kind, hipStream_t s);

}  // namespace cas
