// Host side of beam search's selection and of the reordering of states kept per
// beam: argument validation and launches. Validation runs before any HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <string>
#include <vector>

#include "../../include/cas.h"
#include "cas_host.h"
#include "cas_internal.h"
#include "cas_spans.h"

using namespace cas;

namespace {

constexpr int64_t kMaxVocab = (int64_t)1 << 30;
constexpr int64_t kMaxRows = (int64_t)1 << 20;
constexpr int64_t kMaxStride = (int64_t)1 << 40;   // (with the limits on rows, spans fit 64 bits)

std::string str(int64_t x) { return std::to_string(x); }
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// No exception leaves a C entry (host memory may run out).
template <typename F>
cas_status_t guarded(F &&f) {
  try {
    return f();
  } catch (const std::exception &e) {
    return set_error(CAS_ERR_UNSUPPORTED, std::string("host memory: ") + e.what());
  }
}

cas_status_t check_beam(const cas_beam_problem_t *p) {
  if (!p) return set_error(CAS_ERR_INVALID_ARGUMENT, "problem is NULL");
  if (p->dtype != CAS_DTYPE_BF16 && p->dtype != CAS_DTYPE_FP32) return set_error(CAS_ERR_UNSUPPORTED, "dtype must be bf16 or fp32");
  if (p->batch < 0) return set_error(CAS_ERR_INVALID_ARGUMENT, "batch must be >= 0");
  if (p->beams < 1 || p->k < 1) return set_error(CAS_ERR_INVALID_ARGUMENT, "beams and k must be >= 1");
  if (p->beams > kMaxBeams || p->k > kMaxBeams) return set_error(CAS_ERR_UNSUPPORTED, "more than 64 beams or candidates");
  if ((int64_t)p->batch * p->beams > kMaxRows) return set_error(CAS_ERR_UNSUPPORTED, "more than 2^20 beams in the batch");
  if (p->vocab < 1) return set_error(CAS_ERR_INVALID_ARGUMENT, "vocab must be >= 1");
  if (p->vocab > kMaxVocab) return set_error(CAS_ERR_UNSUPPORTED, "vocab above 2^30");
  if (p->k > p->beams * p->vocab) return set_error(CAS_ERR_INVALID_ARGUMENT, "k above the number of candidates");
  if (p->row_stride < p->vocab || p->row_stride > kMaxStride)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "row_stride must be in [vocab, 2^40]");
  if (p->pad_token < 0 || p->pad_token >= p->vocab) return set_error(CAS_ERR_INVALID_ARGUMENT, "pad_token must be in [0, vocab)");
  return CAS_OK;
}

struct BeamLayout {
  int32_t chunks, per_wave, waves;
  size_t parts, bytes;
};

BeamLayout beam_layout(const cas_beam_problem_t &p) {
  // Chunks of a wave: as many as leave 8,192 waves, twice what is on the GPU at a time (64 x 8 rows of 131,072
  // bf16 before the loads passed by the caches: 30 us, with half or a quarter as many waves 33).
  constexpr int64_t kWaves = 8192;
  const int64_t rows = (int64_t)p.batch * p.beams, piece = p.dtype == CAS_DTYPE_BF16 ? 8 : 4, chunk = 64 * kBeamPieces * piece;
  BeamLayout l;
  l.chunks = (int32_t)((p.vocab + piece - 1 + chunk - 1) / chunk);   // (a row that begins inside a piece reaches further)
  l.per_wave = (int32_t)std::max<int64_t>(1, rows * l.chunks / kWaves);
  l.waves = (l.chunks + l.per_wave - 1) / l.per_wave;
  l.parts = (size_t)rows * (size_t)l.chunks * 256;
  l.bytes = l.parts + align_up((size_t)rows * (size_t)l.waves * sizeof(DevBeamPart), 256);
  return l;
}

cas_status_t select(const cas_beam_problem_t *p, const void *logits, const float *scores, const uint8_t *finished,
                    float *out_scores, int32_t *out_parents, int32_t *out_tokens, void *workspace, size_t ws_bytes,
                    hipStream_t stream) {
  cas_status_t s = check_beam(p);
  if (s != CAS_OK) return s;
  if (p->batch == 0) return CAS_OK;
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens)
    return set_error(CAS_ERR_INVALID_ARGUMENT, "logits, scores and the outputs must be non-NULL");
  const uintptr_t es = p->dtype == CAS_DTYPE_BF16 ? 2 : 4;
  if ((uintptr_t)logits % es || ((uintptr_t)scores | (uintptr_t)out_scores | (uintptr_t)out_parents | (uintptr_t)out_tokens) & 3u)
    return set_error(CAS_ERR_ALIGNMENT, "logits must be aligned to their type, the other tensors to 4 bytes");
  const BeamLayout l = beam_layout(*p);
  if ((s = check_workspace(workspace, ws_bytes, l.bytes)) != CAS_OK) return s;
  const uintptr_t rows = (uintptr_t)p->batch * (uintptr_t)p->beams, out = (uintptr_t)p->batch * (uintptr_t)p->k * 4;
  std::vector<Interval> iv;
  iv.push_back({(uintptr_t)logits, (uintptr_t)logits + ((rows - 1) * (uintptr_t)p->row_stride + (uintptr_t)p->vocab) * es, false, 0, "logits"});
  iv.push_back({(uintptr_t)scores, (uintptr_t)scores + rows * 4, false, 0, "scores"});
  if (finished) iv.push_back({(uintptr_t)finished, (uintptr_t)finished + rows, false, 0, "finished"});
  iv.push_back({(uintptr_t)out_scores, (uintptr_t)out_scores + out, true, 1, "out_scores"});
  iv.push_back({(uintptr_t)out_parents, (uintptr_t)out_parents + out, true, 2, "out_parents"});
  iv.push_back({(uintptr_t)out_tokens, (uintptr_t)out_tokens + out, true, 3, "out_tokens"});
  iv.push_back({(uintptr_t)workspace, (uintptr_t)workspace + l.bytes, true, 4, "workspace"});
  std::string msg;
  if (!overlap_free(iv, msg)) return set_error(CAS_ERR_INVALID_ARGUMENT, msg);
  char *ws = (char *)workspace;
  BeamSelectParams a{};
  a.logits = logits;
  a.scores = scores;
  a.finished = finished;
  a.out_scores = out_scores;
  a.out_parents = out_parents;
  a.out_tokens = out_tokens;
  a.stride = p->row_stride;
  a.vocab = (int32_t)p->vocab;
  a.batch = p->batch;
  a.beams = p->beams;
  a.k = p->k;
  a.pad = p->pad_token;
  a.chunks = l.chunks;
  a.per_wave = l.per_wave;
  a.waves = l.waves;
  a.ln_vocab = std::log((double)p->vocab);
  a.group_max = (float *)ws;
  a.parts = (DevBeamPart *)(ws + l.parts);
  const DType dt = p->dtype == CAS_DTYPE_BF16 ? kBF16 : kFP32;
  // Where the scan of a batch entry has no more waves than its workgroup, that does it itself: 4 beams of 8,000 tokens
  // 11.5 us instead of 12.7 (a call without a graph 11.9 instead of 14.5), 200 x 8 of 4,000 15.0 instead of 19.0. With two
  // rounds of chunks it takes longer, 4 beams of 32,000 17.1 instead of 12.6.
  const bool one_launch = p->batch <= device_topology().cus && (int64_t)p->beams * l.waves <= kBeamPickWaves;
  if (!one_launch) {
    const hipError_t e = timed_launch("beam_scan", stream, [&] { return launch_beam_scan(a, dt, stream); });
    if (e != hipSuccess) return set_hip_error("beam_scan launch", e);
  }
  const hipError_t e = timed_launch("beam_pick", stream, [&] { return launch_beam_pick(a, dt, one_launch, stream); });
  return e == hipSuccess ? CAS_OK : set_hip_error("beam_pick launch", e);
}

// The widest moves that addresses and strides allow: 16, 4 or 1 bytes (their logarithm).
int32_t log_unit(const cas_beam_state_t &t) {
  const uintptr_t all = (uintptr_t)t.x | (uintptr_t)t.y | (uintptr_t)t.x_stride_batch | (uintptr_t)t.x_stride_beam |
                        (uintptr_t)t.y_stride_batch | (uintptr_t)t.y_stride_beam;
  return all % 16 == 0 ? 4 : all % 4 == 0 ? 2 : 0;
}

cas_status_t reorder(const int32_t *parents, int32_t batch, int32_t beams_in, int32_t beams_out, const cas_beam_state_t *ts,
                     int32_t n, hipStream_t stream) {
  if (batch < 0 || beams_in < 1 || beams_out < 1) return set_error(CAS_ERR_INVALID_ARGUMENT, "batch must be >= 0, beams >= 1");
  if (beams_in > kMaxBeams || beams_out > kMaxBeams) return set_error(CAS_ERR_UNSUPPORTED, "more than 64 beams");
  if ((int64_t)batch * std::max(beams_in, beams_out) > kMaxRows) return set_error(CAS_ERR_UNSUPPORTED, "more than 2^20 beams in the batch");
  if (n < 1 || n > kBeamStates || !ts) return set_error(CAS_ERR_INVALID_ARGUMENT, "1 to 8 tensors");
  if (batch == 0) return CAS_OK;
  if (!parents) return set_error(CAS_ERR_INVALID_ARGUMENT, "parents is NULL");
  if ((uintptr_t)parents & 3u) return set_error(CAS_ERR_ALIGNMENT, "parents must be 4-byte aligned");
  BeamReorderParams p{};
  p.parents = parents;
  p.batch = batch;
  p.beams_in = beams_in;
  p.beams_out = beams_out;
  const Footprint par = span_of(parents, (uint64_t)batch * (uint64_t)beams_out * 4);
  Footprint in[kBeamStates], out[kBeamStates];
  int32_t which[kBeamStates];   // the tensors that have something to move
  int m = 0;
  for (int32_t i = 0; i < n; ++i) {
    const cas_beam_state_t &t = ts[i];
    auto refuse = [&](cas_status_t code, const char *why) { return set_error(code, "tensor " + str(i) + ": " + why); };
    if (t.row_bytes < 0 || t.row_bytes > kMaxStride) return refuse(CAS_ERR_INVALID_ARGUMENT, "row_bytes must be in [0, 2^40]");
    for (const int64_t st : {t.x_stride_batch, t.x_stride_beam, t.y_stride_batch, t.y_stride_beam})
      if (st < 0 || st > kMaxStride) return refuse(CAS_ERR_INVALID_ARGUMENT, "strides must be in [0, 2^40]");
    if (t.row_bytes == 0) continue;
    if (!t.x || !t.y) return refuse(CAS_ERR_INVALID_ARGUMENT, "x and y must be non-NULL");
    in[m] = footprint(t.x, batch, beams_in, t.x_stride_batch, t.x_stride_beam, t.row_bytes, 1);
    out[m] = footprint(t.y, batch, beams_out, t.y_stride_batch, t.y_stride_beam, t.row_bytes, 1);
    if (!out[m].distinct) return refuse(CAS_ERR_INVALID_ARGUMENT, "rows of y overlap");
    const bool in_place = t.x == t.y;
    if (in_place && (beams_in != beams_out || (batch > 1 && t.x_stride_batch != t.y_stride_batch) ||
                     (beams_in > 1 && t.x_stride_beam != t.y_stride_beam)))
      return refuse(CAS_ERR_INVALID_ARGUMENT, "in place, x and y must have equal beams and strides");
    which[m] = i;
    p.t[m++] = DevBeamState{(const char *)t.x, (char *)t.y, t.row_bytes, t.x_stride_batch, t.x_stride_beam, t.y_stride_batch,
                            t.y_stride_beam, log_unit(t)};
  }
  if (m == 0) return CAS_OK;
  for (int i = 0; i < m; ++i) {
    auto refuse = [&](const std::string &what) {
      return set_error(CAS_ERR_INVALID_ARGUMENT, "tensor " + str(which[i]) + ": y overlaps " + what);
    };
    if (!apart(out[i], par)) return refuse("parents");
    for (int j = 0; j < m; ++j) {
      if (!(i == j && p.t[i].x == p.t[i].y) && !apart(out[i], in[j])) return refuse("the x of tensor " + str(which[j]));
      if (i != j && !apart(out[i], out[j])) return refuse("the y of tensor " + str(which[j]));
    }
  }
  const hipError_t e = timed_launch("beam_reorder", stream, [&] { return launch_beam_reorder(p, m, stream); });
  return e == hipSuccess ? CAS_OK : set_hip_error("beam_reorder launch", e);
}

}  // namespace

extern "C" {

cas_status_t cas_beam_select_workspace_size(const cas_beam_problem_t *p, size_t *bytes) {
  if (!bytes) return set_error(CAS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  return guarded([&] {
    const cas_status_t s = check_beam(p);
    if (s == CAS_OK) *bytes = beam_layout(*p).bytes;
    return s;
  });
}

cas_status_t cas_beam_select(const cas_beam_problem_t *p, const void *logits, const float *scores, const uint8_t *finished,
                             float *out_scores, int32_t *out_parents, int32_t *out_tokens, void *workspace, size_t ws_bytes,
                             void *hip_stream) {
  return guarded([&] {
    return select(p, logits, scores, finished, out_scores, out_parents, out_tokens, workspace, ws_bytes, (hipStream_t)hip_stream);
  });
}

cas_status_t cas_beam_reorder(const int32_t *parents, int32_t batch, int32_t beams_in, int32_t beams_out,
                              const cas_beam_state_t *states, int32_t n, void *hip_stream) {
  return guarded([&] { return reorder(parents, batch, beams_in, beams_out, states, n, (hipStream_t)hip_stream); });
}

}  // extern "C"
