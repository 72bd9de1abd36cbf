// Beam search: the selection of a step's candidates, and the reordering of states
// kept per beam.
//
// Selection. With the logits x of beam i, m = max x and s = sum exp(x - m), token
// v's score is scores[i] + (x_v - m) - ln s. Within a beam the order is that of the
// logits, so a beam's k best tokens are found without s; a batch entry's k best are
// among those of its beams. Equal scores go by beam, then token.
#include <float.h>

#include "cas_device.h"

namespace cas {

namespace {

constexpr int kRowThreads = 256;
constexpr int kPickThreads = 256;

template <typename T>
__device__ __forceinline__ float logit_at(const T *x, int64_t i) {
  return (float)x[i];
}

// Whether beam `row` has nothing to choose from by its own state.
__device__ __forceinline__ bool out_of_search(const BeamSelectParams &p, int row) {
  const float s = p.scores[row];
  return !(fabsf(s) < INFINITY) || (p.finished && p.finished[row]);
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Before b in a beam's order.
__device__ __forceinline__ bool ahead(float xa, int ta, float xb, int tb) { return xa > xb || (xa == xb && ta < tb); }

// One row: m, ln s and the k best logits above -inf, one after the other.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void beam_rows_kernel(BeamSelectParams p) {
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ float sm_x[kRowThreads / 64];
  __shared__ int sm_t[kRowThreads / 64];
  __shared__ double sm_s[kRowThreads / 64];
  if (out_of_search(p, row)) {
    if (tid == 0) p.list_count[row] = 0;
    return;
  }
  const T *x = (const T *)p.logits + row * p.stride;
  float last_x = INFINITY;
  int last_t = -1, n = 0;
  double m = 0.0;
  for (int i = 0; i <= p.k; ++i) {
    if (i == 1) {   // (the first one found is the maximum)
      double s = 0.0;
      for (int v = tid; v < p.vocab; v += kRowThreads) s += exp((double)logit_at(x, v) - m);
      s = wave_sum(s);
      if (lane == 0) sm_s[wave] = s;
      __syncthreads();
      s = 0.0;
      for (int w = 0; w < kRowThreads / 64; ++w) s += sm_s[w];
      if (!(s < INFINITY)) n = 0;
      if (tid == 0) {
        p.norm[2 * row] = m;
        p.norm[2 * row + 1] = log(s);
      }
      if (n == 0) break;
    }
    if (i == p.k) break;
    float bx = -INFINITY;
    int bt = INT32_MAX;
    for (int v = tid; v < p.vocab; v += kRowThreads) {
      const float y = logit_at(x, v);
      if (y > -INFINITY && ahead(last_x, last_t, y, v) && ahead(y, v, bx, bt)) {
        bx = y;
        bt = v;
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      const float ox = __shfl_xor(bx, o);
      const int ot = __shfl_xor(bt, o);
      if (ahead(ox, ot, bx, bt)) {
        bx = ox;
        bt = ot;
      }
    }
    __syncthreads();
    if (lane == 0) {
      sm_x[wave] = bx;
      sm_t[wave] = bt;
    }
    __syncthreads();
    for (int w = 0; w < kRowThreads / 64; ++w)
      if (ahead(sm_x[w], sm_t[w], bx, bt)) {
        bx = sm_x[w];
        bt = sm_t[w];
      }
    if (bt == INT32_MAX) break;
    if (i == 0) m = bx;
    if (tid == 0) {
      p.list_logit[(int64_t)row * p.k + n] = bx;
      p.list_token[(int64_t)row * p.k + n] = bt;
    }
    last_x = bx;
    last_t = bt;
    ++n;
  }
  if (tid == 0) p.list_count[row] = n;
}

// One batch entry: the lists of its beams in order of their scores. A candidate's
// place is the number of candidates ahead of it; those of another beam are sorted,
// too, so counting stops at the first one behind it.
template <typename T>
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamSelectParams p) {
  extern __shared__ char smem[];
  const int b = blockIdx.x, tid = threadIdx.x, n_beams = p.beams, k = p.k, total = n_beams * k;
  double *score = (double *)smem;                 // [beams][k]
  int *token = (int *)(score + total);            // [beams][k]
  int *count = token + total;                     // [beams]
  int *order = count + n_beams;                   // [k] candidate of each place, or -1
  for (int i = tid; i < n_beams; i += kPickThreads) {
    const int row = b * n_beams + i;
    const bool done = p.finished && p.finished[row] && fabsf(p.scores[row]) < INFINITY;
    count[i] = done ? 1 : p.list_count[row];
    if (done) {
      score[i * k] = p.scores[row];
      token[i * k] = p.pad;
    }
  }
  for (int i = tid; i < k; i += kPickThreads) order[i] = -1;
  __syncthreads();
  for (int c = tid; c < total; c += kPickThreads) {
    const int i = c / k, row = b * n_beams + i;
    if (c - i * k < count[i] && !(p.finished && p.finished[row])) {
      score[c] = (double)p.scores[row] + ((double)p.list_logit[(int64_t)row * k + c - i * k] - p.norm[2 * row]) - p.norm[2 * row + 1];
      token[c] = p.list_token[(int64_t)row * k + c - i * k];
    }
  }
  __syncthreads();
  for (int c = tid; c < total; c += kPickThreads) {
    const int i = c / k;
    int place = c - i * k;
    if (place >= count[i]) continue;
    for (int j = 0; j < n_beams && place < k; ++j) {
      if (j == i) continue;
      for (int e = j * k; e < j * k + count[j] && place < k; ++e, ++place)
        if (!(score[e] > score[c] || (score[e] == score[c] && j < i))) break;
    }
    if (place < k) order[place] = c;
  }
  __syncthreads();
  int n = 0;
  while (n < k && order[n] >= 0) ++n;
  for (int i = tid; i < k; i += kPickThreads) {
    const int64_t at = (int64_t)b * k + i;
    if (i < n) {
      const int c = order[i];
      p.out_scores[at] = (float)score[c];
      p.out_parents[at] = c / k;
      p.out_tokens[at] = token[c];
      continue;
    }
    // The (i - n)-th of the candidates at -inf: of all but the n above.
    int64_t f = i - n;
    for (int64_t g = -1; g != f;) {
      g = f;
      f = i - n;
      for (int e = 0; e < n; ++e) f += (int64_t)(order[e] / k) * p.vocab + token[order[e]] <= g;
    }
    p.out_scores[at] = -INFINITY;
    p.out_parents[at] = (int)(f / p.vocab);
    p.out_tokens[at] = (int)(f % p.vocab);
  }
}

// A thread has the bytes at one place of every row of a batch entry: it loads them
// all before it stores the first, so that a reordering in place needs no copy.
template <typename U, int N>
__device__ __forceinline__ void move(const DevBeamState &t, const int *parents, int n, int n_in, int64_t at, const char *x, char *y) {
  U v[N];
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < n && (unsigned)parents[j] < (unsigned)n_in) v[j] = *reinterpret_cast<const U *>(x + parents[j] * t.xi + at);
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < n && (unsigned)parents[j] < (unsigned)n_in) *reinterpret_cast<U *>(y + j * t.yi + at) = v[j];
}

template <int N>
__global__ __launch_bounds__(256) void beam_reorder_kernel(BeamReorderParams p) {
  const DevBeamState t = p.t[blockIdx.z];
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, whole = t.row_bytes / t.unit, rest = t.row_bytes - whole * t.unit;
  if (i >= whole + rest) return;
  for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
    const int *parents = p.parents + (int64_t)b * p.beams_out;
    const char *x = t.x + b * t.xb;
    char *y = t.y + b * t.yb;
    const int n = p.beams_out, n_in = p.beams_in;
    if (i >= whole) move<uint8_t, N>(t, parents, n, n_in, whole * t.unit + i - whole, x, y);
    else if (t.unit == 16) move<u32x4, N>(t, parents, n, n_in, i * 16, x, y);
    else if (t.unit == 8) move<uint64_t, N>(t, parents, n, n_in, i * 8, x, y);
    else if (t.unit == 4) move<uint32_t, N>(t, parents, n, n_in, i * 4, x, y);
    else if (t.unit == 2) move<uint16_t, N>(t, parents, n, n_in, i * 2, x, y);
    else move<uint8_t, N>(t, parents, n, n_in, i, x, y);
  }
}

}  // namespace

hipError_t launch_beam_rows(const BeamSelectParams &p, DType dt, hipStream_t s) {
  const dim3 grid((unsigned)(p.batch * p.beams)), threads(kRowThreads);
  if (dt == kBF16) hipLaunchKernelGGL(beam_rows_kernel<__bf16>, grid, threads, 0, s, p);
  else hipLaunchKernelGGL(beam_rows_kernel<float>, grid, threads, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_beam_pick(const BeamSelectParams &p, DType dt, hipStream_t s) {
  const size_t lds = (size_t)p.beams * p.k * 12 + (size_t)p.beams * 4 + (size_t)p.k * 4;
  const dim3 grid((unsigned)p.batch), threads(kPickThreads);
  if (dt == kBF16) hipLaunchKernelGGL(beam_pick_kernel<__bf16>, grid, threads, lds, s, p);
  else hipLaunchKernelGGL(beam_pick_kernel<float>, grid, threads, lds, s, p);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorderParams &p, int n, hipStream_t s) {
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t whole = p.t[i].row_bytes / p.t[i].unit;
    most = whole + (p.t[i].row_bytes - whole * p.t[i].unit) > most ? whole + (p.t[i].row_bytes - whole * p.t[i].unit) : most;
  }
  const int64_t blocks = (most + 255) / 256;
  const dim3 grid((unsigned)blocks, (unsigned)(p.batch < 65535 ? p.batch : 65535), (unsigned)n), threads(256);
  if (p.beams_out <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, grid, threads, 0, s, p);
  else if (p.beams_out <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, grid, threads, 0, s, p);
  else if (p.beams_out <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, grid, threads, 0, s, p);
  else if (p.beams_out <= 32) hipLaunchKernelGGL(beam_reorder_kernel<32>, grid, threads, 0, s, p);
  else hipLaunchKernelGGL(beam_reorder_kernel<64>, grid, threads, 0, s, p);
  return hipGetLastError();
}

}  // namespace cas
