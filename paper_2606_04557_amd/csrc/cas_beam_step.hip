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

constexpr int kScanThreads = 256;
constexpr int kListCap = 128;    // groups that a wave has found and not looked at yet

// Whether beam `row` has nothing to choose from by its own state.
__device__ __forceinline__ bool out_of_search(const BeamSelectParams &p, int row) {
  return !(fabsf(p.scores[row]) < INFINITY) || (p.finished && p.finished[row]);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

__device__ __forceinline__ float lane_value(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// What the wave's lanes wrote to LDS before is what they read after.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T>
struct Piece;
template <>
struct Piece<__bf16> {
  static constexpr int N = 8;
  __device__ __forceinline__ static void unpack(const u32x4 &v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  __device__ __forceinline__ static void unpack(const u32x4 &v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
  }
};

// A row in pieces: base is the row's first element moved back to a 16-byte address;
// its elements are those at [begin, end) from there.
template <typename T>
struct Row {
  const T *base;
  int begin, end;
  __device__ __forceinline__ Row(const BeamSelectParams &p, int row) {
    const T *x = (const T *)p.logits + row * p.stride;
    begin = (int)(((uintptr_t)x & 15) / sizeof(T));
    end = begin + p.vocab;
    base = x - begin;
  }
  __device__ __forceinline__ void load(int piece, float *x) const {
    constexpr int N = Piece<T>::N;
    const int at = piece * N;
    if (at >= begin && at + N <= end) {
      Piece<T>::unpack(*reinterpret_cast<const u32x4 *>(base + at), x);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = at + i >= begin && at + i < end ? (float)base[at + i] : -INFINITY;
    }
  }
};

// A wave's chunks of one row: the largest logit of every group, and sum exp(x - ref)
// with ref within 1 of the largest logit. A sum of up to 64 terms is a tree in fp32, sums of those are in fp64.
template <typename T, int J>
__global__ __launch_bounds__(kScanThreads) void beam_scan_kernel(BeamSelectParams p) {
  constexpr int N = Piece<T>::N, E = J * N;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * (kScanThreads / 64) + (threadIdx.x >> 6);
  const int row = (int)(id / p.waves), w = (int)(id - (int64_t)row * p.waves);
  if (row >= p.batch * p.beams || out_of_search(p, row)) return;
  const Row<T> r(p, row);
  const int c0 = w * p.per_wave, c1 = min(c0 + p.per_wave, p.chunks);
  float ref = -FLT_MAX;
  double sum = 0.0;
  for (int c = c0; c < c1; ++c) {
    float x[E];
    const int first = c * 64 * J + lane;
    if (c * 64 * E >= r.begin && (c + 1) * 64 * E <= r.end) {
      u32x4 v[J];
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = *reinterpret_cast<const u32x4 *>(r.base + (first + 64 * j) * N);
#pragma unroll
      for (int j = 0; j < J; ++j) Piece<T>::unpack(v[j], x + j * N);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) r.load(first + 64 * j, x + j * N);
    }
    float m = fmaxf(x[0], x[1]);
#pragma unroll
    for (int i = 2; i < E; i += 2) m = max3(m, x[i], x[i + 1]);
    p.group_max[((int64_t)row * p.chunks + c) * 64 + lane] = m;
    if (__ballot(m > ref + 1.0f)) {
      const float next = wave_max(m);
      sum *= exp((double)ref - (double)next);
      ref = next;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = __builtin_amdgcn_exp2f((x[i] - ref) * kLog2e);
#pragma unroll
    for (int n = E / 2; n; n /= 2)
#pragma unroll
      for (int i = 0; i < n; ++i) x[i] += x[i + n];
    sum += (double)x[0];
  }
  sum = wave_sum(sum);
  if (lane == 0) p.parts[(int64_t)row * p.waves + w] = DevBeamPart{sum, ref, 0.0f};
}

// Before b in a beam's order.
__device__ __forceinline__ bool ahead(float xa, int ta, float xb, int tb) { return xa > xb || (xa == xb && ta < tb); }

// 32-bit keys in the order of the floats.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // (-0 and 0 are alike)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// The k-th largest of the lanes' values.
__device__ __forceinline__ float kth_of_lanes(float x, int k) {
  const uint32_t key = order_key(x);
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t trial = t | 1u << b;
    const int n = __popcll(__ballot(key >= trial));
    if (n >= k) t = trial;
    if (n == k) break;
  }
  return key_value(t > 0x7fffffu ? t : 0x7fffffu);   // (-inf; keys below are those of NaNs)
}

// A beam's best logits so far, one in a lane, in order; (-inf, INT_MAX) where there is none.
struct BeamList {
  float x;
  int token;
  __device__ __forceinline__ void insert(int lane, int k, float nx, int nt) {
    const int at = __popcll(__ballot(ahead(x, token, nx, nt)));
    if (at >= k) return;
    // (From the lane before.)
    const float ux = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x138, 0xf, 0xf, true));
    const int ut = __builtin_amdgcn_update_dpp(0, token, 0x138, 0xf, 0xf, true);
    if (lane > at) {
      x = ux;
      token = ut;
    }
    if (lane == at) {
      x = nx;
      token = nt;
    }
  }
};

// Looks at n listed groups of a row for logits that belong to its k best.
template <typename T, int J>
__device__ __forceinline__ void look_at(const Row<T> &r, const int *groups, int n, int lane, int k, float &least, BeamList &best) {
  constexpr int N = Piece<T>::N, G = 64 / J;   // groups that the wave takes at a time
  for (int g0 = 0; g0 < n; g0 += G) {
    const int g = g0 + lane / J, group = g < n ? groups[g] : 0;
    const int piece = (group >> 6) * 64 * J + lane % J * 64 + (group & 63);
    float x[N];
    r.load(piece, x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int token = piece * N + i - r.begin;
      uint64_t hit = __ballot(g < n && x[i] >= least && x[i] > -INFINITY);
      while (hit) {
        const int l = __builtin_ctzll(hit);
        hit &= hit - 1;
        best.insert(lane, k, lane_value(x[i], l), __builtin_amdgcn_readlane(token, l));
      }
    }
    least = fmaxf(least, lane_value(best.x, k - 1));
  }
}

// The k best logits above -inf of a row. A group with one of them has a maximum
// that is at least the k-th largest of any k groups' maxima; only such groups are
// read again.
template <typename T, int J>
__device__ __forceinline__ BeamList best_of_row(const BeamSelectParams &p, int row, int lane, int *groups) {
  const Row<T> r(p, row);
  const float *gm = p.group_max + (int64_t)row * p.chunks * 64 + lane;
  float m = -INFINITY;
#pragma unroll 8
  for (int c = 0; c < p.chunks; ++c) m = fmaxf(m, gm[c * 64]);
  float least = kth_of_lanes(m, p.k);
  BeamList best{-INFINITY, INT32_MAX};
  int n = 0;
  for (int c = 0; c < p.chunks; ++c) {
    const float g = gm[c * 64];
    const bool mine = g >= least && g > -INFINITY;
    const uint64_t hit = __ballot(mine);
    if (!hit) continue;
    if (mine) groups[n + __popcll(hit & ((1ull << lane) - 1))] = c * 64 + lane;
    n += __popcll(hit);
    if (n > kListCap - 64) {
      wave_lds_fence();
      look_at<T, J>(r, groups, n, lane, p.k, least, best);
      wave_lds_fence();
      n = 0;
    }
  }
  wave_lds_fence();
  look_at<T, J>(r, groups, n, lane, p.k, least, best);
  wave_lds_fence();
  return best;
}

// The exact logarithm's share of a beam's score: how far ln sum may be off by what
// the scan rounds. Relative to its value each term is off by its argument d's two
// roundings (2 |d| 2^-24, and 1 % for log2 e's own), the exponential's unit
// (2 x 2^-24) and six additions; the sum's terms, weighted by it, have at most
// ln V - ln sum + 2 for |d| (the entropy of V tokens is at most ln V, and d is at most 1).
__device__ __forceinline__ double sum_error(int vocab, double ln_sum) {
  return (2.2 * (log((double)vocab) - ln_sum + 2.0) + 9.0) * 0x1p-24;
}

// One batch entry: the best tokens of each beam (a wave to a beam), and then the
// best of all. A candidate's place is the number of candidates ahead of it; those
// of another beam are sorted, too, so counting stops at the first one behind it.
// Where two beams' candidates are closer than their sums are exact, those sums are
// made again in fp64 and the places counted again.
template <typename T, int J>
__global__ __launch_bounds__(1024) void beam_pick_kernel(BeamSelectParams p) {
  extern __shared__ char smem[];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_waves = blockDim.x >> 6;
  const int n_beams = p.beams, k = p.k, total = n_beams * k;
  double *own = (double *)smem;                   // [beams] the score so far
  double *ref = own + n_beams;                    // [beams]
  double *ln = ref + n_beams;                     // [beams] ln sum exp(x - ref)
  double *error = ln + n_beams;                   // [beams] of the latter
  double *partial = error + n_beams;              // [waves]
  float *logit = (float *)(partial + n_waves);    // [beams][k]
  int *token = (int *)(logit + total);            // [beams][k]
  int *count = token + total;                     // [beams]
  int *again = count + n_beams;                   // [beams] to be summed again
  int *order = again + n_beams;                   // [k + 1] candidate of each place, or -1
  int *groups = order + k + 1 + wave * kListCap;  // [waves][kListCap]
  auto score = [&](int c, int i) { return own[i] + ((double)logit[c] - ref[i]) - ln[i]; };
  for (int i = wave; i < n_beams; i += n_waves) {
    const int row = b * n_beams + i;
    const float so_far = p.scores[row];
    const bool done = p.finished && p.finished[row];
    int n = 0;
    if (done && fabsf(so_far) < INFINITY) {
      n = 1;
      if (lane == 0) {
        logit[i * k] = 0.0f;
        token[i * k] = p.pad;
        own[i] = so_far;
        ref[i] = ln[i] = error[i] = 0.0;
      }
    } else if (!out_of_search(p, row)) {
      const DevBeamPart *parts = p.parts + (int64_t)row * p.waves;
      float most = -FLT_MAX;
      for (int w = lane; w < p.waves; w += 64) most = fmaxf(most, parts[w].ref);
      most = wave_max(most);
      double sum = 0.0;
      for (int w = lane; w < p.waves; w += 64) sum += parts[w].sum * exp((double)parts[w].ref - (double)most);
      sum = wave_sum(sum);
      if (sum > 0.0 && sum < INFINITY) {   // (a NaN or +inf among the logits is in the sum)
        const BeamList best = best_of_row<T, J>(p, row, lane, groups);
        n = __popcll(__ballot(lane < k && best.x > -INFINITY));
        if (lane < n) {
          logit[i * k + lane] = best.x;
          token[i * k + lane] = best.token;
        }
        if (lane == 0) {
          own[i] = so_far;
          ref[i] = most;
          ln[i] = log(sum);
          error[i] = sum_error(p.vocab, ln[i]);
        }
      }
    }
    if (lane == 0) {
      count[i] = n;
      again[i] = 0;
    }
  }
  for (int round = 0;; ++round) {
    for (int i = tid; i <= k; i += blockDim.x) order[i] = -1;
    __syncthreads();
    for (int c = tid; c < total; c += blockDim.x) {
      const int i = c / k;
      int place = c - i * k;
      if (place >= count[i]) continue;
      const double mine = score(c, i);
      for (int j = 0; j < n_beams && place <= k; ++j) {
        if (j == i) continue;
        for (int e = j * k; e < j * k + count[j] && place <= k; ++e, ++place) {
          const double other = score(e, j);
          if (!(other > mine || (other == mine && j < i))) break;
        }
      }
      if (place <= k) order[place] = c;
    }
    __syncthreads();
    if (round == 1) break;
    bool near = false;
    for (int i = tid; i < k; i += blockDim.x) {
      const int c0 = order[i], c1 = order[i + 1];
      if (c0 < 0 || c1 < 0) continue;
      const int i0 = c0 / k, i1 = c1 / k;
      if (i0 == i1 || score(c0, i0) - score(c1, i1) >= error[i0] + error[i1]) continue;
      near = true;
      if (error[i0] > 0.0) again[i0] = 1;
      if (error[i1] > 0.0) again[i1] = 1;
    }
    if (!__syncthreads_or(near)) break;
    for (int i = 0; i < n_beams; ++i) {
      if (!again[i]) continue;
      const int row = b * n_beams + i;
      const T *x = (const T *)p.logits + row * p.stride;
      const double most = ref[i];
      double sum = 0.0;
#pragma unroll 4
      for (int v = tid; v < p.vocab; v += blockDim.x) sum += exp((double)(float)x[v] - most);
      sum = wave_sum(sum);
      if (lane == 0) partial[wave] = sum;
      __syncthreads();
      sum = 0.0;
      for (int w = 0; w < n_waves; ++w) sum += partial[w];
      if (tid == 0) ln[i] = log(sum);
      __syncthreads();
    }
  }
  int n = 0;
  while (n < k && order[n] >= 0) ++n;
  for (int i = tid; i < k; i += blockDim.x) {
    const int64_t at = (int64_t)b * k + i;
    if (i < n) {
      const int c = order[i];
      p.out_scores[at] = (float)score(c, c / k);
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

hipError_t launch_beam_scan(const BeamSelectParams &p, DType dt, hipStream_t s) {
  const int64_t waves = (int64_t)p.batch * p.beams * p.waves, per_wg = kScanThreads / 64;
  const dim3 grid((unsigned)((waves + per_wg - 1) / per_wg)), threads(kScanThreads);
  if (dt == kBF16 && p.pieces == 8) hipLaunchKernelGGL((beam_scan_kernel<__bf16, 8>), grid, threads, 0, s, p);
  else if (dt == kBF16) hipLaunchKernelGGL((beam_scan_kernel<__bf16, 2>), grid, threads, 0, s, p);
  else if (p.pieces == 8) hipLaunchKernelGGL((beam_scan_kernel<float, 8>), grid, threads, 0, s, p);
  else hipLaunchKernelGGL((beam_scan_kernel<float, 2>), grid, threads, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_beam_pick(const BeamSelectParams &p, DType dt, hipStream_t s) {
  const int waves = p.beams > 8 ? 16 : 8, total = p.beams * p.k;
  const size_t lds = (size_t)total * 8 + (size_t)p.beams * 40 + (size_t)waves * (8 + 4 * kListCap) + ((size_t)p.k + 1) * 4;
  const dim3 grid((unsigned)p.batch), threads((unsigned)waves * 64);
  if (dt == kBF16 && p.pieces == 8) hipLaunchKernelGGL((beam_pick_kernel<__bf16, 8>), grid, threads, lds, s, p);
  else if (dt == kBF16) hipLaunchKernelGGL((beam_pick_kernel<__bf16, 2>), grid, threads, lds, s, p);
  else if (p.pieces == 8) hipLaunchKernelGGL((beam_pick_kernel<float, 8>), grid, threads, lds, s, p);
  else hipLaunchKernelGGL((beam_pick_kernel<float, 2>), grid, threads, lds, s, p);
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
