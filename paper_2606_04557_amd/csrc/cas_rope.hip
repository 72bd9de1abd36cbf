// Rotary positions, alone (forward and gradient) and on the way into the paged
// cache (paper: paragraph "Pool rotation", the queries' positions are offset by
// the active cartridges' tokens; Su et al. 2021 for the rotation).
//
// A pair (x, y) of a head at position t becomes (x cos a - y sin a, x sin a +
// y cos a), a = 2 pi t turns[i]; the gradient is the same with -a. A thread
// owns 16 channels of a head, 8 pairs: two 16-byte pieces of bf16, rotary_dim/2
// apart or next to each other, so every load and store is 16 bytes wide and the
// eight angles are the same for every head of a token. The thread computes them
// once and walks several heads.
//
// Bound by HBM: an element is read once and written once, and the angles cost
// about 30 operations for each pair and thread. 8,192 tokens of 32 query and 8 key
// heads of 128 (bf16, 168 MB): 27 us, 6.2 TB/s where a 1 GiB device copy reaches
// 5.1 (what the caches still hold counts); 8 requests' 1,000 to 1,024 new tokens
// appended with their queries (198 MB): 34 us, 5.8 TB/s. One new token: 2.7 us, a
// launch's latency.
#include <algorithm>

#include "cas_device.h"

namespace cas {

namespace {

constexpr int kRopeThreads = 256;

// cos and sin of position * turn turns. Whole turns are taken off with the exact
// product (one fused multiply-add in double precision: a rounded one would be off by
// up to 2^-53 of the whole angle, 2.4e-7 at 2^31 radians), so what is left, at most an
// eighth of a turn, is rounded to fp32 once; there the Taylor series are within 2e-9
// (sin, to a^9) and 1e-10 (cos, to a^10).
__device__ __forceinline__ void cos_sin_turns(double position, double turn, float &c, float &s) {
  const double t = __builtin_fma(position, turn, -__builtin_rint(position * turn));
  const double q = __builtin_rint(4.0 * t);
  const float a = (float)((t - 0.25 * q) * 6.283185307179586477);
  const float z = a * a;
  const float sn = a + a * z * (-1.0f / 6 + z * (1.0f / 120 + z * (-1.0f / 5040 + z * (1.0f / 362880))));
  const float cs = 1.0f + z * (-0.5f + z * (1.0f / 24 + z * (-1.0f / 720 + z * (1.0f / 40320 + z * (-1.0f / 3628800)))));
  const int k = (int)q & 3;
  c = k & 1 ? sn : cs;
  s = k & 1 ? cs : sn;
  c = k == 1 || k == 2 ? -c : c;
  s = k >= 2 ? -s : s;
}

template <typename T>
struct Eight;
template <>
struct Eight<__bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const __bf16 *p) { v = *reinterpret_cast<const bf16x8 *>(p); }
  __device__ __forceinline__ void store(__bf16 *p) const { *reinterpret_cast<bf16x8 *>(p) = v; }
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = (__bf16)x; }
};
template <>
struct Eight<float> {
  f32x4 v[2];
  __device__ __forceinline__ void load(const float *p) {
    v[0] = *reinterpret_cast<const f32x4 *>(p);
    v[1] = *reinterpret_cast<const f32x4 *>(p + 4);
  }
  __device__ __forceinline__ void store(float *p) const {
    *reinterpret_cast<f32x4 *>(p) = v[0];
    *reinterpret_cast<f32x4 *>(p + 4) = v[1];
  }
  __device__ __forceinline__ float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ __forceinline__ void set(int i, float x) { v[i >> 2][i & 3] = x; }
};

// A thread's share of every head: 16 channels in two pieces at oa and ob. Unit
// u < rotary / 16 holds pairs 8u .. 8u + 7, a later one channels 16u .. that
// are copied.
template <typename T, bool IL>
struct RopeUnit {
  int oa, ob;
  bool rot;
  float c[8], s[8];

  __device__ __forceinline__ void init(const DevRope &r, int u, int position) {
    rot = r.turns != nullptr && 16 * u < r.rotary;
    oa = rot && !IL ? 8 * u : 16 * u;
    ob = rot && !IL ? r.rotary / 2 + 8 * u : 16 * u + 8;
    if (!rot) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cos_sin_turns((double)position, r.turns[8 * u + e], c[e], s[e]);
      c[e] *= r.scale;
      s[e] *= r.inverse ? -r.scale : r.scale;
    }
  }
  __device__ __forceinline__ void turn(Eight<T> &a, Eight<T> &b) const {
    if (!rot) return;
    if constexpr (IL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        Eight<T> &p = e < 4 ? a : b;
        const int i = 2 * (e & 3);
        const float x = p.get(i), y = p.get(i + 1);
        p.set(i, x * c[e] - y * s[e]);
        p.set(i + 1, x * s[e] + y * c[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = a.get(e), y = b.get(e);
        a.set(e, x * c[e] - y * s[e]);
        b.set(e, x * s[e] + y * c[e]);
      }
    }
  }
  // Heads h0, h0 + step, ... of one token; x and y point at its first head. Up to
  // four heads are loaded before the first is stored.
  __device__ __forceinline__ void heads(const T *x, int64_t x_head, T *y, int64_t y_head, int h0, int step, int n) const {
    int h = h0;
    for (; h + 3 * step < n; h += 4 * step) some<4>(x, x_head, y, y_head, h, step);
    for (; h < n; h += step) some<1>(x, x_head, y, y_head, h, step);
  }
  template <int N>
  __device__ __forceinline__ void some(const T *x, int64_t x_head, T *y, int64_t y_head, int h, int step) const {
    Eight<T> a[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i].load(x + (h + i * step) * x_head + oa);
      b[i].load(x + (h + i * step) * x_head + ob);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      turn(a[i], b[i]);
      a[i].store(y + (h + i * step) * y_head + oa);
      b[i].store(y + (h + i * step) * y_head + ob);
    }
  }
};

template <typename T, int D, bool IL>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeParams p) {
  constexpr int U = D / 16;
  const int u = threadIdx.x % U, w = threadIdx.x / U;
  const DevRopeTensor t = p.t[blockIdx.z];
  const int64_t tok = (int64_t)blockIdx.x * (kRopeThreads / U / t.slots) + w / t.slots;
  const int h0 = w % t.slots;
  if (tok >= p.tokens || h0 >= t.heads) return;
  RopeUnit<T, IL> r;
  r.init(p.rope, u, p.positions[tok]);
  r.heads((const T *)t.x + tok * t.x_tok, t.x_head, (T *)t.y + tok * t.y_tok, t.y_head, h0, t.slots, t.heads);
}

// z: 0 the keys, 1 the values, 2 the queries.
template <int D, bool IL>
__global__ __launch_bounds__(kRopeThreads) void append_kernel(AppendParams p) {
  constexpr int U = D / 16;
  const int u = threadIdx.x % U, w = threadIdx.x / U;
  const uint32_t *words = p.words;
  const int unit = blockIdx.x, per_wg = kRopeThreads / U / p.slots;
  const int which = words[p.map0 + unit / 2] >> (16 * (unit & 1)) & 0xffff;
  const uint32_t *rq = words + which * (int)(sizeof(DevAppendRequest) / 4);
  const DevAppendRequest r{(int)rq[0], (int)rq[1], (int)rq[2], (int)rq[3], (int)rq[4], (int)rq[5]};
  const int i0 = (unit - r.unit0) * per_wg, i = i0 + w / p.slots;
  const int h0 = blockIdx.y * p.slots + w % p.slots, step = gridDim.y * p.slots;
  const int heads = blockIdx.z == 2 ? p.Hkv * p.g : p.Hkv;
  if (i >= r.n || h0 >= heads) return;
  const int64_t tok = (int64_t)r.tok0 + i;
  DevRope rope = p.rope;
  if (blockIdx.z == 1) rope.turns = nullptr;
  RopeUnit<__bf16, IL> turner;
  turner.init(rope, u, r.pos0 + i);
  if (blockIdx.z == 2) {
    turner.heads((const __bf16 *)p.q + tok * p.q_tok, p.q_head, (__bf16 *)p.q_out + tok * heads * D, D, h0, step, heads);
    return;
  }
  // The workgroup's first token's page and the one after it, if its last token is in that.
  const int last = min(i0 + per_wg, r.n) - 1;
  const int e0 = (r.row0 + i0) >> p.page_shift, e1 = (r.row0 + last) >> p.page_shift, e = (r.row0 + i) >> p.page_shift;
  const int page_a = words[p.page0 + r.entry0 + e0], page_b = words[p.page0 + r.entry0 + e1];
  const int64_t row = ((int64_t)(e == e0 ? page_a : page_b) << p.page_shift) + ((r.row0 + i) & ((1 << p.page_shift) - 1));
  const int64_t at = row * p.Hkv * D;
  if (blockIdx.z == 0)
    turner.heads((const __bf16 *)p.k + tok * p.k_tok, p.k_head, (__bf16 *)p.k_pages + at, D, h0, step, heads);
  else
    turner.heads((const __bf16 *)p.v + tok * p.v_tok, p.v_head, (__bf16 *)p.v_pages + at, D, h0, step, heads);
}

template <typename T, int D>
void launch_rope_t(const RopeParams &p, dim3 grid, hipStream_t s) {
  if (p.rope.interleaved) hipLaunchKernelGGL((rope_kernel<T, D, true>), grid, dim3(kRopeThreads), 0, s, p);
  else hipLaunchKernelGGL((rope_kernel<T, D, false>), grid, dim3(kRopeThreads), 0, s, p);
}

template <int D>
void launch_append_t(const AppendParams &p, dim3 grid, hipStream_t s) {
  if (p.rope.interleaved) hipLaunchKernelGGL((append_kernel<D, true>), grid, dim3(kRopeThreads), 0, s, p);
  else hipLaunchKernelGGL((append_kernel<D, false>), grid, dim3(kRopeThreads), 0, s, p);
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, DType dt, int D, int n, hipStream_t s) {
  int slots = 1;   // (the grid is as wide as the tensor with the most workgroups needs)
  for (int i = 0; i < n; ++i) slots = std::max(slots, p.t[i].slots);
  const int64_t per_wg = kRopeThreads / (D / 16) / slots;
  const dim3 grid((unsigned)((p.tokens + per_wg - 1) / per_wg), 1, (unsigned)n);
  if (dt == kBF16) {
    if (D == 64) launch_rope_t<__bf16, 64>(p, grid, s);
    else launch_rope_t<__bf16, 128>(p, grid, s);
  } else {
    if (D == 64) launch_rope_t<float, 64>(p, grid, s);
    else launch_rope_t<float, 128>(p, grid, s);
  }
  return hipGetLastError();
}

hipError_t launch_append(const AppendParams &p, int D, int units, int head_groups, hipStream_t s) {
  const dim3 grid((unsigned)units, (unsigned)head_groups, p.q ? 3u : 2u);
  if (D == 64) launch_append_t<64>(p, grid, s);
  else launch_append_t<128>(p, grid, s);
  return hipGetLastError();
}

}  // namespace cas
