// Beam search: the selection of a step's candidates, and the reordering of states
// kept per beam.
//
// Selection. With the logits x of beam i, m = max x and s = sum exp(x - m), token
// v's score is scores[i] + (x_v - m) - ln s. Within a beam the order is that of the
// logits, so a beam's k best tokens are found without s; a batch entry's k best are
// among those of its beams. Equal scores go by beam, then token.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "cas_beam_error.h"
#include "cas_device.h"

namespace cas {

namespace {

constexpr int kScanThreads = 256;
constexpr int kReorderThreads = 256;
constexpr int kListCap = 128;    // groups that a wave has found and not looked at yet

// The pick's waves, and what their registers hold: the first kTile chunks' group maxima, and kLook pieces of groups
// that are looked at. More than 8 beams have 16 waves: 9 of 32,000 bf16 13.3 us instead of 16.2, 64 of them 33.8
// instead of 45.6.
template <int W>
struct PickShape {
  static constexpr int kThreads = 64 * W, kTile = W == 8 ? 40 : 24, kLook = W == 8 ? 3 : 2;
};

// Whether beam `row` has nothing to choose from by its own state.
__device__ __forceinline__ bool out_of_search(const BeamSelectParams &p, int row) {
  return !(fabsf(p.scores[row]) < INFINITY) || (p.finished && p.finished[row]);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// x of another lane of the wave: lane l +- 1, +- 2 (quad permutations), the mirror of
// 8 and of 16 lanes, and lanes 15 and 31 of the rows before. Rows outside MASK get `old`.
template <int CTRL, int MASK = 0xf>
__device__ __forceinline__ int lane_move(int old, int x) {
  return __builtin_amdgcn_update_dpp(old, x, CTRL, MASK, 0xf, false);
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140, kFrom15 = 0x142, kFrom31 = 0x143;

template <int CTRL, int MASK = 0xf>
__device__ __forceinline__ float max_with(float x) {
  return fmaxf(x, __int_as_float(lane_move<CTRL, MASK>(__float_as_int(x), __float_as_int(x))));
}
__device__ __forceinline__ float wave_max(float x) {
  x = max_with<kMirror16>(max_with<kMirror8>(max_with<kSwap2>(max_with<kSwap1>(x))));
  x = max_with<kFrom31, 0xc>(max_with<kFrom15, 0xa>(x));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

template <int CTRL, int MASK = 0xf>
__device__ __forceinline__ double plus(double x) {
  const int64_t u = __double_as_longlong(x);
  const uint32_t lo = (uint32_t)lane_move<CTRL, MASK>(0, (int)u), hi = (uint32_t)lane_move<CTRL, MASK>(0, (int)(u >> 32));
  return x + __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double wave_min(double x) {   // (rounded towards -inf to fp32)
  float f = (float)x;
  f = (double)f > x ? nextafterf(f, -INFINITY) : f;
  return -(double)wave_max(-f);
}
__device__ __forceinline__ uint64_t lane_value(uint64_t x, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ double wave_sum(double x) {
  x = plus<kMirror16>(plus<kMirror8>(plus<kSwap2>(plus<kSwap1>(x))));
  x = plus<kFrom31, 0xc>(plus<kFrom15, 0xa>(x));
  return __longlong_as_double((int64_t)lane_value((uint64_t)__double_as_longlong(x), 63));
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
  static constexpr uint32_t kEmpty = 0xff80ff80u;   // -inf
  __device__ __forceinline__ static void unpack(const u32x4 &v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static void put(u32x4 &v, int i, __bf16 x) {
    const uint32_t u = __builtin_bit_cast(uint16_t, x);
    v[i / 2] = i & 1 ? (v[i / 2] & 0xffffu) | u << 16 : (v[i / 2] & 0xffff0000u) | u;
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kEmpty = 0xff800000u;
  __device__ __forceinline__ static void unpack(const u32x4 &v, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
  }
  __device__ __forceinline__ static void put(u32x4 &v, int i, float x) { v[i] = __float_as_uint(x); }
};

// A row in pieces: base is the row's first element moved back to a 16-byte address;
// its elements are those at [begin, end) from there, and only those are read. The
// rest of its first and last piece is -inf.
template <typename T>
struct Row {
  static constexpr int N = Piece<T>::N;
  const T *base;
  int begin, end;
  __device__ __forceinline__ Row(const BeamSelectParams &p, int row) {
    const T *x = (const T *)p.logits + row * p.stride;
    begin = (int)(((uintptr_t)x & 15) / sizeof(T));
    end = begin + p.vocab;
    base = x - begin;
  }
  __device__ __forceinline__ bool whole(int piece) const { return piece * N >= begin && (piece + 1) * N <= end; }
  __device__ __forceinline__ u32x4 load(int piece) const { return *reinterpret_cast<const u32x4 *>(base + piece * N); }
  __device__ __forceinline__ u32x4 load_partial(int piece) const {
    u32x4 v = {Piece<T>::kEmpty, Piece<T>::kEmpty, Piece<T>::kEmpty, Piece<T>::kEmpty};
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (piece * N + i >= begin && piece * N + i < end) Piece<T>::put(v, i, base[piece * N + i]);
    return v;
  }
  // A lane's pieces of chunk c, in passing (64 x 8 rows of 131,072 bf16: 27.1 us between events, and 29.2 when the
  // caches are to keep them).
  __device__ __forceinline__ u32x4 load_once(int piece) const {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(base + piece * N));
  }
  __device__ __forceinline__ void load_chunk(int c, int lane, u32x4 *v) const {
    constexpr int J = kBeamPieces;
    const int first = c * 64 * J;
    if (whole(first) && whole(first + 64 * J - 1)) {
#pragma unroll
      for (int j = 0; j < J; ++j) v[j] = load_once(first + 64 * j + lane);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int piece = first + 64 * j + lane;
        v[j] = whole(piece) ? load_once(piece) : load_partial(piece);
      }
    }
  }
};

// What a wave's terms are relative to, see scan().
__device__ __forceinline__ double base_of(float ref) {
  return fabsf(ref) > kFarLogit ? (double)ref : (double)(ref * kLog2e) * 0.6931471805599453;
}

// A wave's chunks of one row: the largest logit of every group, and sum exp(x -
// base). With ref the largest logit of the wave's first 64 pieces, a term is
// 2^(x log2 e - c), one multiply-add and the exponential, where c is ref log2 e
// rounded to fp32 and base = c ln 2. Where ref is beyond +-kFarLogit, so that
// rounding log2 e would count, base = ref and a term is 2^((x - base) log2 e). Eight terms
// (fp32: four) and J / 2 of such sums are added in fp32, the chunks in fp64. A chunk
// with a logit over ref + 16 is done again, with another ref; terms from before keep
// the rounding of the ref that they were made with.
//
// Bound by HBM: 64 x 8 rows of 131,072 bf16 (134 MB) in 25.5 us, 5.3 TB/s (between events 27, without the
// exponentials 26; on data in the cache, so its arithmetic alone, 17.5: an element is
// 7.5 operations of full rate, four of them its exponential's). A wave has 8 KB in
// flight and four waves a SIMD; five, which spill, took 40 us.
template <typename T>
__device__ __forceinline__ void scan(const BeamSelectParams &p, int row, int w, int lane) {
  constexpr int N = Piece<T>::N, J = kBeamPieces;
  const Row<T> r(p, row);
  const int c0 = w * p.per_wave, c1 = min(c0 + p.per_wave, p.chunks);
  float *group_max = p.group_max + (int64_t)row * p.chunks * 64 + lane;
  float ref = 0.0f, low = 0.0f, shift = 0.0f;
  double sum = 0.0;
  bool fresh = true;
  for (int c = c0; c < c1; ++c) {
    u32x4 v[J];
    r.load_chunk(c, lane, v);
    float m = -INFINITY, part;
    for (;;) {
      if (fresh) {   // (by the first piece; by all of them where that was not enough)
        float x[N];
        if (m == -INFINITY) {
          Piece<T>::unpack(v[0], x);
          m = x[0];
#pragma unroll
          for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
        }
        const double was = base_of(ref);
        ref = fmaxf(wave_max(m), -FLT_MAX);
        shift = ref * kLog2e;
        sum *= sum > 0.0 ? exp(was - base_of(ref)) : 0.0;
        if (!(__any(sum > 1e-12))) low = ref;   // (its own term is 1)
        fresh = false;
      }
      float parts[2] = {0.0f, 0.0f};
      m = -INFINITY;
      auto add = [&](auto argument) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          float x[N];
          Piece<T>::unpack(v[j], x);
#pragma unroll
          for (int i = 0; i < N; i += 2) m = max3(m, x[i], x[i + 1]);
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_exp2f(argument(x[i]));
#pragma unroll
          for (int n = N / 2; n; n /= 2)
#pragma unroll
            for (int i = 0; i < n; ++i) x[i] += x[i + n];
          parts[j & 1] += x[0];
        }
      };
      if (fabsf(ref) <= kFarLogit) add([&](float x) { return fmaf(x, kLog2e, -shift); });
      else add([&](float x) { return (x - ref) * kLog2e; });   // (inf - inf: a NaN)
      part = parts[0] + parts[1];
      fresh = __any(m - ref > 16.0f);
      if (!fresh) break;
    }
    group_max[c * 64] = m;
    sum += (double)part;
  }
  sum = wave_sum(sum);
  if (lane == 0) p.parts[(int64_t)row * p.waves + w] = DevBeamPart{sum, ref, low};
}

template <typename T>
__global__ __launch_bounds__(kScanThreads, 4) void beam_scan_kernel(BeamSelectParams p) {
  // (Scalar, so that what the wave begins with is scalar work, too.)
  const unsigned id = blockIdx.x * (kScanThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(id / (unsigned)p.waves), w = (int)(id - (unsigned)row * (unsigned)p.waves);
  if (row >= p.batch * p.beams || out_of_search(p, row)) return;
  scan<T>(p, row, w, threadIdx.x & 63);
}

// 32-bit keys in the order of the floats.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // (-0 and 0 are alike)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// A beam's candidate, the higher the better: equal logits are in the order of their tokens. 0 is none.
__device__ __forceinline__ uint64_t candidate(float x, int token) { return (uint64_t)order_key(x) << 32 | (uint32_t)~token; }
__device__ __forceinline__ float candidate_logit(uint64_t c) { return key_value((uint32_t)(c >> 32)); }
__device__ __forceinline__ int candidate_token(uint64_t c) { return (int)~(uint32_t)c; }

// The k-th largest of N values: each has a key of its own, whose low bits are its index, and counts the keys in LDS that
// are larger.
template <int N>
__device__ __forceinline__ uint32_t distinct_key(float x, int i) {
  return (order_key(x) & ~(uint32_t)(N - 1)) | (N - 1 - i);
}
template <int N>
__device__ __forceinline__ int ahead_of(uint32_t key, const uint32_t *keys) {
  int n = 0;
#pragma unroll 16
  for (int i = 0; i < N / 4; ++i) {
    const u32x4 o = reinterpret_cast<const u32x4 *>(keys)[i];
    n += (o[0] > key) + (o[1] > key) + (o[2] > key) + (o[3] > key);
  }
  return n;
}
// The value, or up to 2^-15 of it less; finite.
template <int N>
__device__ __forceinline__ float finite_value(uint32_t key) {
  key &= ~(uint32_t)(N - 1);
  return key > order_key(-FLT_MAX) ? key_value(key) : -FLT_MAX;
}

// The best logits of a row that a wave has found: `count` (at most k) of them in its
// first lanes, in order, and n more in LDS that have not been compared yet.
struct BeamList {
  uint64_t best;
  uint64_t *found;   // [64]
  int count, n, k;
  float least;       // what is below is not wanted

  // A candidate's place is the number of those ahead of it.
  __device__ __forceinline__ void sort(int lane) {
    wave_lds_fence();
    const uint64_t mine = lane < n ? found[lane] : 0;
    wave_lds_fence();
    int at = lane, at_found = 0;
    for (int i = 0; i < n; ++i) {
      const uint64_t c = lane_value(mine, i);
      at += c > best;
      at_found += c > mine;
    }
    for (int i = 0; i < count; ++i) at_found += lane_value(best, i) > mine;
    if (lane < count && at < k) found[at] = best;
    if (lane < n && at_found < k) found[at_found] = mine;
    count = min(count + n, k);
    n = 0;
    wave_lds_fence();
    best = lane < count ? found[lane] : 0;
    wave_lds_fence();
    if (count == k) least = fmaxf(least, candidate_logit(lane_value(best, k - 1)));
  }
};

// The largest logits of the row's groups, kTile chunks at a time (the first ones stay in registers).
template <int kTile>
struct GroupTile {
  float g[kTile];
  __device__ __forceinline__ void load(const float *at, int chunks) {
    // (By eights, with chunks from the front again behind the row's last: a branch for each would wait for what it loaded.)
#pragma unroll
    for (int c = 0; c < kTile; c += 8) {
      if (c < chunks) {
#pragma unroll
        for (int i = c; i < c + 8; ++i) g[i] = at[(i < chunks ? i : min(i & 3, chunks - 1)) * 64];
      } else {
#pragma unroll
        for (int i = c; i < c + 8; ++i) g[i] = -INFINITY;
      }
    }
  }
};

// The largest of each lane's groups of a row, of which the tile has the first ones, of its chunks i mod 4 (the first
// of them stand in for chunks that the row does not have).
template <int kTile>
__device__ __forceinline__ void largest_of_lane(const float *at, int chunks, const GroupTile<kTile> &tile, float (&m)[4]) {
#pragma unroll
  for (int c = 0; c < kTile; ++c) m[c % 4] = fmaxf(c < 4 ? -INFINITY : m[c % 4], tile.g[c]);
  for (int c = kTile; c < chunks; c += 8) {
    float g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = at[min(c + i, chunks - 1) * 64];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i % 4] = fmaxf(m[i % 4], c + i < chunks ? g[i] : -INFINITY);
  }
}

// The logits of a row that are at least list.least, the k best of them. They are in
// groups whose maximum is at least that, and only such groups are read again, J lanes
// to a group, kLook pieces to a lane at a time. (Sorting is in one place, at the end of
// a loop: 63 KB of code with an insertion wherever a hit is possible took 16.1 us for
// 64 x 8 beams, this 15.0 then.)
template <typename T, int kTile, int kLook>
__device__ __forceinline__ void best_of_row(const BeamSelectParams &p, int row, int lane, int *groups, GroupTile<kTile> &tile,
                                            BeamList &list) {
  constexpr int N = Piece<T>::N, J = kBeamPieces, G = 64 / J, E = kLook * N;
  const Row<T> r(p, row);
  const float *gm = p.group_max + (int64_t)row * p.chunks * 64 + lane;
  for (int c0 = 0;; c0 += kTile) {
    const bool last = c0 + kTile >= p.chunks;
    if (c0) tile.load(gm + c0 * 64, p.chunks - c0);
    uint32_t of[2] = {0, 0};
#pragma unroll
    for (int c = 0; c < kTile; ++c) of[c / 32] |= tile.g[c] >= list.least ? 1u << c % 32 : 0u;
    uint64_t mine = (uint64_t)of[1] << 32 | of[0];   // the lane's groups in the tile that may have something
    if (last) mine &= ~0ull >> (64 - (p.chunks - c0));
    for (bool more = true; more;) {
      int n = 0;   // groups listed
      uint64_t hit;
      while (n <= kListCap - 64 && (hit = __ballot(mine != 0))) {
        if (mine) groups[n + __popcll(hit & ((1ull << lane) - 1))] = (c0 + __builtin_ctzll(mine)) * 64 + lane;
        n += __popcll(hit);
        mine &= mine - 1;
      }
      wave_lds_fence();
      more = n > kListCap - 64;
      for (int g0 = 0;; g0 += G * kLook) {
        float x[E];
        int piece[kLook];
        uint32_t hits = 0;   // the lane's elements that may be among the best
        if (g0 < n) {
          bool partial = false;
#pragma unroll
          for (int u = 0; u < kLook; ++u) {
            const int g = g0 + u * G + lane / J, group = groups[g < n ? g : 0];
            piece[u] = (group >> 6) * 64 * J + lane % J * 64 + (group & 63);
            const bool whole = r.whole(piece[u]);
            partial |= g < n && !whole;
            u32x4 v{};
            if (g < n && whole) v = r.load(piece[u]);
            Piece<T>::unpack(v, x + u * N);
            hits |= (g < n && whole ? (1u << N) - 1 : 0) << u * N;
          }
          if (__builtin_expect(__any(partial), 0)) {
#pragma unroll
            for (int u = 0; u < kLook; ++u)
              if (g0 + u * G + lane / J < n && !r.whole(piece[u])) {
                Piece<T>::unpack(r.load_partial(piece[u]), x + u * N);
                hits |= ((1u << N) - 1) << u * N;
              }
          }
          uint32_t high = 0;
#pragma unroll
          for (int e = 0; e < E; ++e) high |= (uint32_t)(x[e] >= list.least) << e;
          hits &= high;
        }
        const bool end = last && !more && g0 + G * kLook >= n;
        for (;;) {
          // The lane's first one that is left.
          const int e = __builtin_ctz(hits | 1u << 31);
          float y = x[0];
          int at = piece[0];
#pragma unroll
          for (int i = 1; i < E; ++i) y = e == i ? x[i] : y;
#pragma unroll
          for (int u = 1; u < kLook; ++u) at = e / N == u ? piece[u] : at;
          const uint64_t any = __ballot(hits != 0);
          if (!any && !end) break;
          if (!any || list.n + __popcll(any) > 64) {
            list.sort(lane);
            if (!any) return;
            uint32_t high = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) high |= (uint32_t)(x[i] >= list.least) << i;
            hits &= high;
            continue;
          }
          if (hits) list.found[list.n + __popcll(any & ((1ull << lane) - 1))] = candidate(y, at * N + e % N - r.begin);
          list.n += __popcll(any);
          hits &= hits - 1;
        }
        if (g0 + G * kLook >= n) break;
      }
      wave_lds_fence();
    }
  }
}

// One batch entry, a wave to a beam. The largest score of any group with index l mod
// 64 (or 256) is the l-th of 64 (256) values: k groups reach the k-th largest of these,
// and only logits that reach it are looked for. Of k random ones among 64 values that
// is hardly more than k in all while k is small, 44 for 32, but 300 for 64; among 256,
// 74. Then a candidate's place is the number of those ahead of it. Where two beams'
// candidates are closer than their sums are exact, those sums are made again in fp64
// and the places counted again (3 % of the calls for 64 x 8 beams of 131,072 bf16 with
// random logits; 21 us for each such beam, one after the other).
//
// Bound by latency: 64 x 8 beams in 13 us, of which the first loads take a sixth, the
// sums a tenth, the bounds a fifth, listing groups 6 %, their logits 8, sorting them 11, waiting for
// the wave with most of them 8, places and what is close 15, the results 4. 184 scalar
// registers are spilled (8 waves, bf16), in all of these. Equal logits are all looked at, since
// all of them reach the bound: a row of 131,072 takes 7 ms.
template <typename T, int W, bool SCAN>
__global__ __launch_bounds__(PickShape<W>::kThreads) void beam_pick_kernel(BeamSelectParams p) {
  constexpr int kPickThreads = PickShape<W>::kThreads;
  extern __shared__ char smem[];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_beams = p.beams, k = p.k;
  double *score = (double *)smem;                    // [beams][64] of a beam's candidates
  double *own = score + n_beams * 64;                // [beams] the score so far
  double *ref = own + n_beams;                       // [beams]
  double *ln = ref + n_beams;                        // [beams] ln sum exp(x - ref)
  double *error = ln + n_beams;                      // [beams] of the latter
  double *partial = error + n_beams;                 // [W]
  float *values = (float *)(partial + W);            // [W][256], and then
  uint64_t *found = (uint64_t *)(values + wave * 256);   // [W][64]
  int *groups = (int *)(found + 64);                 // [W][kListCap]
  int *pool = (int *)(values + W * 256);             // [kPickThreads] the candidates of all beams, if there are so few
  int *token = pool + kPickThreads;                  // [beams][64]
  int *count = token + n_beams * 64;                 // [beams] -1: candidates of it are looked for
  int *again = count + n_beams;                      // [beams] to be summed again
  int *inside = again + n_beams;                     // [beams] candidates among the k
  int *order = inside + n_beams;                     // [k] candidate of each place
  int *pool_size = order + k;
  static_assert(64 * 2 + kListCap == 256, "a wave's share of the values");
  if (tid == 0) *pool_size = 0;
  auto put = [&](int i, int n) {   // candidates 0 .. n - 1 of beam i into the pool
    int at = lane == 0 ? atomicAdd(pool_size, n) : 0;
    at = __builtin_amdgcn_readfirstlane(at);
    if (lane < n && at + lane < kPickThreads) pool[at + lane] = i * 64 + lane;
  };
  if (SCAN) {   // (otherwise beam_scan_kernel has done it)
    const unsigned items = (unsigned)(n_beams * p.waves);
#pragma unroll 1
    for (unsigned id = __builtin_amdgcn_readfirstlane(wave); id < items; id += W) {
      const int i = (int)(id / (unsigned)p.waves), row = b * n_beams + i;
      if (!out_of_search(p, row)) scan<T>(p, row, (int)(id - (unsigned)i * (unsigned)p.waves), lane);
    }
    __syncthreads();
  }
  GroupTile<PickShape<W>::kTile> tile;
  const bool many = k > 32 && p.chunks >= 4;
  float most_of_lane[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  for (int i = wave; i < n_beams; i += W) {
    const int row = b * n_beams + i;
    // (All that is needed is loaded at once; for a row out of the search it is not used.)
    const DevBeamPart *parts = p.parts + (int64_t)row * p.waves;
    const float *gm = p.group_max + (int64_t)row * p.chunks * 64 + lane;
    const DevBeamPart first = parts[min(lane, p.waves - 1)];
    const float so_far = p.scores[row];
    const bool done = p.finished && p.finished[row];
    tile.load(gm, p.chunks);
    int n = 0;
    if (fabsf(so_far) < INFINITY) {
      double most = 0.0, ln_sum = 0.0, off = 0.0;
      if (done) {
        n = 1;
        if (lane == 0) {
          score[i * 64] = so_far;
          token[i * 64] = p.pad;
          most_of_lane[0] = fmaxf(most_of_lane[0], so_far);
        }
      } else {
        // (A NaN or +inf among the logits is in the sum.)
        float x[4];
        largest_of_lane(gm, p.chunks, tile, x);
        if (!many) x[0] = fmaxf(max3(x[0], x[1], x[2]), x[3]);
        most = wave_max(many ? fmaxf(max3(x[0], x[1], x[2]), x[3]) : x[0]);
        double sum = 0.0, lowest = INFINITY;
        for (int w = lane; w < p.waves; w += 64) {
          const DevBeamPart part = w < 64 ? first : parts[w];
          sum += part.sum > 0.0 ? part.sum * exp(base_of(part.ref) - most) : part.sum;
          if (part.sum > 0.0 && most - part.ref < 60.0) lowest = fmin(lowest, (double)part.low);   // (the others' share is under 1e-10)
        }
        sum = wave_sum(sum);
        if (sum > 0.0 && sum < INFINITY) {
          n = -1;
          ln_sum = fmax(log(sum), 0.0);   // (of a sum that has the term 1: no token is likelier than certain)
          off = sum_error(p.ln_vocab, ln_sum, wave_min(lowest), most);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i == 0 || many) most_of_lane[i] = fmaxf(most_of_lane[i], (float)(so_far + ((double)x[i] - most) - ln_sum));
        }
      }
      if (lane == 0) {
        own[i] = so_far;
        ref[i] = most;
        ln[i] = ln_sum;
        error[i] = off;
      }
    }
    if (lane == 0) {
      count[i] = n;
      again[i] = 0;
      if (n == 0) error[i] = 0.0;
    }
  }
  float *limit = (float *)order;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i == 0 || many) values[wave * 256 + i * 64 + lane] = most_of_lane[i];
  __syncthreads();
  uint32_t *keys = (uint32_t *)pool;
  if (many) {
    float x = values[tid & 255];
    for (int w = 1; w < W; ++w) x = fmaxf(x, values[w * 256 + (tid & 255)]);
    const uint32_t key = distinct_key<256>(x, tid & 255);
    if (tid < 256) keys[tid] = key;
    __syncthreads();
    if (tid < 256 && ahead_of<256>(key, keys) == k - 1) *limit = finite_value<256>(key);
  } else if (wave == 0) {
    float x = values[lane];
#pragma unroll
    for (int w = 1; w < W; ++w) x = fmaxf(x, values[w * 256 + lane]);
    const uint32_t key = distinct_key<64>(x, lane);
    keys[lane] = key;
    wave_lds_fence();
    if (ahead_of<64>(key, keys) == k - 1) *limit = finite_value<64>(key);
  }
  __syncthreads();
  const double reached = *limit;
  for (int i = wave; i < n_beams; i += W) {
    if (count[i] >= 0) {
      put(i, count[i]);
      continue;
    }
    const int row = b * n_beams + i;
    if (n_beams > W) tile.load(p.group_max + (int64_t)row * p.chunks * 64 + lane, p.chunks);
    // (Lower by what the scores, those behind the bound among them, and their rounding to fp32 may be off, and by a step of
    // fp32 for the rounding here.)
    const double bound = reached - own[i] + ref[i] + ln[i], slack = 2.0 * error[i] + 1e-5 + 0x1p-22 * (fabs(reached) + fabs(bound));
    // (Without k values to go by, whatever a beam has may be wanted.)
    const float least = reached > -FLT_MAX ? fmaxf((float)(bound - slack), -FLT_MAX) : -FLT_MAX;
    BeamList list{0, found, 0, 0, k, least};
    best_of_row<T, PickShape<W>::kTile, PickShape<W>::kLook>(p, row, lane, groups, tile, list);
    if (lane < list.count) {
      score[i * 64 + lane] = own[i] + ((double)candidate_logit(list.best) - ref[i]) - ln[i];
      token[i * 64 + lane] = candidate_token(list.best);
    }
    if (lane == 0) count[i] = list.count;
    put(i, list.count);
  }
  // The places. Beams are told apart by sums that are made again where a candidate that may be among the k is closer
  // to another beam's than unsure, twice what a sum may be off.
  double unsure = lane < n_beams ? error[lane] : 0.0;
  unsure = -2.0 * wave_min(-unsure);
  __syncthreads();
  const int total = *pool_size, n = min(total, k);
  for (int round = 0;; ++round) {
    bool near = false;
    if (total <= kPickThreads) {   // (each with every other; four threads to a candidate where there are enough)
      const int share = total <= kPickThreads / 4 ? 2 : 0, q = tid >> share;
      int c = 0;
      double mine = 0.0;
      bool touched = false;
      if (q < total) {
        c = pool[q];
        mine = score[c];
        int place = 0;
#pragma unroll 4
        for (int e = tid & ((1 << share) - 1); e < total; e += 1 << share) {
          const int o = pool[e];
          const double gap = score[o] - mine;
          place += gap > 0.0 || (gap == 0.0 && o < c);
          touched |= fabs(gap) < unsure && (o ^ c) >= 64;
        }
        if (share) place += lane_move<kSwap1>(0, place);
        if (share) place += lane_move<kSwap2>(0, place);
        if (place < k) order[place] = c;
      }
      __syncthreads();
      near = touched && mine > score[order[n - 1]] - unsure;
      if (near) again[c >> 6] = 1;
    } else {
      // Masses of equal candidates. Those of another beam are sorted: how many are ahead is found by doubling steps,
      // then halving them.
      const int log_k = 32 - __builtin_clz(k - 1 | 1), slots = n_beams << log_k;
      for (int i = tid; i < n_beams; i += kPickThreads) inside[i] = 0;
      __syncthreads();
      for (int q = tid; q < slots; q += kPickThreads) {
        const int i = q >> log_k, c = i * 64 + (q & ((1 << log_k) - 1));
        if (c - i * 64 >= count[i]) continue;
        const double mine = score[c];
        int place = c - i * 64;
        for (int j = 0; j < n_beams && place < k; ++j) {
          if (j == i) continue;
          const double *s = score + j * 64;
          auto ahead = [&](int e) { return s[e] > mine || (s[e] == mine && j < i); };
          int lo = 0, hi = count[j];
          for (int step = 1; lo + step <= hi && ahead(lo + step - 1); step *= 2) lo += step;
          for (int step = 32; step; step /= 2)
            if (lo + step <= hi && ahead(lo + step - 1)) lo += step;
          place += lo;
        }
        if (place < k) {
          order[place] = c;
          atomicAdd(&inside[i], 1);
        }
      }
      __syncthreads();
      // Neighbours among the k, and any of the k and the best of another beam's others: whatever else is as close is so
      // by way of such pairs.
      auto tell_apart = [&](int c0, int c1) {
        if (c0 >> 6 == c1 >> 6 || score[c0] - score[c1] >= unsure) return;
        near = true;
        again[c0 >> 6] = again[c1 >> 6] = 1;
      };
      for (int q = tid; q < slots; q += kPickThreads) {
        const int j = q >> log_k, at = q & ((1 << log_k) - 1);
        if (at >= n) continue;
        if (inside[j] < count[j]) tell_apart(order[at], j * 64 + inside[j]);
        if (j == 0 && at + 1 < n) tell_apart(order[at], order[at + 1]);
      }
    }
    if (round == 1 || !__syncthreads_or(near)) break;
    // exp(d) = 2^n 2^(j/32) exp(r), |r| <= ln 2 / 64: a table and a polynomial of degree 5, 17 instructions an element. In
    // units of 2^-53 relative to itself a term is off by 21 for what the polynomial leaves out, 6 for its steps, the table and the
    // product, and 2 |d| (on average at most 2 ln V) for d and r; the sum by an addition for each of a thread's V / 512 and 22 more, its
    // logarithm by 2 ln V: V / 512 + 140 in all. In the order of the tokens, wherever a row begins: rows alike have equal sums.
    double *table = (double *)values;
    if (tid < 32) table[tid] = exp2(tid / 32.0);
    __syncthreads();
    for (int i = 0; i < n_beams; ++i) {
      if (!again[i] || error[i] == 0.0) continue;   // (a finished beam's score is exact)
      const int row = b * n_beams + i;
      const T *x = (const T *)p.logits + row * p.stride;
      const double most = (double)(float)x[token[i * 64]];   // (a beam with a candidate has its first one)
      double sum = 0.0;
#pragma unroll 8
      for (int v = tid; v < p.vocab; v += kPickThreads) {
        const double d = fmax((double)(float)x[v] - most, -700.0);
        const double shifted = fma(d, 32.0 * 1.4426950408889634, 0x1.8p52);   // (its low bits are 32 n + j)
        const int nj = (int)__double_as_longlong(shifted);
        const double r = fma(shifted - 0x1.8p52, -0.6931471805599453 / 32.0, d);
        const double q = fma(r, fma(r, fma(r, fma(r, fma(r, 1.0 / 120.0, 1.0 / 24.0), 1.0 / 6.0), 0.5), 1.0), 1.0);
        sum += ldexp(q * table[nj & 31], nj >> 5);
      }
      sum = wave_sum(sum);
      if (lane == 0) partial[wave] = sum;
      __syncthreads();
      sum = 0.0;
      for (int w = 0; w < W; ++w) sum += partial[w];
      if (tid < count[i]) score[i * 64 + tid] = own[i] + ((double)(float)x[token[i * 64 + tid]] - most) - log(sum);
      __syncthreads();
    }
  }
  for (int i = tid; i < k; i += kPickThreads) {
    const int64_t at = (int64_t)b * k + i;
    if (i < n) {
      const int c = order[i];
      p.out_scores[at] = (float)score[c];
      p.out_parents[at] = c >> 6;
      p.out_tokens[at] = token[c];
      continue;
    }
    // The (i - n)-th of the candidates at -inf: of all but the n above.
    int64_t f = i - n;
    for (int64_t g = -1; g != f;) {
      g = f;
      f = i - n;
      for (int e = 0; e < n; ++e) f += (int64_t)(order[e] >> 6) * p.vocab + token[order[e]] <= g;
    }
    p.out_scores[at] = -INFINITY;
    p.out_parents[at] = (int)(f / p.vocab);
    p.out_tokens[at] = (int)(f % p.vocab);
  }
}

// Reordering. A thread has the bytes at one place of every row of a batch entry: it
// loads them all before it stores the first, so that a reordering in place needs no
// copy. Bound by HBM: every row that is a parent is read once (its further children
// find it in the cache), every one written that is not its own parent in place. Two tensors of
// 32 x 8 rows of 400 KB (329 MB, 120 of the 256 rows parents): 66 us, 4.9 TB/s; with 64 beams, whose
// 64 pieces leave one wave to a SIMD and spill 442 scalar registers, 2.5 TB/s. Rows that are 4 or 1 bytes
// aligned go by such units: 128 x 8 rows of 400 KB in 126, 266 and 624 us (660 MB). Addresses by scalars: with a branch around each
// load and vector addresses the same took 218 us.
template <typename U, int N>
__device__ __forceinline__ void move(const char *x, int64_t xi, char *y, int64_t yi, int parent_of_lane, int n, int n_in, uint32_t at) {
  U v[N];
  const char *row = x;   // (of the last parent that was in range: what has no row of its own loads that, without a branch)
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int parent = __builtin_amdgcn_readlane(parent_of_lane, j);
    row = j < n && (unsigned)parent < (unsigned)n_in ? x + parent * xi : row;
    v[j] = *reinterpret_cast<const U *>(row + at);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int parent = __builtin_amdgcn_readlane(parent_of_lane, j);
    if (j < n && (unsigned)parent < (unsigned)n_in && !(x == y && parent == j)) *reinterpret_cast<U *>(y + j * yi + at) = v[j];
  }
}

template <int N>
__global__ __launch_bounds__(kReorderThreads) void beam_reorder_kernel(BeamReorderParams p) {
  const DevBeamState t = p.t[blockIdx.z];
  const int n = p.beams_out, n_in = p.beams_in, lane = threadIdx.x & 63, log_unit = t.log_unit;
  // Whole units, then (from the next wave on) the bytes behind them.
  const int64_t whole = t.row_bytes >> log_unit, rest0 = (whole + 63) & ~(int64_t)63, rest = t.row_bytes - (whole << log_unit);
#pragma unroll 1
  for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
    const int parent = p.parents[(int64_t)b * n + min(lane, n - 1)];
#pragma unroll 1
    for (int64_t i0 = (int64_t)blockIdx.x * kReorderThreads; i0 < rest0 + rest; i0 += (int64_t)gridDim.x * kReorderThreads) {
      const char *x = t.x + b * t.xb + (i0 << log_unit);
      char *y = t.y + b * t.yb + (i0 << log_unit);
      const int64_t i = i0 + threadIdx.x;
      if (i < whole) {
        const uint32_t at = threadIdx.x << log_unit;
        if (log_unit == 4) move<u32x4, N>(x, t.xi, y, t.yi, parent, n, n_in, at);
        else if (log_unit == 2) move<uint32_t, N>(x, t.xi, y, t.yi, parent, n, n_in, at);
        else move<uint8_t, N>(x, t.xi, y, t.yi, parent, n, n_in, at);
      } else if (i >= rest0 && i < rest0 + rest) {
        const int64_t back = (whole << log_unit) - (i0 << log_unit);   // (may be before this workgroup's first unit)
        move<uint8_t, N>(x + back, t.xi, y + back, t.yi, parent, n, n_in, (uint32_t)(i - rest0));
      }
    }
  }
}

}  // namespace

hipError_t launch_beam_scan(const BeamSelectParams &p, DType dt, hipStream_t s) {
  const int64_t waves = (int64_t)p.batch * p.beams * p.waves, per_wg = kScanThreads / 64;
  const dim3 grid((unsigned)((waves + per_wg - 1) / per_wg)), threads(kScanThreads);
  if (dt == kBF16) hipLaunchKernelGGL(beam_scan_kernel<__bf16>, grid, threads, 0, s, p);
  else hipLaunchKernelGGL(beam_scan_kernel<float>, grid, threads, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_beam_pick(const BeamSelectParams &p, DType dt, bool scan, hipStream_t s) {
  auto launch = [&](auto waves, auto scans) {
    constexpr int W = decltype(waves)::value;
    constexpr bool SCAN = decltype(scans)::value;
    const size_t lds = (size_t)p.beams * (64 * 12 + 44) + (size_t)W * (8 + 1024) + ((size_t)p.k + 1 + PickShape<W>::kThreads) * 4;
    const dim3 grid((unsigned)p.batch), threads(PickShape<W>::kThreads);
    if (dt == kBF16) hipLaunchKernelGGL((beam_pick_kernel<__bf16, W, SCAN>), grid, threads, lds, s, p);
    else hipLaunchKernelGGL((beam_pick_kernel<float, W, SCAN>), grid, threads, lds, s, p);
  };
  using Many = std::integral_constant<int, kBeamPickWaves>;
  if (scan) launch(Many{}, std::true_type{});
  else if (p.beams > 8) launch(Many{}, std::false_type{});
  else launch(std::integral_constant<int, 8>{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const BeamReorderParams &p, int n, hipStream_t s) {
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t whole = p.t[i].row_bytes >> p.t[i].log_unit, rest = p.t[i].row_bytes - (whole << p.t[i].log_unit);
    most = std::max(most, ((whole + 63) & ~(int64_t)63) + rest);
  }
  const int64_t blocks = std::min<int64_t>((most + kReorderThreads - 1) / kReorderThreads, 1 << 20);
  const dim3 grid((unsigned)blocks, (unsigned)std::min(p.batch, 65535), (unsigned)n), threads(kReorderThreads);
  if (p.beams_out <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, grid, threads, 0, s, p);
  else if (p.beams_out <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, grid, threads, 0, s, p);
  else if (p.beams_out <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, grid, threads, 0, s, p);
  else if (p.beams_out <= 32) hipLaunchKernelGGL(beam_reorder_kernel<32>, grid, threads, 0, s, p);
  else hipLaunchKernelGGL(beam_reorder_kernel<64>, grid, threads, 0, s, p);
  return hipGetLastError();
}

}  // namespace cas
