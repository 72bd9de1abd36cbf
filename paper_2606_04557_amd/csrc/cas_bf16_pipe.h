// What the bf16 attention kernels on gfx950 share: tile copies, scheduling and
// barriers, and the two phases of the forward's ping-pong over 64-key tiles (rows
// that read a batch row's segments, cas_bf16.hip, or a request's pages,
// cas_chunk.hip).
#pragma once

#include <type_traits>
#include <utility>

#include "cas_device.h"

namespace cas {

namespace {

constexpr int kNW = 8;                 // waves per workgroup
constexpr int kFastThreads = kNW * 64;
constexpr int kKT = 64;                // keys per tile (forward, dQ)
constexpr int kFastRowsPerWave = 32;
constexpr int kFastRowsPerWg = kNW * kFastRowsPerWave;   // 256
constexpr int kRefMargin = 64;         // forward: row sums below 2^kRefMargin need no exact pass

struct TileInfo {
  const __bf16 *kp;
  const __bf16 *vp;
  int st;      // token stride in elements (the host keeps 128 rows within 32-bit offsets)
  int nvalid;
  int self0;   // first self key of the tile, or -1 for a cartridge tile
};

// f(integral_constant<int, 0>) ... f(integral_constant<int, N-1>), unrolled.
template <typename F, int... Ks>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, Ks...>) {
  (f(std::integral_constant<int, Ks>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// Scheduling groups: the next n MFMAs / LDS reads of the region, in order.
template <int N>
__device__ __forceinline__ void sched_mfma() { __builtin_amdgcn_sched_group_barrier(0x008, N, 0); }
template <int N>
__device__ __forceinline__ void sched_ds_read() { __builtin_amdgcn_sched_group_barrier(0x100, N, 0); }

// Per-lane share of the direct-to-LDS copies of an R-row tile: the tile row
// and element offset (swizzle applied) of each 16-byte chunk this lane moves
// are fixed for the whole kernel, so a tile copy costs one multiply-add and
// one copy instruction per chunk.
template <int D, int R, int NW>
struct CopyLanes {
  static constexpr int CPR = D / 8;
  static constexpr int NI = R * CPR / 64;             // 1 KiB wave instructions per tile
  static constexpr int PER = (NI + NW - 1) / NW;      // instructions per wave
  int row[PER];
  int coff[PER];
  __device__ __forceinline__ void init(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int pos = (wave + i * NW) * 64 + lane;
      const int r = pos / CPR;
      row[i] = r;
      coff[i] = ((pos % CPR) ^ swz<D>(r)) * 8;
    }
  }
  // Rows at or beyond nvalid (>= 1) re-read row nvalid-1 (finite; masked
  // later). The copies go through a buffer resource spanning exactly the
  // tile's rows (an out-of-range offset would read zeros, not fault), and
  // as MUBUF LDS loads they are counted on vmcnt alone.
  __device__ __forceinline__ void issue(char *tile, const __bf16 *base, int st, int nvalid, int wave) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) issue_one(tile, base, st, nvalid, wave, i);
  }
  // Instruction i (< PER) of this wave's share only.
  __device__ __forceinline__ void issue_one(char *tile, const __bf16 *base, int st, int nvalid, int wave,
                                            int i) const {
    issue_rs(tile, make_rsrc(base, ((nvalid - 1) * st + D) * 2), st, nvalid, wave, i);
  }
  // The same through a given resource (an empty one writes zeros).
  __device__ __forceinline__ void issue_rs(char *tile, BufRsrc rs, int st, int nvalid, int wave, int i) const {
    const int inst = wave + i * NW;
    if (NI % NW == 0 || inst < NI) dma16(rs, (min(row[i], nvalid - 1) * st + coff[i]) * 2, tile + inst * 1024);
  }
};

// Pins register values at this point: the compiler may not move their
// computation past it (e.g. across a barrier into the next phase).
template <typename T, int N>
__device__ __forceinline__ void fence_regs(T (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// Workgroup barrier that orders LDS use: this wave's LDS reads have returned,
// and the compiler moves no memory access across it. Outstanding direct
// global->LDS copies are not waited for (wait_vmcnt does that).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0); vmcnt, expcnt untouched
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Matrix phase of the forward as one software-pipelined sequence of MFMAs: the
// PV product of the previous tile (for d = 128 16 MFMAs, two transposed LDS reads
// per fragment), then the scores of this one (16 MFMAs, one LDS read per
// fragment). The fragment of MFMA k+LEAD is read while MFMA k runs, into a ring of
// LEAD+1 registers, and the scheduling groups pin exactly that order, so the LDS
// latency hides behind the MFMA pipe across the PV -> S boundary too.
template <int D>
__device__ __forceinline__ void fwd_matrix_phase(const char *kb, const char *vb, const RowOffsets<D> &ro, const TrOffsets<D> &to,
                                                 const bf16x8 (&qf)[D / 16], const bf16x8 (&pf)[2][2], f32x16 &s0, f32x16 &s1,
                                                 f32x16 (&oacc)[D / 32]) {
  constexpr int NSTEP = D / 16, DT = D / 32;
  constexpr int NPV = 4 * DT;            // PV MFMAs
  constexpr int N = NPV + 2 * NSTEP;     // all MFMAs
  constexpr int LEAD = 4, R = LEAD + 1;
  // MFMA k < NPV: s = k / (2*DT), dt = (k / 2) % DT, key half hh = k % 2.
  // MFMA k >= NPV: st = (k - NPV) / 2, score half hh = (k - NPV) % 2.
  auto load = [&](auto K) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    if constexpr (k < NPV) {
      constexpr int s = k / (2 * DT), dt = (k / 2) % DT, hh = k % 2;
      return tr_frag_at<D>(vb, to, 32 * hh + 16 * s, dt);
    } else {
      constexpr int st = (k - NPV) / 2, hh = (k - NPV) % 2;
      return row_frag_at<D>(kb, ro, 32 * hh, st);
    }
  };
  auto mma = [&](auto K, const bf16x8 &f) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    if constexpr (k < NPV) {
      constexpr int s = k / (2 * DT), dt = (k / 2) % DT, hh = k % 2;
      oacc[dt] = Mma<__bf16>::run(f, pf[hh][s], oacc[dt]);
    } else {
      constexpr int st = (k - NPV) / 2, hh = (k - NPV) % 2;
      if constexpr (hh == 0) s0 = Mma<__bf16>::run(f, qf[st], s0);
      else s1 = Mma<__bf16>::run(f, qf[st], s1);
    }
  };
  s0 = zero16();
  s1 = zero16();
  bf16x8 ring[R];
  static_for<LEAD>([&](auto K) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    ring[k % R] = load(K);
  });
  static_for<N>([&](auto K) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    if constexpr (k + LEAD < N) ring[(k + LEAD) % R] = load(std::integral_constant<int, k + LEAD>{});
    mma(K, ring[k % R]);
  });
  // Scheduling groups: the LEAD first fragments, then per MFMA k the reads
  // of fragment k+LEAD.
  static_for<LEAD>([&](auto K) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    sched_ds_read<(k < NPV ? 2 : 1)>();
  });
  static_for<N>([&](auto K) __attribute__((always_inline)) {
    constexpr int k = decltype(K)::value;
    sched_mfma<1>();
    if constexpr (k + LEAD < N) sched_ds_read<(k + LEAD < NPV ? 2 : 1)>();
  });
}

// Masks a tile's scores. lim: last visible key of this lane's query within the
// tile. Register j of group G holds key crow(j, G) = crow(j, 0) + 4G, so comparing
// lim - 4G against compile-time constants needs no index registers.
__device__ __forceinline__ void fwd_mask(int lim, int G, f32x16 &s0, f32x16 &s1) {
  const int limg = lim - 4 * G;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    s0[j] = crow(j, 0) <= limg ? s0[j] : -INFINITY;
    s1[j] = 32 + crow(j, 0) <= limg ? s1[j] : -INFINITY;
  }
}

// Maximum of a row's scores in the tile, in log2 units.
__device__ __forceinline__ float fwd_tile_max(const f32x16 &s0, const f32x16 &s1, float c) {
  float mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; j += 2) mx = fmaxf(fmaxf(mx, fmaxf(s0[j], s1[j])), fmaxf(s0[j + 1], s1[j + 1]));
  return fmaxf(mx, xor32(mx)) * c;
}

// Weights of a tile from its scores, offset by mu: bf16 for the next product
// (off by up to half a step, 2^-8 of a weight; fp32 products run at a sixteenth of
// the rate), fp32 for the row sum, which the LSE needs to better than that. piece(n), n < PIECES: copy instruction n of
// the phase, spread evenly over the exponentials.
template <int PIECES, typename Piece>
__device__ __forceinline__ float fwd_weights(float c, float mu, f32x16 &s0, f32x16 &s1, bf16x8 (&pf)[2][2], Piece &&piece) {
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    s0[j] = fast_exp2(fmaf(s0[j], c, -mu));
    s1[j] = fast_exp2(fmaf(s1[j], c, -mu));
    constexpr int EPP = 16 / PIECES;
    if (j % EPP == EPP - 1) {
      asm volatile("" : "+v"(s0[j]), "+v"(s1[j]));   // keep the copies spread
      piece(j / EPP);
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    pf[0][s] = pack_bf16x8(s0, s);
    pf[1][s] = pack_bf16x8(s1, s);
  }
  float la = 0.0f, lb = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    la += s0[j];
    lb += s1[j];
  }
  return la + lb;
}

}  // namespace

}  // namespace cas
