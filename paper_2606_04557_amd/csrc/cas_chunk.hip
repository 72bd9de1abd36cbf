// Attention of a chunk of new tokens over a paged KV cache (forward only; paper:
// Section "Inference", cartridges ahead of the prompt, causal masking of what
// follows).
//
// Query i of a request's n new tokens sees keys 0 .. L - n + i of its L. The g
// heads of a group share their KV head's keys, so a row is a (token, head) pair
// and a workgroup of eight waves takes 256 of them, 32 per wave, over a range of
// 64-key tiles, with the phases of the prefix forward: the two waves of a SIMD
// take turns, one in a matrix phase (O += V^T P of the tile before, S = K Q^T of
// this one) while the other is in its softmax phase (cas_bf16.hip). Here the tiles
// are gathered page by page, each group copies its share, and the second pass for
// rows that the fixed softmax reference does not fit is a plain loop. A workgroup
// works through a list of items (blocks of rows, or pieces of their keys), which
// the host makes equally long for all compute units.
//
// Bound by the matrix cores: 2,048 tokens of 32 heads over 18 to 20 thousand keys
// (8 KV heads of 128) take 539 us a call in a long run of them, 1,212 TFLOP/s where an
// 8,192^3 library product reaches 1,388; in turn with it at any pace (10 to 400 calls
// in a row, which change the clock) 0.87 to 0.90 of its rate. A 64-key tile of 256 rows
// takes 1.75 us. With d = 64 it is the softmax (the same exponentials for half the
// products): 1.15 us. A block of at
// most 64 rows would leave most waves idle and one wave's chain of dependent steps
// would set the pace (1.08 us a tile of 32 rows), so there the waves divide the keys
// (0.47 us), as far as memory brings them.
//
// This file is compiled to honour NaN: that second pass also keeps values which
// are not finite from the rows that do not see their keys.
#include "cas_bf16_pipe.h"

namespace cas {

namespace {

__device__ __forceinline__ bool odd16(unsigned bits) { return (bits & 0x7f80u) == 0x7f80u; }   // inf or NaN

// Whether a 64-key tile of V holds a value that is not finite (one wave).
template <int D>
__device__ __forceinline__ bool has_odd(const char *tile, int lane) {
  bool odd = false;
#pragma unroll 1
  for (int i = lane; i < kKT * D / 8; i += 64) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + 16 * i);
#pragma unroll
    for (int k = 0; k < 4; ++k) odd |= odd16(w[k]) || odd16(w[k] >> 16);
  }
  return wave_any(odd);
}

// Adds the values that are not finite of the tile's keys 0 .. lim to a row's O
// (P > 0 times one is itself).
template <int D>
__device__ __forceinline__ void add_odd(const char *tile, int lim, int G, f32x16 (&oacc)[D / 32]) {
#pragma unroll 1
  for (int key = 0; key < kKT; ++key)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int ch = 32 * dt + crow(j, G);
        const __bf16 v = *reinterpret_cast<const __bf16 *>(tile + swz_off<D>(key, ch / 8) + 2 * (ch % 8));
        if (key <= lim && odd16(__builtin_bit_cast(unsigned short, v))) oacc[dt][j] += (float)v;
      }
}

__device__ __forceinline__ bf16x8 finite_only(bf16x8 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] &= (odd16(w[k]) ? 0u : 0xffffu) | (odd16(w[k] >> 16) ? 0u : 0xffff0000u);
  return __builtin_bit_cast(bf16x8, w);
}

// The phases' parts for 32 keys (cas_bf16_pipe.h has those for a tile's 64).
__device__ __forceinline__ void mask_piece(int lim, int G, f32x16 &s) {
  const int limg = lim - 4 * G;
#pragma unroll
  for (int j = 0; j < 16; ++j) s[j] = crow(j, 0) <= limg ? s[j] : -INFINITY;
}

__device__ __forceinline__ float piece_max(const f32x16 &s, float c) {
  float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int j = 0; j < 16; j += 4) {
    mx[0] = fmaxf(fmaxf(mx[0], s[j]), s[j + 1]);
    mx[1] = fmaxf(fmaxf(mx[1], s[j + 2]), s[j + 3]);
  }
  const float m = fmaxf(mx[0], mx[1]);
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * c;
}

__device__ __forceinline__ float piece_weights(float c, float mu, f32x16 &s, bf16x8 (&pf)[2]) {
  float l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 16; ++j) s[j] = fast_exp2(fmaf(s[j], c, -mu));
#pragma unroll
  for (int h = 0; h < 2; ++h) pf[h] = pack_bf16x8(s, h);
#pragma unroll
  for (int j = 0; j < 16; ++j) l[j & 1] += s[j];
  return l[0] + l[1];
}

struct NoTables {};

// The kernel's parameters, with DIRECT the granules' place among them.
template <bool DIRECT>
__device__ __forceinline__ ChunkParams chunk_params() {
  ChunkParams p = load_kernarg<ChunkParams>();
  if constexpr (DIRECT) {
    const ChunkDirect *d = kernarg_at<ChunkDirect>(sizeof(ChunkParams));
    p.granules = d->words + load_const(&d->n, 0) * (int)(sizeof(ChunkDirectRequest) / 4);
  }
  return p;
}

template <bool DIRECT>
__device__ __forceinline__ DevChunkItem chunk_item(const ChunkParams &p, int at) {
  if constexpr (!DIRECT) return load_const(p.items, at);
  const ChunkDirect *d = kernarg_at<ChunkDirect>(sizeof(ChunkParams));
  const auto *requests = reinterpret_cast<const ChunkDirectRequest *>(d->words);
  const int n = load_const(&d->n, 0), rows = load_const(&d->rows, 0);
  const int block = at / p.Hkv;
  int i = 0;
  while (i + 1 < n && block >= load_const(requests, i + 1).block0) ++i;
  const ChunkDirectRequest r = load_const(requests, i);
  const int row0 = (block - r.block0) * rows, row1 = min(r.len * p.g, row0 + rows);
  return DevChunkItem{r.tok0, r.len, r.kv_len, r.granule0, row0, at - block * p.Hkv, 0, (r.kv_len - r.len + (row1 - 1) / p.g) / kKT + 1, -1, -1, row1};
}

template <int D, bool DIRECT>
__global__ __launch_bounds__(kFastThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void chunk_bf16_kernel(ChunkParams, std::conditional_t<DIRECT, ChunkDirect, NoTables>) {
  constexpr int NSTEP = D / 16, DT = D / 32;
  constexpr int TB = kKT * D * 2;
  constexpr int CPR = D / 8, RPI = 64 / CPR;   // 16-byte chunks of a key row, key rows of a copy instruction
  constexpr int PER = kKT / RPI / 4;           // copy instructions of a K or V tile for each of a group's four waves
  __shared__ __attribute__((aligned(1024))) char kb0[TB];
  __shared__ __attribute__((aligned(1024))) char kb1[TB];
  __shared__ __attribute__((aligned(1024))) char kb2[TB];
  __shared__ __attribute__((aligned(1024))) char vb0[TB];
  __shared__ __attribute__((aligned(1024))) char vb1[TB];
  __shared__ __attribute__((aligned(1024))) char vb2[TB];

#pragma unroll 1
  for (int at = blockIdx.x; at >= 0;) {
    // Per item, the lane index and the parameters are read anew: values kept
    // across items would be held in registers through the tile loop.
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const ChunkParams p = chunk_params<DIRECT>();
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wave >> 2, w4 = wave & 3;
    const int G = lane >> 5, n = lane & 31;
    const int g = p.g, Hkv = p.Hkv, Hq = Hkv * g;
    const float c = p.scale_log2;
    RowOffsets<D> ro;
    ro.init(n, G);
    TrOffsets<D> to;
    to.init(lane);
    const DevChunkItem it = chunk_item<DIRECT>(p, at);
    const int nrows = it.row1;   // (the rows of its request that end here)
    // Few rows: the waves share them, in `rgs` groups of 32, and divide the keys.
    const bool narrow = nrows - it.row0 <= kChunkNarrowRows;
    const int rgs = nrows - it.row0 <= kFastRowsPerWave ? 1 : 2;
    const int row0 = it.row0 + (narrow ? wave & (rgs - 1) : wave) * kFastRowsPerWave, my_row = row0 + n;
    const bool wave_active = row0 < nrows;
    const int before = it.kv_len - it.len;       // token t sees keys 0 .. before + t
    const int last_lo = __builtin_amdgcn_readfirstlane(before + row0 / g);
    const int last_hi = __builtin_amdgcn_readfirstlane(before + (min(row0 + kFastRowsPerWave, nrows) - 1) / g);
    const int my_t = my_row / g;
    const int nt = it.tile1 - it.tile0;

    // Copies: group A's waves copy the K tiles, group B's the V tiles. Instruction
    // i of wave w4 moves key rows r0 .. r0 + RPI - 1 of a tile, r0 = RPI (w4 + 4 i),
    // which lie in one granule of 16 rows, and a granule in one page. It has a
    // resource of its own, which ends behind the request's last key: later rows
    // read as zero, and are masked. (With the scalar work of looking up pages and
    // of one group copying both, 215 instructions beside the 120 of the softmax
    // phase, a tile took 1.94 us.) Rows 16 apart share their swizzle, so one lane
    // offset serves every instruction.
    static_assert(4 * RPI % 16 == 0, "the swizzle of a wave's rows is the same for every instruction");
    const int row_bytes = Hkv * D * 2;
    const int lane_off = (lane / CPR) * row_bytes + (((lane % CPR) ^ swz<D>(w4 * RPI + lane / CPR)) << 4);
    const uint64_t pool = (uint64_t)(grp == 0 ? p.k_pages : p.v_pages) + it.kvh * (D * 2) + (w4 * RPI % 16) * row_bytes;
    const int full = (RPI - 1) * row_bytes + D * 2;   // bytes of an instruction's rows
    struct Tile {
      uint32_t at[PER];   // its granules, from the pool's start on, in 2 KiB
    };
    auto tile_at = [&](int j) __attribute__((always_inline)) {
      Tile t;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        t.at[i] = load_const(p.granules, it.granule0 + 4 * (it.tile0 + j) + (w4 * RPI) / 16 + i * (4 * RPI / 16));
      return t;
    };
    // Bytes of tile j's rows from the wave's first one on, up to the last key (none past the last tile).
    auto bytes_left = [&](int j) __attribute__((always_inline)) {
      return j < nt ? min(it.kv_len - (it.tile0 + j) * kKT - w4 * RPI, kKT) * row_bytes - (row_bytes - D * 2) : 0;
    };
    auto copy = [&](char *buf, const Tile &t, int left, int i) __attribute__((always_inline)) {
      dma16(make_rsrc((const void *)(pool + ((uint64_t)t.at[i] << 11)), min(max(left - i * 4 * RPI * row_bytes, 0), full)), lane_off,
            buf + (w4 + 4 * i) * 1024);
    };
    auto copy_tile = [&](char *buf, const Tile &t, int j) __attribute__((always_inline)) {
      const int left = bytes_left(j);
#pragma unroll
      for (int i = 0; i < PER; ++i) copy(buf, t, left, i);
    };
    // On their way together: the first K tile, the queries, the second K and the first V.
    wait_vmcnt<0>();   // (the item before's stores: the partial counts below are of copies alone)
    if (grp == 0 && !narrow) copy_tile(kb0, tile_at(0), 0);
    bf16x8 qf[NSTEP];
    if (my_row < nrows) {
      const __bf16 *rp = (const __bf16 *)p.q + (((int64_t)it.tok0 + my_t) * Hq + it.kvh * g + (my_row - my_t * g)) * D;
#pragma unroll
      for (int st = 0; st < NSTEP; ++st) qf[st] = *reinterpret_cast<const bf16x8 *>(rp + st * 16 + G * 8);
    } else {
#pragma unroll
      for (int st = 0; st < NSTEP; ++st) qf[st] = Mma<__bf16>::zero();
    }
    Tile next;   // granules of the tile copied next, a tile ahead of their use
    if (!narrow) {
      if (grp == 0) copy_tile(kb1, tile_at(min(1, nt - 1)), 1);
      else copy_tile(vb0, tile_at(0), 0);
      next = tile_at(min(grp == 0 ? 2 : 1, nt - 1));
      wait_vmcnt<PER>();   // the first K and the queries
    }

    f32x16 oacc[DT];
    float m_run = -INFINITY, l_run = 0.0f;   // exponent offset of this lane's row, row sum of its keys
    auto live = [&](int j) __attribute__((always_inline)) { return wave_active && (it.tile0 + j) * kKT <= last_hi; };
    constexpr int kPieces = PER;             // copy instructions of a softmax phase
    static_assert(16 % kPieces == 0, "copies spread over the 16 exponential pairs");

#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
    if (narrow) {
      // Of the range's pieces of 32 keys, wave w takes those w / rgs, w / rgs +
      // 8 / rgs, ..., by itself: its K and V rows travel through registers, a piece
      // ahead of their use, to 32 rows of LDS of its own, and no barrier is met.
      constexpr int LOADS = 32 / RPI, HB = 32 * D * 2;   // load instructions and bytes of a piece's K or V rows
      const int strand = wave / rgs, strands = kNW / rgs, pieces = 2 * nt;
      auto tile_of = [&](int i) __attribute__((always_inline)) { return i == 0 ? kb0 : i == 1 ? kb1 : i == 2 ? kb2 : vb0; };
      char *const own = tile_of(wave >> 1) + (wave & 1) * HB;
      int voff[LOADS / 2];
#pragma unroll
      for (int l = 0; l < LOADS / 2; ++l) voff[l] = (l * RPI + lane / CPR) * row_bytes + (lane % CPR) * 16;
      const uint64_t kv_off = (uint64_t)it.kvh * (D * 2);
      uint32_t ga = 0, gb = 0;   // the granules of the piece loaded next
      auto granules_of = [&](int i) __attribute__((always_inline)) {
        const int at = it.granule0 + 4 * it.tile0 + 2 * min(i, pieces - 1);
        ga = load_const(p.granules, at);
        gb = load_const(p.granules, at + 1);
      };
      u32x4 kr[LOADS], vr[LOADS];
      auto load = [&](const void *pages, int i, u32x4 (&r)[LOADS]) __attribute__((always_inline)) {
        const int rows = i < pieces ? it.kv_len - it.tile0 * kKT - 32 * i : 0;   // (rows behind the last key read as zero)
        auto granule = [&](uint32_t gr, int left, int l0) __attribute__((always_inline)) {
          const BufRsrc rs = make_rsrc((const void *)((uint64_t)pages + kv_off + ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(gr) << 11)),
                                       __builtin_amdgcn_readfirstlane(left > 0 ? (min(left, 16) - 1) * row_bytes + D * 2 : 0));
#pragma unroll
          for (int l = 0; l < LOADS / 2; ++l) r[l0 + l] = __builtin_amdgcn_raw_buffer_load_b128(rs, voff[l], 0, 0);
        };
        granule(ga, rows, 0);
        granule(gb, rows - 16, LOADS / 2);
        asm volatile("" ::: "memory");   // (in this order, so that each use waits for its own)
      };
      auto to_lds = [&](const u32x4 (&r)[LOADS]) __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int l = 0; l < LOADS; ++l) *reinterpret_cast<u32x4 *>(own + swz_off<D>(l * RPI + lane / CPR, lane % CPR)) = r[l];
        asm volatile("" ::: "memory");   // (the wave's other lanes read it; its LDS operations stay in order)
      };
      granules_of(strand);
      load(p.k_pages, strand, kr);
      load(p.v_pages, strand, vr);
      granules_of(strand + strands);
#pragma unroll 1
      for (int i = strand; i < pieces; i += strands) {
        const int key0 = it.tile0 * kKT + 32 * i;
        if (!wave_active || key0 > last_hi) break;
        wait_vmcnt<LOADS>();   // (the compiler's own wait is for all loads)
        to_lds(kr);
        load(p.k_pages, i + strands, kr);
        f32x16 s = zero16();
#pragma unroll
        for (int st = 0; st < NSTEP; ++st) s = Mma<__bf16>::run(row_frag_at<D>(own, ro, 0, st), qf[st], s);
        wait_vmcnt<LOADS>();
        to_lds(vr);
        load(p.v_pages, i + strands, vr);
        granules_of(i + 2 * strands);
        if (key0 + 31 > last_lo) mask_piece(before + my_t - key0, G, s);
        const float mt = piece_max(s, c);
        if (wave_any(mt > m_run)) {
          const float m_new = fmaxf(m_run, mt);
          const float alpha = fast_exp2(m_run - m_new);   // (a row that has seen nothing yet: O and l are zero)
          m_run = m_new;
          l_run = m_new == -INFINITY ? 0.0f : l_run * alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) oacc[dt] *= m_new == -INFINITY ? 0.0f : alpha;
        }
        bf16x8 pf[2];
        l_run += piece_weights(c, m_run == -INFINITY ? 0.0f : m_run, s, pf);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) oacc[dt] = Mma<__bf16>::run(tr_frag_at<D>(own, to, 16 * h, dt), pf[h], oacc[dt]);
      }
      // The upper half of the waves gives its sums to the lower half, until one
      // wave has those of each group of rows.
#pragma unroll 1
      for (int h = kNW / 2; h >= rgs; h >>= 1) {
        lds_barrier();
        char *const slot = tile_of(wave & (h - 1)) + lane * 16;   // four registers of 64 lanes are 1 KiB
        float2 *const ml = reinterpret_cast<float2 *>(vb1) + (wave & (h - 1)) * 64 + lane;
        if (wave >= h && wave < 2 * h) {
          *ml = float2{m_run, l_run};
#pragma unroll
          for (int i = 0; i < 4 * DT; ++i) {
            const f32x16 &o = oacc[i / 4];
            const int e = 4 * (i % 4);
            *reinterpret_cast<f32x4 *>(slot + i * 1024) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
          }
        }
        lds_barrier();
        if (wave < h) {
          const float2 other = *ml;
          const float m_new = fmaxf(m_run, other.x), mu = m_new == -INFINITY ? 0.0f : m_new;
          const float wa = fast_exp2(m_run - mu), wb = fast_exp2(other.x - mu);
          m_run = m_new;
          l_run = l_run * wa + other.y * wb;
#pragma unroll
          for (int i = 0; i < 4 * DT; ++i) {
            f32x16 &o = oacc[i / 4];
            const f32x4 x = *reinterpret_cast<const f32x4 *>(slot + i * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[4 * (i % 4) + e] = o[4 * (i % 4) + e] * wa + x[e] * wb;
          }
        }
      }
    } else {
      f32x16 s0 = zero16(), s1 = zero16();
      bf16x8 pf[2][2];
      auto no_weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int s = 0; s < 2; ++s) pf[a][s] = Mma<__bf16>::zero();
      };
      no_weights();
      // (Works on a copy of the scores, as nothing needs them afterwards: written in
      // place they were moved between registers where the variants meet, 2-3 % of all.)
      auto softmax = [&](auto MASK, int lim, auto &&piece) __attribute__((always_inline)) {
        f32x16 t0 = s0, t1 = s1;
        if constexpr (decltype(MASK)::value) fwd_mask(lim, G, t0, t1);
        // Only until every row of the wave has seen a key.
        if (wave_any(m_run == -INFINITY)) {
          const float mt = fwd_tile_max(t0, t1, c);
          m_run = (m_run == -INFINITY) ? mt : m_run;
        }
        const float mu = (m_run == -INFINITY) ? 0.0f : m_run;
        l_run += fwd_weights<kPieces>(c, mu, t0, t1, pf, piece);
      };
      auto gphase = [&](int j, const char *kb, const char *vbp) __attribute__((always_inline)) {
        if (j <= nt && wave_active) fwd_matrix_phase<D>(kb, vbp, ro, to, qf, pf, s0, s1, oacc);
      };
      auto xphase = [&](int j, auto &&piece) __attribute__((always_inline)) {
        auto all_pieces = [&]() __attribute__((always_inline)) {
#pragma unroll
          for (int n = 0; n < kPieces; ++n) piece(n);
        };
        if (j < 0 || j >= nt) {
          all_pieces();
          return;
        }
        if (!live(j)) {
          no_weights();
          all_pieces();
          return;
        }
        const int key0 = (it.tile0 + j) * kKT;
        if (key0 + kKT - 1 > last_lo) softmax(std::true_type{}, before + my_t - key0, piece);
        else softmax(std::false_type{}, kKT - 1, piece);
      };
      // The softmax of tile j, with the copies of this group's tile jc spread over
      // it; at its end the copies of the phase before are waited for.
      auto xcopy = [&](int j, int jc, char *buf) __attribute__((always_inline)) {
        const Tile t = next;
        next = tile_at(min(jc + 1, nt - 1));
        const int left = bytes_left(jc);
        xphase(j, [&](int n) __attribute__((always_inline)) { copy(buf, t, left, n); });
        wait_vmcnt<PER>();
      };

      // (At least one tile: the host lists no empty range.) G_0 multiplies V
      // buffer 2 by P = 0: clear it so no stale bit pattern (a NaN) can reach O.
      for (int i = tid; i < TB / 16; i += kFastThreads) reinterpret_cast<uint4 *>(vb2)[i] = uint4{0, 0, 0, 0};
      lds_barrier();
      // Phase 2i: G_i beside X_{i-1}, phase 2i+1: X_i beside G_i. G_i reads K_i from
      // kb[i%3] and V_{i-1} from vb[(i-1)%3]. V_{i+1} is copied in phase 2i, to where
      // V_{i-2} was read until phase 2i-1, and waited for in phase 2i+2; K_{i+2} in
      // phase 2i+1, to where K_{i-1} was read until phase 2i-1, and waited for in
      // phase 2i+3. Six phases per iteration (three tiles), so every buffer is a
      // fixed LDS address.
      auto run = [&](auto GROUP_A) __attribute__((always_inline)) {
        constexpr bool A = decltype(GROUP_A)::value;
        auto even = [&](int i, const char *kbi, const char *vbp, char *vbn) __attribute__((always_inline)) {
          if constexpr (A) gphase(i, kbi, vbp);
          else xcopy(i - 1, i + 1, vbn);
          lds_barrier();
        };
        auto odd = [&](int i, const char *kbi, const char *vbp, char *kbn) __attribute__((always_inline)) {
          if constexpr (A) xcopy(i, i + 2, kbn);
          else gphase(i, kbi, vbp);
          lds_barrier();
        };
        for (int i = 0; i <= nt; i += 3) {
          even(i, kb0, vb2, vb1);
          odd(i, kb0, vb2, kb2);
          if (i + 1 > nt) break;
          even(i + 1, kb1, vb0, vb2);
          odd(i + 1, kb1, vb0, kb0);
          if (i + 2 > nt) break;
          even(i + 2, kb2, vb1, vb0);
          odd(i + 2, kb2, vb1, kb1);
        }
      };
      if (grp == 0) run(std::true_type{});
      else run(std::false_type{});
      wait_vmcnt<0>();
    }

    // Every wave reaches this point. A row sum that reached 2^kRefMargin or
    // overflowed needs the exact online softmax, an O that is not finite may come
    // from a key that its row does not see: the workgroup takes its tiles again,
    // one after the other.
    bool again = ((__float_as_uint(l_run) >> 23) & 0xffu) >= 127u + (unsigned)kRefMargin;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) again |= (__float_as_uint(oacc[dt][i]) & 0x7f800000u) == 0x7f800000u;
    again = again && (!narrow || wave < rgs);
    if (__syncthreads_or(again ? 1 : 0)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
      m_run = -INFINITY;
      l_run = 0.0f;
#pragma unroll 1
      for (int j = 0; j < nt; ++j) {
        lds_barrier();   // every wave is done with the tile before
        copy_tile(grp == 0 ? kb0 : vb0, tile_at(j), j);
        wait_vmcnt<0>();
        lds_barrier();
        if (!live(j)) continue;
        const int key0 = (it.tile0 + j) * kKT, lim = before + my_t - key0;
        const bool part = key0 + kKT - 1 > last_lo;   // some row sees the tile in part
        f32x16 s0 = zero16(), s1 = zero16();
#pragma unroll
        for (int st = 0; st < NSTEP; ++st) {
          s0 = Mma<__bf16>::run(row_frag_at<D>(kb0, ro, 0, st), qf[st], s0);
          s1 = Mma<__bf16>::run(row_frag_at<D>(kb0, ro, 32, st), qf[st], s1);
        }
        if (part) fwd_mask(lim, G, s0, s1);
        const float m_new = fmaxf(m_run, fwd_tile_max(s0, s1, c));
        const float mu = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = fast_exp2(m_run - mu);
        m_run = m_new;
        bf16x8 pf[2][2];
        l_run = l_run * alpha + fwd_weights<1>(c, mu, s0, s1, pf, [](int) {});
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
        const bool odd = part && has_odd<D>(vb0, lane);
        if (odd) add_odd<D>(vb0, lim, G, oacc);
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              bf16x8 vf = tr_frag_at<D>(vb0, to, 32 * a + 16 * h, dt);
              if (odd) vf = finite_only(vf);
              oacc[dt] = Mma<__bf16>::run(vf, pf[a][h], oacc[dt]);
            }
      }
      lds_barrier();   // (the next item's copies go to the same tiles)
    }

    const float lt = l_run + xor32(l_run);
    const float m_out = m_run;
    // (Read anew, again: nothing of this is held through the tile loop.)
    const ChunkParams pe = load_kernarg<ChunkParams>();
    const DevChunkItem ie = chunk_item<DIRECT>(pe, at);
    at = __builtin_amdgcn_readfirstlane(ie.next);
    int te = threadIdx.x;
    asm volatile("" : "+v"(te));
    const int ge = pe.g, r = ie.row0 + (te >> 6) * kFastRowsPerWave + (te & 31), Ge = te >> 5 & 1;
    if (r >= ie.row1) continue;
    const int t = r / ge, h = ie.kvh * ge + (r - t * ge);
    // (A piece of a split may hold no key that the row sees. A NaN sum stays NaN.)
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    const float lse = lt == 0.0f ? -INFINITY : (m_out + log2f(lt)) * kLn2;
    auto store = [&](auto *op) __attribute__((always_inline)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          store4(op + dt * 32 + crow(j, Ge), oacc[dt][j] * inv, oacc[dt][j + 1] * inv, oacc[dt][j + 2] * inv, oacc[dt][j + 3] * inv);
    };
    if (ie.part < 0) {
      store((__bf16 *)pe.o + (((int64_t)ie.tok0 + t) * (pe.Hkv * ge) + h) * D);
      if (Ge == 0 && pe.lse != nullptr) pe.lse[(int64_t)h * pe.Tq + ie.tok0 + t] = lse;
    } else {
      const int64_t R = (int64_t)ie.part * pe.part_rows + (r - ie.row0);
      store(pe.part_o + R * D);
      if (Ge == 0) pe.part_lse[R] = lse;
    }
  }
}

// The partials of a block of rows, weighted by their LSE. A row is D/4 lanes of 4
// channels each, GR of these groups taking every GR-th partial; their sums meet
// in LDS. Blocks of at most kChunkFewRows rows come first in the list and have
// units for those only, so that single tokens do not cost a chunk's workgroups.
template <int D, int GR>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p, int few) {
  constexpr int CPR = D / 4;
  constexpr int RPW = 256 / (CPR * GR);   // rows per workgroup
  constexpr int UF = kChunkFewRows / RPW, UA = kFastRowsPerWg / RPW;   // units of a block
  __shared__ f32x4 acc_l[256];
  __shared__ float w_l[256];
  const int tid = threadIdx.x, c4 = tid % CPR, gr = (tid / CPR) % GR;
  const int bid = blockIdx.x;
  const int which = bid < few * UF ? bid / UF : few + (bid - few * UF) / UA;
  const int unit = bid < few * UF ? bid % UF : (bid - few * UF) % UA;
  const DevChunkMerge mg = load_const(p.merges, which);
  const int nrows = mg.row1 - mg.row0;
  if (unit * RPW >= nrows) return;
  const int r = unit * RPW + tid / (CPR * GR);
  const int64_t R = (int64_t)mg.part0 * p.part_rows + min(r, nrows - 1);
  const float *lses = p.part_lse + R;
  float mx = -INFINITY;
  for (int i = c4; i < mg.nparts; i += CPR) mx = fmaxf(mx, lses[i * p.part_rows]);
#pragma unroll
  for (int m = CPR / 2; m >= 1; m >>= 1) mx = fmaxf(mx, __shfl_xor(mx, m, CPR));
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float w_sum = 0.0f;
#pragma unroll 4
  for (int i = gr; i < mg.nparts; i += GR) {
    const float ls = lses[i * p.part_rows];
    const float w = ls == -INFINITY ? 0.0f : expf(ls - mx);
    w_sum += w;
    acc += w * *reinterpret_cast<const f32x4 *>(p.part_o + (R + (int64_t)i * p.part_rows) * D + 4 * c4);
  }
  if constexpr (GR > 1) {
    acc_l[tid] = acc;
    w_l[tid] = w_sum;
    __syncthreads();
    if (gr == 0) {
#pragma unroll
      for (int k = 1; k < GR; ++k) {
        acc += acc_l[tid + k * CPR];
        w_sum += w_l[tid + k * CPR];
      }
    }
  }
  if (gr != 0 || r >= nrows) return;
  const float inv = w_sum == 0.0f ? 0.0f : 1.0f / w_sum;
  const int row = mg.row0 + r, t = row / p.g, h = mg.kvh * p.g + (row - t * p.g), Hq = p.Hkv * p.g;
  store4((__bf16 *)p.o + (((int64_t)mg.tok0 + t) * Hq + h) * D + 4 * c4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  if (c4 == 0 && p.lse != nullptr) p.lse[(int64_t)h * p.Tq + mg.tok0 + t] = w_sum == 0.0f ? -INFINITY : mx + logf(w_sum);
}

// Copies the launch tables to the workspace and then says so to the host, which
// may fill their slot anew: a flag of each workgroup in host memory instead of an
// event, whose barrier kept the next kernel waiting for 6 us. Bound by the latency
// of the host link, so a workgroup for every 4 KiB: 53 KB take 4 us, 11 us with
// one workgroup.
__global__ __launch_bounds__(256) void table_flag_kernel(uint4 *dst, const uint4 *src, int64_t n16, uint32_t *flags, uint32_t value) {
#pragma unroll 4
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n16; i += gridDim.x * 256) dst[i] = src[i];
  __syncthreads();   // (every load has returned)
  if (threadIdx.x == 0) __hip_atomic_store(flags + blockIdx.x, value, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_SYSTEM);
}

template <int D, int GR>
void launch_chunk_merge_t(const ChunkParams &p, int few, int n_merges, hipStream_t s) {
  constexpr int RPW = 256 / (D / 4 * GR);
  const int64_t grid = (int64_t)few * (kChunkFewRows / RPW) + (int64_t)(n_merges - few) * (kFastRowsPerWg / RPW);
  hipLaunchKernelGGL((chunk_merge_kernel<D, GR>), dim3((unsigned)grid), dim3(256), 0, s, p, few);
}

}  // namespace

hipError_t launch_chunk_bf16(const ChunkParams &p, const ChunkDirect *direct, int D, int n_wgs, hipStream_t s) {
  const dim3 grid((unsigned)n_wgs), threads(kFastThreads);
  if (direct) {
    if (D == 64) hipLaunchKernelGGL((chunk_bf16_kernel<64, true>), grid, threads, 0, s, p, *direct);
    else hipLaunchKernelGGL((chunk_bf16_kernel<128, true>), grid, threads, 0, s, p, *direct);
  } else {
    if (D == 64) hipLaunchKernelGGL((chunk_bf16_kernel<64, false>), grid, threads, 0, s, p, NoTables{});
    else hipLaunchKernelGGL((chunk_bf16_kernel<128, false>), grid, threads, 0, s, p, NoTables{});
  }
  return hipGetLastError();
}

// Groups a row: eight where each takes two partials or more (few rows, then), one
// where there are few partials but many rows (15.5 us with two and 12.3 with one for
// 16 requests' 15 MB in up to 3 partials; 7.0 and 7.5 for 132 rows in 9).
hipError_t launch_chunk_merge_bf16(const ChunkParams &p, int D, int few, int n_merges, int max_parts, hipStream_t s) {
  auto launch = [&](auto G) {
    constexpr int GR = decltype(G)::value;
    if (D == 64) launch_chunk_merge_t<64, GR>(p, few, n_merges, s);
    else launch_chunk_merge_t<128, GR>(p, few, n_merges, s);
  };
  if (max_parts >= 16) launch(std::integral_constant<int, 8>{});
  else if (max_parts >= 6) launch(std::integral_constant<int, 2>{});
  else launch(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

hipError_t launch_table_flags(void *dst, const void *src, size_t bytes, uint32_t *flags, int n_flags, uint32_t value, hipStream_t s) {
  int64_t n16 = (int64_t)(bytes / 16);
  void *args[] = {&dst, &src, &n16, &flags, &value};
  // (This launch's own status, not an error that was left before: the caller counts on the flags if it succeeds.)
  const hipError_t e = hipLaunchKernel((const void *)table_flag_kernel, dim3((unsigned)n_flags), dim3(256), args, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

}  // namespace cas
