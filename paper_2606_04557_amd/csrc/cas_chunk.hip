// Attention of a chunk of new tokens over a paged KV cache (forward only; paper:
// Section "Inference", cartridges ahead of the prompt, causal masking of what
// follows).
//
// Query i of a request's n new tokens sees keys 0 .. L - n + i of its L. The g
// heads of a group share their KV head's keys, so a row is a (token, head) pair
// and a workgroup of eight waves takes 256 of them, 32 per wave, over a range of
// 64-key tiles: S^T = K Q^T, an online softmax (a lane owns one row; its partner
// lane 32 away the other keys of the tile), O^T += V^T P^T with P^T straight from
// the score registers. Tiles are gathered page by page: a copy instruction moves
// 4 or 8 key rows, which lie in one page since pages are multiples of 16.
#include "cas_device.h"

namespace cas {

namespace {

constexpr int kChunkWaves = 8;
constexpr int kKT = 64;

__device__ __forceinline__ bool odd16(unsigned bits) { return (bits & 0x7f80u) == 0x7f80u; }   // inf or NaN

// Whether a 64-key tile of V holds a value that is not finite (one wave).
template <int D>
__device__ __forceinline__ bool has_odd(const char *tile, int lane) {
  bool odd = false;
#pragma unroll 4
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

template <int D>
__global__ __launch_bounds__(kChunkWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void chunk_bf16_kernel(ChunkParams p) {
  constexpr int NSTEP = D / 16, DT = D / 32, TB = kKT * D * 2;
  constexpr int CPR = D / 8, RPI = 64 / CPR, NI = kKT / RPI / kChunkWaves;   // copy instructions of a tile per wave
  __shared__ __attribute__((aligned(1024))) char kb[2][TB];
  __shared__ __attribute__((aligned(1024))) char vb[2][TB];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = lane >> 5, n = lane & 31;
  const DevChunkItem it = load_const(p.items, (int)blockIdx.x);
  const int g = p.g, Hkv = p.Hkv, Hq = Hkv * g, P = p.page_size;
  const int nrows = min(it.len * g, it.row0 + kChunkWaves * 32);
  const int row0 = it.row0 + wave * 32, my_row = row0 + n;
  const int before = it.kv_len - it.len;                 // token t sees keys 0 .. before + t
  const bool active = row0 < nrows;
  const int lo = before + row0 / g, hi = before + (min(row0 + 32, nrows) - 1) / g;   // last keys of the wave's rows
  const int my_t = my_row / g, my_last = before + my_t;
  const int h = it.kvh * g + (my_row - my_t * g);
  const float c = p.scale_log2;

  RowOffsets<D> ro;
  ro.init(n, G);
  TrOffsets<D> to;
  to.init(lane);
  bf16x8 qf[NSTEP];
#pragma unroll
  for (int st = 0; st < NSTEP; ++st) qf[st] = Mma<__bf16>::zero();
  if (my_row < nrows) {
    const __bf16 *rp = (const __bf16 *)p.q + (((int64_t)it.tok0 + my_t) * Hq + h) * D;
#pragma unroll
    for (int st = 0; st < NSTEP; ++st) qf[st] = *reinterpret_cast<const bf16x8 *>(rp + st * 16 + G * 8);
  }

  // Rows at or past kv_len go through a resource that ends before them: zeros.
  const int row_bytes = Hkv * D * 2;
  auto copy = [&](const void *pool, char *tile_buf, int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int inst = wave + i * kChunkWaves, r0 = inst * RPI, key = tile * kKT + r0;
      const int valid = min(RPI, it.kv_len - key);
      const int page = load_const(p.page_ids, it.page0 + min(key, it.kv_len - 1) / P);
      const __bf16 *base = (const __bf16 *)pool + (((int64_t)page * P + (key & (P - 1))) * Hkv + it.kvh) * D;
      const int r = lane / CPR;
      dma16(make_rsrc(base, valid > 0 ? (valid - 1) * row_bytes + D * 2 : 0),
            r * row_bytes + (((lane % CPR) ^ swz<D>(r0 + r)) << 4), tile_buf + inst * 1024);
    }
  };

  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
  float m = -INFINITY, l = 0.0f;
  copy(p.k_pages, kb[0], it.tile0);
  copy(p.v_pages, vb[0], it.tile0);
  for (int tile = it.tile0; tile < it.tile1; ++tile) {
    const int cur = (tile - it.tile0) & 1;
    wait_vmcnt<0>();
    __syncthreads();
    if (tile + 1 < it.tile1) {
      copy(p.k_pages, kb[cur ^ 1], tile + 1);
      copy(p.v_pages, vb[cur ^ 1], tile + 1);
    }
    const int key0 = tile * kKT;
    if (!active || key0 > hi) continue;
    f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
    for (int st = 0; st < NSTEP; ++st)
#pragma unroll
      for (int a = 0; a < 2; ++a) s[a] = Mma<__bf16>::run(row_frag_at<D>(kb[cur], ro, 32 * a, st), qf[st], s[a]);
    if (key0 + kKT - 1 > lo) {
      const int lim = my_last - key0 - 4 * G;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[a][j] = 32 * a + crow(j, 0) <= lim ? s[a][j] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[a][j]);
    const float m_new = fmaxf(m, fmaxf(mx, xor32(mx)) * c);
    const float mu = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = fast_exp2(m - mu);
    float sum = 0.0f;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        s[a][j] = fast_exp2(fmaf(s[a][j], c, -mu));
        sum += s[a][j];
      }
    l = l * alpha + sum;
    m = m_new;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
    // A value that is not finite would reach, as 0 times it, the rows that do not
    // see its key. In tiles that some rows see in part such values are left out
    // of the product and added to the rows that do see them.
    const bool odd_values = key0 + kKT - 1 > lo && has_odd<D>(vb[cur], lane);
    if (odd_values) add_odd<D>(vb[cur], my_last - key0, G, oacc);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const bf16x8 pf = pack_bf16x8(s[a], st);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          bf16x8 vf = tr_frag_at<D>(vb[cur], to, 32 * a + 16 * st, dt);
          if (odd_values) vf = finite_only(vf);
          oacc[dt] = Mma<__bf16>::run(vf, pf, oacc[dt]);
        }
      }
  }
  if (my_row >= nrows) return;
  const float lt = l + xor32(l);
  const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
  const float lse = lt == 0.0f ? -INFINITY : (m + log2f(lt)) * kLn2;
  if (it.part < 0) {
    __bf16 *op = (__bf16 *)p.o + (((int64_t)it.tok0 + my_t) * Hq + h) * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 16; j += 4)
        store4(op + dt * 32 + crow(j, G), oacc[dt][j] * inv, oacc[dt][j + 1] * inv, oacc[dt][j + 2] * inv, oacc[dt][j + 3] * inv);
    if (G == 0 && p.lse != nullptr) p.lse[(int64_t)h * p.Tq + it.tok0 + my_t] = lse;
  } else {
    const int64_t R = (int64_t)it.part * (kChunkWaves * 32) + (my_row - it.row0);
    float *op = p.part_o + R * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 16; j += 4)
        store4(op + dt * 32 + crow(j, G), oacc[dt][j] * inv, oacc[dt][j + 1] * inv, oacc[dt][j + 2] * inv, oacc[dt][j + 3] * inv);
    if (G == 0) p.part_lse[R] = lse;
  }
}

// The partials of a block of rows, weighted by their LSE: D / 4 lanes per row,
// 4 channels each.
template <int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p) {
  constexpr int CPR = D / 4, RPW = 256 / CPR;
  const DevChunkMerge mg = load_const(p.merges, (int)blockIdx.y);
  const int c4 = threadIdx.x % CPR, r = blockIdx.x * RPW + threadIdx.x / CPR, row = mg.row0 + r;
  if (row >= mg.len * p.g) return;
  const int64_t R = (int64_t)mg.part0 * 256 + r;
  float mx = -INFINITY;
  for (int i = 0; i < mg.nparts; ++i) mx = fmaxf(mx, p.part_lse[R + 256 * i]);
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float w_sum = 0.0f;
  for (int i = 0; i < mg.nparts; ++i) {
    const float ls = p.part_lse[R + 256 * i];
    const float w = ls == -INFINITY ? 0.0f : expf(ls - mx);
    w_sum += w;
    acc += w * *reinterpret_cast<const f32x4 *>(p.part_o + (R + 256 * i) * D + 4 * c4);
  }
  const float inv = w_sum == 0.0f ? 0.0f : 1.0f / w_sum;
  const int t = row / p.g, h = mg.kvh * p.g + (row - t * p.g), Hq = p.Hkv * p.g;
  store4((__bf16 *)p.o + (((int64_t)mg.tok0 + t) * Hq + h) * D + 4 * c4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  if (c4 == 0 && p.lse != nullptr) p.lse[(int64_t)h * p.Tq + mg.tok0 + t] = w_sum == 0.0f ? -INFINITY : mx + logf(w_sum);
}

}  // namespace

hipError_t launch_chunk_bf16(const ChunkParams &p, int D, int n_items, hipStream_t s) {
  if (D == 64) hipLaunchKernelGGL(chunk_bf16_kernel<64>, dim3((unsigned)n_items), dim3(kChunkWaves * 64), 0, s, p);
  else hipLaunchKernelGGL(chunk_bf16_kernel<128>, dim3((unsigned)n_items), dim3(kChunkWaves * 64), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_chunk_merge_bf16(const ChunkParams &p, int D, int n_merges, hipStream_t s) {
  if (D == 64) hipLaunchKernelGGL(chunk_merge_kernel<64>, dim3(256 * 64 / 4 / 256, (unsigned)n_merges), dim3(256), 0, s, p);
  else hipLaunchKernelGGL(chunk_merge_kernel<128>, dim3(256 * 128 / 4 / 256, (unsigned)n_merges), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace cas
