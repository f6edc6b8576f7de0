// Attention over sequences of different lengths in fp32: the three kernels of seq_attention.h (which see for the mathematics)
// on the 32x32x2 fp32 MFMA.  Its accumulator layout is that of the 16-bit instruction; its operands are one value a lane, lane
// l giving row l % 32 at contraction index l / 32, so a product over columns takes columns x and 4 + x of every 8 from
// the two halves (one 16-byte read feeds four instructions), and a product over the other tile's rows takes the rows 8 (r / 4) + r % 4
// and those + 4 that accumulator register r holds in the two halves.
// Bound by the fp32 matrix rate, a sixteenth of the 16-bit one: tiles of 32 rows, loaded through registers one tile ahead.
// PARTS = 2, where the longest sequence has 33 to 64 rows: the waves that have no rows of the workgroup's 128 take every other tile of the
// others' rows, and the two results are put together in LDS.  4 sequences of 64, 2 heads of 64, dropped: forward 9.0 -> 7.1 us,
// dQ 12.3 -> 11.1, dK and dV 13.3 -> 10.6; 256 ragged ones, 12 heads: 56 -> 56, 89 -> 82, 103 -> 83.  (Of 32 or fewer rows there is one
// tile, and the second buffers only cost: 34 -> 45, 54 -> 63, 62 -> 68.)  Its dK / dV kernel at 64 columns takes 257 registers, dropped 262: one wave a SIMD.
#pragma once
#include "seq_attention.h"

namespace sattn {

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <int DP>
struct ImgF {
  static constexpr int ROWS = 32, PITCH = DP + 4;   // floats: 16-byte reads of 32 rows spread over the banks
  static constexpr int FLOATS = ROWS * PITCH, PER = ROWS * DP / 4 / 256;   // 16-byte chunks a thread carries
  f32x4 r[PER];
  __device__ __forceinline__ void load(const float* base, long long ld, int rows, int d) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int u = i * 256 + threadIdx.x, row = u / (DP / 4), col = u % (DP / 4) * 4;
      r[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (row < rows && col < d) r[i] = *(const f32x4*)(base + (long long)row * ld + col);
    }
  }
  __device__ __forceinline__ void put(float* img) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int u = i * 256 + threadIdx.x, row = u / (DP / 4), col = u % (DP / 4) * 4;
      *(f32x4*)(img + row * PITCH + col) = r[i];
    }
  }
  // columns 8 s + 4 (lane / 32) .. of row lane % 32
  static __device__ __forceinline__ f32x4 frag(const float* img, int s, int lane) {
    return *(const f32x4*)(img + (lane & 31) * PITCH + 8 * s + 4 * (lane >> 5));
  }
  // column 32 t + lane % 32 of the row that accumulator register r names
  static __device__ __forceinline__ float across(const float* img, int r, int t, int lane) {
    return img[(8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * PITCH + 32 * t + (lane & 31)];
  }
  static __device__ __forceinline__ void row(const float* p, bool live, int d, int lane, f32x4 (&f)[DP / 8]) {
#pragma unroll
    for (int s = 0; s < DP / 8; ++s) {
      const int col = 8 * s + 4 * (lane >> 5);
      f[s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live && col < d) f[s] = *(const f32x4*)(p + col);
    }
  }
  static __device__ __forceinline__ void store(const f32x16 (&acc)[DP / 32], float* p, int d, int lane, float scale) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        const int col = t * 32 + blk * 8 + 4 * (lane >> 5);
        if (col < d) *(f32x4*)(p + col) = f32x4{acc[t][4 * blk], acc[t][4 * blk + 1], acc[t][4 * blk + 2], acc[t][4 * blk + 3]} * scale;
      }
  }
};
// s += rows of img . f (over columns)
template <int DP>
__device__ __forceinline__ void columns_f32(const float* img, const f32x4 (&f)[DP / 8], f32x16& s, int lane) {
#pragma unroll
  for (int st = 0; st < DP / 8; ++st) {
    const f32x4 x = ImgF<DP>::frag(img, st, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = mfma_f32(x[i], f[st][i], s);
  }
}
// acc += img^T p (over the rows that p's registers hold)
template <int DP>
__device__ __forceinline__ void rows_f32(const float* img, const f32x16& p, f32x16 (&acc)[DP / 32], int lane) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = mfma_f32(ImgF<DP>::across(img, r, t, lane), p[r], acc[t]);
}

// the second part's accumulators (and what else each lane has) to the first: out by the waves with part = 1, in by their neighbours
template <int N>
__device__ __forceinline__ void give(float* to, const f32x16 (&acc)[N], int lane) {
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) to[(t * 16 + r) * 64 + lane] = acc[t][r];
}

template <int DP, bool DROP, int PARTS>
__global__ __launch_bounds__(256) void seq_fwd_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  __shared__ __attribute__((aligned(16))) float lds[PARTS * 2 * I::FLOATS];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group, a.splits_fwd);
  const int split = at.split, blk = nblk - 1 - at.turn, b = at.b, hk = at.hk, h = hk * group + at.head, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = wave / (4 / PARTS), q0 = base_q + wave % (4 / PARTS) * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const float* kb_ = (const float*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const float* vb_ = (const float*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128) : n, all_tiles = (last + 31) / 32;
  const int from = all_tiles * split / a.splits_fwd, tiles = all_tiles * (split + 1) / a.splits_fwd;
  f32x4 qf[DP / 8];
  I::row((const float*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf);
  f32x16 o[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) o[t] = zero16();
  float m = -INFINITY, sum = 0.f;
  const float c = a.scale * LOG2E;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  I kr[PARTS], vr[PARTS];
  const auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const int k0 = (t + u) * 32;   // (n - k0 <= 0: zeros)
      kr[u].load(kb_ + (long long)k0 * a.ldk, a.ldk, n - k0, a.d);
      vr[u].load(vb_ + (long long)k0 * a.ldv, a.ldv, n - k0, a.d);
    }
  };
  const float *Ks = lds + part * 2 * I::FLOATS, *Vs = Ks + I::FLOATS;   // this wave's of the tiles that are in
  fetch(from);
  for (int t = from; t < tiles; t += PARTS) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      kr[u].put(lds + u * 2 * I::FLOATS);
      vr[u].put(lds + u * 2 * I::FLOATS + I::FLOATS);
    }
    __syncthreads();
    if (t + PARTS < tiles) fetch(t + PARTS);
    const int k0 = (t + part) * 32;
    if (!active || t + part >= tiles || (a.causal && k0 >= q0 + 32)) continue;
    f32x16 s = zero16();
    columns_f32<DP>(Ks, qf, s, lane);
    if (k0 + 32 > n || (a.causal && k0 + 31 > q0)) {
      const int lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= lim) s[r] = -INFINITY;
    }
    float cm = m;
#pragma unroll
    for (int r = 0; r < 16; ++r) cm = fmaxf(cm, s[r]);
    cm = half_max(cm);
    if (__any(cm > m)) {
      const float rescale = __builtin_amdgcn_exp2f((m - cm) * c);
      m = cm;
      sum *= rescale;
#pragma unroll
      for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t2][r] *= rescale;
    }
    // (the difference first: an fma with -m c would carry the rounding of that product, up to 2^-24 |m c|, into every exponent)
#pragma unroll
    for (int r = 0; r < 16; ++r) { s[r] = __builtin_amdgcn_exp2f((s[r] - m) * c); sum += s[r]; }
    if (DROP) {
      const u32x4 bytes = drop_bytes<true>(q0, k0, (uint32_t)bh, key, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = drop_keeps(bytes, r, a.drop) ? s[r] : 0.f;
    }
    rows_f32<DP>(Vs, s, o, lane);
  }
  if (PARTS == 2) {   // (the first part has every row's first key)
    float* mine = lds + (wave & 1) * (DP / 32 * 16 + 2) * 64;
    __syncthreads();
    if (part == 1) {
      give(mine, o, lane);
      mine[DP / 32 * 1024 + lane] = m;
      mine[DP / 32 * 1024 + 64 + lane] = sum;
    }
    __syncthreads();
    if (part == 1) return;
    const float m2 = mine[DP / 32 * 1024 + lane], top = fmaxf(m, m2);
    const float f = __builtin_amdgcn_exp2f((m - top) * c), f2 = __builtin_amdgcn_exp2f((m2 - top) * c);
    sum = sum * f + mine[DP / 32 * 1024 + 64 + lane] * f2;
    m = top;
#pragma unroll
    for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t2][r] = o[t2][r] * f + mine[(t2 * 16 + r) * 64 + lane] * f2;
  }
  if (!active) return;
  const float l = half_sum(sum), kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  if (q >= n) return;
  if (a.splits_fwd > 1) {   // (a split without a key that the row sees: l = 0)
    const long long row = (long long)split * a.rows + sq.first + q, stat = ((long long)split * a.heads + h) * a.rows + sq.first + q;
    I::store(o, a.part + row * ((long long)a.heads * a.d) + (long long)h * a.d, a.d, lane, l == 0.f ? 0.f : kept / l);
    if (lane < 32) { a.part_m[stat] = m; a.part_sum[stat] = l; }
    return;
  }
  I::store(o, (float*)a.out + (sq.first + q) * a.ldo + (long long)h * a.d, a.d, lane, kept / l);
  if (a.lse && lane < 32) a.lse[(long long)h * a.rows + sq.first + q] = m * a.scale + __builtin_amdgcn_logf(l) * LN2;
}

template <int DP, bool DROP, int PARTS>
__global__ __launch_bounds__(256) void seq_bwd_dq_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  __shared__ __attribute__((aligned(16))) float lds[PARTS * 2 * I::FLOATS];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group, a.splits_dq);
  const int split = at.split, blk = nblk - 1 - at.turn, b = at.b, hk = at.hk, h = hk * group + at.head, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = wave / (4 / PARTS), q0 = base_q + wave % (4 / PARTS) * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const float* kb_ = (const float*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const float* vb_ = (const float*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128) : n, all_tiles = (last + 31) / 32;
  const int from = all_tiles * split / a.splits_dq, tiles = all_tiles * (split + 1) / a.splits_dq;
  f32x4 qf[DP / 8], gf[DP / 8];
  const float* orow = (const float*)a.o + (sq.first + q) * a.ldo + (long long)h * a.d;
  I::row((const float*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf);
  I::row((const float*)a.dout + (sq.first + q) * a.lddo + (long long)h * a.d, q < n, a.d, lane, gf);
  float D = 0.f, lse = 0.f;
  if (q < n) {
#pragma unroll
    for (int s = 0; s < DP / 8; ++s) {
      const int col = 8 * s + 4 * (lane >> 5);
      if (col < a.d) {
        const f32x4 ov = *(const f32x4*)(orow + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) D = fmaf(gf[s][i], ov[i], D);
      }
    }
    lse = a.lse[(long long)h * a.rows + sq.first + q];
  }
  D = half_sum(D);
  if (q < n && lane < 32 && part == 0 && split == 0) a.delta[(long long)h * a.rows + sq.first + q] = D;
  f32x16 dq[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) dq[t] = zero16();
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  I kr[PARTS], vr[PARTS];
  const auto fetch = [&](int t) {
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const int k0 = (t + u) * 32;   // (n - k0 <= 0: zeros)
      kr[u].load(kb_ + (long long)k0 * a.ldk, a.ldk, n - k0, a.d);
      vr[u].load(vb_ + (long long)k0 * a.ldv, a.ldv, n - k0, a.d);
    }
  };
  const float *Ks = lds + part * 2 * I::FLOATS, *Vs = Ks + I::FLOATS;   // this wave's of the tiles that are in
  fetch(from);
  for (int t = from; t < tiles; t += PARTS) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      kr[u].put(lds + u * 2 * I::FLOATS);
      vr[u].put(lds + u * 2 * I::FLOATS + I::FLOATS);
    }
    __syncthreads();
    if (t + PARTS < tiles) fetch(t + PARTS);
    const int k0 = (t + part) * 32;
    if (!active || t + part >= tiles || (a.causal && k0 >= q0 + 32)) continue;
    f32x16 s = zero16(), g = zero16();
    columns_f32<DP>(Ks, qf, s, lane);
    columns_f32<DP>(Vs, gf, g, lane);
    const int lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
    u32x4 bytes;
    if (DROP) bytes = drop_bytes<true>(q0, k0, (uint32_t)bh, key, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float p = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -lse) * LOG2E);
      p = 8 * (r >> 2) + (r & 3) >= lim ? 0.f : p;
      g[r] = p * (DROP ? (drop_keeps(bytes, r, a.drop) ? fmaf(g[r], kept, -D) : -D) : g[r] - D);
    }
    rows_f32<DP>(Ks, g, dq, lane);
  }
  if (PARTS == 2) {
    float* mine = lds + (wave & 1) * DP / 32 * 1024;
    __syncthreads();
    if (part == 1) give(mine, dq, lane);
    __syncthreads();
    if (part == 1) return;
#pragma unroll
    for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[t2][r] += mine[(t2 * 16 + r) * 64 + lane];
  }
  if (!active || q >= n) return;
  if (a.splits_dq > 1) {
    const long long row = (long long)split * a.rows + sq.first + q;
    I::store(dq, a.part + row * ((long long)a.heads * a.d) + (long long)h * a.d, a.d, lane, a.scale);
    return;
  }
  I::store(dq, (float*)a.dq + (sq.first + q) * a.lddq + (long long)h * a.d, a.d, lane, a.scale);
}

template <int DP, bool DROP, int PARTS>
__global__ __launch_bounds__(256) void seq_bwd_dkv_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  constexpr int STAGE = 2 * I::FLOATS + 64;   // Q, dO, and 32 rows' lse and D
  __shared__ __attribute__((aligned(16))) float lds[PARTS * STAGE];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, 1, a.splits_dkv);
  const int split = at.split, blk = at.turn, b = at.b, hk = at.hk;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_k = blk * 128;
  if (base_k >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = wave / (4 / PARTS), key0 = base_k + wave % (4 / PARTS) * 32, kk = key0 + (lane & 31);
  const bool active = key0 < n;
  const int t0 = a.causal ? base_k / 32 : 0, per_head = (n + 31) / 32 - t0, all_tiles = per_head * group;
  const int from = all_tiles * split / a.splits_dkv, tiles = all_tiles * (split + 1) / a.splits_dkv;   // this split's, of all heads' in turn
  I qr[PARTS], gr[PARTS];
  float stat = 0.f;
  const auto fetch = [&](int i) {
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const bool live = i + u < tiles;
      const int h = hk * group + (live ? (i + u) / per_head : 0), row0 = (t0 + (live ? (i + u) % per_head : 0)) * 32, rows = live ? n - row0 : 0;
      const long long tok = sq.first + row0;
      qr[u].load((const float*)a.q + tok * a.ldq + (long long)h * a.d, a.ldq, rows, a.d);
      gr[u].load((const float*)a.dout + tok * a.lddo + (long long)h * a.d, a.lddo, rows, a.d);
      if (threadIdx.x / 64 == u) {   // lse and D; rows past the sequence are zeros, which add nothing
        const int row = threadIdx.x & 31;
        stat = row < rows ? (lane < 32 ? a.lse : a.delta)[(long long)h * a.rows + tok + row] : 0.f;
      }
    }
  };
  fetch(from);
  f32x4 kf[DP / 8], vf[DP / 8];
  I::row((const float*)a.k + (sq.first + kk) * a.ldk + (long long)hk * a.d, kk < n, a.d, lane, kf);
  I::row((const float*)a.v + (sq.first + kk) * a.ldv + (long long)hk * a.d, kk < n, a.d, lane, vf);
  f32x16 dv[DP / 32], dk[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) { dv[t] = zero16(); dk[t] = zero16(); }
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  const float *Qs = lds + part * STAGE, *Gs = Qs + I::FLOATS, *Ls = Gs + I::FLOATS, *Ds = Ls + 32;
  for (int i0 = from; i0 < tiles; i0 += PARTS) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      qr[u].put(lds + u * STAGE);
      gr[u].put(lds + u * STAGE + I::FLOATS);
      if (threadIdx.x / 64 == u) lds[u * STAGE + 2 * I::FLOATS + lane] = stat;   // (Ds follows Ls)
    }
    __syncthreads();
    if (i0 + PARTS < tiles) fetch(i0 + PARTS);
    const int i = i0 + part;
    if (!active || i >= tiles) continue;
    const int h = hk * group + i / per_head, row0 = (t0 + i % per_head) * 32;
    if (a.causal && row0 + 32 <= key0) continue;
    f32x16 s = zero16(), g = zero16();
    columns_f32<DP>(Qs, kf, s, lane);
    columns_f32<DP>(Gs, vf, g, lane);
    const int lim = a.causal ? kk - row0 - 4 * (lane >> 5) : -32;
    u32x4 bytes;
    if (DROP) bytes = drop_bytes<false>(row0, key0, (uint32_t)(b * a.heads + h), key, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
      const float D = Ds[row];
      float p = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -Ls[row]) * LOG2E);
      p = 8 * (r >> 2) + (r & 3) < lim ? 0.f : p;
      const bool keep = !DROP || drop_keeps(bytes, r, a.drop);
      g[r] = p * (DROP ? (keep ? fmaf(g[r], kept, -D) : -D) : g[r] - D);
      s[r] = keep ? p : 0.f;
    }
    rows_f32<DP>(Gs, s, dv, lane);
    rows_f32<DP>(Qs, g, dk, lane);
  }
  if (PARTS == 2) {
    float* mine = lds + (wave & 1) * DP / 32 * 2048;
    __syncthreads();
    if (part == 1) {
      give(mine, dv, lane);
      give(mine + DP / 32 * 1024, dk, lane);
    }
    __syncthreads();
    if (part == 1) return;
#pragma unroll
    for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dv[t2][r] += mine[(t2 * 16 + r) * 64 + lane];
        dk[t2][r] += mine[DP / 32 * 1024 + (t2 * 16 + r) * 64 + lane];
      }
  }
  if (!active || kk >= n) return;
  if (a.splits_dkv > 1) {
    const long long width = (long long)a.kv_heads * a.d, row = 2LL * split * a.rows + sq.first + kk;
    I::store(dv, a.part + row * width + (long long)hk * a.d, a.d, lane, kept);
    I::store(dk, a.part + (row + a.rows) * width + (long long)hk * a.d, a.d, lane, a.scale);
    return;
  }
  I::store(dv, (float*)a.dv + (sq.first + kk) * a.lddv + (long long)hk * a.d, a.d, lane, kept);
  I::store(dk, (float*)a.dk + (sq.first + kk) * a.lddk + (long long)hk * a.d, a.d, lane, a.scale);
}

}  // namespace sattn
