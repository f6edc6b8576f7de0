// Attention over sequences of different lengths in fp32: the three kernels of seq_attention.h (which see for the mathematics)
// on the 32x32x2 fp32 MFMA.  Its accumulator layout is that of the 16-bit instruction; its operands are one value a lane, lane
// l giving row l % 32 at contraction index l / 32, so a product over columns takes columns x and 4 + x of every 8 from
// the two halves (one 16-byte read feeds four instructions), and a product over the other tile's rows takes the rows 8 (r / 4) + r % 4
// and those + 4 that accumulator register r holds in the two halves.
// Bound by the fp32 matrix rate, a sixteenth of the 16-bit one: tiles of 32 rows, loaded through registers one tile ahead.
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

template <int DP, bool DROP>
__global__ __launch_bounds__(256) void seq_fwd_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  __shared__ __attribute__((aligned(16))) float lds[2 * I::FLOATS];
  float *Ks = lds, *Vs = lds + I::FLOATS;
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group * nblk);
  const int blk = nblk - 1 - at.block % nblk;
  const int b = at.unit / a.kv_heads, hk = at.unit % a.kv_heads, h = hk * group + at.block / nblk, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const float* kb_ = (const float*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const float* vb_ = (const float*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128) : n, tiles = (last + 31) / 32;
  f32x4 qf[DP / 8];
  I::row((const float*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf);
  f32x16 o[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) o[t] = zero16();
  float m = -INFINITY, sum = 0.f;
  const float c = a.scale * LOG2E;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  I kr, vr;
  kr.load(kb_, a.ldk, min(32, n), a.d);
  vr.load(vb_, a.ldv, min(32, n), a.d);
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();
    kr.put(Ks);
    vr.put(Vs);
    __syncthreads();
    const int k0 = t * 32;
    if (t + 1 < tiles) {
      kr.load(kb_ + (long long)(k0 + 32) * a.ldk, a.ldk, min(32, n - k0 - 32), a.d);
      vr.load(vb_ + (long long)(k0 + 32) * a.ldv, a.ldv, min(32, n - k0 - 32), a.d);
    }
    if (!active || (a.causal && k0 >= q0 + 32)) continue;
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
  if (!active) return;
  const float l = half_sum(sum), kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  if (q >= n) return;
  I::store(o, (float*)a.out + (sq.first + q) * a.ldo + (long long)h * a.d, a.d, lane, kept / l);
  if (a.lse && lane < 32) a.lse[(long long)h * a.rows + sq.first + q] = m * a.scale + __builtin_amdgcn_logf(l) * LN2;
}

template <int DP, bool DROP>
__global__ __launch_bounds__(256) void seq_bwd_dq_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  __shared__ __attribute__((aligned(16))) float lds[2 * I::FLOATS];
  float *Ks = lds, *Vs = lds + I::FLOATS;
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group * nblk);
  const int blk = nblk - 1 - at.block % nblk;
  const int b = at.unit / a.kv_heads, hk = at.unit % a.kv_heads, h = hk * group + at.block / nblk, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const float* kb_ = (const float*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const float* vb_ = (const float*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128) : n, tiles = (last + 31) / 32;
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
  if (q < n && lane < 32) a.delta[(long long)h * a.rows + sq.first + q] = D;
  f32x16 dq[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) dq[t] = zero16();
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  I kr, vr;
  kr.load(kb_, a.ldk, min(32, n), a.d);
  vr.load(vb_, a.ldv, min(32, n), a.d);
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();
    kr.put(Ks);
    vr.put(Vs);
    __syncthreads();
    const int k0 = t * 32;
    if (t + 1 < tiles) {
      kr.load(kb_ + (long long)(k0 + 32) * a.ldk, a.ldk, min(32, n - k0 - 32), a.d);
      vr.load(vb_ + (long long)(k0 + 32) * a.ldv, a.ldv, min(32, n - k0 - 32), a.d);
    }
    if (!active || (a.causal && k0 >= q0 + 32)) continue;
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
  if (!active || q >= n) return;
  I::store(dq, (float*)a.dq + (sq.first + q) * a.lddq + (long long)h * a.d, a.d, lane, a.scale);
}

template <int DP, bool DROP>
__global__ __launch_bounds__(256) void seq_bwd_dkv_f32_kernel(const SeqAttnArgs a) {
  using I = ImgF<DP>;
  __shared__ __attribute__((aligned(16))) float lds[2 * I::FLOATS + 64];
  float *Qs = lds, *Gs = lds + I::FLOATS, *Ls = lds + 2 * I::FLOATS, *Ds = Ls + 32;
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, nblk);
  const int blk = at.block, b = at.unit / a.kv_heads, hk = at.unit % a.kv_heads;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_k = blk * 128;
  if (base_k >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key0 = base_k + wave * 32, kk = key0 + (lane & 31);
  const bool active = key0 < n;
  const int t0 = a.causal ? base_k / 32 : 0, per_head = (n + 31) / 32 - t0, tiles = per_head * group;
  I qr, gr;
  float stat = 0.f;
  const auto fetch = [&](int i) {
    const int h = hk * group + i / per_head, row0 = (t0 + i % per_head) * 32, rows = min(32, n - row0);
    const long long tok = sq.first + row0;
    qr.load((const float*)a.q + tok * a.ldq + (long long)h * a.d, a.ldq, rows, a.d);
    gr.load((const float*)a.dout + tok * a.lddo + (long long)h * a.d, a.lddo, rows, a.d);
    if (threadIdx.x < 64) {   // lse and D; rows past the sequence are zeros, which add nothing
      const int row = threadIdx.x & 31;
      stat = row < rows ? (threadIdx.x < 32 ? a.lse : a.delta)[(long long)h * a.rows + tok + row] : 0.f;
    }
  };
  fetch(0);
  f32x4 kf[DP / 8], vf[DP / 8];
  I::row((const float*)a.k + (sq.first + kk) * a.ldk + (long long)hk * a.d, kk < n, a.d, lane, kf);
  I::row((const float*)a.v + (sq.first + kk) * a.ldv + (long long)hk * a.d, kk < n, a.d, lane, vf);
  f32x16 dv[DP / 32], dk[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) { dv[t] = zero16(); dk[t] = zero16(); }
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  for (int i = 0; i < tiles; ++i) {
    __syncthreads();
    qr.put(Qs);
    gr.put(Gs);
    if (threadIdx.x < 64) Ls[threadIdx.x] = stat;   // (Ds follows Ls)
    __syncthreads();
    if (i + 1 < tiles) fetch(i + 1);
    const int h = hk * group + i / per_head, row0 = (t0 + i % per_head) * 32;
    if (!active || (a.causal && row0 + 32 <= key0)) continue;
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
  if (!active || kk >= n) return;
  I::store(dv, (float*)a.dv + (sq.first + kk) * a.lddv + (long long)hk * a.d, a.d, lane, kept);
  I::store(dk, (float*)a.dk + (sq.first + kk) * a.lddk + (long long)hk * a.d, a.d, lane, a.scale);
}

}  // namespace sattn
