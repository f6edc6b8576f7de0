// Attention over sequences of different lengths, 16-bit formats (element type E = bf16 or fp16), head widths up to 128 padded to DP:
//   S = scale Q K^T over the visible keys, P = softmax rows, O = (P . Z) V, lse = log of the row's sum of e^S;
//   D = rowsum(dO . O), dV = (P . Z)^T dO, dP = (dO V^T) . Z, dS = P . (dP - D), dQ = scale dS K, dK = scale dS^T Q,
// with Z the dropout factors (0 or 1 / kept share; dropout.h) and P taken again from S and lse in the backward pass, so
// that nothing of size length^2 is stored.  Sequence b owns `len[b]` consecutive token rows from `first[b]` on; a query
// sees the keys of its sequence, with `causal` those up to its own position.  Query head h reads key and value head
// h / (heads / kv_heads); the gradients of a shared head are summed over its query heads in one workgroup's accumulators,
// in a fixed order, so results do not depend on timing.
//
// Tiles, fragments and LDS images are those of attention.h: S^T = K Q^T with queries along the lanes in the forward and
// dQ kernels, S = Q K^T with keys along the lanes in the dK / dV kernel, so that P and dS leave the accumulators as the B
// operand of the next product.
#pragma once
#include "attention.h"
#include "dropout.h"
#include "ops.h"

namespace sattn {

using attn::Any;
using attn::Vec;
using attn::CHA;
using attn::pack8;
using attn::zero16;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// over lanes l and l ^ 32 (the swap leaves the lower half's values in one register and the upper half's in the other)
struct Halves { float lo, hi; };
__device__ __forceinline__ Halves halves(float v) {
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t lo = r.x, hi = r.y;
  return Halves{__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}
__device__ __forceinline__ float half_max(float v) { const Halves h = halves(v); return fmaxf(h.lo, h.hi); }
__device__ __forceinline__ float half_sum(float v) { const Halves h = halves(v); return h.lo + h.hi; }

// Workgroup order: consecutive workgroups go to the 8 XCDs in turn; here each XCD gets a contiguous share of the logical
// order instead, so that the blocks of one head, which read the same keys, meet in one L2.  The grid is a multiple of 8.
__device__ __forceinline__ long long xcd_order() { return (long long)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }

struct Seq { long long first; int n; };
// rows of sequence b; n = 0 for one that does not fit the rows or the longest length (reported, not followed)
__device__ __forceinline__ Seq sequence(const SeqAttnArgs& a, int b) {
  Seq s;
  s.first = a.first ? (long long)a.first[b] : (long long)b * a.max_len;
  s.n = a.len ? a.len[b] : a.max_len;
  if (s.n < 0 || s.n > a.max_len || s.first < 0 || s.first + s.n > a.rows) {
    if (threadIdx.x == 0 && s.n != 0) atomicOr(a.bad, 2);
    s.n = 0;
  }
  return s;
}

// transposed accumulators (lane = row) of 32 rows on their way to memory through 32 rows of LDS that only this wave touches:
// whole rows per store instead of 16 bytes of 32 rows
template <typename E, int DP>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[DP / 32], char* stage, E* out, long long ld, int rows, int d, int lane, float scale) {
  using I = Any<DP>;
  attn::wave_lds_order();
  const int q = lane & 31;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      typename Vec<E>::x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = from_f32<E>(acc[t][blk * 4 + i] * scale);
      *(typename Vec<E>::x4*)(stage + q * I::PITCH + I::slot(q, t * 4 + blk) * 16 + 8 * (lane >> 5)) = v;
    }
  attn::wave_lds_order();
#pragma unroll
  for (int i = 0; i < I::NC / 2; ++i) {
    const int idx = i * 64 + lane, r = idx / I::NC, c = idx % I::NC;
    if (r < rows && c * 8 < d) *(bf16x8*)(out + (long long)r * ld + c * 8) = *(const bf16x8*)(stage + r * I::PITCH + I::slot(r, c) * 16);
  }
}

// ---- forward -----------------------------------------------------------------------------------------------------------
// A workgroup owns 128 NQ queries of one (sequence, head), each of its four waves 32 NQ of them, and walks the keys in tiles of 64; the next
// tile's K and V are on their way into the other half of the LDS while one is computed.
template <typename E, int DP, int NQ, bool DROP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void seq_fwd_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  __shared__ __attribute__((aligned(1024))) char lds[4 * I::IMG];
  const int nblk = (a.max_len + 128 * NQ - 1) / (128 * NQ);
  const long long id = xcd_order();
  if (id >= (long long)a.sequences * a.heads * nblk) return;
  const int blk = nblk - 1 - (int)(id % nblk);   // (a causal sequence's longest blocks first)
  const int bh = (int)(id / nblk), b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv_heads);
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128 * NQ;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32 * NQ;
  const bool active = q0 < n;   // (per wave)
  const E* kb_ = (const E*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const E* vb_ = (const E*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128 * NQ) : n, tiles = (last + CHA - 1) / CHA;
  const auto fetch = [&](int t) {
    char* dst = lds + (t & 1) * 2 * I::IMG;
    const int rows = min(CHA, n - t * CHA);
    I::load(kb_ + (long long)t * CHA * a.ldk, (uint32_t)a.ldk, rows, a.d, dst, wave, lane);
    I::load(vb_ + (long long)t * CHA * a.ldv, (uint32_t)a.ldv, rows, a.d, dst + I::IMG, wave, lane);
  };
  fetch(0);
  bf16x8 qf[NQ][DP / 16];
  f32x16 o[NQ][DP / 32];
  float m[NQ], sum[NQ];
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    const int q = q0 + u * 32 + (lane & 31);
    I::template row_frags<E>((const E*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf[u]);
    m[u] = -INFINITY;
    sum[u] = 0.f;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[u][t] = zero16();
  }
  const float c = a.scale * LOG2E;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  for (int t = 0; t < tiles; ++t) {
    wait_vm0();
    __syncthreads();   // this tile is in, and every wave has left the one whose place the next one takes
    if (t + 1 < tiles) fetch(t + 1);
    const int k0 = t * CHA;
    if (!active || (a.causal && k0 >= q0 + 32 * NQ)) continue;
    const char* Ks = lds + (t & 1) * 2 * I::IMG;
    const char* Vs = Ks + I::IMG;
    f32x16 s[NQ][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int u = 0; u < NQ; ++u) s[u][kb] = zero16();
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        const bf16x8 kf = I::rows_frag(Ks, kb * 32 + (lane & 31), st, lane);
#pragma unroll
        for (int u = 0; u < NQ; ++u) s[u][kb] = mfma_32x32x16<E>(kf, qf[u][st], s[u][kb]);
      }
    }
    if (k0 + CHA > n || (a.causal && k0 + CHA - 1 > q0)) {   // keys that a query does not see
#pragma unroll
      for (int u = 0; u < NQ; ++u) {
        const int q = q0 + u * 32 + (lane & 31), lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kb * 32 + 8 * (r >> 2) + (r & 3) >= lim) s[u][kb][r] = -INFINITY;
      }
    }
#pragma unroll
    for (int u = 0; u < NQ; ++u) {
      float cm = s[u][0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) cm = fmaxf(cm, s[u][kb][r]);
      cm = fmaxf(half_max(cm), m[u]);
      // The row's maximum only keeps the exponents in range: it moves, and the accumulators are rescaled, when some row of
      // the wave has exceeded its own by 2^8, which the first tile does and few after it (fp32 sums hold 2^8 as well as 1,
      // and so does P in either 16-bit format).
      if (__any((cm - m[u]) * c > 8.0f)) {
        const float rescale = __builtin_amdgcn_exp2f((m[u] - cm) * c);   // 0 on the first tile
        m[u] = cm;
        sum[u] *= rescale;
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[u][t2][r] *= rescale;
      }
      const float mc = m[u] * c;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[u][kb][r] = __builtin_amdgcn_exp2f(fmaf(s[u][kb][r], c, -mc));
          sum[u] += s[u][kb][r];
        }
        if (DROP) {
          const u32x4 bytes = drop_bytes<true>(q0 + u * 32, k0 + kb * 32, (uint32_t)bh, key, lane);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[u][kb][r] = drop_keeps(bytes, r, a.drop) ? s[u][kb][r] : 0.f;
        }
      }
    }
    // (P is rounded to the format here, as the matrix cores take it: half a step relative, of either sign, per probability)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        bf16x8 pf[NQ];
#pragma unroll
        for (int u = 0; u < NQ; ++u) pf[u] = pack8<E>(s[u][kb], 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) {
          const bf16x8 vf = I::rows_T(Vs, kb, s2, t2, lane);
#pragma unroll
          for (int u = 0; u < NQ; ++u) o[u][t2] = mfma_32x32x16<E>(vf, pf[u], o[u][t2]);
        }
      }
  }
  __syncthreads();   // the images are no longer read: a quarter of them is each wave's way out
  if (!active) return;
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    const int qr = q0 + u * 32, q = qr + (lane & 31);
    if (qr >= n) break;
    const float l = half_sum(sum[u]);
    store_rows<E, DP>(o[u], lds + wave * I::IMG, (E*)a.out + (sq.first + qr) * a.ldo + (long long)h * a.d, a.ldo, n - qr, a.d, lane, kept / l);
    if (a.lse && lane < 32 && q < n) a.lse[(long long)h * a.rows + sq.first + q] = (m[u] * c + __builtin_amdgcn_logf(l)) * LN2;
  }
}

// ---- dQ, and what the dK / dV kernel needs of each row ----------------------------------------------------------------
template <typename E, int DP, bool DROP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void seq_bwd_dq_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  __shared__ __attribute__((aligned(1024))) char lds[4 * I::IMG];
  const int nblk = (a.max_len + 127) / 128;
  const long long id = xcd_order();
  if (id >= (long long)a.sequences * a.heads * nblk) return;
  const int blk = nblk - 1 - (int)(id % nblk);
  const int bh = (int)(id / nblk), b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv_heads);
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const E* kb_ = (const E*)a.k + sq.first * a.ldk + (long long)hk * a.d;
  const E* vb_ = (const E*)a.v + sq.first * a.ldv + (long long)hk * a.d;
  const int last = a.causal ? min(n, base_q + 128) : n, tiles = (last + CHA - 1) / CHA;
  const auto fetch = [&](int t) {
    char* dst = lds + (t & 1) * 2 * I::IMG;
    const int rows = min(CHA, n - t * CHA);
    I::load(kb_ + (long long)t * CHA * a.ldk, (uint32_t)a.ldk, rows, a.d, dst, wave, lane);
    I::load(vb_ + (long long)t * CHA * a.ldv, (uint32_t)a.ldv, rows, a.d, dst + I::IMG, wave, lane);
  };
  fetch(0);
  bf16x8 qf[DP / 16], gf[DP / 16];
  const E* grow = (const E*)a.dout + (sq.first + q) * a.lddo + (long long)h * a.d;
  const E* orow = (const E*)a.o + (sq.first + q) * a.ldo + (long long)h * a.d;
  I::template row_frags<E>((const E*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf);
  I::template row_frags<E>(grow, q < n, a.d, lane, gf);
  float D = 0.f, nl = 0.f;
  if (q < n) {
#pragma unroll
    for (int st = 0; st < DP / 16; ++st) {
      const int col = st * 16 + (lane >> 5) * 8;
      if (col < a.d) {
        const typename Vec<E>::x8 gv = __builtin_bit_cast(typename Vec<E>::x8, gf[st]);
        const typename Vec<E>::x8 ov = *(const typename Vec<E>::x8*)(orow + col);
#pragma unroll
        for (int i = 0; i < 8; ++i) D = fmaf(to_f32(gv[i]), to_f32(ov[i]), D);
      }
    }
    nl = -a.lse[(long long)h * a.rows + sq.first + q] * LOG2E;
  }
  D = half_sum(D);
  if (q < n && lane < 32) {
    a.nlse2[(long long)h * a.rows + sq.first + q] = nl;
    a.delta[(long long)h * a.rows + sq.first + q] = D;
  }
  f32x16 dq[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) dq[t] = zero16();
  const float c = a.scale * LOG2E, kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  for (int t = 0; t < tiles; ++t) {
    wait_vm0();
    __syncthreads();
    if (t + 1 < tiles) fetch(t + 1);
    const int k0 = t * CHA;
    if (!active || (a.causal && k0 >= q0 + 32)) continue;
    const char* Ks = lds + (t & 1) * 2 * I::IMG;
    const char* Vs = Ks + I::IMG;
    const bool edge = k0 + CHA > n || (a.causal && k0 + CHA - 1 > q0);
    const int lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s = zero16(), g = zero16();
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        s = mfma_32x32x16<E>(I::rows_frag(Ks, kb * 32 + (lane & 31), st, lane), qf[st], s);
        g = mfma_32x32x16<E>(I::rows_frag(Vs, kb * 32 + (lane & 31), st, lane), gf[st], g);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, nl));
      if (edge) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kb * 32 + 8 * (r >> 2) + (r & 3) >= lim) s[r] = 0.f;
      }
      if (DROP) {
        const u32x4 bytes = drop_bytes<true>(q0, k0 + kb * 32, (uint32_t)bh, key, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] = s[r] * (drop_keeps(bytes, r, a.drop) ? fmaf(g[r], kept, -D) : -D);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] = s[r] * (g[r] - D);
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 df = pack8<E>(g, 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) dq[t2] = mfma_32x32x16<E>(I::rows_T(Ks, kb, s2, t2, lane), df, dq[t2]);
      }
    }
  }
  __syncthreads();
  if (!active) return;
  store_rows<E, DP>(dq, lds + wave * I::IMG, (E*)a.dq + (sq.first + q0) * a.lddq + (long long)h * a.d, a.lddq, n - q0, a.d, lane, a.scale);
}

// ---- dK, dV -----------------------------------------------------------------------------------------------------------
// A workgroup owns 128 keys of one (sequence, key head) and walks the queries of all the head's query heads in tiles of 64.
template <typename E, int DP, bool DROP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP > 96 ? 1 : 2)))
void seq_bwd_dkv_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  constexpr int STAGE = 2 * I::IMG + 512;   // Q, dO, and 64 rows' -lse and D
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  const int nblk = (a.max_len + 127) / 128;
  const long long id = xcd_order();
  if (id >= (long long)a.sequences * a.kv_heads * nblk) return;
  const int blk = (int)(id % nblk);
  const int bk = (int)(id / nblk), b = bk / a.kv_heads, hk = bk % a.kv_heads, group = a.heads / a.kv_heads;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_k = blk * 128;
  if (base_k >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key0 = base_k + wave * 32, kk = key0 + (lane & 31);
  const bool active = key0 < n;
  // query tiles of one head: with a causal mask from the one that holds this block's first key on
  const int t0 = a.causal ? base_k / CHA : 0, per_head = (n + CHA - 1) / CHA - t0, tiles = per_head * group;
  const auto fetch = [&](int i) {
    char* dst = lds + (i & 1) * STAGE;
    const int h = hk * group + i / per_head, row0 = (t0 + i % per_head) * CHA, rows = min(CHA, n - row0);
    const long long tok = sq.first + row0;
    I::load((const E*)a.q + tok * a.ldq + (long long)h * a.d, (uint32_t)a.ldq, rows, a.d, dst, wave, lane);
    I::load((const E*)a.dout + tok * a.lddo + (long long)h * a.d, (uint32_t)a.lddo, rows, a.d, dst + I::IMG, wave, lane);
    if (wave < 2) {   // rows past the sequence: zeros, which add nothing (their Q and dO are zeros too)
      const float* src = (wave ? a.delta : a.nlse2) + (long long)h * a.rows + tok;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(src, (uint32_t)rows * 4), (__attribute__((address_space(3))) void*)(dst + 2 * I::IMG + wave * 256),
                                               4, lane * 4, 0, 0, 0);
    }
  };
  fetch(0);
  bf16x8 kf[DP / 16], vf[DP / 16];
  I::template row_frags<E>((const E*)a.k + (sq.first + kk) * a.ldk + (long long)hk * a.d, kk < n, a.d, lane, kf);
  I::template row_frags<E>((const E*)a.v + (sq.first + kk) * a.ldv + (long long)hk * a.d, kk < n, a.d, lane, vf);
  f32x16 dv[DP / 32], dk[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) { dv[t] = zero16(); dk[t] = zero16(); }
  const float c = a.scale * LOG2E, kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  for (int i = 0; i < tiles; ++i) {
    wait_vm0();
    __syncthreads();
    if (i + 1 < tiles) fetch(i + 1);
    const int h = hk * group + i / per_head, row0 = (t0 + i % per_head) * CHA;
    if (!active || (a.causal && row0 + CHA <= key0)) continue;
    const char* Qs = lds + (i & 1) * STAGE;
    const char* Gs = Qs + I::IMG;
    const float* Ls = (const float*)(Gs + I::IMG);
    const float* Ds = Ls + 64;
    const bool edge = a.causal && row0 < key0 + 31;
    const int lim = kk - row0 - 4 * (lane >> 5);   // causal: rows below it do not see this lane's key
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      f32x16 s = zero16(), g = zero16();
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        s = mfma_32x32x16<E>(I::rows_frag(Qs, qb * 32 + (lane & 31), st, lane), kf[st], s);
        g = mfma_32x32x16<E>(I::rows_frag(Gs, qb * 32 + (lane & 31), st, lane), vf[st], g);
      }
      u32x4 bytes;
      if (DROP) bytes = drop_bytes<false>(row0 + qb * 32, key0, (uint32_t)(b * a.heads + h), key, lane);
#pragma unroll
      for (int blk4 = 0; blk4 < 4; ++blk4) {
        const f32x4 L4 = *(const f32x4*)(Ls + qb * 32 + 8 * blk4 + 4 * (lane >> 5));
        const f32x4 D4 = *(const f32x4*)(Ds + qb * 32 + 8 * blk4 + 4 * (lane >> 5));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 4 * blk4 + j;
          float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, L4[j]));
          if (edge) p = qb * 32 + 8 * blk4 + j < lim ? 0.f : p;
          if (DROP) {
            const bool keep = drop_keeps(bytes, r, a.drop);
            g[r] = p * (keep ? fmaf(g[r], kept, -D4[j]) : -D4[j]);
            s[r] = keep ? p : 0.f;
          } else {
            g[r] = p * (g[r] - D4[j]);
            s[r] = p;
          }
        }
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 pf = pack8<E>(s, 8 * s2), df = pack8<E>(g, 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) {
          dv[t2] = mfma_32x32x16<E>(I::rows_T(Gs, qb, s2, t2, lane), pf, dv[t2]);
          dk[t2] = mfma_32x32x16<E>(I::rows_T(Qs, qb, s2, t2, lane), df, dk[t2]);
        }
      }
    }
  }
  __syncthreads();
  if (!active) return;
  char* stage = lds + wave * (STAGE / 2);
  store_rows<E, DP>(dv, stage, (E*)a.dv + (sq.first + key0) * a.lddv + (long long)hk * a.d, a.lddv, n - key0, a.d, lane, kept);
  store_rows<E, DP>(dk, stage, (E*)a.dk + (sq.first + key0) * a.lddk + (long long)hk * a.d, a.lddk, n - key0, a.d, lane, a.scale);
}

}  // namespace sattn
