// Attention over sequences of different lengths, 16-bit formats (element type E = bf16 or fp16), head widths up to 128 padded to DP:
//   S = scale Q K^T over the visible keys, P = softmax rows, O = (P . Z) V, lse = log of the row's sum of e^S;
//   D = rowsum(dO . O), dV = (P . Z)^T dO, dP = (dO V^T) . Z, dS = P . (dP - D), dQ = scale dS K, dK = scale dS^T Q,
// with Z the dropout factors (0 or 1 / kept share; dropout.h) and P taken again from S and lse in the backward pass, so
// that nothing of size length^2 is stored.  Sequence b owns `len[b]` consecutive token rows from `first[b]` on; a query
// sees the keys of its sequence, with `causal` those up to its own position.  Query head h reads key and value head
// h / (heads / kv_heads); the gradients of a shared head are summed over its query heads in one workgroup's accumulators or in
// several whose partial results a second kernel adds up, in a fixed order either way, so results do not depend on timing.
//
// Tiles, fragments and LDS images are those of attention.h: S^T = K Q^T with queries along the lanes in the forward and
// dQ kernels, S = Q K^T with keys along the lanes in the dK / dV kernel, so that P and dS leave the accumulators as the B
// operand of the next product.
//
// Rounded to E, for the matrix cores: P and dS; everything else between inputs and results is fp32 (scores, maxima, sums, D, accumulators, partial
// results).  Each rounds once, by half a step at most, and with the result's own rounding a result is 1.4 times as far from 64 bits as that one
// alone (bf16 0.0023 to 0.0027 of a matrix's norm); P and dS in two halves each would double the products that read them.  D comes from
// the rounded O, which is seen where rows have few keys (dQ kernel).
#pragma once
#include <type_traits>

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
constexpr float NEAR = 1024.f;   // scores, in powers of two, whose products may be rounded (by 2^-15 at most) before their differences are taken

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

// Workgroup order.  Blocks in the order of the launch's `blocks` (the longest walks first, where the mask makes them differ), and of one block
// all heads of all sequences: long and short sequences then spread over the chip, the longest walks begin first, and the blocks that
// a short sequence does not have end at once.  (Head by head, the 8 XCDs that take workgroups in turn each get the same blocks of every
// head, some the long and some the short ones: one causal sequence of 4096, 32 heads on 8 of 64: forward 144 us, 99 so; dQ 180 and 117.
// 64 ragged sequences of up to 512, 16 heads, dropped: 88 and 80, 112 and 100, dK and dV 134 and 122.)
// Of these heads an XCD takes runs of neighbours, as far as they come in eights:
// - the query heads that share a key head, whose keys and values then meet in its L2, where all of them are more than two L2s.  7 causal
//   sequences of up to 1999, 12 heads on 4 of 96: forward 79 us one by one and 62 in threes, dQ 78 and 66; 6 of up to 1700, 32 heads on 8 of 128:
//   143 and 139, 185 and 180; but 12 of up to 1200, 16 heads on 2 of 64, 4 MB: 44 and 49, 50 and 59.
// - eight, where sequences have one block: heads side by side in memory are read by one XCD at a time.  256 of 128 tokens, 16 heads of
//   64: forward 74 and 61, backward 155 and 149.  (With 64 of 512: 80 and 85, 100 and 106: XCDs get unequal shares of ragged sequences.)
struct Place { int b, hk, head, turn, split; };   // sequence, key head, query head of it, block in order, split of it
__device__ __forceinline__ Place place(const SeqAttnArgs& a, int group, int splits) {
  const int run = a.max_len <= 128 ? 8 : a.by_group ? group : 1, of_turn = a.sequences * a.kv_heads * group * splits;
  const int turn = blockIdx.x / of_turn, in = blockIdx.x % of_turn;
  const int at = in < of_turn / (8 * run) * (8 * run) ? in / (8 * run) * (8 * run) + (in & 7) * run + (in >> 3) % run : in;
  const int head = at / splits, unit = head / group;
  return Place{unit / a.kv_heads, unit % a.kv_heads, head % group, turn, at % splits};
}

struct Seq { long long first; int n; };
// rows of sequence b; n = 0 for one that does not fit the rows or the longest length (reported, not followed)
__device__ __forceinline__ Seq sequence(const SeqAttnArgs& a, int b) {
  typedef const __attribute__((address_space(4))) int32_t* Scalar;   // (through the scalar cache, which other workgroups have filled)
  Seq s;
  s.first = a.first ? (long long)((Scalar)(uintptr_t)a.first)[b] : (long long)b * a.max_len;
  s.n = a.len ? ((Scalar)(uintptr_t)a.len)[b] : a.max_len;
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

// Loads from memory straight into LDS (lane l's 16 or 4 bytes to `dst` + 16 l or 4 l), which have no register to be waited for: the
// waits are the kernels' own (wait_vm0 at the head of a tile).  As built-ins, the compiler counts them before every transposing LDS read,
// whose place it does not know, and so takes the next tile's loads for this tile's.  The no-op is the wait state between M0 and
// its use.  M0 is a reserved register, which no clobber list can name: nothing else in these kernels may use it, and in what is compiled from them
// nothing does.
__device__ __forceinline__ i32x4 lds_source(const void* base, uint32_t bytes) {
  const uint64_t p = (uint64_t)base;
  return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) & 0xFFFF,
               __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}
__device__ __forceinline__ uint32_t lds_place(const __attribute__((address_space(3))) char* p) { return (uint32_t)(uintptr_t)p; }
__device__ __forceinline__ void lds_load16(i32x4 from, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(off), "s"(from) : "memory");
}
__device__ __forceinline__ void lds_load4(i32x4 from, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(off), "s"(from) : "memory");
}

// 64 rows of a matrix into an LDS image, 16 bytes a lane and instruction, by the four waves of a workgroup: the lanes' places within a tile
// are worked out once, a tile moves only the descriptor.  Rows past the sequence and columns past the head lie outside the descriptor
// and arrive as zeros.
template <typename E, int DP>
struct Tiles {
  using I = Any<DP>;
  static constexpr int PER = I::IMG / 4096;
  const E* base;   // row 0 of the sequence, first column of the head
  long long ld;
  int n, d;
  uint32_t off[PER];
  __device__ __forceinline__ Tiles(const void* p, long long first, long long ld_, int head, int n_, int d_, int wave, int lane)
      : base((const E*)p + first * ld_ + (long long)head * d_), ld(ld_), n(n_), d(d_) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int idx = (i * 4 + wave) * 64 + lane, row = idx / I::NC, c = I::chunk(row, idx % I::NC);
      off[i] = c * 8 < d ? ((uint32_t)row * (uint32_t)ld + (uint32_t)c * 8) * 2u : BUF_OOB;
    }
  }
  // to: the image's place in LDS
  __device__ __forceinline__ void fetch(int row0, uint32_t to, int wave) const {
    const i32x4 from = lds_source(base + (long long)row0 * ld, (uint32_t)(((long long)(min(CHA, n - row0) - 1) * ld + d) * 2));
#pragma unroll
    for (int i = 0; i < PER; ++i) lds_load16(from, off[i], to + wave * 1024 + i * 4096);
  }
};
// fp16 ends at 6e-5 below (6e-8 with few bits), where bf16 has the range of fp32; the dS of a long row is smaller than dO by its length.  P and dS of the backward
// kernels are therefore taken times 2^up, a power for each lane, whose row or key all of its accumulators belong to: UP_MOST, which keeps P in
// range, until a dS outgrows it (dQ kernel), or less from the start by dS's bound, the largest |dO| |v| + |D| (dK / dV kernel, which knows both and
// whose registers leave no room for a look at every dS).  (3000 keys, dO of 1e-3: dQ off by 3.9e-3 of its norm without, 6e-4 with, which is its own rounding.)
constexpr float UP_MOST = 14.f, UP_LIMIT = 32768.f;
// the power of two to take a number beyond UP_LIMIT down by, with two bits to spare (infinity: by all there is)
__device__ __forceinline__ float power_down(float x, float up) {
  const float by = (float)((int)(__builtin_bit_cast(uint32_t, x) >> 23) - (127 + 12));
  return x > UP_LIMIT ? fminf(by, up) : 0.f;
}
// the largest of 32 rows' kept |dO| and |D|, rounded up to 16 bits each
__device__ __forceinline__ uint32_t pack_bounds(float norm, float D) {
  const uint32_t a = __builtin_bit_cast(uint32_t, wave_max(norm)) + 0xFFFFu, b = __builtin_bit_cast(uint32_t, wave_max(fabsf(D))) + 0xFFFFu;
  return (a >> 16) | (b & 0xFFFF0000u);
}
__device__ __forceinline__ float largest16(const f32x16& g) {
  float x = fabsf(g[0]);
#pragma unroll
  for (int r = 1; r < 16; ++r) x = fmaxf(x, fabsf(g[r]));
  return x;
}
template <int N>
__device__ __forceinline__ void times(f32x16 (&acc)[N], float f) {
#pragma unroll
  for (int t = 0; t < N; ++t) acc[t] *= f;
}
__device__ __forceinline__ f32x16 splat16(float x) { return f32x16{x, x, x, x, x, x, x, x, x, x, x, x, x, x, x, x}; }

// the same rows as fp32 partial results, straight from the registers (16 bytes a lane; few of them are written)
template <int DP>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[DP / 32], float* row, bool live, int d, int lane, float scale) {
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      const int col = t * 32 + blk * 8 + 4 * (lane >> 5);
      if (live && col < d) *(f32x4*)(row + col) = f32x4{acc[t][4 * blk], acc[t][4 * blk + 1], acc[t][4 * blk + 2], acc[t][4 * blk + 3]} * scale;
    }
}

// ---- forward -----------------------------------------------------------------------------------------------------------
// A workgroup owns 128 queries of one (sequence, head), each of its four waves 32 of them, and walks the keys in tiles of 64; the next
// tile's K and V are on their way into the other half of the LDS while one is computed.  A tile's keys are taken in halves, which costs a second
// look at the rows' maxima and saves 16 registers: a fourth wave a SIMD at 64 columns also with dropped probabilities.
// Bound at 64 columns by vector instructions (109 of them, 16 exponentials, to 8 MFMA per wave and 32 keys; 62 % of the SIMDs' clocks at
// three or more waves), at 128 by the matrix cores.  256 sequences of 128 tokens, 16 heads of 64: 60 us, 4.5 TB/s of the 5.1 that a copy
// reaches; 64 of up to 512, ragged and dropped: 81 us, with vector instructions in 0.55 of the SIMDs' clocks and 2.3 waves a SIMD.  One causal sequence of 16384, 32
// heads on 8 of 128: 2200 to 2300 us, 970 TFLOP/s of the visible half (a library product of 8192^3: 1221).
template <typename E, int DP, bool DROP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 64 ? 4 : DP <= 96 && DROP ? 3 : 2)))
void seq_fwd_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  __shared__ __attribute__((aligned(1024))) char lds[4 * I::IMG];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group, a.splits_fwd);
  const int split = at.split, blk = nblk - 1 - at.turn;   // (a causal sequence's longest blocks first)
  const int b = at.b, hk = at.hk, h = hk * group + at.head, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;   // (per wave)
  const Tiles<E, DP> kt(a.k, sq.first, a.ldk, hk, n, a.d, wave, lane), vt(a.v, sq.first, a.ldv, hk, n, a.d, wave, lane);
  const int last = a.causal ? min(n, base_q + 128) : n, all_tiles = (last + CHA - 1) / CHA;
  const int from = all_tiles * split / a.splits_fwd, tiles = all_tiles * (split + 1) / a.splits_fwd;   // this split's
  const uint32_t lds0 = lds_place((const __attribute__((address_space(3))) char*)lds);
  const auto fetch = [&](int t) {
    const uint32_t to = lds0 + (t & 1) * 2 * I::IMG;
    kt.fetch(t * CHA, to, wave);
    vt.fetch(t * CHA, to + I::IMG, wave);
  };
  if (from < tiles) fetch(from);
  bf16x8 qf[DP / 16];
  f32x16 o[DP / 32];
  // No maximum yet: below any score, and finite with its product, as a split's first tile may have no key that the row sees.
  const float c = a.scale * LOG2E;
  float m = -3e38f / fmaxf(c, 1.0f), sum = 0.f;
  bool far = false;   // a maximum of the wave's rows is not near
  I::template row_frags<E>((const E*)a.q + (sq.first + q) * a.ldq + (long long)h * a.d, q < n, a.d, lane, qf);
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) o[t] = zero16();
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  const auto arrive = [&](int t) {
    wait_vm0();
    __syncthreads();   // this tile is in, and every wave has left the one whose place the next one takes
    if (t + 1 < tiles) fetch(t + 1);
  };
  const auto compute = [&](int t, auto edge) {
    const int k0 = t * CHA;
    const char* Ks = lds + (t & 1) * 2 * I::IMG;
    const char* Vs = Ks + I::IMG;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s = zero16();
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) s = mfma_32x32x16<E>(I::rows_frag(Ks, kb * 32 + (lane & 31), st, lane), qf[st], s);
      if constexpr (decltype(edge)::value) {   // keys that a query does not see
        const int lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (kb * 32 + 8 * (r >> 2) + (r & 3) >= lim) s[r] = -INFINITY;
      }
      float cm = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) cm = fmaxf(cm, s[r]);
      cm = fmaxf(half_max(cm), m);
      if (__any((cm - m) * c > 8.0f)) {
        const float rescale = __builtin_amdgcn_exp2f((m - cm) * c);   // 0 on the first tile
        m = cm;
        far = __any(fabsf(m * c) > NEAR);
        sum *= rescale;
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t2][r] *= rescale;
      }
      // Near zero one fma a score, whose second product is rounded; far from it the difference first: half a step of m c, a factor of
      // every P of the row, is 2^128 where m c is 2^31.
      if (far) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] -= m;
      }
      const float mc = far ? 0.f : m * c;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -mc));
        sum += s[r];
      }
      if (DROP) {
        const u32x4 bytes = drop_bytes<true>(q0, k0 + kb * 32, (uint32_t)bh, key, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = drop_select(drop_keeps(bytes, r, a.drop), s[r]);
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 pf = pack8<E>(s, 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) o[t2] = mfma_32x32x16<E>(I::rows_T(Vs, kb, s2, t2, lane), pf, o[t2]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The wave's tiles: those that all of its queries see whole, those with a mask, and those of its neighbours', where it only helps to
  // load.  In loops of their own: with the mask and the way round the work as branches inside one, the accumulators are copied back and forth.
  const int mine = !active ? 0 : a.causal ? min(tiles, (q0 + 32 + CHA - 1) / CHA) : tiles;
  const int whole = min(mine, (a.causal ? min(n, q0 + 1) : n) / CHA);   // (counted from the first key, whatever the split)
  int t = from;
  for (; t < whole; ++t) { arrive(t); compute(t, std::false_type{}); }
  for (; t < mine; ++t) { arrive(t); compute(t, std::true_type{}); }
  for (; t < tiles; ++t) arrive(t);
  __syncthreads();   // the images are no longer read: a quarter of them is each wave's way out
  if (!active) return;
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  const float l = half_sum(sum), mc = m * c;
  const float rest = fabsf(mc) <= NEAR ? fmaf(m, c, -mc) : 0.f;   // (what the rounded product left out, in l)
  if (a.splits_fwd > 1) {   // (a split without a key that the row sees: l = 0)
    const long long row = (long long)split * a.rows + sq.first + q, stat = ((long long)split * a.heads + h) * a.rows + sq.first + q;
    store_part<DP>(o, a.part + row * ((long long)a.heads * a.d) + (long long)h * a.d, q < n, a.d, lane, l == 0.f ? 0.f : kept / l);
    if (lane < 32 && q < n) { a.part_m[stat] = m; a.part_sum[stat] = l * __builtin_amdgcn_exp2f(-rest); }
    return;
  }
  store_rows<E, DP>(o, lds + wave * I::IMG, (E*)a.out + (sq.first + q0) * a.ldo + (long long)h * a.d, a.ldo, n - q0, a.d, lane, kept / l);
  if (a.lse && lane < 32 && q < n) a.lse[(long long)h * a.rows + sq.first + q] = fmaf(m, a.scale, (__builtin_amdgcn_logf(l) - rest) * LN2);
}

// ---- dQ, and what the dK / dV kernel needs of each row ----------------------------------------------------------------
// As the forward kernel, with dP beside S and dS K in the place of P V.  Bound by vector instructions and the latency of its three dependent
// products at 64 columns (64 sequences of up to 512, 16 heads, dropped: 97 to 101 us; at two waves a SIMD a tenth more), by
// the matrix cores at 128 (one causal sequence of 16384, 32 heads on 8: 2850 to 2990 us, 1100 to 1160 TFLOP/s).
template <typename E, int DP, bool DROP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP <= 32 ? 4 : DP <= 64 ? 3 : 2)))
void seq_bwd_dq_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  constexpr bool SCALED = std::is_same<E, fp16>::value;
  __shared__ __attribute__((aligned(1024))) char lds[4 * I::IMG];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, group, a.splits_dq);
  const int split = at.split, blk = nblk - 1 - at.turn;   // (a causal sequence's longest blocks first)
  const int b = at.b, hk = at.hk, h = hk * group + at.head, bh = b * a.heads + h;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_q = blk * 128;
  if (base_q >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int q0 = base_q + wave * 32, q = q0 + (lane & 31);
  const bool active = q0 < n;
  const Tiles<E, DP> kt(a.k, sq.first, a.ldk, hk, n, a.d, wave, lane), vt(a.v, sq.first, a.ldv, hk, n, a.d, wave, lane);
  const int last = a.causal ? min(n, base_q + 128) : n, all_tiles = (last + CHA - 1) / CHA;
  const int from = all_tiles * split / a.splits_dq, tiles = all_tiles * (split + 1) / a.splits_dq;
  const uint32_t lds0 = lds_place((const __attribute__((address_space(3))) char*)lds);
  const auto fetch = [&](int t) {
    const uint32_t to = lds0 + (t & 1) * 2 * I::IMG;
    kt.fetch(t * CHA, to, wave);
    vt.fetch(t * CHA, to + I::IMG, wave);
  };
  if (from < tiles) fetch(from);
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
    nl = -a.lse[(long long)h * a.rows + sq.first + q] / a.scale;
  }
  D = half_sum(D);
  const bool stats = q < n && lane < 32 && from == 0 && tiles > 0;   // (one of the splits writes them)
  const float kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  if (stats) {
    a.nlse2[(long long)h * a.rows + sq.first + q] = nl;
    a.delta[(long long)h * a.rows + sq.first + q] = -D;
  }
  if constexpr (SCALED) {
    float norm = 0.f;
#pragma unroll
    for (int st = 0; st < DP / 16; ++st) {
      const typename Vec<E>::x8 x = __builtin_bit_cast(typename Vec<E>::x8, gf[st]);
#pragma unroll
      for (int i = 0; i < 8; ++i) norm = fmaf(to_f32(x[i]), to_f32(x[i]), norm);
    }
    const uint32_t bounds = pack_bounds(kept * __builtin_amdgcn_sqrtf(half_sum(norm)), D);
    if (stats && lane == 0) a.bounds[(long long)h * a.rows + sq.first + q] = bounds;
  }
  f32x16 dq[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) dq[t] = zero16();
  const float c = a.scale * LOG2E;
  float nlc = nl * c, up = 0.f;
  if (SCALED) { up = UP_MOST; nlc += up; }
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  const auto arrive = [&](int t) {
    wait_vm0();
    __syncthreads();
    if (t + 1 < tiles) fetch(t + 1);
  };
  const auto compute = [&](int t, auto edge) {
    const int k0 = t * CHA;
    const char* Ks = lds + (t & 1) * 2 * I::IMG;
    const char* Vs = Ks + I::IMG;
    const int lim = (a.causal ? min(n, q + 1) : n) - k0 - 4 * (lane >> 5);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s = zero16(), g = splat16(DROP ? 0.f : -D);   // (from -D instead of zero, which leaves one product for dS)
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        s = mfma_32x32x16<E>(I::rows_frag(Ks, kb * 32 + (lane & 31), st, lane), qf[st], s);
        g = mfma_32x32x16<E>(I::rows_frag(Vs, kb * 32 + (lane & 31), st, lane), gf[st], g);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, nlc));
      if constexpr (decltype(edge)::value) {
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
        for (int r = 0; r < 16; ++r) g[r] *= s[r];
      }
      if constexpr (SCALED) {
        const float largest = largest16(g);
        if (__any(largest > UP_LIMIT)) {
          const float by = power_down(half_max(largest), up), f = __builtin_amdgcn_exp2f(-by);   // (lanes l and l ^ 32 share a row)
          up -= by;
          nlc -= by;
          s *= f;
          g *= f;
          times(dq, f);
        }
      }
      // D comes from O as it was stored, off by its rounding: noise in every dS of the row, which is one over the square root of the number of keys of
      // what dS's own rounding does, but all of it where rows see few.  A row of dS has the sum zero (P has the sum 1): where these 32
      // keys are all that the rows see, its sum is D's error, and is taken out.  (Two to four keys: the gradients' error falls from
      // 1.6 times that of their rounding alone, against 64 bits, to the 1.4 of long rows.)
      if constexpr (decltype(edge)::value) {
        if (kb == 0 && q0 == 0 && (a.causal || n <= 32)) {
          float off = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) off += g[r];
          off = half_sum(off);
          if (SCALED) off *= __builtin_amdgcn_exp2f(-up);
#pragma unroll
          for (int r = 0; r < 16; ++r) g[r] = fmaf(-s[r], off, g[r]);
          if (stats) a.delta[(long long)h * a.rows + sq.first + q] = -(D + off);
        }
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 df = pack8<E>(g, 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) dq[t2] = mfma_32x32x16<E>(I::rows_T(Ks, kb, s2, t2, lane), df, dq[t2]);
      }
      __builtin_amdgcn_sched_barrier(0);   // (the halves side by side want more registers than the waves of a SIMD have)
    }
  };
  const int mine = !active ? 0 : a.causal ? min(tiles, (q0 + 32 + CHA - 1) / CHA) : tiles;   // (as in the forward kernel)
  const int whole = min(mine, (a.causal ? min(n, q0 + 1) : n) / CHA);
  int t = from;
  for (; t < whole; ++t) { arrive(t); compute(t, std::false_type{}); }
  for (; t < mine; ++t) { arrive(t); compute(t, std::true_type{}); }
  for (; t < tiles; ++t) arrive(t);
  __syncthreads();
  if (!active) return;
  const float out_scale = SCALED ? a.scale * __builtin_amdgcn_exp2f(-up) : a.scale;
  if (a.splits_dq > 1) {
    const long long row = (long long)split * a.rows + sq.first + q;
    store_part<DP>(dq, a.part + row * ((long long)a.heads * a.d) + (long long)h * a.d, q < n, a.d, lane, out_scale);
    return;
  }
  store_rows<E, DP>(dq, lds + wave * I::IMG, (E*)a.dq + (sq.first + q0) * a.lddq + (long long)h * a.d, a.lddq, n - q0, a.d, lane, out_scale);
}

// ---- dK, dV -----------------------------------------------------------------------------------------------------------
// A workgroup owns 128 keys of one (sequence, key head) and walks the queries of all the head's query heads in tiles of 64.
// WHOLE, where no sequence is longer than 128: the workgroup has all keys of its head, so that dQ of a tile can be made here as well, from dS
// that the waves lay side by side in LDS, and the dQ kernel with its second pass over scores, probabilities and masks is not run.  The
// rows' D and lse are taken from O, dO and lse at the head's start.  (256 sequences of up to 128, 16 heads of 64, dropped: 119 to 122 us, the
// two kernels 143; wider heads leave no registers for it.)
// Bound at 64 columns by latency at two waves a SIMD (226 and 240 registers; at three they spill): 64 ragged sequences of up to 512, dropped, 115 to
// 121 us; WHOLE by its first loads, half of a workgroup's life (256 of 128 tokens: 148 us, 3.6 TB/s).  WHOLE takes 245 registers; dropped it takes
// all 256 and spills 14 vector and 67 scalar ones (at 32 columns 192, and 62 scalar ones).  At 128 columns one wave a SIMD (292 registers, dropped
// 314), bound by the matrix cores and what that wave waits for (one causal sequence of 16384, 32 heads on 8: 4830 to 5220 us, 840 to 910 TFLOP/s).
template <typename E, int DP, bool DROP, bool WHOLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DP > 96 ? 1 : 2)))
void seq_bwd_dkv_kernel(const SeqAttnArgs a) {
  using I = Any<DP>;
  constexpr bool SCALED = std::is_same<E, fp16>::value && !WHOLE;   // (WHOLE: at most 128 keys, and dQ's sums want one power for all of them)
  using IS = Any<64>;                       // dS: [key][64 queries]
  constexpr int STAGE = 2 * I::IMG + 512;   // Q, dO, and 64 rows' -lse and D
  constexpr int KIMG = 2 * STAGE, SIMG = KIMG + 2 * I::IMG, STAT = SIMG + 2 * IS::IMG;   // (WHOLE) K, dS, two heads' -lse and D of 128 rows
  __shared__ __attribute__((aligned(1024))) char lds[WHOLE ? STAT + 2 * 1024 : 2 * STAGE];
  const int nblk = (a.max_len + 127) / 128, group = a.heads / a.kv_heads;
  const Place at = place(a, 1, a.splits_dkv);
  const int split = at.split, blk = at.turn, b = at.b, hk = at.hk;
  const Seq sq = sequence(a, b);
  const int n = sq.n, base_k = blk * 128;
  if (base_k >= n) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key0 = base_k + wave * 32, kk = key0 + (lane & 31);
  const bool active = key0 < n;
  // query tiles of one head: with a causal mask from the one that holds this block's first key on
  const int t0 = a.causal ? base_k / CHA : 0, per_head = (n + CHA - 1) / CHA - t0, all_tiles = per_head * group;
  const int from = all_tiles * split / a.splits_dkv, tiles = all_tiles * (split + 1) / a.splits_dkv - from;   // this split's, of all heads' in turn
  const int h0 = hk * group + from / per_head;
  Tiles<E, DP> qt(a.q, sq.first, a.ldq, h0, n, a.d, wave, lane), gt(a.dout, sq.first, a.lddo, h0, n, a.d, wave, lane);
  const float* stats = (wave ? a.delta : a.nlse2) + (long long)h0 * a.rows + sq.first;
  int next_t = t0 + from % per_head;   // the next tile to be fetched, of the head that the three point at
  const uint32_t lds0 = lds_place((const __attribute__((address_space(3))) char*)lds);
  const auto fetch = [&](int i) {
    const uint32_t to = lds0 + (i & 1) * STAGE;
    qt.fetch(next_t * CHA, to, wave);
    gt.fetch(next_t * CHA, to + I::IMG, wave);
    if (!WHOLE && wave < 2)   // rows past the sequence: zeros, which add nothing (their Q and dO are zeros too)
      lds_load4(lds_source(stats + next_t * CHA, (uint32_t)min(CHA, n - next_t * CHA) * 4), lane * 4, to + 2 * I::IMG + wave * 256);
    if (++next_t == t0 + per_head) {
      next_t = t0;
      qt.base += a.d;
      gt.base += a.d;
      stats += a.rows;
    }
  };
  if (tiles > 0) fetch(0);
  // WHOLE: -lse / scale and -D of the head's rows (zeros past the sequence), whole rows per load
  const auto head_stats = [&](int h) {
    constexpr int CH = DP / 8;   // lanes to a row
    const int col = threadIdx.x % CH * 8;
    float* st = (float*)(lds + STAT + (h & 1) * 1024);
#pragma unroll
    for (int u = 0; u < CH / 2; ++u) {
      const int row = u * (256 / CH) + threadIdx.x / CH;
      float D = 0.f;
      if (row < n && col < a.d) {
        const typename Vec<E>::x8 gv = *(const typename Vec<E>::x8*)((const E*)a.dout + (sq.first + row) * a.lddo + (long long)h * a.d + col);
        const typename Vec<E>::x8 ov = *(const typename Vec<E>::x8*)((const E*)a.o + (sq.first + row) * a.ldo + (long long)h * a.d + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) D = fmaf(to_f32(gv[j]), to_f32(ov[j]), D);
      }
      D += dpp_move<0xB1>(D);
      D += dpp_move<0x4E>(D);
      if (CH == 8) D += dpp_move<0x141>(D);
      if (col == 0) st[128 + row] = -D;
    }
    if (threadIdx.x < 128) st[threadIdx.x] = threadIdx.x < n ? -a.lse[(long long)h * a.rows + sq.first + threadIdx.x] / a.scale : 0.f;
  };
  const bool few = key0 == 0 && (a.causal || n <= 32);   // the wave's keys are all that the first 32 rows see
  bf16x8 kf[DP / 16], vf[DP / 16];
  if constexpr (WHOLE) {   // through LDS, V where dS will be: loads of 16 bytes of 32 rows each are evicted and fetched again before the rows' other parts are read
    const Tiles<E, DP> kt(a.k, sq.first, a.ldk, hk, n, a.d, wave, lane), vt(a.v, sq.first, a.ldv, hk, n, a.d, wave, lane);
    kt.fetch(0, lds0 + KIMG, wave);
    vt.fetch(0, lds0 + SIMG, wave);
    if (n > CHA) {
      kt.fetch(CHA, lds0 + KIMG + I::IMG, wave);
      vt.fetch(CHA, lds0 + SIMG + I::IMG, wave);
    }
    head_stats(h0);
    wait_vm0();
    __syncthreads();
#pragma unroll
    for (int st = 0; st < DP / 16; ++st) {
      kf[st] = I::rows_frag(lds + KIMG + (wave >> 1) * I::IMG, (wave & 1) * 32 + (lane & 31), st, lane);
      vf[st] = I::rows_frag(lds + SIMG + (wave >> 1) * I::IMG, (wave & 1) * 32 + (lane & 31), st, lane);
    }
  } else {
    I::template row_frags<E>((const E*)a.k + (sq.first + kk) * a.ldk + (long long)hk * a.d, kk < n, a.d, lane, kf);
    I::template row_frags<E>((const E*)a.v + (sq.first + kk) * a.ldv + (long long)hk * a.d, kk < n, a.d, lane, vf);
  }
  f32x16 dv[DP / 32], dk[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) { dv[t] = zero16(); dk[t] = zero16(); }
  const float c = a.scale * LOG2E, kept = DROP ? 256.0f / (256.0f - (float)a.drop) : 1.0f;
  DropKey key;
  if (DROP) key = drop_key(a.seed, a.site, a.step);
  float up = 0.f;
  if constexpr (SCALED) {
    float v_norm = 0.f, norm = 0.f, most_D = 0.f;
    for (int h = hk * group; h < (hk + 1) * group; ++h)
      for (int row = lane * 32; row < n; row += 64 * 32) {
        const uint32_t b2 = a.bounds[(long long)h * a.rows + sq.first + row];
        norm = fmaxf(norm, __builtin_bit_cast(float, b2 << 16));
        most_D = fmaxf(most_D, __builtin_bit_cast(float, b2 & 0xFFFF0000u));
      }
#pragma unroll
    for (int st = 0; st < DP / 16; ++st) {
      const typename Vec<E>::x8 x = __builtin_bit_cast(typename Vec<E>::x8, vf[st]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v_norm = fmaf(to_f32(x[j]), to_f32(x[j]), v_norm);
    }
    const float bound = fmaf(wave_max(norm), __builtin_amdgcn_sqrtf(half_sum(v_norm)), wave_max(most_D));
    up = UP_MOST - power_down(bound * 0x1p14f, UP_MOST);
  }
  int i = 0;   // tiles so far, of all heads
  const auto arrive = [&] {
    wait_vm0();
    __syncthreads();
    if (i + 1 < tiles) fetch(i + 1);
  };
  const auto compute = [&](int h, int row0, auto edge) {
    const char* Qs = lds + (i & 1) * STAGE;
    const char* Gs = Qs + I::IMG;
    const float* Ls = WHOLE ? (const float*)(lds + STAT + (h & 1) * 1024) + row0 : (const float*)(Gs + I::IMG);
    const float* Ds = Ls + (WHOLE ? 128 : 64);
    const int lim = a.causal ? kk - row0 - 4 * (lane >> 5) : 0;   // causal: rows below it do not see this lane's key
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      f32x16 s, g;   // (from -lse / scale and -D, as in the dQ kernel)
#pragma unroll
      for (int blk4 = 0; blk4 < 4; ++blk4) {
        const f32x4 L4 = *(const f32x4*)(Ls + qb * 32 + 8 * blk4 + 4 * (lane >> 5));
        const f32x4 D4 = *(const f32x4*)(Ds + qb * 32 + 8 * blk4 + 4 * (lane >> 5));
#pragma unroll
        for (int j = 0; j < 4; ++j) { s[4 * blk4 + j] = L4[j]; g[4 * blk4 + j] = DROP ? 0.f : D4[j]; }
      }
#pragma unroll
      for (int st = 0; st < DP / 16; ++st) {
        s = mfma_32x32x16<E>(I::rows_frag(Qs, qb * 32 + (lane & 31), st, lane), kf[st], s);
        g = mfma_32x32x16<E>(I::rows_frag(Gs, qb * 32 + (lane & 31), st, lane), vf[st], g);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(SCALED ? fmaf(s[r], c, up) : s[r] * c);
      if constexpr (decltype(edge)::value) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (qb * 32 + 8 * (r >> 2) + (r & 3) < lim) s[r] = 0.f;
      }
      u32x4 bytes;
      if (DROP) {
        bytes = drop_bytes<false>(row0 + qb * 32, key0, (uint32_t)(b * a.heads + h), key, lane);
#pragma unroll
        for (int blk4 = 0; blk4 < 4; ++blk4) {
          const f32x4 D4 = *(const f32x4*)(Ds + qb * 32 + 8 * blk4 + 4 * (lane >> 5));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = 4 * blk4 + j;
            const bool keep = drop_keeps(bytes, r, a.drop);
            g[r] = s[r] * (keep ? fmaf(g[r], kept, D4[j]) : D4[j]);
            if (!(WHOLE && decltype(edge)::value)) s[r] = drop_select(keep, s[r]);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] *= s[r];
      }
      if constexpr (WHOLE && decltype(edge)::value) {
        if (qb == 0 && few && row0 == 0) {   // D's error, as in the dQ kernel: the row's keys are this wave's lanes
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float off = kk < n ? g[r] : 0.f;
            off += dpp_move<0xB1>(off);
            off += dpp_move<0x4E>(off);
            off += dpp_move<0x141>(off);
            off += dpp_move<0x140>(off);
            off += __shfl_xor(off, 16);
            g[r] = fmaf(-s[r], off, g[r]);
          }
        }
        if (DROP) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = drop_select(drop_keeps(bytes, r, a.drop), s[r]);
        }
      }
      if (WHOLE && key0 + 32 > n) {   // a key past the sequence has a row of K that is zero, and a dS that may be anything
#pragma unroll
        for (int r = 0; r < 16; ++r) g[r] = kk < n ? g[r] : 0.f;
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8 pf = pack8<E>(s, 8 * s2), df = pack8<E>(g, 8 * s2);
#pragma unroll
        for (int t2 = 0; t2 < DP / 32; ++t2) {
          dv[t2] = mfma_32x32x16<E>(I::rows_T(Gs, qb, s2, t2, lane), pf, dv[t2]);
          dk[t2] = mfma_32x32x16<E>(I::rows_T(Qs, qb, s2, t2, lane), df, dk[t2]);
        }
        if constexpr (WHOLE) {   // registers 8 s2 .. of this key's row: queries 16 s2 + 8 {0, 1} + 4 (lane / 32) + 0..3
          const int row = key0 + (lane & 31);
          const u32x4 w = __builtin_bit_cast(u32x4, df);
#pragma unroll
          for (int x = 0; x < 2; ++x)
            *(u32x2*)(lds + SIMG + row * IS::PITCH + IS::slot(row & 63, qb * 4 + 2 * s2 + x) * 16 + 8 * (lane >> 5)) = x ? u32x2{w.z, w.w} : u32x2{w.x, w.y};
        }
      }
      if (WHOLE) __builtin_amdgcn_sched_barrier(0);   // (the halves side by side want more registers than two waves a SIMD have)
    }
  };
  // WHOLE: dQ^T = K^T dS^T of the tile, a 32 x 32 block of (columns, queries) to a wave at a time
  const auto query_grads = [&](int h, int row0) {
    __syncthreads();   // every wave's dS is in
    const int nkb = min((n + 31) / 32, a.causal ? (row0 + CHA) / 32 : 4);   // (the keys behind have no weight and no dS)
#pragma unroll
    for (int j = 0; j < (2 * (DP / 32) + 3) / 4; ++j) {
      const int idx = wave + 4 * j, qb = idx & 1, t2 = idx >> 1, q = row0 + qb * 32 + (lane & 31);
      if (t2 >= DP / 32) break;
      f32x16 dq = zero16();
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
        if (kb < nkb) {
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2)
            dq = mfma_32x32x16<E>(I::rows_T(lds + KIMG + (kb >> 1) * I::IMG, kb & 1, s2, t2, lane),
                                  IS::rows_T(lds + SIMG + (kb >> 1) * IS::IMG, kb & 1, s2, qb, lane), dq);
        }
      if (q < n) {
        E* out = (E*)a.dq + (sq.first + q) * a.lddq + (long long)h * a.d;
#pragma unroll
        for (int blk4 = 0; blk4 < 4; ++blk4) {
          const int col = t2 * 32 + blk4 * 8 + 4 * (lane >> 5);
          typename Vec<E>::x4 v;
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] = from_f32<E>(dq[blk4 * 4 + x] * a.scale);
          if (col < a.d) *(typename Vec<E>::x4*)(out + col) = v;
        }
      }
    }
  };
  // per head: tiles before the wave's first key, where it only helps to load, those with a mask, those whole
  const int idle = !active ? per_head : a.causal ? min(per_head, key0 / CHA - t0) : 0;
  const int masked = a.causal ? min(per_head, (key0 + 31 + CHA - 1) / CHA - t0) : WHOLE && few ? 1 : 0;   // (the first tile: D's error)
  for (int h = h0; i < tiles; ++h) {
    int t = h == h0 ? from % per_head : 0;
    const int end = min(per_head, t + tiles - i);
    if (WHOLE && h != h0) head_stats(h);
    const auto grads = [&] {
      if constexpr (WHOLE) query_grads(h, (t0 + t) * CHA);
    };
    for (; t < min(idle, end); ++t, ++i) { arrive(); grads(); }
    for (; t < min(masked, end); ++t, ++i) { arrive(); compute(h, (t0 + t) * CHA, std::true_type{}); grads(); }
    for (; t < end; ++t, ++i) { arrive(); compute(h, (t0 + t) * CHA, std::false_type{}); grads(); }
  }
  __syncthreads();
  if (!active) return;
  const float down = SCALED ? __builtin_amdgcn_exp2f(-up) : 1.f, scale_v = kept * down, scale_k = a.scale * down;
  if (a.splits_dkv > 1) {
    const long long width = (long long)a.kv_heads * a.d, row = 2LL * split * a.rows + sq.first + kk;
    store_part<DP>(dv, a.part + row * width + (long long)hk * a.d, kk < n, a.d, lane, scale_v);
    store_part<DP>(dk, a.part + (row + a.rows) * width + (long long)hk * a.d, kk < n, a.d, lane, scale_k);
    return;
  }
  char* stage = lds + wave * (STAGE / 2);
  store_rows<E, DP>(dv, stage, (E*)a.dv + (sq.first + key0) * a.lddv + (long long)hk * a.d, a.lddv, n - key0, a.d, lane, scale_v);
  store_rows<E, DP>(dk, stage, (E*)a.dk + (sq.first + key0) * a.lddk + (long long)hk * a.d, a.lddk, n - key0, a.d, lane, scale_k);
}

// ---- partial results of the splits together -------------------------------------------------------------------------------
// out = sum over the splits of part, or with WEIGHTED (forward) of w_s part_s / sum w with w_s = sum_s e^(scale (m_s - m)), from the maxima and sums
// themselves (weights from an lse per split would carry its last bit, 2^-24 of the score, into O).  A workgroup takes 64 rows of one
// (sequence, head), eight columns a thread; splits in their order.  Bound by memory, the splits' share of it.
struct JoinArgs {
  const float* part[2];     // of dV and dK; otherwise one
  long long split_stride;   // elements from a split to the next
  const float *part_m, *part_sum;   // WEIGHTED
  float* lse;               // WEIGHTED: or null
  void* out[2];
  long long ldo[2];
  int splits, heads;        // heads of `out`
};
template <typename E, bool WEIGHTED>
__global__ __launch_bounds__(256) void seq_join_kernel(const SeqAttnArgs a, const JoinArgs j) {
  const int nblk = (a.max_len + 63) / 64, blk = blockIdx.x % nblk, bh = blockIdx.x / nblk, b = bh / j.heads, h = bh % j.heads;
  const float* part = j.part[blockIdx.y];
  E* out = (E*)j.out[blockIdx.y];
  const long long ldo = j.ldo[blockIdx.y];
  const Seq sq = sequence(a, b);
  const int chunks = a.d / 8;
  for (int u = threadIdx.x; u < 64 * chunks; u += 256) {
    const int i = blk * 64 + u / chunks, col = u % chunks * 8;
    if (i >= sq.n) return;
    const long long row = sq.first + i, at = row * ((long long)j.heads * a.d) + (long long)h * a.d + col;
    // four splits' loads at a time, without a branch between them: places past the last split are read again and count nothing
    float top = -INFINITY, total = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const auto stat_of = [&](const float* stat, int s) { return stat[((long long)min(s, j.splits - 1) * j.heads + h) * a.rows + row]; };
    if (WEIGHTED) {
      for (int s0 = 0; s0 < j.splits; s0 += 4) {
        float m[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) m[x] = stat_of(j.part_m, s0 + x);
        top = fmaxf(fmaxf(top, fmaxf(m[0], m[1])), fmaxf(m[2], m[3]));
      }
    }
    for (int s0 = 0; s0 < j.splits; s0 += 4) {
      float v[4][8], m[4], w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        load8(part + min(s0 + x, j.splits - 1) * j.split_stride + at, v[x]);
        if (WEIGHTED) { m[x] = stat_of(j.part_m, s0 + x); w[x] = stat_of(j.part_sum, s0 + x); }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (s0 + x >= j.splits) continue;
        if (WEIGHTED) {
          if (w[x] != 0.f) w[x] *= __builtin_amdgcn_exp2f((m[x] - top) * (a.scale * LOG2E));   // (0: a split without a key that the row sees)
          total += w[x];
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] = WEIGHTED ? fmaf(v[x][c], w[x], acc[c]) : acc[c] + v[x][c];
      }
    }
    if (WEIGHTED) {
#pragma unroll
      for (int x = 0; x < 8; ++x) acc[x] /= total;
      if (j.lse && col == 0) j.lse[(long long)h * a.rows + row] = fmaf(top, a.scale, __builtin_amdgcn_logf(total) * LN2);
    }
    store8(out + row * ldo + (long long)h * a.d + col, acc);
  }
}

}  // namespace sattn
