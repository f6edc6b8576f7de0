// Dropout with bias and residual, and token log probabilities with entropy and top alternatives: kernels and launchers of the
// single operations that pass over memory once (entry points and checks: l2l.hip).
#include <algorithm>
#include <type_traits>

#include "dropout.h"
#include "ops.h"

namespace {

// 16 bytes at any element boundary: rows of an odd length start anywhere, and the memory path takes such accesses whole
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Vec16 { T v[N]; };
template <typename T>
struct Line {
  static constexpr int N = 16 / (int)sizeof(T);
  Vec16<T, N> r;
};

// ---- dropout -------------------------------------------------------------------------------------------------------------
// y = resid + Z (x + bias); backward dx = Z dy and the column sums of dx (the bias gradient).  Z = 0 or 1 / kept share from
// the generator in dropout.h: 16 bits an element, eight neighbours of a row from one call, nothing stored.
// Bound by memory.  A thread owns eight columns and walks every (256 / CW)-th row of a block of rows, up to four rows requested at
// a time; CW threads lie along the columns.  The column sums stay in fp32 registers, then add up across the workgroup's row lanes and leave as
// one row of partial sums per block, which a second kernel adds in a fixed order: no atomics, so the same call gives the same bits.

struct DropGrid { int cw, lanes, groups, per, blocks; };   // threads along columns, row lanes, column groups, rows per thread, row blocks
DropGrid drop_grid(int rows, int n) {
  DropGrid g;
  const int chunks = (n + 7) / 8;
  // threads along the columns: a power of two up to 64, the one that leaves the fewest without columns
  const auto covered = [&](int cw) { return (long long)(chunks + cw - 1) / cw * cw; };
  g.cw = 64;
  for (int cw = 32; cw >= std::min(16, chunks); cw /= 2)
    if (covered(cw) < covered(g.cw)) g.cw = cw;
  g.lanes = 256 / g.cw;
  g.groups = (chunks + g.cw - 1) / g.cw;
  // rows per thread: 1, 2 or a multiple of 4, as many as leave two thousand workgroups, at most 16 (the partial sums are then a
  // sixtieth of the traffic at most)
  const long long share = (long long)rows * g.groups / g.lanes / 2048;
  g.per = share >= 4 ? (int)std::min<long long>(16, share / 4 * 4) : share >= 2 ? 2 : 1;
  g.blocks = (rows + g.lanes * g.per - 1) / (g.lanes * g.per);
  return g;
}

// Column sums of few rows: a workgroup to every eight columns, with a row to a thread, has all that goes into them, and the second kernel is
// not run.  256 rows of 128 columns: 4.9 us instead of 4.1 + 2.5 and a launch; with four rows to a thread, 1024 of 1024, 8.0 against 4.9 + 2.9.
constexpr int DROP_ONE_BLOCK_ROWS = 256;
DropGrid drop_grid_one_block(int n) { return DropGrid{1, DROP_ONE_BLOCK_ROWS, (n + 7) / 8, 1, 1}; }

// v[i] = v[i + by], 0 <= by < 8 (what comes from behind is not looked at)
__device__ __forceinline__ void move_down(float (&v)[8], int by) {
#pragma unroll
  for (int step = 4; step; step >>= 1)
#pragma unroll
    for (int i = 0; i + step < 8; ++i) v[i] = by & step ? v[i + step] : v[i];
}

// ROWS: rows in flight per thread
template <typename T, int ROWS, bool RESID, bool SUMS, bool TINY>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4)))
void dropout_kernel(const DropoutArgs a, int cw, int lanes, int groups, int per) {
  using Line8 = Vec16<T, 8>;
  const int group = blockIdx.x % groups, block = blockIdx.x / groups;
  const int chunk = group * cw + threadIdx.x % cw, row_lane = threadIdx.x / cw, col = chunk * 8;
  const int count = min(8, a.n - col);   // <= 0: this thread has no columns
  // Every line of every row is loaded, without a branch between the loads: a thread whose own would pass the end of the row takes the
  // row's last eight columns and moves its own to the front (TINY, fewer than eight in all: one by one), one whose row would pass
  // the last row takes that.
  const int at = min(col, a.n - 8), by = min(7, col - at);
  const long long row0 = (long long)block * lanes * per + row_lane;
  const DropKey key = drop_key(a.seed, a.site, a.step);
  const float kept = 65536.0f / (65536.0f - (float)a.drop);
  const auto load = [&](const void* base, long long row, long long ld) {
    const T* p = (const T*)base + row * ld;
    Line8 x;
    if constexpr (TINY) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x.v[i] = p[min(i, a.n - 1)];
    } else {
      x = *(const Line8*)(p + at);
    }
    return x;
  };
  const auto widen = [&](const Line8& x, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(x.v[i]);
    if (!TINY && by) move_down(v, by);
  };
  float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sums[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (a.bias) widen(load(a.bias, 0, 0), bias);
  for (int j = 0; j < per; j += ROWS) {
    Line8 x[ROWS], res[RESID ? ROWS : 1];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long row = min(row0 + (long long)(j + u) * lanes, (long long)a.rows - 1);
      x[u] = load(a.x, row, a.ldx);
      if constexpr (RESID) res[u] = load(a.resid, row, a.ldr);
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      const long long row = row0 + (long long)(j + u) * lanes;
      const bool live = row < a.rows;
      const u32x4 w = philox7((uint32_t)chunk, (uint32_t)row, key);
      float v[8], r[8];
      widen(x[u], v);
      if constexpr (RESID) widen(res[u], r);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t bits = (w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
        const float z = bits >= a.drop ? (v[i] + bias[i]) * kept : 0.f;
        if (SUMS) sums[i] += live ? z : 0.f;
        v[i] = RESID ? r[i] + z : z;
      }
      if (!live) continue;
      T* out = (T*)a.y + row * a.ldy + col;
      if (count >= 8) {
        Line8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = from_f32<T>(v[i]);
        *(Line8*)out = y;
      } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
          if (i < count) out[i] = from_f32<T>(v[i]);
      }
    }
  }
  if constexpr (SUMS) {
    __shared__ float red[256][9];   // (9: the eight values of 64 lanes spread over the banks)
#pragma unroll
    for (int i = 0; i < 8; ++i) red[threadIdx.x][i] = sums[i];
    __syncthreads();
    if (a.rows <= DROP_ONE_BLOCK_ROWS) {   // all rows are here, of eight columns: 32 threads to a column, then one
      __shared__ float red2[32][9];
      const int i = threadIdx.x & 7, l0 = threadIdx.x >> 3;
      float s = 0.f;
#pragma unroll
      for (int l = 0; l < 8; ++l) s += red[l0 + 32 * l][i];
      red2[l0][i] = s;
      __syncthreads();
      if (threadIdx.x < 8 && group * 8 + i < a.n) {
        const float old = a.accumulate ? a.dbias[group * 8 + i] : 0.f;
        s = 0.f;
#pragma unroll
        for (int l = 0; l < 32; ++l) s += red2[l][i];
        a.dbias[group * 8 + i] = old + s;
      }
      return;
    }
    for (int u = threadIdx.x; u < cw * 8; u += 256) {
      const int c = u / 8, i = u % 8, to = (group * cw + c) * 8 + i;
      float s = 0.f;
      for (int l = 0; l < lanes; ++l) s += red[l * cw + c][i];
      if (to < a.n) a.part[(long long)block * a.n + to] = s;
    }
  }
}

// dbias (+)= the partial sums: 16 columns a workgroup, 64 lanes down the blocks.  Bound by the latency of one round of loads (eight
// at a time, unconditional ones: places past the end are read again and count nothing) and of the sum over the lanes.
constexpr int DROP_SUM_NT = 1024;
__global__ __launch_bounds__(DROP_SUM_NT) void dropout_sum_kernel(const float* part, int blocks, int n, float* dbias, int accumulate) {
  __shared__ float red[64][17], red2[16][17];
  const int c = threadIdx.x & 15, l = threadIdx.x >> 4, col = blockIdx.x * 16 + c, from = min(col, n - 1);
  const float old = accumulate ? dbias[from] : 0.f;
  float s = 0.f;
  for (int b0 = l; b0 < blocks; b0 += 64 * 8) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = part[(long long)min(b0 + 64 * u, blocks - 1) * n + from];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += b0 + 64 * u < blocks ? v[u] : 0.f;
  }
  red[l][c] = s;
  __syncthreads();
  if (l < 16) red2[l][c] = (red[4 * l][c] + red[4 * l + 1][c]) + (red[4 * l + 2][c] + red[4 * l + 3][c]);
  __syncthreads();
  if (l == 0 && col < n) {
    s = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) s += red2[j][c];
    dbias[col] = old + s;
  }
}

template <typename T>
void launch_dropout_t(const DropoutArgs& a, hipStream_t s) {
  const bool one_block = a.dbias && a.rows <= DROP_ONE_BLOCK_ROWS;
  const DropGrid g = one_block ? drop_grid_one_block(a.n) : drop_grid(a.rows, a.n);
  const dim3 grid((unsigned)((long long)g.groups * g.blocks));
  const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, g.cw, g.lanes, g.groups, g.per); };
  const auto rows = [&](auto resid, auto sums) {
    constexpr bool R = decltype(resid)::value, S = decltype(sums)::value;
    if (a.n < 8) go(dropout_kernel<T, 1, R, S, true>);
    else if (g.per >= 4) go(dropout_kernel<T, 4, R, S, false>);
    else if (g.per == 2) go(dropout_kernel<T, 2, R, S, false>);
    else go(dropout_kernel<T, 1, R, S, false>);
  };
  if (a.dbias) {
    rows(std::false_type{}, std::true_type{});
    if (!one_block) hipLaunchKernelGGL(dropout_sum_kernel, dim3((a.n + 15) / 16), dim3(DROP_SUM_NT), 0, s, a.part, g.blocks, a.n, a.dbias, a.accumulate);
  } else if (a.resid) {
    rows(std::true_type{}, std::false_type{});
  } else {
    rows(std::false_type{}, std::false_type{});
  }
}

// ---- token log probabilities ---------------------------------------------------------------------------------------------
// Of a row of logits x, with m = max, s = sum e^(x - m), t = sum e^(x - m) (x - m): lse = m + log s, log p(id) = x[id] - m - log s, entropy
// = log s - t / s; and the `top` largest by (value, lowest index first).  One pass over memory: a workgroup holds a slab of the row in
// registers, from which it takes the sums and the candidates for the top.  A value can be among the top k only if it is not
// below the k-th largest of any 64 values of the row; each wave takes that bound from its lanes' own maxima (a binary search by
// ballots over their leading bits), and what reaches the highest bound known goes to a list in LDS: some dozens of the row, of
// which each counts in the end how many are before it, its place.  Where equal values overflow the list, the workgroup searches the top one by one.
// Bound by memory: two workgroups of 512 threads share a compute unit and load under each other's reductions.
// Rows too few to fill the chip are split over workgroups, whose parts a second kernel joins.
constexpr int LP_LIST = 1024, LP_TOP = 32;
constexpr float LP_NEAR = 0x1p20f;   // (half a step of x log2(e) is 1/16 at most below it)
constexpr float LP_FAR = -1.0e4f;   // 2^x is 0 from here down, and 0 * x has to be 0 as well for x = -inf
constexpr float LP_LOG2E = 1.4426950408889634f, LP_LN2 = 0.6931471805599453f;

// whole numbers in the order of the values (-0 and 0 alike, every NaN before everything)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return x != x ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// larger = earlier in the top: the value, then the lower index
__device__ __forceinline__ uint64_t rank_key(uint32_t key, uint32_t index) { return (uint64_t)key << 32 | (0xFFFFFFFFu - index); }

// m = the largest x, s = sum 2^d, t = sum 2^d d with d = (x - m) log2(e).  m is a logit itself and every difference is taken before its
// product: a rounded m log2(e) is off by half a step of its own, which is a factor of the sums wherever logits are far from zero (a
// vocabulary masked with -1e10 or the type's lowest value: 2^128 and more), and overflows from 2.4e38 on.
struct Stat { float m, s, t; };
__device__ __forceinline__ float log2_ratio(float x, float m) { return fmaxf((x - m) * LP_LOG2E, LP_FAR); }   // (NaN becomes LP_FAR)
// both relative to their own maximum; an empty one (m = -inf, s = t = 0) changes nothing
__device__ __forceinline__ Stat join(Stat a, Stat b) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  if (r.m == -INFINITY) return Stat{r.m, a.s + b.s, a.t + b.t};
  const float da = log2_ratio(a.m, r.m), db = log2_ratio(b.m, r.m), fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  r.s = a.s * fa + b.s * fb;
  r.t = (a.t + a.s * da) * fa + (b.t + b.s * db) * fb;
  return r;
}
__device__ __forceinline__ Stat wave_join(Stat a) {
  Stat r;
  r.m = wave_max(a.m);
  const float d = r.m == -INFINITY ? 0.f : log2_ratio(a.m, r.m), f = __builtin_amdgcn_exp2f(d);
  r.s = wave_sum(a.s * f);
  r.t = wave_sum((a.t + a.s * d) * f);
  return r;
}

// each lane's entry to its place among the first `found` lanes' if that is one of the `top` first
__device__ __forceinline__ void place_64(uint64_t k, int found, int lane, int top, uint64_t* best) {
  int before = 0;
  for (int o = 0; o < found; ++o) {
    const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), o) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, o);
    before += other > k;
  }
  if (lane < found && before < top) best[before] = k;
}

// the largest number, to 13 leading bits, that `count` lanes' keys reach
__device__ __forceinline__ uint32_t lanes_reach(uint32_t key, int count) {
  uint32_t reach = 0;
#pragma unroll
  for (int bit = 31; bit >= 19; --bit)
    if (__popcll(__ballot(key >= (reach | 1u << bit))) >= count) reach |= 1u << bit;
  return reach;
}

// every logit is -inf (a NaN among them, which no maximum shows, is in the sum)
__device__ __forceinline__ bool nothing(Stat st) { return st.m == -INFINITY && st.s == 0.f; }
// log p of a logit x of the row
__device__ __forceinline__ float log_prob(Stat st, float x) {
  return nothing(st) ? -INFINITY : (x - st.m) - log2f(st.s) * LP_LN2;
}
__device__ __forceinline__ void write_row(const LogprobArgs& a, int row, Stat st, int id, float x_id) {
  const bool none = nothing(st);
  const float log_s = log2f(st.s);
  a.lse[row] = none ? -INFINITY : fmaf(log_s, LP_LN2, st.m);
  a.entropy[row] = none ? 0.f : (log_s - st.t / st.s) * LP_LN2;
  if (id >= a.vocab) atomicOr(a.bad, 1);   // (clamped)
  if (a.ids) a.logp[row] = id < 0 ? 0.f : log_prob(st, x_id);
}

// NT threads, NV lines of 16 bytes each; AHEAD: for rows of several slabs, the next one's lines on their way while one is worked on (else
// the slab is the whole range), and the next row's behind the last slab; TINY: vocabularies shorter than a line
template <typename T, int NT, int NV, bool AHEAD, bool TINY = false>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4)))
void logprob_kernel(const LogprobArgs a) {
  constexpr int N = Line<T>::N, SLAB = NT * N * NV, WAVES = NT / 64;
  static_assert(N * NV <= 64, "a thread's values are bits of a word");
  __shared__ uint64_t lists[AHEAD ? 2 : 1][LP_LIST], best[LP_TOP];   // (two lists, taken in turn: a wave may be a row ahead of another)
  __shared__ Stat wave_stat[WAVES];
  __shared__ int counts[2];
  __shared__ uint32_t bounds[2], wave_bound[WAVES];
  const int split = blockIdx.x % a.splits, stride = gridDim.x / a.splits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, top = a.top;
  // (splits begin at whole lines, so that all but the last one are of equal length)
  const int chunks = (a.vocab + N - 1) / N, per_split = (chunks + a.splits - 1) / a.splits * N;
  const int begin = min(a.vocab, split * per_split), end = min(a.vocab, begin + per_split), last = max(0, end - N);
  // Every line is loaded, the last whole one of the range where a thread's own would pass the end (no branch between the
  // loads, so that all are under way at once); what it holds of other threads' values becomes -inf.
  using Line16 = Vec16<T, N>;
  Line16 r[NV], next[AHEAD ? NV : 1];
  const auto load = [&](Line16 (&to)[NV], const T* x, int from) {
    if constexpr (!TINY) {
#pragma unroll
      for (int j = 0; j < NV; ++j) to[j] = *(const Line16*)(x + min(from + (j * NT + tid) * N, last));
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) to[j].v[i] = i < a.vocab ? x[i] : from_f32<T>(-INFINITY);
    }
  };
  int row = blockIdx.x / a.splits;
  load(r, (const T*)a.logits + (long long)row * a.ld, begin);
  if (tid < 2) { counts[tid] = 0; bounds[tid] = 0; }
  if (top) __syncthreads();
  int turn = 0;
  do {
    const T* x = (const T*)a.logits + (long long)row * a.ld;
    // (through the scalar cache, and its logit by every thread: neither is waited for before the lines, and the logit not before the end)
    const int id = a.ids ? *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.ids + row) : -1;
    const float x_id = to_f32(x[max(0, min(id, a.vocab - 1))]);
    uint64_t* list = lists[turn];
    Stat st = {-INFINITY, 0.f, 0.f};   // of this wave's values
    for (int slab = begin; slab < end; slab += SLAB) {
      // (behind the last row's last slab every thread asks for one line of it: under a condition, the loads of both paths would be waited for here)
      if constexpr (AHEAD) {
        const bool more = slab + SLAB < end, rows = row + stride < a.rows;
        load(next, more || !rows ? x : x + (long long)stride * a.ld, more ? slab + SLAB : rows ? begin : end);
      }
      int own0 = slab + tid * N;
      const auto own = [&](int j) { return own0 + j * NT * N; };   // the first index this thread answers for,
      const auto at = [&](int j) { return min(own(j), last); };    // and where its line starts
      float lm = -INFINITY;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (own(j) + N > end) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (at(j) + i < own(j)) r[j].v[i] = from_f32<T>(-INFINITY);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) lm = fmaxf(lm, to_f32(r[j].v[i]));
      }
      // (what is derived from the values is derived again where it is used next: kept, it would take a multiple of their registers)
      const auto forget = [&] {
        asm("" : "+v"(own0));
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          u32x4 raw = __builtin_bit_cast(u32x4, r[j]);
          asm("" : "+v"(raw));
          r[j] = __builtin_bit_cast(Line16, raw);
        }
      };
      forget();
      // One fma a value, x log2(e) - lm log2(e) with the second product rounded, and what that rounding left out (up to 1/16) taken out of the
      // sums behind; where a maximum of the wave lies too far from zero for it, the difference first.  (4915 rows of 30522 in fp32: 117 us; the
      // difference first everywhere 120; 16-bit rows take as long either way.)
      Stat mine = {lm, 0.f, 0.f};
      const float own_m = lm == -INFINITY ? 0.f : lm;
      const auto add = [&](float d) {
        const float e = __builtin_amdgcn_exp2f(d);
        mine.s += e;
        mine.t = fmaf(e, fmaxf(d, LP_FAR), mine.t);
      };
      if (__any(!(fabsf(own_m) < LP_NEAR))) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          u32x4 raw = __builtin_bit_cast(u32x4, r[j]);   // (a copy that shares nothing with the other branch)
          asm("" : "+v"(raw));
          const Line16 line = __builtin_bit_cast(Line16, raw);
#pragma unroll
          for (int i = 0; i < N; ++i) add((to_f32(line.v[i]) - own_m) * LP_LOG2E);
        }
      } else {
        const float base = own_m * LP_LOG2E, rest = fmaf(own_m, LP_LOG2E, -base);   // own_m log2(e) = base + rest
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < N; ++i) add(fmaf(to_f32(r[j].v[i]), LP_LOG2E, -base));
        const float back = __builtin_amdgcn_exp2f(-rest);
        mine.t = (mine.t - mine.s * rest) * back;
        mine.s *= back;
      }
      st = join(st, wave_join(mine));
      if (top) {
        // The bound may be any that is one: if each of t waves has q lanes whose maxima reach b, and t q >= top, then b is.  The first
        // slab's is the t-th largest of the waves' own, each the largest, to 13 leading bits, that q lanes reach; with q near top / (half
        // the waves) it leaves a fraction of the candidates that the best wave's alone would (q = top).  Behind it waves
        // raise it by that one, and read it, without waiting for each other.
        const uint32_t key = order_key(lm);
        uint32_t least;
        if (slab == begin) {
          const int half = max(1, min(WAVES, (end - begin + 64 * N - 1) / (64 * N)) / 2);   // (of the waves that have values)
          const int q = (top + half - 1) / half, t = (top + q - 1) / q;
          const uint32_t reach = lanes_reach(key, q);
          if (lane == 0) wave_bound[wave] = reach;
          __syncthreads();
          const uint32_t b = lane < WAVES ? wave_bound[lane] : 0;
          int reached_by = 0;
#pragma unroll
          for (int o = 0; o < WAVES; ++o) reached_by += (uint32_t)__builtin_amdgcn_readlane((int)b, o) >= b;
          const uint32_t cand = reached_by >= t ? b : 0;
          least = 0;
#pragma unroll
          for (int o = 0; o < WAVES; ++o) least = max(least, (uint32_t)__builtin_amdgcn_readlane((int)cand, o));
          if (tid == 0) atomicMax(&bounds[turn], least);
        } else {
          least = *(volatile uint32_t*)&bounds[turn];
          if (__popcll(__ballot(key > least)) >= top) {
            const uint32_t reach = lanes_reach(key, top);
            if (lane == 0) atomicMax(&bounds[turn], reach);
            least = max(least, reach);
          }
        }
        const float least_value = key_value(least);
        if (!(lm < least_value)) {   // (few threads)
          // which of the lines' values, as bits; then one at a time, read again (a line's place in registers cannot be computed)
          forget();
          uint64_t reached = 0;
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) reached |= (uint64_t)!(to_f32(r[j].v[i]) < least_value) << (j * N + i);
          while (reached) {
            const int e = __builtin_ctzll(reached), index = at(e / N) + e % N;
            reached &= reached - 1;
            if (index >= own(e / N) && index < end) {
              const int slot = atomicAdd(&counts[turn], 1);
              if (slot < LP_LIST) list[slot] = rank_key(order_key(to_f32(x[index])), (uint32_t)index);
            }
          }
        }
      }
      if constexpr (AHEAD) {
#pragma unroll
        for (int j = 0; j < NV; ++j) r[j] = next[j];
      }
    }
    if (lane == 0) wave_stat[wave] = st;
    __syncthreads();
    st = wave_stat[0];
    for (int j = 1; j < WAVES; ++j) st = join(st, wave_stat[j]);
    if (tid == 0) { counts[turn ^ 1] = 0; bounds[turn ^ 1] = 0; }
    int have = 0;
    if (top) {
      const int found = counts[turn];
      have = min(found, top);
      if (found <= 64) {   // (one wave, whose lanes read each other)
        if (wave == 0) place_64(lane < found ? list[lane] : 0, found, lane, top, best);
      } else if (found <= LP_LIST) {
        for (int u = tid; u < found; u += NT) {
          const uint64_t k = list[u];
          int before = 0;
#pragma unroll 8
          for (int o = 0; o < found; ++o) before += list[o] > k;
          if (before < top) best[before] = k;
        }
      } else {
        // too many equal ones: one by one, the largest after the previous one, from memory
        uint64_t prev = ~0ull;
        for (int n = 0; n < top; ++n) {
          uint64_t k = 0;
          for (int index = begin + tid; index < end; index += NT) {
            const uint64_t o = rank_key(order_key(to_f32(x[index])), (uint32_t)index);
            if (o < prev && o > k) k = o;
          }
#pragma unroll
          for (int off = 32; off; off >>= 1) {
            const uint64_t o = (uint64_t)__shfl_xor((unsigned)(k >> 32), off, 64) << 32 | __shfl_xor((unsigned)k, off, 64);
            k = o > k ? o : k;
          }
          __syncthreads();
          if (lane == 0) list[wave] = k;
          __syncthreads();
          for (int j = 0; j < WAVES; ++j) k = max(k, list[j]);
          if (tid == 0) best[n] = k;
          prev = k;
        }
      }
    }
    __syncthreads();
    if (a.splits == 1) {
      if (tid == 0) write_row(a, row, st, id, x_id);
      if (tid < top) {
        const uint64_t k = best[tid];
        a.top_ids[(long long)row * top + tid] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
        a.top_logp[(long long)row * top + tid] = log_prob(st, key_value((uint32_t)(k >> 32)));
      }
    } else {
      // [rows][splits] of: m, s, t, x[id]; then `top` ranks (fewer: zeros, which are behind everything)
      float* part = (float*)a.work + ((long long)row * a.splits + split) * 4;
      uint64_t* ranks = (uint64_t*)((float*)a.work + (long long)a.rows * a.splits * 4) + ((long long)row * a.splits + split) * top;
      if (tid == 0) { part[0] = st.m; part[1] = st.s; part[2] = st.t; part[3] = x_id; }
      if (tid < top) ranks[tid] = tid < have ? best[tid] : 0;
    }
    row += stride;
    turn ^= 1;
  } while (AHEAD && row < a.rows);
}

__global__ __launch_bounds__(256) void logprob_join_kernel(const LogprobArgs a) {
  __shared__ uint64_t list[LP_LIST];
  const int row = blockIdx.x, tid = threadIdx.x, top = a.top, n = a.splits * top;
  const float* part = (const float*)a.work + (long long)row * a.splits * 4;
  const uint64_t* ranks = (const uint64_t*)((const float*)a.work + (long long)a.rows * a.splits * 4) + (long long)row * n;
  for (int u = tid; u < n; u += 256) list[u] = ranks[u];
  Stat st = {-INFINITY, 0.f, 0.f};
  for (int j = 0; j < a.splits; ++j) st = join(st, Stat{part[4 * j], part[4 * j + 1], part[4 * j + 2]});
  __syncthreads();
  if (tid == 0) write_row(a, row, st, a.ids ? a.ids[row] : -1, part[3]);
  for (int u = tid; u < n; u += 256) {
    const uint64_t k = list[u];
    int before = 0;
    for (int o = 0; o < n; ++o) before += list[o] > k;
    if (k && before < top) {
      a.top_ids[(long long)row * top + before] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
      a.top_logp[(long long)row * top + before] = log_prob(st, key_value((uint32_t)(k >> 32)));
    }
  }
}

// From which |lse| on its last bit, half a step of 2^-23 |lse|, is too coarse for log p: it may be off by 2^-17 in fp32, by 2^-13 (a quarter
// of the half step that fp16 rounds by) in 16-bit formats.
template <typename T>
constexpr float kFarLse = sizeof(T) == 4 ? 256.f : 4096.f;

// The lines of a row, four at a time, by a workgroup of 256 threads: f(first index, values, their number).
template <typename T, typename F>
__device__ __forceinline__ void row_lines(const T* x, int vocab, F&& f) {
  constexpr int N = Line<T>::N, PER = 4;
  for (int from = threadIdx.x * N; from < vocab; from += PER * 256 * N) {
    Vec16<T, N> r[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int at = from + j * 256 * N;
      if (at + N <= vocab) {
        r[j] = *(const Vec16<T, N>*)(x + at);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r[j].v[i] = at + i < vocab ? x[at + i] : from_f32<T>(-INFINITY);
      }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int at = from + j * 256 * N;
      if (at < vocab) f(at, r[j], min(N, vocab - at));
    }
  }
}

// max and log sum e^(x - max) of a row, by a workgroup of 256 threads
template <typename T>
__device__ __forceinline__ void row_stat(const T* x, int vocab, float& m, float& log_s) {
  constexpr int N = Line<T>::N;
  __shared__ Stat waves[4];
  Stat st = {-INFINITY, 0.f, 0.f};
  row_lines(x, vocab, [&](int, const Vec16<T, N>& r, int) {
    Stat line = {to_f32(r.v[0]), 0.f, 0.f};
#pragma unroll
    for (int i = 1; i < N; ++i) line.m = fmaxf(line.m, to_f32(r.v[i]));
    const float own_m = line.m == -INFINITY ? 0.f : line.m;
#pragma unroll
    for (int i = 0; i < N; ++i) line.s += __builtin_amdgcn_exp2f((to_f32(r.v[i]) - own_m) * LP_LOG2E);
    st = join(st, line);
  });
  st = wave_join(st);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = st;
  __syncthreads();
  st = join(join(waves[0], waves[1]), join(waves[2], waves[3]));
  m = st.m;
  log_s = log2f(st.s) * LP_LN2;
}

// d logits = g (onehot - p) - h p (log p + H): g, h the gradients of log p(id) and of the entropy.  Element-wise; in place allowed.
// A row too far from zero for lse to hold log p (one that is masked as a whole, with -1e9 or the type's lowest value, say) is left to one of
// its workgroups, which takes the maximum and the sum from the logits again, before it writes any (in place, another one's would be gone).
// 1024 rows of 128257 in bf16: 103 to 116 us; all of them too far 310.  One row of 30522 in fp32: 6 and 16.
template <typename T>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(const LogprobArgs a, int blocks_per_row) {
  constexpr int N = Line<T>::N, PER = 4;
  const int row = blockIdx.x / blocks_per_row, block = blockIdx.x % blocks_per_row;
  const T* x = (const T*)a.logits + (long long)row * a.ld;
  T* dx = (T*)a.dlogits + (long long)row * a.ldd;
  int id = a.ids ? a.ids[row] : -1;
  if (id >= a.vocab) id = a.vocab - 1;
  const float g = id >= 0 && a.dlogp ? a.dlogp[row] : 0.f, h = a.dentropy ? a.dentropy[row] : 0.f;
  const float lse = a.lse[row], H = a.dentropy ? a.entropy[row] : 0.f;
  const bool none = lse == -INFINITY;
  const auto grad_of = [&](float lp, int at) { return (at == id ? g : 0.f) - __expf(lp) * fmaf(h, fmaxf(lp, LP_FAR) + H, g); };
  if (fabsf(lse) >= kFarLse<T> && !none) {
    if (block != row % blocks_per_row) return;   // (the XCDs take blocks in turn: the first ones of all rows may be one XCD's)
    float m, log_s;
    row_stat(x, a.vocab, m, log_s);
    row_lines(x, a.vocab, [&](int at, Vec16<T, N> r, int count) {   // (in place: what a thread reads is its own to write)
#pragma unroll
      for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(grad_of((to_f32(r.v[i]) - m) - log_s, at + i));
      if (count == N) {
        *(Vec16<T, N>*)(dx + at) = r;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < count) dx[at + i] = r.v[i];
      }
    });
    return;
  }
  const auto grad = [&](float v, int at) {
    const float d = grad_of(v - lse, at);
    return none ? 0.f : d;
  };
  Vec16<T, N> r[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int at = ((block * PER + j) * 256 + threadIdx.x) * N;
    if (at + N <= a.vocab) r[j] = *(const Vec16<T, N>*)(x + at);
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int at = ((block * PER + j) * 256 + threadIdx.x) * N;
    if (at + N <= a.vocab) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[j].v[i] = from_f32<T>(grad(to_f32(r[j].v[i]), at + i));
      *(Vec16<T, N>*)(dx + at) = r[j];
    } else {
      for (int i = at; i < a.vocab; ++i) dx[i] = from_f32<T>(grad(to_f32(x[i]), i));
    }
  }
}

template <typename T>
void launch_logprobs_t(const LogprobArgs& a, hipStream_t s) {
  constexpr int N = Line<T>::N;
  const int per = (a.vocab + a.splits - 1) / a.splits + N;
  const long long wgs = (long long)a.rows * a.splits;
  const auto go = [&](auto kern, int threads, long long most = 1LL << 31) {
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min(wgs, most)), dim3(threads), 0, s, a);
  };
  if (a.vocab < N) go(logprob_kernel<T, 512, 1, false, true>, 512);
  else if (wgs > 256) {   // two workgroups of 512 threads to a compute unit
    if (per <= 512 * N) go(logprob_kernel<T, 512, 1, false>, 512);
    else if (per <= 512 * 16) go(logprob_kernel<T, 512, 16 / N, false>, 512);
    else if (N == 4 && per <= 512 * 64) go(logprob_kernel<T, 512, 64 / N, false>, 512);
    else go(logprob_kernel<T, 512, 8, true>, 512, a.splits == 1 ? 512 : wgs);
  } else {              // a compute unit to each: as many threads as fit one workgroup
    if (per <= 1024 * N) go(logprob_kernel<T, 1024, 1, false>, 1024);
    else if (per <= 1024 * 32) go(logprob_kernel<T, 1024, 32 / N, false>, 1024);
    else go(logprob_kernel<T, 1024, 8, true>, 1024);
  }
  if (a.splits > 1) hipLaunchKernelGGL(logprob_join_kernel, dim3(a.rows), dim3(256), 0, s, a);
}

template <typename T>
void launch_logprobs_bwd_t(const LogprobArgs& a, hipStream_t s) {
  const int per_block = 256 * 4 * Line<T>::N, blocks = (a.vocab + per_block - 1) / per_block;
  hipLaunchKernelGGL(logprob_bwd_kernel<T>, dim3((unsigned)((long long)a.rows * blocks)), dim3(256), 0, s, a, blocks);
}

}  // namespace

int dropout_row_blocks(int rows, int n) { return drop_grid(rows, n).blocks; }

void l2l_launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) launch_dropout_t<float>(a, s);
  else if (dtype == 1) launch_dropout_t<bf16>(a, s);
  else launch_dropout_t<fp16>(a, s);
}

int logprob_splits(int rows, int vocab) {
  const int want = (256 + rows - 1) / rows, most = std::max(1, vocab / 32768);
  return std::max(1, std::min(std::min(want, most), 32));
}
size_t logprob_work_bytes(int rows, int splits, int top) {
  return splits > 1 ? (size_t)rows * splits * (16 + 8 * (size_t)top) : 0;
}

void l2l_launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) launch_logprobs_t<float>(a, s);
  else if (dtype == 1) launch_logprobs_t<bf16>(a, s);
  else launch_logprobs_t<fp16>(a, s);
}
void l2l_launch_logprobs_bwd(const LogprobArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) launch_logprobs_bwd_t<float>(a, s);
  else if (dtype == 1) launch_logprobs_bwd_t<bf16>(a, s);
  else launch_logprobs_bwd_t<fp16>(a, s);
}
