// Dropout with bias and residual, and token log probabilities with entropy and top alternatives: kernels and launchers of the
// single operations that pass over memory once (entry points and checks: l2l.hip).
#include <algorithm>

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
// Bound by memory.  A thread owns eight columns and walks every (256 / CW)-th row of a block of rows, four rows requested at a
// time; CW threads lie along the columns.  The column sums stay in fp32 registers, then add up across the workgroup's row lanes and leave as
// one row of partial sums per block, which a second kernel adds in a fixed order: no atomics, so the same call gives the same bits.
constexpr int DROP_ROWS = 4;      // rows in flight per thread

struct DropGrid { int cw, lanes, groups, per, blocks; };   // threads along columns, row lanes, column groups, rows per thread, row blocks
DropGrid drop_grid(int rows, int n) {
  DropGrid g;
  const int chunks = (n + 7) / 8;
  g.cw = 1;
  while (g.cw < chunks && g.cw < 64) g.cw *= 2;
  g.lanes = 256 / g.cw;
  g.groups = (chunks + g.cw - 1) / g.cw;
  // rows per thread: as many as leave two thousand workgroups, at most 16 (the partial sums are then a sixtieth of the traffic at most)
  const long long threads_rows = (long long)rows * g.groups / g.lanes / 2048;
  g.per = (int)std::min<long long>(16, std::max<long long>(1, threads_rows));
  g.per = g.per > DROP_ROWS ? (g.per + DROP_ROWS - 1) / DROP_ROWS * DROP_ROWS : g.per;
  g.blocks = (rows + g.lanes * g.per - 1) / (g.lanes * g.per);
  return g;
}

template <typename T>
__device__ __forceinline__ void load_cols(const T* p, int count, float (&v)[8]) {
  if (count >= 8) {
    const Vec16<T, 8> x = *(const Vec16<T, 8>*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(x.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? to_f32(p[i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_cols(T* p, int count, const float (&v)[8]) {
  if (count >= 8) {
    Vec16<T, 8> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = from_f32<T>(v[i]);
    *(Vec16<T, 8>*)p = x;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = from_f32<T>(v[i]);
  }
}

template <typename T, bool RESID, bool SUMS>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a, int cw, int lanes, int groups, int per) {
  const int group = blockIdx.x % groups, block = blockIdx.x / groups;
  const int chunk = group * cw + threadIdx.x % cw, row_lane = threadIdx.x / cw, col = chunk * 8;
  const int count = min(8, a.n - col);   // <= 0: this thread has no columns
  const long long row0 = (long long)block * lanes * per + row_lane;
  const DropKey key = drop_key(a.seed, a.site, a.step);
  const float kept = 65536.0f / (65536.0f - (float)a.drop);
  float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sums[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (a.bias && count > 0) load_cols((const T*)a.bias + col, count, bias);
  if (count > 0) {
    for (int j = 0; j < per; j += DROP_ROWS) {
      float x[DROP_ROWS][8], res[RESID ? DROP_ROWS : 1][8];
      bool live[DROP_ROWS];
#pragma unroll
      for (int u = 0; u < DROP_ROWS; ++u) {
        const long long row = row0 + (long long)(j + u) * lanes;
        live[u] = j + u < per && row < a.rows;
        if (live[u]) {
          load_cols((const T*)a.x + row * a.ldx + col, count, x[u]);
          if (RESID) load_cols((const T*)a.resid + row * a.ldr + col, count, res[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < DROP_ROWS; ++u) {
        if (!live[u]) continue;
        const long long row = row0 + (long long)(j + u) * lanes;
        const u32x4 w = philox7((uint32_t)chunk, (uint32_t)row, key);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t bits = (w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
          const float v = x[u][i] + bias[i];
          const float z = bits >= a.drop ? v * kept : 0.f;
          if (SUMS) sums[i] += z;
          x[u][i] = RESID ? res[u][i] + z : z;
        }
        store_cols((T*)a.y + row * a.ldy + col, count, x[u]);
      }
    }
  }
  if (SUMS) {
    __shared__ float red[256][9];   // (9: the eight values of 64 lanes spread over the banks)
#pragma unroll
    for (int i = 0; i < 8; ++i) red[threadIdx.x][i] = sums[i];
    __syncthreads();
    for (int u = threadIdx.x; u < cw * 8; u += 256) {
      const int c = u / 8, i = u % 8, at = (group * cw + c) * 8 + i;
      float s = 0.f;
      for (int l = 0; l < lanes; ++l) s += red[l * cw + c][i];
      if (at < a.n) a.part[(long long)block * a.n + at] = s;
    }
  }
}

// dbias (+)= the partial sums: 16 columns a workgroup, 16 lanes to a column
__global__ __launch_bounds__(256) void dropout_sum_kernel(const float* part, int blocks, int n, float* dbias, int accumulate) {
  __shared__ float red[16][17];
  const int c = threadIdx.x & 15, l = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float s = 0.f;
  if (col < n)
    for (int b = l; b < blocks; b += 16) s += part[(long long)b * n + col];
  red[l][c] = s;
  __syncthreads();
  if (l == 0 && col < n) {
    for (int j = 1; j < 16; ++j) s += red[j][c];
    dbias[col] = accumulate ? dbias[col] + s : s;
  }
}

template <typename T>
void launch_dropout_t(const DropoutArgs& a, hipStream_t s) {
  const DropGrid g = drop_grid(a.rows, a.n);
  const dim3 grid((unsigned)((long long)g.groups * g.blocks));
  const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a, g.cw, g.lanes, g.groups, g.per); };
  if (a.dbias) {
    go(dropout_kernel<T, false, true>);
    hipLaunchKernelGGL(dropout_sum_kernel, dim3((a.n + 15) / 16), dim3(256), 0, s, a.part, g.blocks, a.n, a.dbias, a.accumulate);
  } else if (a.resid) {
    go(dropout_kernel<T, true, false>);
  } else {
    go(dropout_kernel<T, false, false>);
  }
}

// ---- token log probabilities ---------------------------------------------------------------------------------------------
// Of a row of logits x: m = max, s = sum e^(x - m), t = sum e^(x - m) (x - m); lse = m + log s, log p(id) = x[id] - m - log s, entropy
// = log s - t / s, and the `top` largest by (value, lowest index first).  One pass over memory: a workgroup holds a slab of the row in
// registers, from which it takes the sums and the candidates for the top.  A value can be among the top k only if it is not
// below the k-th largest of any 64 values of the row; each wave takes that bound from its lanes' own maxima (a binary search by
// ballots over their leading bits), the workgroup the highest of them, and what reaches it (some dozens of the slab) goes to a list in LDS,
// where every candidate counts how many are before it: its place.  Where equal values overflow the list, the workgroup searches the top one by one.
// Bound by memory: two workgroups of 512 threads share a compute unit and load under each other's reductions.
// Rows too few to fill the chip are split over workgroups, whose parts a second kernel joins.
constexpr int LP_NT = 512, LP_WAVES = LP_NT / 64, LP_LIST = 1024, LP_TOP = 32;
constexpr float LP_FAR = -1.0e4f;   // e^x is 0 from here down, and 0 * x has to be 0 as well for x = -inf

// whole numbers in the order of the values (-0 and 0 alike)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// larger = earlier in the top: the value, then the lower index
__device__ __forceinline__ uint64_t rank_key(uint32_t key, uint32_t index) { return (uint64_t)key << 32 | (0xFFFFFFFFu - index); }

struct Stat { float m, s, t; };
// both relative to their own maximum; an empty one (m = -inf, s = t = 0) changes nothing
__device__ __forceinline__ Stat join(Stat a, Stat b) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  if (r.m == -INFINITY) return Stat{r.m, a.s + b.s, a.t + b.t};
  const float da = fmaxf(a.m - r.m, LP_FAR), db = fmaxf(b.m - r.m, LP_FAR), fa = __expf(da), fb = __expf(db);
  r.s = a.s * fa + b.s * fb;
  r.t = (a.t + a.s * da) * fa + (b.t + b.s * db) * fb;
  return r;
}
__device__ __forceinline__ Stat wave_join(Stat a) {
  Stat r;
  r.m = wave_max(a.m);
  const float d = r.m == -INFINITY ? 0.f : fmaxf(a.m - r.m, LP_FAR), f = __expf(d);
  r.s = wave_sum(a.s * f);
  r.t = wave_sum((a.t + a.s * d) * f);
  return r;
}

__device__ __forceinline__ void write_row(const LogprobArgs& a, int row, Stat st, float x_id) {
  const bool none = st.m == -INFINITY;   // every logit is -inf
  const float log_s = logf(st.s);
  a.lse[row] = none ? -INFINITY : st.m + log_s;
  a.entropy[row] = none ? 0.f : log_s - st.t / st.s;
  if (a.ids) a.logp[row] = a.ids[row] < 0 ? 0.f : none ? -INFINITY : (x_id - st.m) - log_s;
}

template <typename T, int NV>
__global__ __launch_bounds__(LP_NT) __attribute__((amdgpu_waves_per_eu(4)))
void logprob_kernel(const LogprobArgs a) {
  constexpr int N = Line<T>::N, SLAB = LP_NT * N * NV;
  __shared__ uint64_t list[LP_LIST], best[LP_TOP];
  __shared__ Stat wave_stat[LP_WAVES];
  __shared__ uint32_t bound[LP_WAVES];
  __shared__ int count;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, top = a.top;
  // splits of whole slabs' worth of threads' chunks, so that all but the last one are full
  const int chunks = (a.vocab + N - 1) / N, per_split = (chunks + a.splits - 1) / a.splits * N;
  const int begin = min(a.vocab, split * per_split), end = min(a.vocab, begin + per_split);
  const T* x = (const T*)a.logits + (long long)row * a.ld;
  float x_id = 0.f;
  if (tid == 0 && split == 0 && a.ids) {
    int id = a.ids[row];
    if (id >= a.vocab) { atomicOr(a.bad, 1); id = a.vocab - 1; }
    if (id >= 0) x_id = to_f32(x[id]);
  }
  Stat st = {-INFINITY, 0.f, 0.f};
  int have = 0;                // entries of list that earlier slabs left, in order
  uint32_t floor_key = 0;      // the top-th of them, once there are as many
  for (int slab = begin; slab < end; slab += SLAB) {
    float v[NV][N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = slab + (j * LP_NT + tid) * N;
      if (at + N <= end) {
        const Vec16<T, N> r = *(const Vec16<T, N>*)(x + at);
#pragma unroll
        for (int i = 0; i < N; ++i) v[j][i] = to_f32(r.v[i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[j][i] = at + i < end ? to_f32(x[at + i]) : -INFINITY;
      }
    }
    float lm = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) lm = fmaxf(lm, v[j][i]);
    Stat mine = {lm, 0.f, 0.f};
    const float base = lm == -INFINITY ? 0.f : lm;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = v[j][i] - base, e = __expf(d);
        mine.s += e;
        mine.t = fmaf(e, fmaxf(d, LP_FAR), mine.t);
      }
    const Stat w = wave_join(mine);
    // the largest bound, to 16 leading bits, that `top` lanes' maxima reach
    uint32_t reach = 0;
    if (top) {
      const uint32_t key = order_key(lm);
#pragma unroll
      for (int bit = 31; bit >= 16; --bit)
        if (__popcll(__ballot(key >= (reach | 1u << bit))) >= top) reach |= 1u << bit;
    }
    if (lane == 0) { wave_stat[wave] = w; bound[wave] = reach; }
    if (tid == 0) count = have;
    __syncthreads();
    for (int j = 0; j < LP_WAVES; ++j) st = join(st, wave_stat[j]);
    if (top) {
      uint32_t least = floor_key;
#pragma unroll
      for (int j = 0; j < LP_WAVES; ++j) least = max(least, bound[j]);
      if (order_key(lm) >= least) {   // (few threads)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const uint32_t key = order_key(v[j][i]), at = slab + (j * LP_NT + tid) * N + i;
            if (key >= least && at < (uint32_t)end) {
              const int slot = atomicAdd(&count, 1);
              if (slot < LP_LIST) list[slot] = rank_key(key, at);
            }
          }
      }
      __syncthreads();
      const int found = count;
      if (found <= LP_LIST) {
        for (int u = tid; u < found; u += LP_NT) {
          const uint64_t k = list[u];
          int before = 0;
          for (int o = 0; o < found; ++o) before += list[o] > k;
          if (before < top) best[before] = k;
        }
        have = min(found, top);
      } else {
        // one by one: the largest after the previous one, over the slab and what earlier slabs left
        const int earlier = have;
        uint64_t prev = ~0ull;
        have = 0;
        while (have < top) {
          uint64_t k = tid < earlier && list[tid] < prev ? list[tid] : 0;
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const uint32_t at = slab + (j * LP_NT + tid) * N + i;
              const uint64_t o = rank_key(order_key(v[j][i]), at);
              if (at < (uint32_t)end && o < prev && o > k) k = o;
            }
#pragma unroll
          for (int off = 32; off; off >>= 1) {
            const uint64_t o = (uint64_t)__shfl_xor((unsigned)(k >> 32), off, 64) << 32 | __shfl_xor((unsigned)k, off, 64);
            k = o > k ? o : k;
          }
          __syncthreads();   // (the slots at the end of the list, past what earlier slabs left, carry the waves' results)
          if (lane == 0) list[LP_LIST - LP_WAVES + wave] = k;
          __syncthreads();
          for (int j = 0; j < LP_WAVES; ++j) k = max(k, list[LP_LIST - LP_WAVES + j]);
          if (tid == 0) best[have] = k;
          ++have;
          prev = k;
        }
      }
      __syncthreads();
      if (tid < have) list[tid] = best[tid];
      floor_key = have == top ? (uint32_t)(best[top - 1] >> 32) : 0;
    }
    __syncthreads();   // the list and the waves' results are free again, and what is left of the list can be read
  }
  if (a.splits == 1) {
    if (tid == 0) write_row(a, row, st, x_id);
    if (tid < top) {
      const uint64_t k = list[tid];
      a.top_ids[(long long)row * top + tid] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
      a.top_logp[(long long)row * top + tid] = st.m == -INFINITY ? -INFINITY : (key_value((uint32_t)(k >> 32)) - st.m) - logf(st.s);
    }
  } else {
    // [rows][splits] of: m, s, t, x[id]; then `top` ranks (fewer: zeros, which are behind everything)
    float* part = (float*)a.work + ((long long)row * a.splits + split) * 4;
    uint64_t* ranks = (uint64_t*)((float*)a.work + (long long)a.rows * a.splits * 4) + ((long long)row * a.splits + split) * top;
    if (tid == 0) { part[0] = st.m; part[1] = st.s; part[2] = st.t; part[3] = x_id; }
    if (tid < top) ranks[tid] = tid < have ? list[tid] : 0;
  }
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
  if (tid == 0) write_row(a, row, st, part[3]);
  for (int u = tid; u < n; u += 256) {
    const uint64_t k = list[u];
    int before = 0;
    for (int o = 0; o < n; ++o) before += list[o] > k;
    if (k && before < top) {
      a.top_ids[(long long)row * top + before] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
      a.top_logp[(long long)row * top + before] = st.m == -INFINITY ? -INFINITY : (key_value((uint32_t)(k >> 32)) - st.m) - logf(st.s);
    }
  }
}

// d logits = g (onehot - p) - h p (log p + H): g, h the gradients of log p(id) and of the entropy.  Element-wise; in place allowed.
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
  const auto grad = [&](float v, int at) {
    const float lp = fmaxf(v - lse, LP_FAR), p = __expf(v - lse);
    const float d = (at == id ? g : 0.f) - p * fmaf(h, lp + H, g);
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
  const dim3 grid((unsigned)((long long)a.rows * a.splits));
  const int per = (a.vocab + a.splits - 1) / a.splits + N;
  // registers for the slab by what a workgroup has to hold: 32768 values at most at a time
  if (per <= LP_NT * N) hipLaunchKernelGGL((logprob_kernel<T, 1>), grid, dim3(LP_NT), 0, s, a);
  else if (per <= LP_NT * 16) hipLaunchKernelGGL((logprob_kernel<T, 16 / N>), grid, dim3(LP_NT), 0, s, a);
  else hipLaunchKernelGGL((logprob_kernel<T, 64 / N>), grid, dim3(LP_NT), 0, s, a);
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
  // as many as give 256 compute units a workgroup each, of 2048 values or more, and 32 at most (32 parts of 32 fill the joining list)
  const int want = (256 + rows - 1) / rows, most = std::max(1, vocab / 2048);
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
