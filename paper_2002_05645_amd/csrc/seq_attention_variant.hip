// Attention over sequences of different lengths for one element type and padded head width (-DL2L_DP=32, 64, 96 or 128; -DL2L_ELEM=0 fp32,
// 1 bf16, 2 fp16): each pair is a translation unit of its own, so that the build runs in parallel.
#if L2L_ELEM == 0
#include "seq_attention_f32.h"
#else
#include "seq_attention.h"
#endif

#define L2L_CAT2(a, b) a##b
#define L2L_CAT(a, b) L2L_CAT2(a, b)
#if L2L_ELEM == 0
typedef float Elem;
#define L2L_NAME(x) L2L_CAT(L2L_CAT(x, f), L2L_DP)
#elif L2L_ELEM == 1
typedef bf16 Elem;
#define L2L_NAME(x) L2L_CAT(L2L_CAT(x, v), L2L_DP)
#else
typedef fp16 Elem;
#define L2L_NAME(x) L2L_CAT(L2L_CAT(x, h), L2L_DP)
#endif

namespace {

// one workgroup per `rows_per` rows of every (sequence, head)
dim3 blocks(const SeqAttnArgs& a, int heads, int rows_per) {
  return dim3((unsigned)((long long)a.sequences * heads * ((a.max_len + rows_per - 1) / rows_per)));
}

// the splits' partial results together, where there are any
template <bool WEIGHTED>
void join(const SeqAttnArgs& a, const sattn::JoinArgs& j, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.sequences * j.heads * ((a.max_len + 63) / 64)), j.out[1] ? 2 : 1);
  hipLaunchKernelGGL((sattn::seq_join_kernel<Elem, WEIGHTED>), grid, dim3(256), 0, s, a, j);
}
void join_fwd(const SeqAttnArgs& a, hipStream_t s) {
  if (a.splits_fwd > 1) join<true>(a, {{a.part}, a.rows * a.heads * a.d, a.part_m, a.part_sum, a.lse, {a.out}, {a.ldo}, a.splits_fwd, a.heads}, s);
}
void join_dq(const SeqAttnArgs& a, hipStream_t s) {
  if (a.splits_dq > 1) join<false>(a, {{a.part}, a.rows * a.heads * a.d, nullptr, nullptr, nullptr, {a.dq}, {a.lddq}, a.splits_dq, a.heads}, s);
}
void join_dkv(const SeqAttnArgs& a, hipStream_t s) {
  const long long one = a.rows * a.kv_heads * a.d;
  if (a.splits_dkv > 1)
    join<false>(a, {{a.part, a.part + one}, 2 * one, nullptr, nullptr, nullptr, {a.dv, a.dk}, {a.lddv, a.lddk}, a.splits_dkv, a.kv_heads}, s);
}

template <typename K>
void go(K kern, dim3 grid, const SeqAttnArgs& a, hipStream_t s) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, a); }

#if L2L_ELEM == 0
// dropped or not; waves without rows of their own on the others' tiles, where no sequence is longer than 64 (but the longest has two tiles)
template <typename F>
void pick_f32(const SeqAttnArgs& a, F f) {
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  if (a.max_len > 32 && a.max_len <= 64) a.drop ? f(std::true_type{}, Two{}) : f(std::false_type{}, Two{});
  else a.drop ? f(std::true_type{}, One{}) : f(std::false_type{}, One{});
}
#endif

}  // namespace

void L2L_NAME(l2l_seq_attn_fwd_)(const SeqAttnArgs& a, hipStream_t s) {
#if L2L_ELEM == 0
  pick_f32(a, [&](auto drop, auto parts) {
    go(sattn::seq_fwd_f32_kernel<L2L_DP, decltype(drop)::value, decltype(parts)::value>, blocks(a, a.heads * a.splits_fwd, 128), a, s);
  });
#else
  if (a.drop) go(sattn::seq_fwd_kernel<Elem, L2L_DP, true>, blocks(a, a.heads * a.splits_fwd, 128), a, s);
  else go(sattn::seq_fwd_kernel<Elem, L2L_DP, false>, blocks(a, a.heads * a.splits_fwd, 128), a, s);
#endif
  join_fwd(a, s);
}

void L2L_NAME(l2l_seq_attn_bwd_)(const SeqAttnArgs& a, hipStream_t s) {
#if L2L_ELEM == 0
  pick_f32(a, [&](auto drop, auto parts) {
    go(sattn::seq_bwd_dq_f32_kernel<L2L_DP, decltype(drop)::value, decltype(parts)::value>, blocks(a, a.heads * a.splits_dq, 128), a, s);
    join_dq(a, s);
    go(sattn::seq_bwd_dkv_f32_kernel<L2L_DP, decltype(drop)::value, decltype(parts)::value>, blocks(a, a.kv_heads * a.splits_dkv, 128), a, s);
    join_dkv(a, s);
  });
#else
  const auto both = [&](auto drop) {
    constexpr bool D = decltype(drop)::value;
    if constexpr (L2L_DP <= 64) {
      if (a.in_one) {
        go(sattn::seq_bwd_dkv_kernel<Elem, L2L_DP, D, true>, blocks(a, a.kv_heads * a.splits_dkv, 128), a, s);
        join_dkv(a, s);
        return;
      }
    }
    {
      go(sattn::seq_bwd_dq_kernel<Elem, L2L_DP, D>, blocks(a, a.heads * a.splits_dq, 128), a, s);
      join_dq(a, s);
      go(sattn::seq_bwd_dkv_kernel<Elem, L2L_DP, D, false>, blocks(a, a.kv_heads * a.splits_dkv, 128), a, s);
      join_dkv(a, s);
    }
  };
  if (a.drop) both(std::true_type{});
  else both(std::false_type{});
#endif
}
