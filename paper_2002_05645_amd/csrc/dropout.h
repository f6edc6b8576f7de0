// Counter-based dropout: which elements a site drops is a function of (seed, site, element) alone, so that the layer
// forward that the backward pass recomputes, and the backward pass itself, see the forward pass's mask without anybody
// having stored it.
//
// Generator: Philox-4x32 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011) with seven
// rounds, the fewest that its authors report as passing BigCrush.  Key = seed; counter = (element group, row or pair, site low, site
// high); one call gives 128 bits.
//  - element-wise dropout: 16 bits an element, eight neighbouring elements of a row from one call (counter words 0, 1 =
//    column / 8, row).  The pass over memory has the time for it.
//  - attention probabilities: 8 bits an element, a 4 x 4 patch (query / 4, key / 4) from one call (word 0 = query / 4 << 16 |
//    key / 4, word 1 = 2^31 | pair of sequence and head).  Here the generator is what bounds the kernels, and a patch serves the tiles of both
//    orientations, queries or keys along the lanes, with whole calls.
#pragma once
#include "common.h"

struct DropKey {
  uint32_t k0, k1;   // seed
  uint32_t s0, s1;   // site
};

// the site of a launch: as given, plus the caller's step counter in device memory (captured launches take a new mask per replay that way)
__device__ __forceinline__ DropKey drop_key(uint64_t seed, uint64_t site, const uint64_t* step) {
  if (step) site += *step;
  return DropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)site, (uint32_t)(site >> 32)};
}

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }   // one instruction

__device__ __forceinline__ u32x4 philox7(uint32_t c0, uint32_t c1, const DropKey& key) {
  uint32_t c2 = key.s0, c3 = key.s1, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t n0 = xor3((uint32_t)(b >> 32), c1, k0), n2 = xor3((uint32_t)(a >> 32), c3, k1);
    c0 = n0; c1 = (uint32_t)b; c2 = n2; c3 = (uint32_t)a;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}

// Transposes a 4 x 4 matrix of words held by four neighbouring lanes (row = lane % 4): two exchanges with the neighbours
// at distance 1 and 2.
__device__ __forceinline__ u32x4 quad_transpose(u32x4 a, int lane) {
  const bool odd = lane & 1, high = lane & 2;
  uint32_t x = dpp_move_u32<0xB1>(odd ? a.x : a.y), y = dpp_move_u32<0xB1>(odd ? a.z : a.w);   // quad_perm [1,0,3,2]
  if (odd) { a.x = x; a.z = y; } else { a.y = x; a.w = y; }
  x = dpp_move_u32<0x4E>(high ? a.x : a.z); y = dpp_move_u32<0x4E>(high ? a.y : a.w);          // quad_perm [2,3,0,1]
  if (high) { a.x = x; a.y = y; } else { a.z = x; a.w = y; }
  return a;
}
// Transposes the 4 x 4 matrix of bytes in a lane's four words.
__device__ __forceinline__ u32x4 byte_transpose(u32x4 a) {
  // perm(hi, lo, sel): selector values 0..3 name lo's bytes, 4..7 hi's
  const uint32_t p = __builtin_amdgcn_perm(a.y, a.x, 0x05010400u), q = __builtin_amdgcn_perm(a.w, a.z, 0x05010400u);
  const uint32_t r = __builtin_amdgcn_perm(a.y, a.x, 0x07030602u), s = __builtin_amdgcn_perm(a.w, a.z, 0x07030602u);
  return u32x4{__builtin_amdgcn_perm(q, p, 0x05040100u), __builtin_amdgcn_perm(q, p, 0x07060302u),
               __builtin_amdgcn_perm(s, r, 0x05040100u), __builtin_amdgcn_perm(s, r, 0x07060302u)};
}

// The random bytes of a lane's 16 elements of a 32 x 32 tile of probabilities whose accumulator register r holds index
// 8 (r / 4) + 4 (lane / 32) + r % 4 of one axis at index lane % 32 of the other: word r / 4, byte r % 4.  The four lanes of
// a quad need the same four patches, each a quarter of every one: each computes one of them and they exchange.
// i0 / j0: first query / key of the tile (multiples of 32).  QL: queries along the lanes (else keys).
template <bool QL>
__device__ __forceinline__ u32x4 drop_bytes(int i0, int j0, uint32_t pair, const DropKey& key, int lane) {
  const uint32_t along = (uint32_t)(lane & 31) >> 2, across = 2u * (lane & 3) + ((uint32_t)lane >> 5);
  const uint32_t I = (uint32_t)i0 / 4 + (QL ? along : across), J = (uint32_t)j0 / 4 + (QL ? across : along);
  const u32x4 w = philox7(I << 16 | J, 0x80000000u | pair, key);
  return quad_transpose(QL ? w : byte_transpose(w), lane);
}
// keeps ? x : 0, done here and in 32 bits: left to itself the compiler makes the choice behind the rounding to 16 bits, value by value
__device__ __forceinline__ float drop_select(bool keeps, float x) {
  x = keeps ? x : 0.f;
  asm("" : "+v"(x));
  return x;
}
__device__ __forceinline__ bool drop_keeps(const u32x4& bytes, int r, uint32_t drop) {
  return ((bytes[r >> 2] >> (8 * (r & 3))) & 255u) >= drop;
}
