// What the grouped GEMMs of the expert FFN share, whatever their operand type:
// vector types, the activations, and the walk over the groups' tiles and rows.
#pragma once
#include "common.h"

namespace moeca {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;  // 16 bytes, a native vector
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_t;

// kProj: a dense projection of listed token rows (the attention path of a
// block): row r reads token list[r] and writes row list[r] of the output.
enum { kUp = 0, kDown = 1, kProj = 2 };
constexpr int kXcds = 8;

// Activation of the up projection.  tanh GELU:
//   0.5 z (1 + tanh(u)) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3),
// with exp(-2u) = 2^(-2u log2 e) from the hardware exp2 (about 1 ulp) and a
// hardware reciprocal; the erf form uses erff.  (A branch-free polynomial for
// z Phi(z) took 24 of 685 us off a threshold-mode refresh cycle of 3 x 1000
// tokens, 16 experts, and is not used: other last bits, twice erff's relative
// error for 0 < z < 3 and -6e-9 where the function goes to zero.)
// kActSwiglu marks the gated epilogue (silu below), which pairs columns
// instead of mapping each one.
enum { kActGeluTanh = 0, kActGeluErf = 1, kActNone = 2, kActSwiglu = 3, kActBias = 4 };

// silu(z) = z / (1 + exp(-z)), exp(-z) = 2^(-z log2 e) by the hardware exp2.
__device__ __forceinline__ float silu_f(float z) {
  return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

template <int ACT>
__device__ __forceinline__ float act_fn(float z) {
  if constexpr (ACT == kActGeluTanh) {
    const float u = 0.7978845608028654f * (z + 0.044715f * z * z * z);
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-2.8853900817779268f * u));
  } else if constexpr (ACT == kActGeluErf) {
    return 0.5f * z * (1.0f + erff(z * 0.7071067811865476f));
  } else {
    return z;
  }
}

// Group of logical tile L: the number of group tile prefixes <= L, minus
// one, from two ballots (groups 0-63 in toff0, 64-127 in toff1: lane l holds
// the prefixes of groups l and 64 + l, INT_MAX past the last group); also
// returns the group's first tile.
__device__ __forceinline__ int tile_group(int L, int toff0, int toff1, int& first) {
  const int n0 = __popcll(__ballot(toff0 <= L));
  const int n1 = __popcll(__ballot(toff1 <= L));
  const int e = n0 + n1 - 1;
  first = e < 64 ? __shfl(toff0, e, 64) : __shfl(toff1, e - 64, 64);
  return e;
}

// Row table entry r of a tile of group e (first list row r0, `rows` rows):
// the A-operand source row and the output row (-1: padding, never stored;
// padding rows re-read the tile's first row).  Routed groups (e < E): up
// reads token list[r]/k and writes intermediate row r; down reads
// intermediate row r and writes row row_dst[r] of the cache (of `fresh`, in list
// order, where the cache is in 8 bits).  Shared groups: up
// reads token r - off[e] and writes intermediate row r; down reads
// intermediate row r and writes shared-output row r - off[E].
template <int KIND>
__device__ __forceinline__ void group_row(int e, int E, int r0, int rows, int r, int k,
                                          const int32_t* __restrict__ off,
                                          const int32_t* __restrict__ list,
                                          const int32_t* __restrict__ row_dst, int& src,
                                          int& dst) {
  const int rr = r < rows ? r : 0;
  if (KIND == kProj) {
    src = list[r0 + rr];
    dst = r < rows ? list[r0 + r] : -1;
  } else if (e < E) {
    if (KIND == kUp) {
      src = list[r0 + rr] / k;
      dst = r < rows ? r0 + r : -1;
    } else {
      src = r0 + rr;
      dst = r < rows ? row_dst[r0 + r] : -1;
    }
  } else {
    if (KIND == kUp) {
      src = r0 + rr - off[e];
      dst = r < rows ? r0 + r : -1;
    } else {
      src = r0 + rr;
      dst = r < rows ? r0 + r - off[E] : -1;
    }
  }
}

}  // namespace
}  // namespace moeca
