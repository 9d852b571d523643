// 8-bit rows: quantising them as they are written into slots, reading them
// back, and the combine of a layer whose cache is held that way.
//
// All three move bytes: a row of K elements is 2 K (bf16) or 4 K (fp32) bytes
// on one side and K + K / 128 on the other.  One wavefront per row, eight
// elements a lane, so that a block of 128 is one 16-lane row of the wave and
// its largest magnitude four DPP steps; every element is loaded once and kept
// in registers between the maximum and the conversion.  Measured, 16384 rows of
// 1152, bf16: written with their norms in 12.9 us, 4.4 TB/s; read in 12.0 us, 4.7 TB/s
// (a copy of 1 GiB: 5.2), among other passes; under a kernel trace 14.2 and 13.0.
// There, asking for three groups of a row before using the first took 0.8 us more
// (14.3 -> 15.1).  154 rows take 4.2 us, a launch and two round trips.
#include <algorithm>

#include "common.h"
#include "internal.h"
#include "q8.h"

#pragma clang fp contract(off)

namespace moeca {
namespace {

constexpr int kRowWaves = 4;
constexpr int kMaxRowBlocks = 1 << 20;  // grid bound; rows beyond it by a stride

// q[slot[r]], s[slot[r]], norm[slot[r]] = src row r; a slot outside [0, slots)
// leaves its row out.  The last block's elements past K are zeros.
template <typename T, bool VEC>
__global__ __launch_bounds__(kRowWaves * kWave) void quant_rows_kernel(
    const T* __restrict__ src, int64_t rows, int K, int64_t ld, const int32_t* __restrict__ slot,
    const uint8_t* __restrict__ mask, int64_t slots, uint8_t* __restrict__ q,
    uint8_t* __restrict__ s, float* __restrict__ norm) {
  const int lane = threadIdx.x & (kWave - 1);
  const int pitch = static_cast<int>(q8_pitch(K)), spitch = static_cast<int>(q8_spitch(K));
  for (int64_t r = int64_t(blockIdx.x) * kRowWaves + threadIdx.x / kWave; r < rows;
       r += int64_t(gridDim.x) * kRowWaves) {
    const int64_t to = slot != nullptr ? slot[r] : r;
    if (to < 0 || to >= slots) continue;  // uniform across the wave
    if (mask != nullptr && mask[r] == 0) continue;
    const T* const row = src + r * ld;
    uint8_t* const qr = q + to * pitch;
    uint8_t* const sr = s + to * spitch;
    double ss = 0.0;
    for (int c = lane * 8; c < pitch; c += 8 * kWave) {  // whole 16-lane rows in or out
      float v[8];
      load8<T, VEC>(row + c, K - c, v);
      int byte;
      const uint2 p = q8_quant8(v, byte);
      *reinterpret_cast<uint2*>(qr + c) = p;
      if ((lane & 15) == 0) sr[c / kBlk] = static_cast<uint8_t>(byte);
      if (norm != nullptr) ss += q8_square8(p, byte);
    }
    if (norm != nullptr) {
      ss = wave_sum_f64(ss);
      if (lane == 0) norm[to] = static_cast<float>(sqrt(ss));
    }
  }
}

// dst row r = the values of row slot[r]; a slot outside [0, slots) gives zeros.
template <typename T, bool VEC>
__global__ __launch_bounds__(kRowWaves * kWave) void dequant_rows_kernel(
    const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int64_t slots, int K,
    const int32_t* __restrict__ slot, int64_t rows, T* __restrict__ dst, int64_t ld) {
  const int lane = threadIdx.x & (kWave - 1);
  const int pitch = static_cast<int>(q8_pitch(K)), spitch = static_cast<int>(q8_spitch(K));
  for (int64_t r = int64_t(blockIdx.x) * kRowWaves + threadIdx.x / kWave; r < rows;
       r += int64_t(gridDim.x) * kRowWaves) {
    const int64_t at = slot != nullptr ? slot[r] : r;
    const bool in = at >= 0 && at < slots;
    for (int c = lane * 8; c < K; c += 8 * kWave) {
      float v[8];
      if (in) {
        const uint2 p = *reinterpret_cast<const uint2*>(q + at * pitch + c);
        const float two = q8_two(s[at * spitch + c / kBlk]);
        q8_unpack4(p.x, v);
        q8_unpack4(p.y, v + 4);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] *= two;
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = 0.0f;
      }
      store8<T, VEC>(dst + r * ld + c, K - c, v);
    }
  }
}

// Weights [count][N][K] (dense) to q [count][N][pitch], s [count][ceil(N / 128)]
// [spitch]: a block per 128 x 128 of a matrix, its 64 elements a thread kept in
// registers between the maximum and the conversion.  16 x 4608 x 1152, bf16: 50 us,
// 5.1 TB/s.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_matrix_kernel(const T* __restrict__ W, int N, int K,
                                                           uint8_t* __restrict__ q,
                                                           uint8_t* __restrict__ s) {
  __shared__ uint32_t s_top[4];
  const int pitch = static_cast<int>(q8_pitch(K)), spitch = static_cast<int>(q8_spitch(K));
  const int nb = (N + kBlk - 1) / kBlk;
  const int kb = blockIdx.x, n0 = blockIdx.y * kBlk;
  const int64_t i = blockIdx.z;
  const int tid = threadIdx.x;
  const int c = kb * kBlk + (tid & 15) * 8;
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const int n = n0 + (tid >> 4) + 16 * h;
    if (n < N) {
      load8<T, VEC>(W + (i * N + n) * K + c, K - c, v[h]);
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u) v[h][u] = 0.0f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) top = max(top, q8_finite(v[h][u]));
  }
  top = row_max_u32(top);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16, kWave)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32, kWave)));
  if ((tid & (kWave - 1)) == 0) s_top[tid / kWave] = top;
  __syncthreads();
  top = max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3]));
  const int byte = q8_scale_byte(top);
  const float inv = q8_inv(byte);
  if (tid == 0) s[(i * nb + blockIdx.y) * spitch + kb] = static_cast<uint8_t>(byte);
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const int n = n0 + (tid >> 4) + 16 * h;
    if (n >= N) continue;
    const float* x = v[h];
    *reinterpret_cast<uint2*>(q + (i * N + n) * pitch + c) =
        make_uint2(q8_pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                   q8_pack4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
  }
}

// ---------------------------------------------------------------------------
// Combine of a layer whose cache is held in 8 bits (Sec. 4.1):
//
//   y_i = sum_s h_s + sum_p f32(w_p * hhat_p)
//
// as in combine.hip, with hhat_p the row that the down projection just left in
// `fresh` (list order, activation type) for a recomputed branch, unrounded by
// the cache, and the stored value q 2^e of slot sigma(p) for a reused one.
// A recomputed row is quantised into its slot on the way, with the norm of
// what is stored; a synchronised token's attention feature goes into its row of
// the 8-bit attention cache.
// ---------------------------------------------------------------------------
// One wave per token.  Where a row is loaded from depends on the branch: a recomputed
// one costs two round trips, what the decision left, then the row's elements (GI
// groups of 512 a lane's eight of each; GI = 0: any width, a group at a time), all
// asked for before any is used.  The token's own slots need no decision: with GI > 0
// (two of them at most) they are asked for first, `reuse` (a step that may reuse
// some).  8192 tokens of 1152, two branches: a full step 28 us (104 MB), a cache step
// 16.5 us, 18.3 us on average over a cycle (20.4 with the slots after the decision, and
// then 21.7 and 32.5 in registers for six and eight waves a SIMD).
template <typename T> struct Raw;  // eight elements as loaded; 8-bit rows use the first two words
template <> struct Raw<uint16_t> {
  typedef __attribute__((ext_vector_type(4))) unsigned int v;
  static __device__ __forceinline__ void widen(v x, float* f) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f[2 * u] = __uint_as_float(x[u] << 16);
      f[2 * u + 1] = __uint_as_float(x[u] & 0xffff0000u);
    }
  }
};
template <> struct Raw<float> {
  typedef __attribute__((ext_vector_type(8), aligned(16))) unsigned int v;  // as rows are
  static __device__ __forceinline__ void widen(v x, float* f) {
#pragma unroll
    for (int u = 0; u < 8; ++u) f[u] = __uint_as_float(x[u]);
  }
};

template <typename T, int KMAX, int GI>
__global__ __launch_bounds__(kRowWaves * kWave) void combine_q8_kernel(
    const float* __restrict__ w_t, const int32_t* __restrict__ e_t,
    const int32_t* __restrict__ sigma, const uint8_t* __restrict__ mask,
    const uint8_t* __restrict__ sync, const int32_t* __restrict__ pos,
    const T* __restrict__ fresh, uint8_t* __restrict__ h_c, uint8_t* __restrict__ s_c,
    int32_t* __restrict__ e_c, float* __restrict__ w_c, float* __restrict__ n_c,
    T* __restrict__ out, const T* __restrict__ attn_in, uint8_t* __restrict__ attn_q,
    uint8_t* __restrict__ attn_s, const T* __restrict__ h_sh, int S, int64_t T_tokens, int d,
    int k, int reuse) {
  typedef typename Raw<T>::v raw;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t t = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x)) *
                        int64_t(kRowWaves) +
                    __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  if (t >= T_tokens) return;
  const int pitch = static_cast<int>(q8_pitch(d)), spitch = static_cast<int>(q8_spitch(d));
  static_assert(GI == 0 || KMAX == 2, "a slot is one of two");
  constexpr int G = GI > 0 ? GI : 1;
  uint2 own[KMAX][G];  // the token's slots
  int own_s[KMAX][G];
  float wp[KMAX];
  int slot[KMAX], from[KMAX];  // from: row of `fresh`, -1 for a reused branch
  double ss[KMAX];
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    wp[p] = 0.0f;
    slot[p] = 0;
    from[p] = -1;
    ss[p] = 0.0;
    if (p < k) {
      const int64_t f = t * k + p;
      wp[p] = w_t[f];
      slot[p] = sigma[f];
      const int at = pos[f];
      from[p] = mask[f] != 0 ? at : -1;
    }
  }
  int syn_v = 0;
  if (attn_in != nullptr) syn_v = sync[t];
  if constexpr (GI > 0) {
#pragma unroll
    for (int p = 0; p < KMAX; ++p)
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        own[p][gi] = make_uint2(0, 0);
        own_s[p][gi] = 0;
        const int c = (gi * kWave + lane) * 8;
        if (reuse != 0 && p < k && c < d) {
          own[p][gi] = *reinterpret_cast<const uint2*>(h_c + (t * k + p) * pitch + c);
          own_s[p][gi] = s_c[(t * k + p) * spitch + c / kBlk];
        }
      }
  }
  // the same for the whole wave: say so, so that branches on it are scalar
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    from[p] = __builtin_amdgcn_readfirstlane(from[p]);
    slot[p] = __builtin_amdgcn_readfirstlane(slot[p]);
  }
  const bool syn = __builtin_amdgcn_readfirstlane(syn_v) != 0;

  for (int base = 0; base < (GI > 0 ? 1 : pitch); base += 8 * kWave) {
    raw h[KMAX][G], a[G];
    int sb[KMAX][G];
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const int c = base + (gi * kWave + lane) * 8;
      const bool in = c < d;  // d is a multiple of 64: eight or none
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        h[p][gi] = raw{};
        sb[p][gi] = 0;
        if (p >= k || !in) continue;
        if (from[p] >= 0) {  // uniform across the wave
          h[p][gi] = __builtin_nontemporal_load(
              reinterpret_cast<const raw*>(fresh + int64_t(from[p]) * d + c));
        } else if constexpr (GI > 0) {
          const uint2 q = slot[p] == 0 ? own[0][gi] : own[1][gi];
          h[p][gi][0] = q.x;
          h[p][gi][1] = q.y;
          sb[p][gi] = slot[p] == 0 ? own_s[0][gi] : own_s[1][gi];
        } else {
          const int64_t r = t * k + slot[p];
          const uint2 q = *reinterpret_cast<const uint2*>(h_c + r * pitch + c);
          h[p][gi][0] = q.x;
          h[p][gi][1] = q.y;
          sb[p][gi] = s_c[r * spitch + c / kBlk];
        }
      }
      a[gi] = raw{};
      if (syn && in)
        a[gi] = __builtin_nontemporal_load(reinterpret_cast<const raw*>(attn_in + t * d + c));
    }
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const int c = base + (gi * kWave + lane) * 8;
      if (c >= pitch) continue;  // whole 16-lane rows in or out
      float acc[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[u] = 0.0f;
      for (int sh = 0; sh < S; ++sh) {
        float v[8];
        load8<T, true>(h_sh + (sh * T_tokens + t) * d + c, d - c, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] = __fadd_rn(acc[u], v[u]);
      }
#pragma unroll
      for (int p = 0; p < KMAX; ++p) {
        if (p >= k) continue;
        float v[8];
        if (from[p] >= 0) {
          Raw<T>::widen(h[p][gi], v);
          int byte;
          const uint2 q = q8_quant8(v, byte);
          const int64_t r = t * k + slot[p];
          *reinterpret_cast<uint2*>(h_c + r * pitch + c) = q;
          if ((lane & 15) == 0) s_c[r * spitch + c / kBlk] = static_cast<uint8_t>(byte);
          ss[p] += q8_square8(q, byte);
        } else {
          const float two = q8_two(sb[p][gi]);
          q8_unpack4(h[p][gi][0], v);
          q8_unpack4(h[p][gi][1], v + 4);
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] = __fmul_rn(v[u], two);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] = __fadd_rn(acc[u], __fmul_rn(wp[p], v[u]));
      }
      if (c < d) store8<T, true>(out + t * d + c, d - c, acc);
      if (syn) {
        float v[8];
        Raw<T>::widen(a[gi], v);
        int byte;
        *reinterpret_cast<uint2*>(attn_q + t * pitch + c) = q8_quant8(v, byte);
        if ((lane & 15) == 0) attn_s[t * spitch + c / kBlk] = static_cast<uint8_t>(byte);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < KMAX; ++p) {
    if (p >= k || from[p] < 0) continue;  // uniform across the wave
    const double sq = wave_sum_f64(ss[p]);
    if (lane == 0) {
      const int64_t c = t * k + slot[p];
      n_c[c] = static_cast<float>(sqrt(sq));
      e_c[c] = e_t[t * k + p];
      w_c[c] = wp[p];
    }
  }
}

bool vec_rows(const void* p, int64_t ld, size_t elem) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * elem % 16 == 0;
}

unsigned row_blocks(int64_t rows) {
  return static_cast<unsigned>(
      std::min<int64_t>((rows + kRowWaves - 1) / kRowWaves, kMaxRowBlocks));
}

}  // namespace

hipError_t launch_quant_rows(const void* src, bool bf16, int64_t rows, int K, int64_t ld,
                             const int32_t* slot, const uint8_t* mask, int64_t slots, uint8_t* q,
                             uint8_t* s, float* norm, hipStream_t st) {
  const dim3 grid(row_blocks(rows)), block(kRowWaves * kWave);
#define MOECA_QROWS(T, V)                                                                        \
  launch_kernel(&quant_rows_kernel<T, V>, grid, block, 0, st, static_cast<const T*>(src), rows, \
                K, ld, slot, mask, slots, q, s, norm)
  if (bf16) {
    if (vec_rows(src, ld, 2)) MOECA_QROWS(uint16_t, true);
    else MOECA_QROWS(uint16_t, false);
  } else {
    if (vec_rows(src, ld, 4)) MOECA_QROWS(float, true);
    else MOECA_QROWS(float, false);
  }
#undef MOECA_QROWS
  return hipGetLastError();
}

hipError_t launch_dequant_rows(const uint8_t* q, const uint8_t* s, int64_t slots, int K,
                               const int32_t* slot, int64_t rows, void* dst, bool bf16,
                               int64_t ld, hipStream_t st) {
  const dim3 grid(row_blocks(rows)), block(kRowWaves * kWave);
#define MOECA_DROWS(T, V)                                                                   \
  launch_kernel(&dequant_rows_kernel<T, V>, grid, block, 0, st, q, s, slots, K, slot, rows, \
                static_cast<T*>(dst), ld)
  if (bf16) {
    if (vec_rows(dst, ld, 2)) MOECA_DROWS(uint16_t, true);
    else MOECA_DROWS(uint16_t, false);
  } else {
    if (vec_rows(dst, ld, 4)) MOECA_DROWS(float, true);
    else MOECA_DROWS(float, false);
  }
#undef MOECA_DROWS
  return hipGetLastError();
}

hipError_t launch_quant_matrix(const void* W, bool bf16, int count, int N, int K, uint8_t* q,
                               uint8_t* s, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(q8_pitch(K) / kBlk),
                  static_cast<unsigned>((N + kBlk - 1) / kBlk), static_cast<unsigned>(count));
#define MOECA_QMAT(T, V)                                                                       \
  launch_kernel(&quant_matrix_kernel<T, V>, grid, dim3(256), 0, st, static_cast<const T*>(W), N, \
                K, q, s)
  if (bf16) {
    if (vec_rows(W, K, 2)) MOECA_QMAT(uint16_t, true);
    else MOECA_QMAT(uint16_t, false);
  } else {
    if (vec_rows(W, K, 4)) MOECA_QMAT(float, true);
    else MOECA_QMAT(float, false);
  }
#undef MOECA_QMAT
  return hipGetLastError();
}

hipError_t launch_combine_q8(const Shape& s, void* out, const void* attn_in, uint8_t* attn_q,
                             uint8_t* attn_s, bool full, const Buffers& b, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>((s.tokens() + kRowWaves - 1) / kRowWaves));
  const dim3 block(kRowWaves * kWave);
#define MOECA_CQ8(T, KM, GI)                                                                     \
  launch_kernel(&combine_q8_kernel<T, KM, GI>, grid, block, 0, st, b.w_t, b.e_t, b.sigma, b.mask, \
                b.sync, b.pos, static_cast<const T*>(b.fresh), static_cast<uint8_t*>(b.h_c),     \
                b.s_c, b.e_c, b.w_c, b.n_c, static_cast<T*>(out), static_cast<const T*>(attn_in), \
                attn_q, attn_s, static_cast<const T*>(b.h_sh), s.S, s.tokens(), s.d, s.k,     \
                full ? 0 : 1)
  const int64_t gi = (q8_pitch(s.d) + 8 * kWave - 1) / (8 * kWave);
  if (s.bf16 && s.k <= 2 && gi <= 2) MOECA_CQ8(uint16_t, 2, 2);
  else if (s.bf16 && s.k <= 2 && gi <= 3) MOECA_CQ8(uint16_t, 2, 3);
  else if (s.bf16 && s.k <= 2 && gi <= 4) MOECA_CQ8(uint16_t, 2, 4);
  else if (s.bf16) MOECA_CQ8(uint16_t, 8, 0);
  else if (s.k <= 2 && gi <= 2) MOECA_CQ8(float, 2, 2);
  else MOECA_CQ8(float, 8, 0);
#undef MOECA_CQ8
  return hipGetLastError();
}

}  // namespace moeca
