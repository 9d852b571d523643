// Products of 8-bit operands: rows X (a scale per 128 of a row) times weights
// W (a scale per 128 x 128), both e4m3 with power-of-two scales (q8.h),
//
//   y[m][n] = sum_b 2^(ex[m][b] + ew[n / 128][b]) sum_{j in block b} x[m][j] w[n][j],
//
// as the grouped GEMMs of a layer's experts (Sec. 2.3) and as a dense product.
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 128 of K, one block, and takes
// both scales as operand bytes, so that the sum over blocks stays in the fp32
// accumulators and no vector instruction is spent on a scale.
//
// Two ways to multiply.  The 8-bit matrix instructions of gfx950 (this one, the
// 32x32x64 and the unscaled forms alike) align the products of eight
// consecutive k to the largest of them and keep 2^-13 of it; only across such
// groups the sum is fp32.  Measured: dots of 128 normal values are off by 1.5e-5
// of their 2-norm (bf16 instructions on the same numbers: 8e-9), rows with a few
// elements twenty times the others by 4e-5.  Next to a bf16 result's rounding
// (4e-3) that is nothing, and they run at twice the bf16 rate.  Where it does
// show, EXACT converts the operands in registers to bf16, which holds every
// e4m3 number and power of two, and takes the bf16 instructions with fp32 sums:
//  - fp32 results;
//  - hidden rows of a layer whose cache is 8-bit too: a hidden element that
//    moves over a rounding border (1 in 200 does, at 1.5e-5) moves the down
//    projection's row by 1.4e-3, and 1.6 % of the cached elements by a whole
//    step of 2^-3: reused branches were 5.7e-3 off the 64-bit definition
//    instead of 1.7e-3.
//
//   up   : mid[r]  = q8(act(x[token(r)] . W_up[e]^T))   rows by the expert lists
//   down : row of r = mid[r] . W_down[e]^T
//   dense: y[m] = x[m] . W^T + bias
//
// The up projection's epilogue quantises what it has in its accumulators: the
// hidden rows are never held in more than 8 bits, and the activation's value
// is rounded once, from fp32.
#include <algorithm>

#include "common.h"
#include "gemm.h"
#include "internal.h"
#include "moeca.h"
#include "q8.h"

namespace moeca {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

enum { kDense = 3 };

// One product's operands (by value).
struct QArgs {
  const uint8_t *X, *Xs;      // rows [.][pitch], scales [.][spitch]
  const uint8_t *W, *Ws;      // routed experts (or the dense matrix)
  const uint8_t *Wsh, *Wssh;  // shared experts
  const int32_t *off, *tile_off, *list, *row_dst;
  int E, G, k;     // routed groups, all groups, branches a token
  int M;           // dense: rows
  int pitch, spitch;
  int Nout;        // weight rows of a group
  int64_t ldo;     // elements of an output row (down, dense)
  const float* bias;
  void *dst, *dst_sh;  // down, dense
  uint8_t *q, *s;      // up: hidden rows
  int qpitch, qspitch;
};

__device__ __forceinline__ i32x8_t join(u32x4_t a, u32x4_t b) {
  return i32x8_t{static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]),
                 static_cast<int>(a[3]), static_cast<int>(b[0]), static_cast<int>(b[1]),
                 static_cast<int>(b[2]), static_cast<int>(b[3])};
}

// The operands of one 16 x 128 piece: a lane has 32 elements of row (lane & 15),
// 16-byte chunks (lane / 16) and (lane / 16) + 4 of the row's 128 bytes (which k
// a lane holds is free as long as both operands agree).  EXACT: as bf16, already
// times their scale.
template <bool EXACT> struct Piece;
template <> struct Piece<false> {
  i32x8_t v;
  int s;
  __device__ __forceinline__ void set(u32x4_t a, u32x4_t b, int byte) {
    v = join(a, b);
    s = byte;
  }
};
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_q;
template <> struct Piece<true> {
  bf16x8_t v[4];
  __device__ __forceinline__ void set(u32x4_t a, u32x4_t b, int byte) {
    const float two = q8_two(byte);
    const u32x4_t* const in[2] = {&a, &b};
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      u32x4_t o;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int w = static_cast<int>((*in[h / 2])[2 * (h & 1) + u]);
        o[2 * u] = __builtin_bit_cast(
            uint32_t, bf16x2_q(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, two, false)));
        o[2 * u + 1] = __builtin_bit_cast(
            uint32_t, bf16x2_q(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, two, true)));
      }
      v[h] = __builtin_bit_cast(bf16x8_t, o);
    }
  }
};

__device__ __forceinline__ f32x4_t mfma_q8(const Piece<false>& w, const Piece<false>& x,
                                           f32x4_t c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, c, 0, 0, 0, w.s, 0, x.s);
}
__device__ __forceinline__ f32x4_t mfma_q8(const Piece<true>& w, const Piece<true>& x, f32x4_t c) {
#pragma unroll
  for (int h = 0; h < 4; ++h) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[h], x.v[h], c, 0, 0, 0);
  return c;
}

// Four consecutive outputs of a row from column c on; whole: all four exist and
// the address is a multiple of their size.
template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4_t v, int n, bool whole) {
  if (whole) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x2_t*>(p) =
          u32x2_t{f32_to_bf16(v[0]) | (uint32_t(f32_to_bf16(v[1])) << 16),
                  f32_to_bf16(v[2]) | (uint32_t(f32_to_bf16(v[3])) << 16)};
    } else {
      *reinterpret_cast<f32x4_t*>(p) = v;
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (u < n) p[u] = Act<T>::from_f32(v[u]);
}

// ---------------------------------------------------------------------------
// 128-row tiles, 128 columns (gated: 256 weight rows, 128 hidden columns, so
// that a tile has whole blocks of the hidden rows).  256 threads as 2 x 2
// waves, k-tile 128, LDS double buffered in rows of 144 bytes (no two of the
// 16 rows of a read share a bank), the next k-tile loaded into registers
// while this one is multiplied.
// ---------------------------------------------------------------------------
constexpr int kQTM = 128;
constexpr int kQThreads = 256;
constexpr int kQRow = kBlk + 16;

template <int KIND, int ACT, typename T, bool EXACT>
__global__ __launch_bounds__(kQThreads, 1) void qgemm_kernel(QArgs a) {
  constexpr bool kGated = ACT == kActSwiglu;
  constexpr int TN = kGated ? 256 : 128;
  constexpr int WN = TN / 2;          // wave columns
  constexpr int FM = 4, FN = WN / 16;  // 16 x 16 tiles of a wave
  constexpr int LA = kQTM / 32, LB = TN / 32;
  __shared__ __attribute__((aligned(16))) uint8_t Xl[2][kQTM * kQRow];
  __shared__ __attribute__((aligned(16))) uint8_t Wl[2][TN * kQRow];
  __shared__ int s_src[kQTM], s_dst[kQTM];
  __shared__ float s_top[2][kQTM];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wv = tid >> 6;
  const int wm = wv >> 1, wn = wv & 1;
  const int nt = (a.Nout + TN - 1) / TN;
  const int total = KIND == kDense ? (a.M + kQTM - 1) / kQTM * nt : a.tile_off[a.G];
  const int per = (total + kXcds - 1) / kXcds;
  const int lo = (blockIdx.x % kXcds) * per;
  const int hi = min(total, lo + per);
  const int stride = gridDim.x / kXcds;
  int toff0 = 0, toff1 = 0;
  if constexpr (KIND != kDense) {
    toff0 = lane < a.G ? a.tile_off[lane] : 0x7fffffff;
    toff1 = lane + 64 < a.G ? a.tile_off[lane + 64] : 0x7fffffff;
  }
  const int KT = a.pitch / kBlk;
  const int nbw = (a.Nout + kBlk - 1) / kBlk;
  const int lrow = tid >> 3, lcol = (tid & 7) * 16;

  for (int L = lo + static_cast<int>(blockIdx.x) / kXcds; L < hi; L += stride) {
    int e = 0, e_base = 0, o0 = 0, cnt = a.M;
    if constexpr (KIND != kDense) {
      e = tile_group(L, toff0, toff1, e_base);
      o0 = a.off[e];
      cnt = a.off[e + 1] - o0;
    }
    const int mt = (cnt + kQTM - 1) / kQTM;
    const int local = L - e_base;
    const int m = local % mt;
    const int r0 = o0 + m * kQTM;
    const int rows = min(kQTM, cnt - m * kQTM);
    const int n0 = (local / mt) * TN;
    const bool routed = KIND == kDense || e < a.E;
    const int64_t g = routed ? e : e - a.E;
    const uint8_t* const Wg = (routed ? a.W : a.Wsh) + g * a.Nout * a.pitch;
    const uint8_t* const Wsg = (routed ? a.Ws : a.Wssh) + g * nbw * a.spitch;

    for (int r = tid; r < kQTM; r += kQThreads) {
      if constexpr (KIND == kDense) {
        s_src[r] = r < rows ? r0 + r : r0;
        s_dst[r] = r < rows ? r0 + r : -1;
      } else {
        group_row<KIND>(e, a.E, r0, rows, r, a.k, a.off, a.list, a.row_dst, s_src[r], s_dst[r]);
      }
    }
    __syncthreads();

    const uint8_t *xp[LA], *wp[LB], *xsp[FM];
#pragma unroll
    for (int i = 0; i < LA; ++i) xp[i] = a.X + int64_t(s_src[lrow + 32 * i]) * a.pitch + lcol;
#pragma unroll
    for (int i = 0; i < LB; ++i)
      wp[i] = Wg + int64_t(min(n0 + lrow + 32 * i, a.Nout - 1)) * a.pitch + lcol;
#pragma unroll
    for (int i = 0; i < FM; ++i)
      xsp[i] = a.Xs + int64_t(s_src[wm * 64 + i * 16 + (lane & 15)]) * a.spitch;
    const uint8_t* const wsp = Wsg + int64_t(min((n0 + wn * WN) / kBlk, nbw - 1)) * a.spitch;

    f32x4_t acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[j][i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    u32x4_t R[LA + LB];
    int sx[FM], sw, sxn[FM], swn;
    auto gload = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LA; ++i) R[i] = *reinterpret_cast<const u32x4_t*>(xp[i] + kt * kBlk);
#pragma unroll
      for (int i = 0; i < LB; ++i)
        R[LA + i] = *reinterpret_cast<const u32x4_t*>(wp[i] + kt * kBlk);
#pragma unroll
      for (int i = 0; i < FM; ++i) sxn[i] = xsp[i][kt];
      swn = wsp[kt];
    };
    auto lstore = [&](int b) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < LA; ++i)
        *reinterpret_cast<u32x4_t*>(&Xl[b][(lrow + 32 * i) * kQRow + lcol]) = R[i];
#pragma unroll
      for (int i = 0; i < LB; ++i)
        *reinterpret_cast<u32x4_t*>(&Wl[b][(lrow + 32 * i) * kQRow + lcol]) = R[LA + i];
#pragma unroll
      for (int i = 0; i < FM; ++i) sx[i] = sxn[i];
      sw = swn;
    };
    gload(0);
    lstore(0);
    __syncthreads();
    const int fr = (lane & 15) * kQRow + (lane >> 4) * 16;
    for (int kt = 0; kt < KT; ++kt) {
      const int b = kt & 1;
      if (kt + 1 < KT) gload(kt + 1);
      Piece<EXACT> fx[FM];
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const uint8_t* p = &Xl[b][(wm * 64 + i * 16) * kQRow + fr];
        fx[i].set(*reinterpret_cast<const u32x4_t*>(p),
                  *reinterpret_cast<const u32x4_t*>(p + 64), sx[i]);
      }
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const uint8_t* p = &Wl[b][(wn * WN + j * 16) * kQRow + fr];
        Piece<EXACT> fw;
        fw.set(*reinterpret_cast<const u32x4_t*>(p), *reinterpret_cast<const u32x4_t*>(p + 64),
               sw);
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = mfma_q8(fw, fx[i], acc[j][i]);
      }
      if (kt + 1 < KT) lstore(b ^ 1);
      __syncthreads();
    }

    // the lane holds columns c .. c + 3 (c = 16 j + 4 (lane / 16)) of row
    // (lane & 15) of each 16 x 16 tile
    const int c0 = n0 + wn * WN + 4 * (lane >> 4);
    if constexpr (KIND == kUp) {
      const int No = kGated ? a.Nout / 2 : a.Nout;
      // activation in place, then each row's largest magnitude over the block:
      // the lane's, the four lanes of a row, the two waves of a row
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          f32x4_t& v = acc[j][i];
          const int c = c0 + 16 * j;
          if constexpr (kGated) {
            v[0] = c < a.Nout ? silu_f(v[0]) * v[1] : 0.0f;
            v[1] = c + 2 < a.Nout ? silu_f(v[2]) * v[3] : 0.0f;
            top = fmaxf(top, fmaxf(q8_mag(v[0]), q8_mag(v[1])));
          } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              v[u] = c + u < No ? act_fn<ACT>(v[u]) : 0.0f;
              top = fmaxf(top, q8_mag(v[u]));
            }
          }
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        if (lane < 16) s_top[wn][wm * 64 + i * 16 + lane] = top;
      }
      __syncthreads();
      const int blk = (kGated ? n0 / 2 : n0) / kBlk;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int row = wm * 64 + i * 16 + (lane & 15);
        const int byte = q8_scale_byte(fmaxf(s_top[0][row], s_top[1][row]));
        const float inv = q8_inv(byte);
        const int64_t drow = s_dst[row];
        if (drow < 0) continue;
        if (wn == 0 && lane < 16) a.s[drow * a.qspitch + blk] = static_cast<uint8_t>(byte);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const f32x4_t v = acc[j][i];
          const int c = c0 + 16 * j;
          uint8_t* const p = a.q + drow * a.qpitch + (kGated ? c / 2 : c);
          if constexpr (kGated)
            *reinterpret_cast<uint16_t*>(p) =
                static_cast<uint16_t>(q8_pack4(v[0] * inv, v[1] * inv, 0.0f, 0.0f));
          else
            *reinterpret_cast<uint32_t*>(p) =
                q8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        }
      }
    } else {
      T* const og = static_cast<T*>(routed ? a.dst : a.dst_sh);
      const bool vec = (reinterpret_cast<uintptr_t>(og) & 15u) == 0 && a.ldo % 4 == 0;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int64_t drow = s_dst[wm * 64 + i * 16 + (lane & 15)];
        if (drow < 0) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int c = c0 + 16 * j;
          f32x4_t v = acc[j][i];
          if (KIND == kDense && a.bias != nullptr) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (c + u < a.Nout) v[u] += a.bias[c + u];
          }
          store4(og + drow * a.ldo + c, v, a.Nout - c, vec && c + 4 <= a.Nout);
        }
      }
    }
    __syncthreads();
  }
}

constexpr int kQBlocksPerCu = 1;

template <int KIND, int ACT, typename T, bool EXACT>
hipError_t launch(const QArgs& a, hipStream_t st) {
  launch_kernel(&qgemm_kernel<KIND, ACT, T, EXACT>, dim3(device_cus() * kQBlocksPerCu), dim3(kQThreads),
                0, st, a);
  return hipGetLastError();
}

template <bool EXACT>
hipError_t launch_act(int act, const QArgs& a, hipStream_t st) {
  if (act == MOECA_ACT_SWIGLU) return launch<kUp, kActSwiglu, float, EXACT>(a, st);
  if (act == MOECA_ACT_GELU_ERF) return launch<kUp, kActGeluErf, float, EXACT>(a, st);
  return launch<kUp, kActGeluTanh, float, EXACT>(a, st);
}

// Whether the up projection takes the exact products (above).
bool exact_up(const Shape& s) { return !s.bf16 || s.cache8; }

}  // namespace

size_t q8_bytes(int64_t rows, int64_t K) {
  const int64_t q = (rows * q8_pitch(K) + 255) / 256 * 256;
  return static_cast<size_t>(q + (rows * q8_spitch(K) + 255) / 256 * 256);
}

Q8 q8_view(void* base, int64_t rows, int64_t K) {
  auto* p = static_cast<uint8_t*>(base);
  return Q8{p, p + (rows * q8_pitch(K) + 255) / 256 * 256};
}

FfnPlan q8_plan(const Shape& s, StepKind kind, int64_t rows) {
  (void)kind;
  (void)rows;
  FfnPlan p;
  p.tm = p.tm_up = kQTM;
  p.tn_up = s.swiglu ? 256 : 128;
  p.tn_down = 128;
  return p;
}

hipError_t launch_q8_up(const Shape& s, int act, const FfnPlan& plan, const QuantWeights& w,
                        const Buffers& b, hipStream_t st) {
  (void)plan;
  QArgs a{};
  const Q8 x = q8_view(b.x8, s.tokens(), s.d), mid = q8_view(b.mid, s.mid_rows(), s.d_ff);
  a.X = x.q;
  a.Xs = x.s;
  a.W = static_cast<const uint8_t*>(w.up);
  a.Ws = static_cast<const uint8_t*>(w.up_s);
  a.Wsh = static_cast<const uint8_t*>(w.up_sh);
  a.Wssh = static_cast<const uint8_t*>(w.up_sh_s);
  a.off = b.off;
  a.tile_off = b.tiles;
  a.list = b.list;
  a.row_dst = b.row_dst;
  a.E = s.E;
  a.G = s.groups();
  a.k = s.k;
  a.pitch = static_cast<int>(q8_pitch(s.d));
  a.spitch = static_cast<int>(q8_spitch(s.d));
  a.Nout = s.up_rows();
  a.q = mid.q;
  a.s = mid.s;
  a.qpitch = static_cast<int>(q8_pitch(s.d_ff));
  a.qspitch = static_cast<int>(q8_spitch(s.d_ff));
  if (exact_up(s)) return launch_act<true>(act, a, st);
  return launch_act<false>(act, a, st);
}

hipError_t launch_q8_down(const Shape& s, const FfnPlan& plan, const QuantWeights& w,
                          const Buffers& b, hipStream_t st) {
  (void)plan;
  QArgs a{};
  const Q8 mid = q8_view(b.mid, s.mid_rows(), s.d_ff);
  a.X = mid.q;
  a.Xs = mid.s;
  a.W = static_cast<const uint8_t*>(w.down);
  a.Ws = static_cast<const uint8_t*>(w.down_s);
  a.Wsh = static_cast<const uint8_t*>(w.down_sh);
  a.Wssh = static_cast<const uint8_t*>(w.down_sh_s);
  a.off = b.off;
  a.tile_off = b.tiles + s.groups() + 1;
  a.list = b.list;
  a.row_dst = b.row_dst;
  a.E = s.E;
  a.G = s.groups();
  a.k = s.k;
  a.pitch = static_cast<int>(q8_pitch(s.d_ff));
  a.spitch = static_cast<int>(q8_spitch(s.d_ff));
  a.Nout = s.d;
  a.ldo = s.d;
  a.dst = s.cache8 ? b.fresh : b.h_c;
  a.dst_sh = b.h_sh;
  if (s.bf16) return launch<kDown, kActNone, uint16_t, false>(a, st);
  return launch<kDown, kActNone, float, true>(a, st);
}

hipError_t launch_q8_linear(const Q8& x, int64_t M, int K, const void* W, const void* Ws, int N,
                            const float* bias, void* out, bool bf16, int64_t ldo,
                            hipStream_t st) {
  QArgs a{};
  a.X = x.q;
  a.Xs = x.s;
  a.W = static_cast<const uint8_t*>(W);
  a.Ws = static_cast<const uint8_t*>(Ws);
  a.M = static_cast<int>(M);
  a.pitch = static_cast<int>(q8_pitch(K));
  a.spitch = static_cast<int>(q8_spitch(K));
  a.Nout = N;
  a.ldo = ldo;
  a.bias = bias;
  a.dst = out;
  if (bf16) return launch<kDense, kActNone, uint16_t, false>(a, st);
  return launch<kDense, kActNone, float, true>(a, st);
}

}  // namespace moeca
