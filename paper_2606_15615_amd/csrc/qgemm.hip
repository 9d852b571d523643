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
// e4m3 number times a power of two down to 2^-133 (scales from 2^-124 on), and
// takes the bf16 instructions with fp32 sums:
//  - fp32 results, and those of at most 16 rows (a matter of latency, not of rate);
//  - both products of a layer whose cache is 8-bit too, since what is cached is
//    rounded to 8 bits once more.  Up: a hidden element that moves over a rounding
//    border (1 in 200 does, at 1.5e-5) moves the down projection's row by 1.4e-3,
//    and 1.6 % of the cached elements by a whole step of 2^-3: reused branches were
//    5.7e-3 off the 64-bit definition instead of 1.7e-3.  Down: one or two cached
//    elements in 10^4 moved by a step, and one scale in 10^5 by a power of two.  A
//    cycle of 8 x 1024 tokens, 16 experts of 1152 x 4608, takes 755 us with its down
//    projections exact, 672 without.
//
//   up   : mid[r]  = q8(act(x[token(r)] . W_up[e]^T))   rows by the expert lists
//   down : row of r = mid[r] . W_down[e]^T
//   dense: y[m] = x[m] . W^T + bias
//
// The up projection's epilogue quantises what it has in its accumulators: the
// hidden rows are never held in more than 8 bits, and the activation's value
// is rounded once, from fp32.
#include <algorithm>
#include <type_traits>

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
  // of the 256-column tiles: rows, at most, and (tm[2]) whether they are 128
  // columns wide (from the lists kernel; dense: rows from the host)
  const int32_t* tm;
  int dense_tm;
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
  // computed by here, whatever the compiler would rather
  __device__ __forceinline__ void pin() {}
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
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int h = 0; h < 4; ++h) asm volatile("" : "+v"(v[h]));
  }
};

typedef __attribute__((ext_vector_type(2))) float f32x2_q;
// Two fp32 -> two bf16 (hardware round to nearest even), packed in 4 bytes.
__device__ __forceinline__ uint32_t pack2_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_q{a, b}, bf16x2_q));
}

// ---------------------------------------------------------------------------
// What the tiles' epilogues share.  A wave has FN x FM accumulator tiles, FN of
// columns; the matrix instruction leaves four columns of row (lane & 15) of each
// with a lane, group g = lane / 16.  The weight rows are laid into LDS in an order
// that gives a lane V consecutive columns, as many as fill a 16-byte store (16
// hidden bytes, 8 bf16, 4 fp32; at most its 4 FN), and the four groups of a row
// the V after each other: no exchange, and a store covers whole runs of a row.
// Column of the wave's: tile j, group g, element u.
// ---------------------------------------------------------------------------
template <int V>
__device__ __forceinline__ constexpr int tile_column(int j, int g) {
  return j / (V / 4) * (4 * V) + V * g + 4 * (j % (V / 4));
}
// The tile's column that weight row r of its LDS rows holds.
template <int FN, int V>
__device__ __forceinline__ int weight_column(int r) {
  constexpr int WN = 16 * FN;
  const int t = r & (WN - 1);
  return r - t + tile_column<V>(t >> 4, (t >> 2) & 3) + (t & 3);
}
// V of an epilogue: hidden rows take 4 FN columns together, others 16 bytes.
template <int KIND, typename T, int FN>
__device__ __host__ constexpr int run_columns() {
  constexpr int most = KIND == kUp ? 16 : 16 / static_cast<int>(sizeof(T));
  return 4 * FN < most ? 4 * FN : most;
}

// The activation of an accumulator tile in place (gated: the two hidden values
// in v[0], v[1]), zeros in hidden columns past the width (their weight rows are
// clamped; whole: there are none), and the largest magnitude's bits.
template <int ACT>
__device__ __forceinline__ uint32_t hidden4(f32x4_t& v, int c, int Nout, bool whole) {
  if constexpr (ACT == kActSwiglu) {
    v[0] = silu_f(v[0]) * v[1];
    v[1] = silu_f(v[2]) * v[3];
    if (!whole) {
      if (c >= Nout) v[0] = 0.0f;
      if (c + 2 >= Nout) v[1] = 0.0f;
    }
    return max(q8_mag(v[0]), q8_mag(v[1]));
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[u] = act_fn<ACT>(v[u]);
      if (!whole && c + u >= Nout) v[u] = 0.0f;
    }
    return max(max(q8_mag(v[0]), q8_mag(v[1])), max(q8_mag(v[2]), q8_mag(v[3])));
  }
}
// The largest finite magnitude of a tile's hidden values.
template <int ACT>
__device__ __forceinline__ uint32_t hidden_finite4(const f32x4_t& v) {
  const uint32_t t = max(q8_finite(v[0]), q8_finite(v[1]));
  return ACT == kActSwiglu ? t : max(t, max(q8_finite(v[2]), q8_finite(v[3])));
}
// Largest over the four lanes of a row.
__device__ __forceinline__ uint32_t quad_max(uint32_t t) {
  t = max(t, static_cast<uint32_t>(__shfl_xor(static_cast<int>(t), 16, kWave)));
  return max(t, static_cast<uint32_t>(__shfl_xor(static_cast<int>(t), 32, kWave)));
}

// The hidden values of a row's accumulator tiles (columns c .. c + 4 FN - 1), their
// largest finite magnitude in the lane.
template <int ACT, int FN>
__device__ __forceinline__ uint32_t hidden_row(f32x4_t* const (&v)[FN], int c, int Nout,
                                               bool whole) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < FN; ++j) top = max(top, hidden4<ACT>(*v[j], c + 4 * j, Nout, whole));
  if (__builtin_expect(__any(top >= kInfBits), 0)) {
    top = 0;
#pragma unroll
    for (int j = 0; j < FN; ++j) top = max(top, hidden_finite4<ACT>(*v[j]));
  }
  return quad_max(top);
}

// Them quantised, into hidden columns c .. (gated: c / 2 ..) of their row.
template <int ACT, int FN>
__device__ __forceinline__ void store_hidden(uint8_t* row, int c, f32x4_t* const (&v)[FN],
                                             float inv) {
  constexpr int ND = ACT == kActSwiglu ? FN / 2 : FN;  // dwords
  uint32_t d[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) {
    if constexpr (ACT == kActSwiglu) {
      const f32x4_t &x = *v[2 * j], &y = *v[2 * j + 1];
      d[j] = q8_pack4(x[0] * inv, x[1] * inv, y[0] * inv, y[1] * inv);
    } else {
      const f32x4_t& x = *v[j];
      d[j] = q8_pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    }
  }
  uint8_t* const p = row + (ACT == kActSwiglu ? c / 2 : c);
  if constexpr (ND == 4) *reinterpret_cast<u32x4_t*>(p) = u32x4_t{d[0], d[1], d[2], d[3]};
  else if constexpr (ND == 2) *reinterpret_cast<u32x2_t*>(p) = u32x2_t{d[0], d[1]};
  else *reinterpret_cast<uint32_t*>(p) = d[0];
}

// The bias of a lane's columns (zeros without one, and past the last); c: the
// wave's first column.
template <int FN, int V>
__device__ __forceinline__ void load_bias(const QArgs& a, int c, int g, f32x4_t (&b)[FN]) {
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int n = c + tile_column<V>(j, g) + u;
      b[j][u] = a.bias != nullptr && n < a.Nout ? a.bias[n] : 0.0f;
    }
}

// A lane's columns of an output row; vec: rows are 16-byte aligned.
template <typename T, int FN, int V>
__device__ __forceinline__ void store_out(const QArgs& a, T* row, int c, int g,
                                          const f32x4_t* const (&v)[FN], const f32x4_t (&b)[FN],
                                          bool vec) {
  f32x4_t x[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) x[j] = *v[j] + b[j];
  if (vec && c + 16 * FN <= a.Nout) {
#pragma unroll
    for (int j = 0; j < FN; j += V / 4) {
      T* const p = row + c + tile_column<V>(j, g);
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x4_t*>(p) =
            u32x4_t{pack2_bf16(x[j][0], x[j][1]), pack2_bf16(x[j][2], x[j][3]),
                    pack2_bf16(x[j + 1][0], x[j + 1][1]), pack2_bf16(x[j + 1][2], x[j + 1][3])};
      else
        *reinterpret_cast<f32x4_t*>(p) = x[j];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int n = c + tile_column<V>(j, g) + u;
      if (n < a.Nout) row[n] = Act<T>::from_f32(x[j][u]);
    }
}

// The four (or two) waves' largest magnitudes of a row.
typedef __attribute__((ext_vector_type(4))) unsigned int top4_t;

// Tile `local` of a group of mt x nt tiles: bands of at most eight row tiles, equal
// ones, in a band the column tiles in turn, each with all of the band's rows.  The
// 32 CUs of an XCD, on consecutive tiles, then share some eight row and four column
// tiles in its L2 (without bands, and 64 row tiles, each CU had rows of its own).
__device__ __forceinline__ void band_order(int local, int mt, int nt, int& m, int& n) {
  const int nb = (mt + 7) / 8, h = mt / nb, tall = mt - nb * h;  // `tall` bands of h + 1, then h
  const int at = local / nt, edge = tall * (h + 1);
  const bool in_tall = at < edge;
  const int hb = in_tall ? h + 1 : h;
  const int first = in_tall ? at / (h + 1) * (h + 1) : edge + (at - edge) / h * h;
  const int in = local - first * nt;
  n = in / hb;
  m = first + in - n * hb;
}

// Source and destination row of row r of a tile (`rows` rows from r0 on).
template <int KIND>
__device__ __forceinline__ void tile_row(const QArgs& a, int e, int r0, int rows, int r, int& src,
                                         int& dst) {
  if constexpr (KIND == kDense) {
    src = r0 + (r < rows ? r : 0);
    dst = r < rows ? r0 + r : -1;
  } else {
    group_row<KIND>(e, a.E, r0, rows, r, a.k, a.off, a.list, a.row_dst, src, dst);
  }
}

// ---------------------------------------------------------------------------
// Two groups of four waves take turns: a group's memory slot (LDS reads, loads of
// the ring, one wait) runs beside the other's matrix slot, a barrier after each,
// so that on every SIMD one wave multiplies while the other reads.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void slot_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// One wait for both: at most N loads of this wave in flight (N < 16), every LDS
// read returned.
template <int N>
__device__ __forceinline__ void slot_wait() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// c += w x with the accumulator in place.  The builtin leaves the compiler free to
// put the sum elsewhere and to move the instruction past branches, barriers and
// waits; with 128 accumulator registers of 256 that ended in spills between the
// loads of the ring.  The operands' LDS reads are waited for by the caller
// (slot_wait), two wait states follow any vector instruction that wrote one, each
// accumulator is used once between two barriers, and the epilogue's first read is
// held off (below): the distances that the hardware leaves to the program.
__device__ __forceinline__ void mfma_q8_tied(f32x4_t& c, const i32x8_t& w, const i32x8_t& x,
                                             int sw, int sx) {
  asm volatile(
      "s_nop 1\n\t"
      "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
      : "+v"(c)
      : "v"(w), "v"(x), "v"(sw), "v"(sx));
}

__device__ __forceinline__ void mfma_q8(const Piece<false>& w, const Piece<false>& x, f32x4_t& c) {
  mfma_q8_tied(c, w.v, x.v, w.s, x.s);
}
__device__ __forceinline__ void mfma_q8(const Piece<true>& w, const Piece<true>& x, f32x4_t& c) {
#pragma unroll
  for (int h = 0; h < 4; ++h) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[h], x.v[h], c, 0, 0, 0);
}

// ---------------------------------------------------------------------------
// 128 rows x 256 weight rows for gated up projections, whose block of 128 hidden
// columns takes 256 weight rows: 8 waves (2 x 4) of 64 x 64, 4 x 4 tiles of 16 x 16
// each (weights the A operand).  A k-tile is 128 bytes of every row, one
// block; three of them (48 KB each) are in LDS or on their way, brought by direct
// global -> LDS loads in the XOR-swizzled order of the bf16 kernels: position p
// of row r holds 16-byte chunk p ^ ((r >> 1) & 7).  The scales come the same
// way, 16 bytes (16 k-tiles) of each row at a time, into one of two buffers; a
// k-tile's are read as bytes.  The two groups are the tile's halves of rows; EXACT
// converts its operands in the memory slot.  A block of 128 hidden columns lies
// with four waves of a row, which exchange their largest magnitudes through LDS.
// Persistent, one block per CU; the next tile's first loads start before this
// tile's epilogue.  Measured, 64 experts of 2048 x 1408, 4 x 1024 tokens, eight
// branches each: 256 us with the quantising of x, 1.48 PFLOP/s (EXACT 451 us, 0.84
// PFLOP/s: the conversions fill the memory slot).  For few rows an
// expert the kernel below has tiles of 64 x 256 (q8_plan).
// ---------------------------------------------------------------------------
constexpr int kMidTM = 128;
constexpr int kMidTN = 256;
constexpr int kMidWaves = 8;
constexpr int kMidThreads = kMidWaves * kWave;
constexpr int kMidStages = 3;
constexpr int kMidTileX = kMidTM * kBlk;               // bytes
constexpr int kMidStage = kMidTileX + kMidTN * kBlk;   // 48 KB
constexpr int kMidLoadsX = kMidTM / 8 / kMidWaves;     // 2 per wave and stage
constexpr int kMidLoadsW = kMidTN / 8 / kMidWaves;     // 4
constexpr int kMidScales = (kMidTM + 2) * 16;          // bytes of a scale buffer: rows, two blocks
template <bool EXACT>
__global__ __launch_bounds__(kMidThreads, 1) void qgemm_gated_kernel(QArgs a) {
  constexpr int FM = 4, FN = 4, V = run_columns<kUp, uint8_t, FN>();
  __shared__ __attribute__((aligned(16))) uint8_t lds[kMidStages * kMidStage];
  __shared__ __attribute__((aligned(16))) uint8_t s_sc[2][kMidScales];
  __shared__ int s_src[kMidTM], s_dst[kMidTM];
  __shared__ __attribute__((aligned(16))) uint32_t s_top[kMidTM][4];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wv >> 2, wn = wv & 3;
  const int nt = (a.Nout + kMidTN - 1) / kMidTN;
  const int total = a.tile_off[a.G];
  const int per = (total + kXcds - 1) / kXcds;
  const int lo = (blockIdx.x % kXcds) * per;
  const int hi = min(total, lo + per);
  const int stride = gridDim.x / kXcds;
  const int toff0 = lane < a.G ? a.tile_off[lane] : 0x7fffffff;
  const int toff1 = lane + 64 < a.G ? a.tile_off[lane + 64] : 0x7fffffff;
  const int KT = a.pitch / kBlk;
  const int nbw = (a.Nout + kBlk - 1) / kBlk;
  const int chunk = (lane & 7) ^ (4 * (wv & 1) + (lane >> 4));
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds) + wv * 1024);
  const uint32_t sc0 = __builtin_amdgcn_readfirstlane(lds_addr(&s_sc[0][0]) + wv * 1024);

  struct Tile {
    int e, r0, rows, n0;
  };
  auto tile = [&](int L) __attribute__((always_inline)) {
    Tile t;
    int e_base;
    t.e = tile_group(L, toff0, toff1, e_base);
    const int o0 = a.off[t.e];
    const int cnt = a.off[t.e + 1] - o0;
    const int mt = (cnt + kMidTM - 1) / kMidTM;
    int m, n;
    band_order(L - e_base, mt, nt, m, n);
    t.e = __builtin_amdgcn_readfirstlane(t.e);
    t.r0 = __builtin_amdgcn_readfirstlane(o0 + m * kMidTM);
    t.rows = __builtin_amdgcn_readfirstlane(min(kMidTM, cnt - m * kMidTM));
    t.n0 = __builtin_amdgcn_readfirstlane(n * kMidTN);
    return t;
  };

  const uint8_t *gx[kMidLoadsX], *gw[kMidLoadsW], *gs = nullptr;
  auto start = [&](const Tile& t, int src, int dst) __attribute__((always_inline)) {
    if (tid < kMidTM) {
      s_src[tid] = src;
      s_dst[tid] = dst;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMidLoadsX; ++u)
      gx[u] = a.X + int64_t(s_src[8 * (wv + kMidWaves * u) + (lane >> 3)]) * a.pitch + chunk * 16;
    const bool routed = t.e < a.E;
    const int64_t g = routed ? t.e : t.e - a.E;
    const uint8_t* const W = (routed ? a.W : a.Wsh) + g * a.Nout * a.pitch;
#pragma unroll
    for (int u = 0; u < kMidLoadsW; ++u) {
      const int n =
          min(t.n0 + weight_column<FN, V>(8 * (wv + kMidWaves * u) + (lane >> 3)), a.Nout - 1);
      gw[u] = W + int64_t(n) * a.pitch + chunk * 16;
    }
    // scales: waves 0 and 1 the rows', two lanes of wave 2 the weight blocks'
    if (wv < 2)
      gs = a.Xs + int64_t(s_src[64 * wv + lane]) * a.spitch;
    else if (wv == 2)
      gs = (routed ? a.Ws : a.Wssh) +
           (g * nbw + min(t.n0 / kBlk + (lane & 1), nbw - 1)) * a.spitch;
  };
  auto issue = [&](int kt, int st) __attribute__((always_inline)) {
    const uint32_t base = lds0 + st * kMidStage;
#pragma unroll
    for (int u = 0; u < kMidLoadsX; ++u)
      dma16(reinterpret_cast<const uint16_t*>(gx[u] + int64_t(kt) * kBlk),
            base + u * kMidWaves * 1024);
#pragma unroll
    for (int u = 0; u < kMidLoadsW; ++u)
      dma16(reinterpret_cast<const uint16_t*>(gw[u] + int64_t(kt) * kBlk),
            base + kMidTileX + u * kMidWaves * 1024);
  };
  auto issue_scales = [&](int c) __attribute__((always_inline)) {
    // the LDS address is the wave's: say so inside the lanes' branch too
    if (wv < 2 || (wv == 2 && lane < 2))
      dma16(reinterpret_cast<const uint16_t*>(gs + c * 16),
            __builtin_amdgcn_readfirstlane(sc0 + (c & 1) * kMidScales));
  };
  // the first two k-tiles and 16 k-tiles' scales of a tile
  auto begin = [&]() __attribute__((always_inline)) {
    issue_scales(0);
    issue(0, 0);
    if (KT > 1) issue(1, 1);
  };
  auto first_landed = [&]() __attribute__((always_inline)) {
    if (KT > 1) slot_wait<kMidLoadsX + kMidLoadsW>();
    else slot_wait<0>();
    slot_barrier();
  };

  int L = lo + static_cast<int>(blockIdx.x) / kXcds;
  if (L >= hi) return;
  Tile cur = tile(L);
  {
    int src = 0, dst = -1;
    if (tid < kMidTM) tile_row<kUp>(a, cur.e, cur.r0, cur.rows, tid, src, dst);
    start(cur, src, dst);
  }
  begin();
  const uint32_t fr = (lane & 15) * kBlk + (((lane >> 4) ^ ((lane >> 1) & 7)) * 16);

  for (;;) {
    const int Ln = L + stride;
    const bool has_next = Ln < hi;
    Tile nxt = cur;
    int nsrc = 0, ndst = -1;
    if (has_next) {
      nxt = tile(Ln);
      if (tid < kMidTM) tile_row<kUp>(a, nxt.e, nxt.r0, nxt.rows, tid, nsrc, ndst);
    }
    f32x4_t acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[j][i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // a wave without rows or columns of the tile only loads and waits
    const bool active = wm * 64 < cur.rows && cur.n0 + wn * 64 < a.Nout;
    first_landed();
    if (wm == 1) slot_barrier();
    int st = 0;
    for (int kt = 0; kt < KT; ++kt) {
      // memory slot
      Piece<EXACT> px[FM], pw[FN];
      if (active) {
        const uint32_t xo = st * kMidStage + wm * 64 * kBlk + fr;
        const uint32_t wo = st * kMidStage + kMidTileX + wn * 64 * kBlk + fr;
        const uint8_t* const sc = s_sc[(kt >> 4) & 1] + (kt & 15);
        const int sw = sc[(kMidTM + (wn >> 1)) * 16];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const uint32_t o = xo + i * 16 * kBlk;  // and chunk (lane / 16) + 4: bit 6 flipped
          px[i].set(*reinterpret_cast<const u32x4_t*>(lds + o),
                    *reinterpret_cast<const u32x4_t*>(lds + (o ^ 64u)),
                    sc[(wm * 64 + i * 16 + (lane & 15)) * 16]);
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const uint32_t o = wo + j * 16 * kBlk;
          pw[j].set(*reinterpret_cast<const u32x4_t*>(lds + o),
                    *reinterpret_cast<const u32x4_t*>(lds + (o ^ 64u)), sw);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) px[i].pin();
#pragma unroll
        for (int j = 0; j < FN; ++j) pw[j].pin();
      }
      if (kt + 2 < KT) {
        issue(kt + 2, st == 0 ? 2 : st - 1);
        if ((kt & 15) == 0 && kt + 16 < KT) issue_scales((kt >> 4) + 1);
        slot_wait<kMidLoadsX + kMidLoadsW>();
      } else {
        slot_wait<0>();
      }
      slot_barrier();
      // matrix slot
      if (active) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int i = 0; i < FM; ++i) mfma_q8(pw[j], px[i], acc[j][i]);
        __builtin_amdgcn_s_setprio(0);
      }
      slot_barrier();
      st = st == 2 ? 0 : st + 1;
    }
    if (wm == 0) slot_barrier();
    if (!EXACT) {
      // what reads the accumulators comes after this
      asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) asm volatile("" : "+v"(acc[j][i]));
    }

    int drow[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) drow[i] = s_dst[wm * 64 + i * 16 + (lane & 15)];
    __syncthreads();
    if (has_next) {
      start(nxt, nsrc, ndst);
      begin();
    }
    const int c0 = cur.n0 + wn * 64 + 16 * (lane >> 4);
    const bool whole = cur.n0 + kMidTN <= a.Nout;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      f32x4_t* const v[FN] = {&acc[0][i], &acc[1][i], &acc[2][i], &acc[3][i]};
      const uint32_t top = hidden_row<kActSwiglu, FN>(v, c0, a.Nout, whole);
      if (lane < 16) s_top[wm * 64 + i * 16 + lane][wn] = top;
    }
    __syncthreads();
    const int blk = cur.n0 / 2 / kBlk;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const top4_t t = *reinterpret_cast<const top4_t*>(s_top[wm * 64 + i * 16 + (lane & 15)]);
      const int byte = q8_scale_byte(max(max(t[0], t[1]), max(t[2], t[3])));
      if (drow[i] < 0) continue;
      f32x4_t* const v[FN] = {&acc[0][i], &acc[1][i], &acc[2][i], &acc[3][i]};
      store_hidden<kActSwiglu, FN>(a.q + int64_t(drow[i]) * a.qpitch, c0, v, q8_inv(byte));
      if (wn == 0 && lane < 16)
        a.s[int64_t(drow[i]) * a.qspitch + blk] = static_cast<uint8_t>(byte);
    }
    if (!has_next) break;
    L = Ln;
    cur = nxt;
  }
}

// ---------------------------------------------------------------------------
// Tiles of TM = 128, 64 or 32 rows by 128 columns (gated: 256 weight rows, TM = 64) in
// blocks of four waves, two blocks per CU (gated: one): what one block waits for,
// its loads, its conversions, its epilogue, runs beside the other's matrix
// instructions.  Waves are 2 x 2 of 64 x 64 (TM = 128) or 1 x 4 of TM x 32; a ring
// of kStages k-tiles, one barrier each, in the swizzled order of the gated kernel,
// scales in two buffers of 16 k-tiles.  A tile of TM = 64 skips the 16-row tiles
// that it has no rows for.
//
// What bounds it: with many rows, EXACT, what a CU can load (20 bytes a clock; 16
// experts of 1152 x 4608, 8 x 1024 tokens, up 206 us, 0.85 PFLOP/s of bf16
// instructions, down 167 us, 1.04); with few, the stream of the weights (256 tokens
// of the same layer: up 85 MB in 21 to 25 us, 576 tiles for 512 places; down 20.5 us,
// 4.1 TB/s).  A ring of six k-tiles instead of three left down at 21 and slowed up to
// 33 us (one block per CU).  Four stages of half a k-tile, three ahead, in the LDS of
// the two stages of 128 EXACT rows took 7 % longer.  Dense 333 x 1152 x 4608 10.9 us,
// 1000 rows 17.6 us.
// ---------------------------------------------------------------------------
template <int TM, bool GATED> struct Duo {
  static constexpr int TN = GATED ? 256 : 128;
  static constexpr int kWaves = 4, kThreads = kWaves * kWave;
  static constexpr int kStages = TM == 128 ? 2 : 3;
  static constexpr int kTileX = TM * kBlk, kStage = (TM + TN) * kBlk;
  static constexpr int kLoadsX = TM / 8 / kWaves, kLoadsW = TN / 8 / kWaves;
  static constexpr int kScales = (TM + TN / kBlk) * 16;
  static constexpr int kBlocks = GATED ? 1 : 2;
  static constexpr int kWavesM = TM == 128 ? 2 : 1, kWavesN = kWaves / kWavesM;
  static constexpr int FM = TM / kWavesM / 16, FN = TN / kWavesN / 16;
};

template <int KIND, int ACT, typename T, bool EXACT, int TM>
__global__ __launch_bounds__(256, (Duo<TM, ACT == kActSwiglu>::kBlocks)) void qgemm_duo_kernel(
    QArgs a) {
  constexpr bool kGated = ACT == kActSwiglu;
  typedef Duo<TM, kGated> D;
  constexpr int FM = D::FM, FN = D::FN, WN = FN * 16, V = run_columns<KIND, T, FN>();
  __shared__ __attribute__((aligned(16))) uint8_t lds[D::kStages * D::kStage];
  __shared__ __attribute__((aligned(16))) uint8_t s_sc[2][D::kScales];
  __shared__ int s_src[TM], s_dst[TM];
  __shared__ __attribute__((aligned(16))) uint32_t s_top[KIND == kUp ? TM : 1][D::kWavesN];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wv / D::kWavesN, wn = wv % D::kWavesN;
  const int nt = (a.Nout + D::TN - 1) / D::TN;
  const int total = KIND == kDense ? (a.M + TM - 1) / TM * nt : a.tile_off[a.G];
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
  const int chunk = (lane & 7) ^ (4 * (wv & 1) + (lane >> 4));
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds) + wv * 1024);
  // the scales' rows are loaded by the first waves, 64 each, the weight blocks' by
  // the next one
  constexpr int kRowWavesX = TM == 128 ? 2 : 1;
  const uint32_t sc0 = __builtin_amdgcn_readfirstlane(
      lds_addr(&s_sc[0][0]) + (wv < kRowWavesX ? wv * 1024 : TM * 16));
  const uint32_t fr = (lane & 15) * kBlk + (((lane >> 4) ^ ((lane >> 1) & 7)) * 16);

  for (int L = lo + static_cast<int>(blockIdx.x) / kXcds; L < hi; L += stride) {
    int e = 0, e_base = 0, o0 = 0, cnt = a.M;
    if constexpr (KIND != kDense) {
      e = tile_group(L, toff0, toff1, e_base);
      o0 = a.off[e];
      cnt = a.off[e + 1] - o0;
    }
    const int mt = (cnt + TM - 1) / TM;
    int m, n;
    band_order(L - e_base, mt, nt, m, n);
    e = __builtin_amdgcn_readfirstlane(e);
    const int r0 = __builtin_amdgcn_readfirstlane(o0 + m * TM);
    const int rows = __builtin_amdgcn_readfirstlane(min(TM, cnt - m * TM));
    const int n0 = __builtin_amdgcn_readfirstlane(n * D::TN);
    const bool routed = KIND == kDense || e < a.E;
    const int64_t g = routed ? e : e - a.E;
    const uint8_t* const W = (routed ? a.W : a.Wsh) + g * a.Nout * a.pitch;
    const uint8_t* const Ws = (routed ? a.Ws : a.Wssh) + g * nbw * a.spitch;
    const uint8_t *gx[D::kLoadsX], *gw[D::kLoadsW], *gs;
#pragma unroll
    for (int u = 0; u < D::kLoadsW; ++u)
      gw[u] = W +
              int64_t(min(n0 + weight_column<FN, V>(8 * (wv + D::kWaves * u) + (lane >> 3)),
                          a.Nout - 1)) * a.pitch +
              chunk * 16;
    auto issue_w = [&](int kt, int st) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < D::kLoadsW; ++u)
        dma16(reinterpret_cast<const uint16_t*>(gw[u] + int64_t(kt) * kBlk),
              lds0 + st * D::kStage + D::kTileX + u * D::kWaves * 1024);
    };
    // nx: of the loads' 32-row groups, those that the tile has rows in
    auto issue_x = [&](int kt, int st, auto nx) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < decltype(nx)::value; ++u)
        dma16(reinterpret_cast<const uint16_t*>(gx[u] + int64_t(kt) * kBlk),
              lds0 + st * D::kStage + u * D::kWaves * 1024);
    };
    auto issue_scales = [&](int c) __attribute__((always_inline)) {
      if (wv <= kRowWavesX && lane < (wv < kRowWavesX ? TM : D::TN / kBlk))
        dma16(reinterpret_cast<const uint16_t*>(gs + c * 16),
              __builtin_amdgcn_readfirstlane(sc0 + (c & 1) * D::kScales));
    };
    // the weights need no row table: their first k-tiles are asked for before it
    issue_w(0, 0);
    if (tid < TM) {
      int src, dst;
      tile_row<KIND>(a, e, r0, rows, tid, src, dst);
      s_src[tid] = src;
      s_dst[tid] = dst;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < D::kLoadsX; ++u)
      gx[u] = a.X + int64_t(s_src[8 * (wv + D::kWaves * u) + (lane >> 3)]) * a.pitch + chunk * 16;
    gs = wv < kRowWavesX ? a.Xs + int64_t(s_src[(64 * wv + lane) & (TM - 1)]) * a.spitch
                      : Ws + int64_t(min(n0 / kBlk + (lane & 1), nbw - 1)) * a.spitch;
    issue_scales(0);

    f32x4_t acc[FN][FM];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[j][i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // the k-loop for a wave with NI 16-row tiles
    auto run = [&](auto ni_c) __attribute__((always_inline)) {
      constexpr int NI = decltype(ni_c)::value;
      typedef std::integral_constant<int, (TM == 64 && NI > 0 && NI <= 2 ? 1 : D::kLoadsX)> NX;
      issue_x(0, 0, NX{});
      if (D::kStages > 2 && KT > 1) {
        issue_w(1, 1);
        issue_x(1, 1, NX{});
      }
      int st = 0;
      for (int kt = 0; kt < KT; ++kt) {
        if (D::kStages > 2 && kt + 1 < KT) slot_wait<D::kLoadsW + NX::value>();
        else slot_wait<0>();
        slot_barrier();
        constexpr int kAhead = D::kStages - 1;
        if (kt + kAhead < KT) {
          const int to = st + kAhead >= D::kStages ? st + kAhead - D::kStages : st + kAhead;
          issue_w(kt + kAhead, to);
          issue_x(kt + kAhead, to, NX{});
          if ((kt & 15) == 0 && kt + 16 < KT) issue_scales((kt >> 4) + 1);
        }
        if constexpr (NI > 0) {
          const uint32_t xo = st * D::kStage + wm * 64 * kBlk + fr;
          const uint32_t wo = st * D::kStage + D::kTileX + wn * WN * kBlk + fr;
          const uint8_t* const sc = s_sc[(kt >> 4) & 1] + (kt & 15);
          const int sw = sc[(TM + (wn * WN) / kBlk) * 16];
          Piece<EXACT> px[NI > 0 ? NI : 1];
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const uint32_t o = xo + i * 16 * kBlk;
            px[i].set(*reinterpret_cast<const u32x4_t*>(lds + o),
                      *reinterpret_cast<const u32x4_t*>(lds + (o ^ 64u)),
                      sc[(wm * 64 + i * 16 + (lane & 15)) * 16]);
          }
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            const uint32_t o = wo + j * 16 * kBlk;
            Piece<EXACT> pw;
            pw.set(*reinterpret_cast<const u32x4_t*>(lds + o),
                   *reinterpret_cast<const u32x4_t*>(lds + (o ^ 64u)), sw);
#pragma unroll
            for (int i = 0; i < NI; ++i) mfma_q8(pw, px[i], acc[j][i]);
          }
        }
        st = st + 1 == D::kStages ? 0 : st + 1;
      }
    };
    const int mine = rows - wm * 64;
    if (n0 + wn * WN >= a.Nout || mine <= 0) run(std::integral_constant<int, 0>{});
    else if (TM == 64 && mine <= 16) run(std::integral_constant<int, 1>{});
    else if (TM == 64 && mine <= 32) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, FM>{});
    if (!EXACT) {
      asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) asm volatile("" : "+v"(acc[j][i]));
    }

    const int cw = n0 + wn * WN, c0 = cw + 4 * FN * (lane >> 4);
    if constexpr (KIND == kUp) {
      const bool whole = n0 + D::TN <= a.Nout;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        if (TM == 64 && i * 16 >= rows) continue;
        f32x4_t* v[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
        const uint32_t top = hidden_row<ACT, FN>(v, c0, a.Nout, whole);
        if (lane < 16) s_top[wm * 64 + i * 16 + lane][wn] = top;
      }
      __syncthreads();
      const int blk = (kGated ? n0 / 2 : n0) / kBlk;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int row = wm * 64 + i * 16 + (lane & 15);
        const int64_t drow = s_dst[row];
        uint32_t top = s_top[row][0];
#pragma unroll
        for (int w = 1; w < D::kWavesN; ++w) top = max(top, s_top[row][w]);
        const int byte = q8_scale_byte(top);
        if (drow < 0) continue;
        f32x4_t* v[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
        store_hidden<ACT, FN>(a.q + drow * a.qpitch, c0, v, q8_inv(byte));
        if (wn == 0 && lane < 16) a.s[drow * a.qspitch + blk] = static_cast<uint8_t>(byte);
      }
    } else {
      T* const og = static_cast<T*>(routed ? a.dst : a.dst_sh);
      const bool vec =
          (reinterpret_cast<uintptr_t>(og) & 15u) == 0 && a.ldo * sizeof(T) % 16 == 0;
      f32x4_t bias[FN];
      load_bias<FN, V>(a, cw, lane >> 4, bias);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int64_t drow = s_dst[wm * 64 + i * 16 + (lane & 15)];
        if (drow < 0) continue;
        const f32x4_t* v[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
        store_out<T, FN, V>(a, og + drow * a.ldo, cw, lane >> 4, v, bias, vec);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// 256 x 256 tiles for many rows, 8-bit products only: 64 KB of a k-tile per 16.8
// MFLOP, where 128 x 128 take 32 KB per 4.2 and 128 x 256 take 48 KB per 8.4, so
// that neither what a CU can load nor its LDS bounds the matrix instructions.
//
// The schedule is the 256 x 256 bf16 kernel's (ffn.hip), whose k-tile has the
// same bytes: eight waves of 128 rows x 64 columns (2 x 4), two LDS buffers of a
// k-tile, each in four 16 KB regions, rows X0 X1 and columns W0 W1; a k-tile is
// four phases, X0 W0, X0 W1, X1 W1, X1 W0, each a memory slot (LDS reads, two
// loads, one wait) and a matrix slot (8 instructions of 16 x 16 x 128); waves 4-7
// run one slot behind waves 0-3.  A region is refilled one phase after its last
// read and has seven phases to land.  The load stream goes on into the next tile.
//
// Scales: 16 k-tiles of a tile's rows and two weight blocks (258 x 16 bytes) come
// in one piece, three buffers in turn (the next piece, or the next tile's first,
// is on its way while one is read).  The extra load only makes the counted waits
// a little longer.
//
// The rows of a tile, 256, 192 or 128, come from the lists kernel's table (dense:
// from the host) as for the bf16 kernel, and so do its columns: 128 where tiles of
// 256 would leave half of the CUs without one (a threshold step that recomputes few
// branches, which the host cannot know); the second columns' region is not loaded
// then (16 experts of 1152 x 4608, 8 x 1024 tokens, down projections of a full step and
// three such steps 49.1 -> 46.5 us on average).
//
// Measured: 16384 x 4608 x 4608 300 us, 2.3 PFLOP/s; 16 experts of 1152 x 4608, 8 x
// 1024 tokens, up 180 us and down 98 us, 0.97 and 1.77 PFLOP/s; 64 gated experts of
// 2048 x 1408, 4 x 4096 tokens, up 930 us and down 615 us, 2.0 and 1.5 PFLOP/s.  A
// k-tile takes 1.2 to 1.4 us a tile (the matrix instructions alone 0.9), a tile some 10 us
// besides: 128 KB of results leave every CU at about the same time.  Letting the next
// tile's counted waits pass those stores changed nothing (340 and 340 us with
// the quantising).
// ---------------------------------------------------------------------------
constexpr int kTallTM = 256;
constexpr int kTallTN = 256;
constexpr int kTallWaves = 8;
constexpr int kTallThreads = kTallWaves * kWave;
constexpr int kTallHalf = 128 * kBlk;    // bytes of a region
constexpr int kTallBuf = 4 * kTallHalf;  // X0 X1 W0 W1
constexpr int kTallMinKT = 4;            // k-tiles
constexpr int kTallScales = (kTallTM + 2) * 16;

// The column, of the tile's, that row r of region h of the weights holds.  A wave
// has rows 32 wn .. of either region, two 16-column tiles in each.  wide: the
// tile has columns past 128, and a wave 64 consecutive ones; else the first region
// has them all, and a wave 32.
template <int KIND, typename T>
__device__ __forceinline__ int tall_column(int r, int h, bool wide) {
  const int wn = r >> 5, j = (r >> 4) & 1, g = (r >> 2) & 3, u = r & 3;
  return wide ? 64 * wn + tile_column<run_columns<KIND, T, 4>()>(2 * h + j, g) + u
              : 32 * wn + tile_column<run_columns<KIND, T, 2>()>(j, g) + u;
}

template <int KIND, int ACT, typename T>
__global__ __launch_bounds__(kTallThreads, 1) void qgemm_tall_kernel(QArgs a) {
  constexpr bool kGated = ACT == kActSwiglu;
  constexpr bool kListed = KIND == kUp;  // token rows come through the list
  constexpr bool kTable = KIND != kDense;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kTallBuf];
  __shared__ __attribute__((aligned(16))) uint8_t s_sc[3 * kTallScales];
  __shared__ int s_list[2][kTallTM];
  __shared__ int s_toff[128];
  __shared__ __attribute__((aligned(16))) uint32_t s_top[KIND == kUp ? kTallTM : 1][4];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wv >> 2, wn = wv & 3;  // wm is also the ping-pong group
  const int TM = kTable ? a.tm[0] : a.dense_tm;
  const bool half = kTable && !kGated && a.tm[2] != 0;
  const int TN = half ? 128 : kTallTN;
  const int nt = (a.Nout + TN - 1) / TN;
  const int total = kTable ? a.tile_off[a.G] : (a.M + TM - 1) / TM * nt;
  const int per = (total + kXcds - 1) / kXcds;
  const int lo = (blockIdx.x % kXcds) * per;
  const int hi = min(total, lo + per);
  const int stride = gridDim.x / kXcds;
  if constexpr (kTable) {
    if (tid < 128) s_toff[tid] = tid < a.G ? a.tile_off[tid] : 0x7fffffff;
    __syncthreads();
  }
  const int KT = a.pitch / kBlk;
  const int nbw = (a.Nout + kBlk - 1) / kBlk;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds) + wv * 1024);
  const uint32_t sl0 = __builtin_amdgcn_readfirstlane(lds_addr(&s_list[0][0]) + (wv & 3) * 256);
  const uint32_t sc0 = __builtin_amdgcn_readfirstlane(lds_addr(&s_sc[0]) + wv * 1024);

  // the lane number, opaque to the compiler: what is derived from it at a tile's
  // ends is computed there and not kept in registers across the k-loop
  auto fresh_lane = [&]() __attribute__((always_inline)) {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  struct TTile {
    int e, r0, rows, n0;
  };
  auto tile = [&](int L) __attribute__((always_inline)) {
    TTile t;
    int e_base = 0, o0 = 0, cnt = a.M;
    t.e = 0;
    if constexpr (kTable) {
      const int toff0 = s_toff[fresh_lane()], toff1 = s_toff[64 + fresh_lane()];
      t.e = __builtin_amdgcn_readfirstlane(tile_group(L, toff0, toff1, e_base));
      o0 = a.off[t.e];
      cnt = a.off[t.e + 1] - o0;
    }
    const int mt = (cnt + TM - 1) / TM;
    int m, n;
    band_order(__builtin_amdgcn_readfirstlane(L - e_base), mt, nt, m, n);
    t.r0 = __builtin_amdgcn_readfirstlane(o0 + static_cast<int>(int64_t(m) * cnt / mt));
    t.rows = __builtin_amdgcn_readfirstlane(o0 + static_cast<int>(int64_t(m + 1) * cnt / mt) - t.r0);
    t.n0 = __builtin_amdgcn_readfirstlane(n * TN);
    return t;
  };

  // gated tiles are always wide: they fill whole blocks of the hidden rows
  auto wide = [&](const TTile& t) __attribute__((always_inline)) {
    return kGated || (!half && t.n0 + 128 < a.Nout);
  };
  // the load stream's tile: byte offsets of this lane's rows, and of its scales'
  uint32_t va[4], vw[4];
  const uint8_t* wbase = a.W;
  auto source = [&](const TTile& t, int lb, int r) __attribute__((always_inline)) {
    const int rr = r < t.rows ? r : 0;
    if (KIND == kDense) return t.r0 + rr;
    if (KIND == kDown) return t.r0 + rr;
    if (t.e >= a.E) return t.r0 + rr - a.off[t.e];
    return s_list[lb][rr] / a.k;
  };
  auto aim = [&](const TTile& t, int lb) __attribute__((always_inline)) {
    const int lane = fresh_lane();
    const int chunk = (lane & 7) ^ (4 * (wv & 1) + (lane >> 4));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = 128 * (q >> 1) + 8 * (wv + kTallWaves * (q & 1)) + (lane >> 3);
      va[q] = static_cast<uint32_t>(source(t, lb, r)) * static_cast<uint32_t>(a.pitch) + chunk * 16;
      const int n = min(tall_column<KIND, T>(r & 127, q >> 1, wide(t)), a.Nout - 1 - t.n0);
      vw[q] = static_cast<uint32_t>(n) * static_cast<uint32_t>(a.pitch) + chunk * 16;
    }
    const bool routed = !kTable || t.e < a.E;
    wbase = (routed ? a.W : a.Wsh) + (int64_t(routed ? t.e : t.e - a.E) * a.Nout + t.n0) * a.pitch;
  };
  // piece c of a tile's scales into buffer b: waves 0-3 the rows', two lanes of
  // wave 4 the weight blocks'
  auto issue_scales = [&](const TTile& t, int lb, int c, int b) __attribute__((always_inline)) {
    const int lane = fresh_lane();
    const uint32_t to = __builtin_amdgcn_readfirstlane(sc0 + b * kTallScales);
    if (wv < 4) {
      dma16(reinterpret_cast<const uint16_t*>(
                a.Xs + int64_t(source(t, lb, 64 * wv + lane)) * a.spitch + c * 16),
            to);
    } else if (wv == 4 && lane < 2) {
      const bool routed = !kTable || t.e < a.E;
      dma16(reinterpret_cast<const uint16_t*>(
                (routed ? a.Ws : a.Wssh) +
                (int64_t(routed ? t.e : t.e - a.E) * nbw + min(t.n0 / kBlk + lane, nbw - 1)) *
                    a.spitch + c * 16),
            __builtin_amdgcn_readfirstlane(to));
    }
  };
  // row table of a tile into s_list[lb]: the list entries, fetched one tile ahead
  // (up), or the output rows of the current tile (down)
  auto fetch_list = [&](const TTile& t, int lb) __attribute__((always_inline)) {
    const int lane = fresh_lane();
    if (wv < 4 && t.e < a.E)
      dma4((kListed ? a.list : a.row_dst) + t.r0 + min(64 * wv + lane, t.rows - 1),
           sl0 + lb * (kTallTM * 4));
  };
  auto issue_x = [&](int kt, int b, int h, int nr) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (h == 0 || 128 + 64 * u < nr)
        dma16_s(a.X + kt * kBlk, va[2 * h + u], lds0 + b * kTallBuf + h * kTallHalf + u * 8192);
  };
  auto issue_w = [&](int kt, int b, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      dma16_s(wbase + kt * kBlk, vw[2 * h + u],
              lds0 + b * kTallBuf + (2 + h) * kTallHalf + u * 8192);
  };

  const uint32_t fr = (lane & 15) * kBlk + (((lane >> 4) ^ ((lane >> 1) & 7)) * 16);
  const uint8_t* const xl = lds + wm * 2048;
  const uint8_t* const wl = lds + 2 * kTallHalf + wn * 4096;
  const uint32_t sl = (lane & 15) * 16 + wm * 256;

  i32x8_t fx[4], fa[2], fb[2];
  int sx[4], sw;
  auto read_x = [&](int b, int h, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= n) continue;
      const uint8_t* const p = xl + b * kTallBuf + h * kTallHalf + i * 4096;
      fx[i] = join(*reinterpret_cast<const u32x4_t*>(p + fr),
                   *reinterpret_cast<const u32x4_t*>(p + (fr ^ 64)));
    }
  };
  auto read_w = [&](i32x8_t (&f)[2], int b, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint8_t* const p = wl + b * kTallBuf + h * kTallHalf + j * 2048;
      f[j] = join(*reinterpret_cast<const u32x4_t*>(p + fr),
                  *reinterpret_cast<const u32x4_t*>(p + (fr ^ 64)));
    }
  };
  // sb: the scale buffer's offset plus the k-tile's byte
  auto read_sx = [&](int sb, int h, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) sx[i] = s_sc[sb + sl + h * 2048 + i * 512];
  };

  int L = lo + static_cast<int>(blockIdx.x) / kXcds;
  if (L >= hi) return;
  TTile cur = tile(L);
  int lb = 0, sb = 0;      // row table and first buffer of the tile
  int sc = 0;              // scale buffer of the k-tile (0, 1, 2)
  if (kListed) fetch_list(cur, 0);
  slot_wait<0>();
  slot_barrier();
  aim(cur, 0);
  issue_scales(cur, 0, 0, 0);
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    issue_w(p, p, 0);
    issue_x(p, p, 0, kTallTM);
    issue_w(p, p, 1);
    issue_x(p, p, 1, kTallTM);
  }
  slot_wait<0>();
  slot_barrier();
  read_w(fa, 0, 0);
  slot_wait<0>();
  slot_barrier();
  if (wm == 1) slot_barrier();

  f32x4_t acc[4][8];  // [column tile][row tile]
  for (;;) {
    const int Ln = L + stride;
    const bool has_next = Ln < hi;
    TTile nxt = cur;
    if (has_next) nxt = tile(Ln);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[j][i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // one instantiation per tile height (NX = 0, 2 or 4 16-row tiles per wave in
    // the second half), with or without columns past 128 (CA: wide)
    auto run = [&](auto nx_c, auto ca_c) __attribute__((always_inline)) {
      constexpr int NX = decltype(nx_c)::value;
      constexpr bool CA = decltype(ca_c)::value;
      auto mfma_q = [&](int h, int c, const i32x8_t (&f)[2]) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (h == 0 || i < NX)
              mfma_q8_tied(acc[2 * c + j][4 * h + i], f[j], fx[i], sw, sx[i]);
        __builtin_amdgcn_s_setprio(0);
      };
      auto ktile = [&](int t, int b, i32x8_t (&p)[2], i32x8_t (&q)[2], auto tail_c)
          __attribute__((always_inline)) {
        constexpr bool kTail = decltype(tail_c)::value;
        const int lt = kTail ? t + 2 - KT : t + 2;
        constexpr int nx = kTail || NX == 4 ? 256 : NX == 2 ? 192 : 128;
        const int so = __builtin_amdgcn_readfirstlane(sc * kTallScales + (t & 15));
        auto settle = [&]() __attribute__((always_inline)) {
          slot_wait<kTail ? 8 : (CA ? 8 : 4) + NX>();
          slot_barrier();
        };
        // phase 0: X0 x W0
        read_x(b, 0, 4);
        read_sx(so, 0, 4);
        sw = s_sc[so + kTallTM * 16 + (CA ? (wn >> 1) * 16 : 0)];
        issue_w(lt, b, 0);
        settle();
        mfma_q(0, 0, p);
        slot_barrier();
        // phase 1: X0 x W1
        if (CA) read_w(q, b, 1);
        issue_x(lt, b, 0, nx);
        settle();
        if (CA) mfma_q(0, 1, q);
        slot_barrier();
        // phase 2: X1 x W1
        if (NX > 0) {
          read_x(b, 1, NX);
          read_sx(so, 1, NX);
        }
        if (CA || kTail) issue_w(lt, b, 1);
        settle();
        if (CA && NX > 0) mfma_q(1, 1, q);
        slot_barrier();
        // phase 3: X1 x W0, and the next k-tile's W0
        read_w(q, b ^ 1, 0);
        issue_x(lt, b, 1, nx);
        settle();
        if (NX > 0) mfma_q(1, 0, p);
        slot_barrier();
      };
      // No branches inside a k-tile: tables and scales are asked for between them,
      // and the last tile's last two k-tiles load as the others' do (its own first
      // ones, again).
      auto advance = [&](int done) __attribute__((always_inline)) {
        sc = (done & 15) != 15 ? sc : sc == 2 ? 0 : sc + 1;
      };
      int t = 0;
      for (; t < KT - 3; t += 2) {
        if ((t & 15) == 0) {
          // the row table of this tile (down) or the next one (up), in the buffer
          // that the previous tile's epilogue does not read
          if (t == 0 && KIND == kDown) fetch_list(cur, lb);
          if (t == 0 && kListed && has_next) fetch_list(nxt, lb ^ 1);
          if (t + 16 < KT) issue_scales(cur, lb, (t >> 4) + 1, sc == 2 ? 0 : sc + 1);
        }
        ktile(t, sb, fa, fb, std::false_type{});
        ktile(t + 1, sb ^ 1, fb, fa, std::false_type{});
        advance(t + 1);
      }
      if (t == KT - 3) {
        // odd count: one more, and its roles exchanged back
        ktile(t, sb, fa, fb, std::false_type{});
#pragma unroll
        for (int j = 0; j < 2; ++j) fa[j] = fb[j];
        sb ^= 1;
        advance(t);
      }
      if (has_next) {
        aim(nxt, lb ^ 1);
        // into the next buffer, or past the one that this tile's last k-tile reads
        issue_scales(nxt, lb ^ 1, 0, (sc + (((KT - 2) & 15) == 15 ? 2 : 1)) % 3);
      }
      ktile(KT - 2, sb, fa, fb, std::true_type{});
      advance(KT - 2);
      ktile(KT - 1, sb ^ 1, fb, fa, std::true_type{});
      // what reads the accumulators comes after this
      asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(acc[j][i]));
    };
    if (wide(cur)) {
      if (cur.rows > 192) run(std::integral_constant<int, 4>{}, std::true_type{});
      else if (cur.rows > 128) run(std::integral_constant<int, 2>{}, std::true_type{});
      else run(std::integral_constant<int, 0>{}, std::true_type{});
    } else {
      if (cur.rows > 192) run(std::integral_constant<int, 4>{}, std::false_type{});
      else if (cur.rows > 128) run(std::integral_constant<int, 2>{}, std::false_type{});
      else run(std::integral_constant<int, 0>{}, std::false_type{});
    }

    // epilogue: tile i of rows starts at 128 (i / 4) + 16 (2 (i % 4) + wm); the
    // wave has 64 columns, or 32 (tall_column)
    const int lane = fresh_lane();
    const int g = lane >> 4;
    auto finish = [&](auto fn_c) __attribute__((always_inline)) {
      constexpr int FN = decltype(fn_c)::value;
      constexpr int V = run_columns<KIND, T, FN>();
      const int cw = cur.n0 + 16 * FN * wn, c0 = cw + 4 * FN * g;
      if constexpr (KIND == kUp) {
        const bool whole = cur.n0 + 64 * FN <= a.Nout;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f32x4_t* v[FN];
#pragma unroll
          for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
          const uint32_t top = hidden_row<ACT, FN>(v, c0, a.Nout, whole);
          if (lane < 16) s_top[128 * (i >> 2) + 16 * (2 * (i & 3) + wm) + lane][wn] = top;
        }
        slot_wait<15>();
        slot_barrier();
        // a block of 128 hidden columns lies with two waves, or four (gated, not wide)
        constexpr bool kPair = FN == 4 && !kGated;
        const int blk = kGated ? cur.n0 / 2 / kBlk : cur.n0 / kBlk + (kPair ? wn >> 1 : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = 128 * (i >> 2) + 16 * (2 * (i & 3) + wm) + (lane & 15);
          const top4_t t = *reinterpret_cast<const top4_t*>(s_top[row]);
          const uint32_t t01 = max(t[0], t[1]), t23 = max(t[2], t[3]);
          const int byte = q8_scale_byte(kPair ? (wn < 2 ? t01 : t23) : max(t01, t23));
          const int64_t drow = cur.r0 + row;
          f32x4_t* v[FN];
#pragma unroll
          for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
          if (row < cur.rows && blk * kBlk < a.qpitch) {
            store_hidden<ACT, FN>(a.q + drow * a.qpitch, c0, v, q8_inv(byte));
            if ((wn & (kPair ? 1 : 3)) == 0 && lane < 16)
              a.s[drow * a.qspitch + blk] = static_cast<uint8_t>(byte);
          }
        }
      } else {
        T* const og = static_cast<T*>(!kTable || cur.e < a.E ? a.dst : a.dst_sh);
        const bool vec =
            (reinterpret_cast<uintptr_t>(og) & 15u) == 0 && a.ldo * sizeof(T) % 16 == 0;
        f32x4_t bias[FN];
        load_bias<FN, V>(a, cw, g, bias);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = 128 * (i >> 2) + 16 * (2 * (i & 3) + wm) + (lane & 15);
          if (row >= cur.rows) continue;
          int64_t drow = cur.r0 + row;
          if (KIND == kDown) drow = cur.e < a.E ? s_list[lb][row] : drow - a.off[a.E];
          const f32x4_t* v[FN];
#pragma unroll
          for (int j = 0; j < FN; ++j) v[j] = &acc[j][i];
          store_out<T, FN, V>(a, og + drow * a.ldo, cw, g, v, bias, vec);
        }
      }
    };
    if (wide(cur)) finish(std::integral_constant<int, 4>{});
    else finish(std::integral_constant<int, 2>{});
    if (!has_next) break;
    // the next tile's first piece of scales
    sc = sc == 2 ? 0 : sc + 1;
    L = Ln;
    cur = nxt;
    lb ^= 1;
  }
  if (wm == 0) slot_barrier();
  slot_wait<0>();  // the last loads have landed before the LDS is given up
}

// ---------------------------------------------------------------------------
// y = x W^T for up to 16 rows straight from the activations: one launch, no
// workspace.  A block has 16 columns (weight rows), its four waves every fourth
// k-tile; a wave loads its weights from memory into the operand registers,
// quantises the block of every row itself (a lane has 32 of a row's 128 elements),
// and the waves' sums meet in LDS, added in wave order.  What bounds it is how many
// loads are in flight: at M = 1 the grid covers every CU from N = 4096 on, and all
// of a wave's loads up to K = 1536 are asked for at once.  1 x 1152 x 4608 6.6 us, 16
// rows 7.3 us; quantising first, then 64-row tiles, takes 7.8 and 8.4 us.
// ---------------------------------------------------------------------------
constexpr int kFewWaves = 4;
constexpr int kFewAhead = 3;  // k-tiles of a wave in flight

template <typename T, bool VEC>
__global__ __launch_bounds__(kFewWaves * kWave) void qlinear_few_kernel(
    const T* __restrict__ x, int M, int K, int64_t ldx, const uint8_t* __restrict__ W,
    const uint8_t* __restrict__ Ws, int N, const float* __restrict__ bias, T* __restrict__ out,
    int64_t ldo) {
  __shared__ f32x4_t s_acc[kFewWaves - 1][kWave];
  const int lane = threadIdx.x & (kWave - 1);
  const int wv = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int g = lane >> 4, r = lane & 15;
  const int pitch = static_cast<int>(q8_pitch(K)), spitch = static_cast<int>(q8_spitch(K));
  const int KT = pitch / kBlk;
  const int n0 = blockIdx.x * 16;
  const uint8_t* const wrow = W + int64_t(min(n0 + r, N - 1)) * pitch + g * 16;
  const uint8_t* const wsc = Ws + int64_t(n0 / kBlk) * spitch;
  const bool in = r < M;
  const T* const xr = x + int64_t(in ? r : 0) * ldx;  // lanes without a row: the first, as zeros
  f32x4_t acc{0.0f, 0.0f, 0.0f, 0.0f};

  for (int k0 = wv; k0 < KT; k0 += kFewWaves * kFewAhead) {
    u32x4_t w[kFewAhead][2];
    int sw[kFewAhead];
    float v[kFewAhead][32];
#pragma unroll
    for (int t = 0; t < kFewAhead; ++t) {
      const int kt = k0 + kFewWaves * t;
      if (kt >= KT) continue;  // uniform
      w[t][0] = *reinterpret_cast<const u32x4_t*>(wrow + int64_t(kt) * kBlk);
      w[t][1] = *reinterpret_cast<const u32x4_t*>(wrow + int64_t(kt) * kBlk + 64);
      sw[t] = wsc[kt];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int c = kt * kBlk + 64 * (h >> 1) + g * 16 + 8 * (h & 1);
        load8<T, VEC>(xr + c, K - c, &v[t][8 * h]);
      }
    }
#pragma unroll
    for (int t = 0; t < kFewAhead; ++t) {
      if (k0 + kFewWaves * t >= KT) continue;
      Piece<true> pw, px;
      pw.set(w[t][0], w[t][1], sw[t]);
      const float* const e = v[t];
      uint32_t top = 0;
#pragma unroll
      for (int u = 0; u < 32; ++u) top = max(top, q8_mag(e[u]));
      if (__builtin_expect(__any(top >= kInfBits), 0)) {
        top = 0;
#pragma unroll
        for (int u = 0; u < 32; ++u) top = max(top, q8_finite(e[u]));
      }
      const int byte = q8_scale_byte(quad_max(top));
      const float inv = q8_inv(byte);
      u32x4_t q[2];
#pragma unroll
      for (int d = 0; d < 8; ++d)
        q[d >> 2][d & 3] = in ? q8_pack4(e[4 * d] * inv, e[4 * d + 1] * inv, e[4 * d + 2] * inv,
                                         e[4 * d + 3] * inv)
                              : 0u;
      px.set(q[0], q[1], byte);
      mfma_q8(pw, px, acc);
    }
  }
  if (wv > 0) s_acc[wv - 1][lane] = acc;
  __syncthreads();
  if (wv > 0 || !in) return;
#pragma unroll
  for (int w = 0; w < kFewWaves - 1; ++w) acc += s_acc[w][lane];
  const int c = n0 + 4 * g;
  T* const o = out + int64_t(r) * ldo;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (c + u >= N) continue;
    o[c + u] = Act<T>::from_f32(bias != nullptr ? acc[u] + bias[c + u] : acc[u]);
  }
}

template <int KIND, int ACT, typename T>
hipError_t launch_tall(const QArgs& a, hipStream_t st) {
  launch_kernel(&qgemm_tall_kernel<KIND, ACT, T>, dim3(device_cus()), dim3(kTallThreads), 0, st,
                a);
  return hipGetLastError();
}

template <int KIND, int ACT, typename T, bool EXACT, int TM>
hipError_t launch_duo(const QArgs& a, hipStream_t st) {
  launch_kernel(&qgemm_duo_kernel<KIND, ACT, T, EXACT, TM>,
                dim3(device_cus() * Duo<TM, ACT == kActSwiglu>::kBlocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int ACT>
hipError_t launch_up(const QArgs& a, bool exact, const FfnPlan& plan, hipStream_t st) {
  if (plan.tall_up) return launch_tall<kUp, ACT, float>(a, st);
  if (plan.tm_up == 128) {
    if constexpr (ACT == kActSwiglu) {
      const dim3 grid(device_cus()), block(kMidThreads);
      if (exact) launch_kernel(&qgemm_gated_kernel<true>, grid, block, 0, st, a);
      else launch_kernel(&qgemm_gated_kernel<false>, grid, block, 0, st, a);
      return hipGetLastError();
    } else {
      return exact ? launch_duo<kUp, ACT, float, true, 128>(a, st)
                   : launch_duo<kUp, ACT, float, false, 128>(a, st);
    }
  }
  return exact ? launch_duo<kUp, ACT, float, true, 64>(a, st)
               : launch_duo<kUp, ACT, float, false, 64>(a, st);
}

template <typename T, bool EXACT>
hipError_t launch_down(const QArgs& a, const FfnPlan& plan, hipStream_t st) {
  return plan.tm == 64 ? launch_duo<kDown, kActNone, T, EXACT, 64>(a, st)
                       : launch_duo<kDown, kActNone, T, EXACT, 128>(a, st);
}

// Whether the 256 x 256 tiles can take a product: rows addressed by 32-bit byte
// offsets, K long enough for the load stream's lookahead.
bool tall_capable(int64_t rows, int K) {
  return q8_pitch(K) / kBlk >= kTallMinKT && rows * q8_pitch(K) < (int64_t(1) << 32);
}

// Whether a layer's products are the exact ones (above).
bool exact_products(const Shape& s) { return !s.bf16 || s.exact8; }

// The tile height (32, 64, 128, or 256 for the 256-column tiles) that takes least
// time: blocks come in rounds of two per CU, the last one perhaps of one, which is
// over sooner; the 256-column tiles one per CU.  Times of a round in tenths of a
// microsecond, per k-tile and fixed, one block and two per CU, fitted to dense
// products of 17 to 16384 rows, 640 to 4608 columns, K 640 to 9216: of 84 bf16 sizes
// the tile chosen is the fastest but for a few within 8 %.  Measured, us, 32 / 64 /
// 128 rows / 256 columns: 129 x 1152 x 4608 9.7 11.0 13.4 19.6; 700 x 4608 x 4608
// 44 33 37 48; 1500 x 1152 x 4608 25.3 22.2 19.5 23.9; 8192 x 4608 x 4608
// 320 229 189 179.  (Gated up projections, which have tiles of their own, are weighed
// against the 256-row tiles by the same figures.)
// tiles(tm, tn): tiles of a height and width; least: the lowest height there is.
template <typename F>
int q8_tile(F tiles, int kt, bool exact, bool tall, int least) {
  struct Cost {
    int tm, one_kt, one, two_kt, two;
  };
  constexpr Cost kFast[3] = {{32, 37, 370, 62, 260}, {64, 60, 300, 74, 430}, {128, 67, 500, 98, 340}};
  constexpr Cost kExact[3] = {{32, 53, 350, 87, 380}, {64, 77, 390, 108, 680}, {128, 140, 480, 187, 660}};
  const int64_t cus = device_cus();
  int best = 0;
  int64_t cost = 0;
  for (const Cost& c : exact ? kExact : kFast) {
    if (c.tm < least) continue;
    const int64_t n = tiles(c.tm, 128), rest = n % (2 * cus);
    const int64_t one = c.one_kt * kt + c.one, two = c.two_kt * kt + c.two;
    const int64_t t = n / (2 * cus) * two + (rest == 0 ? 0 : rest <= cus ? one : two);
    if (best == 0 || t < cost) {
      best = c.tm;
      cost = t;
    }
  }
  if (tall) {
    const int64_t t = (tiles(kTallTM, kTallTN) + cus - 1) / cus * (123 * kt + 1040);
    if (t < cost) best = kTallTM;
  }
  return best;
}

}  // namespace

size_t q8_bytes(int64_t rows, int64_t K) {
  const int64_t q = (rows * q8_pitch(K) + 255) / 256 * 256;
  return static_cast<size_t>(q + (rows * q8_spitch(K) + 255) / 256 * 256);
}

Q8 q8_view(void* base, int64_t rows, int64_t K) {
  auto* p = static_cast<uint8_t*>(base);
  return Q8{p, p + (rows * q8_pitch(K) + 255) / 256 * 256};
}

FfnPlan q8_plan(const Shape& s, int64_t rows) {
  FfnPlan p;
  const bool exact = exact_products(s);
  // the rows of an expert vary: an eighth above the mean
  const int64_t mean = rows / s.E + rows / s.E / 8;
  auto tiles = [&](int n) {
    return [&s, mean, n](int tm, int tn) {
      return (s.E * std::max<int64_t>(1, (mean + tm - 1) / tm) +
              s.S * ((s.tokens() + tm - 1) / tm)) * ((n + tn - 1) / tn);
    };
  };
  const int ku = static_cast<int>(q8_pitch(s.d) / kBlk), kd = static_cast<int>(q8_pitch(s.d_ff) / kBlk);
  p.tm_up = q8_tile(tiles(s.up_rows()), ku, exact, !exact && tall_capable(s.tokens(), s.d), 64);
  p.tm = q8_tile(tiles(s.d), kd, exact, !exact && tall_capable(s.mid_rows(), s.d_ff), 64);
  p.tall_up = p.tm_up == kTallTM;
  p.tall_down = p.tm == kTallTM;
  // Gated: 64-row tiles, one block per CU, where most experts have one.  Up, us, 64
  // against 128 rows, 64 experts of 2048 x 1408 with 18, 36 and 72 rows (an eighth above
  // the mean), EXACT: 75 84, 85 86, 124 105; not EXACT, 36 and 72: 74 76, 97 80.  (16
  // of 1152 x 2304 with 72 would rather have 64: 37 46, 29 33.)
  if (s.swiglu && !p.tall_up) p.tm_up = mean <= 48 ? 64 : kMidTM;
  p.tn_up = p.tall_up || s.swiglu ? 256 : 128;
  p.tn_down = p.tall_down ? kTallTN : 128;
  p.half_up = !s.swiglu;
  p.half_down = true;
  return p;
}

hipError_t launch_q8_up(const Shape& s, int act, const FfnPlan& plan, const QuantWeights& w,
                        const Buffers& b, hipStream_t st) {
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
  a.tm = b.tiles + 2 * (s.groups() + 1);
  const bool exact = exact_products(s);
  if (act == MOECA_ACT_SWIGLU) return launch_up<kActSwiglu>(a, exact, plan, st);
  if (act == MOECA_ACT_GELU_ERF) return launch_up<kActGeluErf>(a, exact, plan, st);
  return launch_up<kActGeluTanh>(a, exact, plan, st);
}

hipError_t launch_q8_down(const Shape& s, const FfnPlan& plan, const QuantWeights& w,
                          const Buffers& b, hipStream_t st) {
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
  a.tm = b.tiles + 2 * (s.groups() + 1) + 1;
  if (plan.tall_down) return launch_tall<kDown, kActNone, uint16_t>(a, st);
  if (!s.bf16) return launch_down<float, true>(a, plan, st);
  return exact_products(s) ? launch_down<uint16_t, true>(a, plan, st)
                           : launch_down<uint16_t, false>(a, plan, st);
}

int64_t q8_few_rows() { return 16; }

hipError_t launch_q8_few(const void* x, bool bf16, int64_t M, int K, int64_t ldx, const void* W,
                         const void* Ws, int N, const float* bias, void* out, int64_t ldo,
                         hipStream_t st) {
  if (M > q8_few_rows()) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>((N + 15) / 16)), block(kFewWaves * kWave);
  const size_t elem = bf16 ? 2 : 4;
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ldx * elem % 16 == 0;
#define MOECA_FEW(T, V)                                                                      \
  launch_kernel(&qlinear_few_kernel<T, V>, grid, block, 0, st, static_cast<const T*>(x),     \
                static_cast<int>(M), K, ldx, static_cast<const uint8_t*>(W),                 \
                static_cast<const uint8_t*>(Ws), N, bias, static_cast<T*>(out), ldo)
  if (bf16) {
    if (vec) MOECA_FEW(uint16_t, true);
    else MOECA_FEW(uint16_t, false);
  } else {
    if (vec) MOECA_FEW(float, true);
    else MOECA_FEW(float, false);
  }
#undef MOECA_FEW
  return hipGetLastError();
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
  auto tiles = [&](int tm, int tn) { return (M + tm - 1) / tm * ((int64_t(N) + tn - 1) / tn); };
  switch (q8_tile(tiles, a.pitch / kBlk, !bf16, bf16 && tall_capable(M, K), 32)) {
    case 32:
      return bf16 ? launch_duo<kDense, kActNone, uint16_t, false, 32>(a, st)
                  : launch_duo<kDense, kActNone, float, true, 32>(a, st);
    case 64:
      return bf16 ? launch_duo<kDense, kActNone, uint16_t, false, 64>(a, st)
                  : launch_duo<kDense, kActNone, float, true, 64>(a, st);
    case 128:
      return bf16 ? launch_duo<kDense, kActNone, uint16_t, false, 128>(a, st)
                  : launch_duo<kDense, kActNone, float, true, 128>(a, st);
    default:
      a.dense_tm = tall_rows_one(M, (N + kTallTN - 1) / kTallTN, device_cus());
      return launch_tall<kDense, kActNone, uint16_t>(a, st);
  }
}

}  // namespace moeca
