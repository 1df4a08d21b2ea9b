// Product of matrices in 8 bits with a power-of-two scale for each 128 columns (svdcache_matmul8).
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 columns of 16 rows of W and of 16 rows of A, that is one block of scales of each, and applies the
// scales itself: the sum over blocks is a plain chain of these instructions.  Operand layout per lane l (r = l % 16, g = l / 16):
//     W: 32 bytes of row r,  A: 32 bytes of row r,  result: 4 float32 = z[n = 4 g .. 4 g + 3][m = r]
// The 128 columns may be dealt out to the lanes of a row in any order as long as W and A use the same one; each lane hands over the scale of its own
// row, and as all four lanes of a row lie in one block of scales the order does not matter to the scales either.
//
// The instruction adds the products of 8 consecutive bytes with 13 bits below the largest exponent among them (the operands' own added up, -6 for subnormal values; measured: smaller
// bits are cut off), then those sums in float32.  That is less than 2^-10 of sum |a w|, and some 2e-5 of sums of random signs (measured at K = 11072): nothing beside the rounding
// of a result to bfloat16 or e4m3 but where large terms cancel, and not float32.  So are the partial sums of such results made.  Results in float32 are made with
// bfloat16 instructions, at half the rate: e4m3 values are bfloat16 values exactly, and their products are summed with 24 bits.  With their scales they are bfloat16 values
// too, but for scales near the ends of their range (448 * 2^126 is above the largest bfloat16, 2^-9 * 2^-126 below the smallest): there a block's sums are made without
// scales and enter the others times 2^(exponent of A + exponent of W), which is in range wherever the result is.
#include <algorithm>

#include "eight_bit.h"
#include "matmul8_plan.h"
#include "svdc_internal.h"

namespace svdc {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MatmulArgs {
  const uint8_t *A, *As, *W, *Ws;
  const float* bias;
  void* Out;
  uint8_t* Os;
  int64_t M, ldo;
  int N, K, dtype, act, splits;
};

__device__ __forceinline__ f32x4 mfma8(const i32x8& w, const i32x8& a, const f32x4& c, int sw, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, sw, 0, sa);
}

// 8 e4m3 values times `scale`, a power of two, as bfloat16: exactly for scales with in_range
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
// 2^-9 * scale is a normal number (byte >= 10) and 448 * scale a finite one (byte <= 246)
__device__ __forceinline__ bool in_range(int byte) { return (uint32_t)byte - 10 <= 236; }

// Exponents of the scales of the sums of a column: `a` of its row of A, and of rows of W that lie in one block of 128 up to row `edge` (one number for all lanes), in the
// next from there on.  All as bytes, of W's a lane's for its own row.
struct Exponents {
  int below, above, edge;
  __device__ __forceinline__ Exponents(int w, int a) : below(w + a - 254), above(0), edge(INT32_MAX) {}
  __device__ __forceinline__ Exponents(int w, int a, int edge, int last)
      : below(__builtin_amdgcn_readlane(w, 0) + a - 254), above(__builtin_amdgcn_readlane(w, last) + a - 254), edge(edge) {}
  __device__ __forceinline__ int operator[](int row) const { return row < edge ? below : above; }
};

// c += t * 2^exponent: sums of a block of columns, of which the e-th lies in row row_of(e) of the tile
template <typename Sums, typename Row>
__device__ __forceinline__ void add_scaled(Sums& c, const Sums& t, const Exponents& exponent, Row&& row_of) {
#pragma unroll
  for (int e = 0; e < (int)(sizeof(Sums) / sizeof(float)); ++e) c[e] += __builtin_amdgcn_ldexpf(t[e], exponent[row_of(e)]);
}

// 128 columns of 16 rows of W and of A, without scales and with float32 sums
__device__ __forceinline__ f32x4 widened(const i32x8& w, const i32x8& a) {
  f32x4 t = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * i], w[2 * i + 1], 1.f), widen8(a[2 * i], a[2 * i + 1], 1.f), t, 0, 0, 0);
  return t;
}

// x / (1 + exp(-t)), with the hardware's power of two and reciprocal (one step of the last place each): half the instructions of a division
__device__ __forceinline__ float times_sigmoid(float x, float t_log2e) {
  return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-t_log2e));
}
__device__ __forceinline__ float silu(float x) { return times_sigmoid(x, 1.4426950408889634f * x); }
// with t = 2 sqrt(2 / pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu(float x) { return times_sigmoid(x, x * __builtin_fmaf(0.10294324f, x * x, 2.3022082f)); }

// Column `col` of Out from its sum z (and the sum u that it gates); zero beyond the last column
__device__ __forceinline__ float finished(const MatmulArgs& a, int col, float z, float u) {
  if (col >= a.N) return 0.f;
  if (a.bias) {
    z += a.bias[col];
    if (a.act == SVDC_ACT_SWIGLU) u += a.bias[a.N + col];
  }
  return a.act == SVDC_ACT_GELU ? gelu(z) : a.act == SVDC_ACT_SWIGLU ? silu(z) * u : z;
}

// ---- few rows, or few tiles ------------------------------------------------------------------------------------------
//
// Where there are not enough large tiles to occupy the card, a workgroup makes 16 TM rows by 16 TN columns and its eight waves share the blocks of columns of
// A and W: wave w takes blocks w, w + 8, ... straight from memory into registers (nothing is used twice within a wave), and the eight sums are added through
// LDS, always in the same order.
//
// What bounds it: the look-ups of lines by the loads.  A load of an operand takes 64 bytes of 16 rows, and lines are looked up one at a time: 54 MB of weights in this
// pattern take 13.6 us alone, in 128 bytes of 8 rows 9.8 us, but the matrix instructions want 16 rows (instructions that waste half their work on the other pattern were no
// faster).  1 x 18432 x 3072 into bfloat16 12.3 us (4.6 TB/s of weights; a read of as many bytes 8.7 us), 1 x 3072 x 3072 4.4 us.

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }   // a value that all lanes hold, as a scalar

// a buffer for bounds-checked accesses: loads beyond its end give zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bounded(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

constexpr int kShareWaves = 8;

// GATED: TN tiles of gates and TN of what they gate.  EXACT: float32 sums.  EIGHT: the result is in 8 bits (TN = 8).
template <int TM, int TN, bool EXACT, bool GATED, bool EIGHT>
__device__ __forceinline__ void shared_sums(const MatmulArgs& a) {
  constexpr int NW = GATED ? 2 * TN : TN, COLUMNS = 16 * TN, ROWS = 16 * TM;
  constexpr int FREE = 190 - TM * NW * 4 - (EXACT ? 40 : 0), EACH = (TM + NW) * 9;   // registers: for operands, and those of a block
  constexpr int DEPTH = FREE / EACH < 1 ? 1 : FREE / EACH > 3 ? 3 : FREE / EACH;     // blocks in flight
  __shared__ f32x4 sums[kShareWaves][NW * TM][kWave];
  __shared__ float tops[TM * 16][8];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  const int64_t Kp = q8_row_bytes(a.K);
  const int blocks = uniform(q8_blocks(a.K)), ss = uniform(q8_scale_row_bytes(a.K));
  const int column_tiles = (a.N + COLUMNS - 1) / COLUMNS;
  const int row_tile = uniform(blockIdx.x / column_tiles), column_tile = uniform(blockIdx.x % column_tiles);
  const int64_t m0 = (int64_t)row_tile * ROWS;
  const int n0 = column_tile * COLUMNS, rows = (int)min<int64_t>(ROWS, a.M - m0), columns = min(COLUMNS, a.N - n0);

  const int a_bytes = uniform((int)(rows * Kp)), w_bytes = uniform((int)(columns * Kp));
  const int as_bytes = uniform(rows * ss), ws_bytes = uniform((int)((int64_t)q8_blocks(GATED ? 2 * a.N : a.N) * ss));
  // a lane's 32 bytes of a row are 16 from each half of a block, so that a load takes 64 bytes in a row
  uint32_t at[TM + NW];
#pragma unroll
  for (int t = 0; t < TM + NW; ++t) at[t] = (uint32_t)(((t < TM ? t : (t - TM) % TN) * 16 + r) * Kp + 16 * g);
  // scales: of TM tiles of A; one for all columns, as they lie in one block of 128; of what the gates gate, whose blocks begin anywhere, each row's own
  constexpr int SCALES = TM + 1 + (GATED ? TN : 0);
  uint32_t scale_at[SCALES];
#pragma unroll
  for (int t = 0; t < SCALES; ++t)
    scale_at[t] = (uint32_t)(t < TM    ? (t * 16 + r) * ss
                             : t == TM ? n0 / kScaleBlock * ss
                                       : (a.N + min(n0 + (t - TM - 1) * 16 + r, a.N - 1)) / kScaleBlock * ss);
  struct Operands {
    i32x8 x[TM + NW];
    int s[SCALES];
  };
  const auto load = [&](int b, Operands& o) {
    const int any = b < blocks ? -1 : 0;
    const auto A = bounded(a.A + m0 * Kp, a_bytes & any), W = bounded(a.W + n0 * Kp, w_bytes & any),
               U = bounded(a.W + ((GATED ? (int64_t)a.N : 0) + n0) * Kp, w_bytes & any);
    const auto As = bounded(a.As + m0 * ss, as_bytes & any), Ws = bounded(a.Ws, ws_bytes & any);
#pragma unroll
    for (int t = 0; t < SCALES; ++t) o.s[t] = __builtin_amdgcn_raw_buffer_load_b32(t < TM ? As : Ws, scale_at[t], uniform(b & ~3), 0);
#pragma unroll
    for (int t = 0; t < TM + NW; ++t) {
      const auto from = t < TM ? A : t < TM + TN ? W : U;
      const auto lo = __builtin_amdgcn_raw_buffer_load_b128(from, at[t], uniform(b * 128), 0),
                 hi = __builtin_amdgcn_raw_buffer_load_b128(from, at[t], uniform(b * 128 + 64), 0);
      o.x[t] = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    }
  };
  f32x4 c[NW][TM] = {};
  // rows of tile i of what the gates gate that lie before the next block of 128 rows
  const auto edge = [&](int i) { return kScaleBlock - (a.N + n0 + 16 * i) % kScaleBlock; };
  const auto multiply = [&](int b, const Operands& o) {
    int s[SCALES];                         // the block's byte, lowest
#pragma unroll
    for (int t = 0; t < SCALES; ++t) {
      s[t] = o.s[t];
      asm volatile("" : "+v"(s[t]));       // not before this block's turn, or it would wait for the loads of all of them
      s[t] = (int)((uint32_t)s[t] >> (b & 3) * 8);
      if (EXACT) s[t] &= 255;
    }
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        const int sw = s[i < TN ? TM : TM + 1 + i - TN];
        if (!EXACT) {
          c[i][j] = mfma8(o.x[TM + i], o.x[j], c[i][j], sw, s[j]);
        } else {
          add_scaled(c[i][j], widened(o.x[TM + i], o.x[j]), i < TN ? Exponents(sw, s[j]) : Exponents(sw, s[j], edge(i - TN), 15), [&](int e) { return 4 * g + e; });
        }
      }
  };
  Operands o[DEPTH];
  int b = wave;
  if (b + DEPTH * kShareWaves < blocks) {
    // Loads and products of a round are made whether its blocks are there or not (behind the last one the buffers have no bytes and give zeros): behind
    // conditions, the compiler would wait for each block's loads before the next block's were of any use.
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      load(b + d * kShareWaves, o[d]);
      __builtin_amdgcn_sched_barrier(0);
    }
    for (; b + DEPTH * kShareWaves < blocks; b += DEPTH * kShareWaves) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        multiply(b + d * kShareWaves, o[d]);
        __builtin_amdgcn_sched_barrier(0);
        load(b + (d + DEPTH) * kShareWaves, o[d]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) multiply(b + d * kShareWaves, o[d]);
  } else {
    // all at once, and no loads for nothing: they cost as much as others
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (b + d * kShareWaves < blocks) load(b + d * kShareWaves, o[d]);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (b + d * kShareWaves < blocks) multiply(b + d * kShareWaves, o[d]);
  }
#pragma unroll
  for (int i = 0; i < NW; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) sums[wave][i * TM + j][lane] = c[i][j];
  __syncthreads();

  // wave w finishes tiles w, w + 8, ... of 16 columns by 16 rows: lane (r, g) columns 4 g .. 4 g + 3 of row r
  constexpr int TURNS = (TN * TM + kShareWaves - 1) / kShareWaves;
  float v[TURNS][4];
#pragma unroll
  for (int turn = 0; turn < TURNS; ++turn) {
    const int tile = turn * kShareWaves + wave, i = tile / TM, j = tile % TM;
    if (TN * TM % kShareWaves && tile >= TN * TM) break;
    f32x4 z = {}, u = {};
#pragma unroll
    for (int w = 0; w < kShareWaves; ++w) {
      z += sums[w][tile][lane];
      if (GATED) u += sums[w][TN * TM + tile][lane];
    }
    const int col = n0 + 16 * i + 4 * g;
    const int64_t row = m0 + 16 * j + r;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[turn][e] = finished(a, col + e, z[e], GATED ? u[e] : 0.f);
    if (EIGHT) {
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[turn][e]));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (g == 0) tops[16 * j + r][i] = top;
    } else if (row < a.M) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.N) {
          if (EXACT)
            static_cast<float*>(a.Out)[row * a.ldo + col + e] = v[turn][e];
          else
            static_cast<bf16_t*>(a.Out)[row * a.ldo + col + e] = (bf16_t)v[turn][e];
        }
    }
  }
  if (EIGHT) {
    static_assert(!EIGHT || TN == 8, "");
    __syncthreads();
#pragma unroll
    for (int turn = 0; turn < TURNS; ++turn) {
      const int tile = turn * kShareWaves + wave, i = tile / TM, j = tile % TM;
      const int col = n0 + 16 * i + 4 * g;
      const int64_t row = m0 + 16 * j + r;
      float top = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) top = fmaxf(top, tops[16 * j + r][w]);
      const int byte = scale_byte(top);
      const float inv = inverse_scale(byte);
      if (row < a.M) {
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.Out) + row * q8_row_bytes(a.N) + col) =
            pack_e4m3(v[turn][0] * inv, v[turn][1] * inv, v[turn][2] * inv, v[turn][3] * inv);
        uint8_t* os = a.Os + row * q8_scale_row_bytes(a.N);
        if (i == 0 && g == 0) os[column_tile] = (uint8_t)byte;
        if (i == 1 && g == 0 && column_tile == column_tiles - 1)
          for (int s = column_tiles; s < q8_scale_row_bytes(a.N); ++s) os[s] = 127;
      }
    }
  }
}

template <int TM, int TN, bool EXACT, bool GATED, bool EIGHT>
__global__ __launch_bounds__(kShareWaves* kWave) void matmul8_shared_kernel(MatmulArgs a) {
#ifdef __HIP_DEVICE_COMPILE__          // buffer descriptors mean nothing to the host's pass
  shared_sums<TM, TN, EXACT, GATED, EIGHT>(a);
#endif
}

// ---- tiles ----------------------------------------------------------------------------------------------------------
//
// A workgroup of four waves makes BM = 64 TM rows by BN = 64 TN rows of W; a wave 32 TM by 32 TN of them, with 32 x 32 x 64 instructions (the same rate as
// 16 x 16 x 128, half the operand words).  Two or four stages of 128 columns of both operands lie in LDS, written by direct loads one or three blocks ahead; a wave's operands
// lie in two register sets, one read from LDS while the other is multiplied.  Rows of 128 bytes are eight 16-byte slots; slot s of row r holds columns
// 16 (s ^ swizzle(r)): eight consecutive rows and the rows of one parity of sixteen have different slots of a column, so that reads meet no bank twice.
//
// What bounds it.  Tiles of 256, one workgroup on a compute unit: the matrix cores and their clock, which the card lowers under this load to 1.76 GHz: 4608 x 3072 x
// 12288 148 us, 2350 TFLOP/s, matrix cores 83 % busy; and the tile's ends, when they stand still (first loads 3.5 us, sums to results 4 us, GELU 3.5 us, stores 2 us in
// 8 bits and 8 us in bfloat16, all units at once): 18432 x 12288 x 3072 with GELU into 8 bits 602 us, 2310 TFLOP/s, 63 % busy.  Tiles of 64 and 128: the latency of loads
// for each block, less of it with four stages (where they pay: see deep() in matmul8_plan.h).  Results in float32: widening, 64 conversions a block and wave; 256 x 3072 x 3072
// 12.4 us, 22 % busy.
__device__ __forceinline__ int swizzle(int row) { return (row & 7) ^ (row >> 3 & 1); }

typedef float f32x16 __attribute__((ext_vector_type(16)));

// c += the sums of 64 columns of 32 rows of W and of A, in float32, from operands with their scales
__device__ __forceinline__ void widened32(f32x16& c, const i32x8& w, const i32x8& a, float sw, float sa) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w[2 * i], w[2 * i + 1], sw), widen8(a[2 * i], a[2 * i + 1], sa), c, 0, 0, 0);
}

// An instruction is issued here and not where the compiler would move it, with its sums in accumulation registers
__device__ __forceinline__ void hold(f32x16& c) {
  asm volatile("" : "+a"(c));
}

// Writes 16 bytes of Out, ES bytes an element, from column col on; `n` elements are in range
template <int ES>
__device__ __forceinline__ void store16(void* Out, int64_t at, int n, const u32x4& v) {
  if (n >= 16 / ES) {
    *reinterpret_cast<u32x4_any*>(static_cast<uint8_t*>(Out) + at * ES) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 16 / ES; ++i) {
      if (i >= n) break;
      if (ES == 4) static_cast<uint32_t*>(Out)[at + i] = v[i];
      if (ES == 2) static_cast<uint16_t*>(Out)[at + i] = (uint16_t)(v[i / 2] >> 16 * (i % 2));
    }
  }
}

// Finished rows of a wave, v[i][4 q + e] = Out[row lane % 32][column 32 i + 8 q + 4 (lane / 32) + e], go to memory through its own part of LDS, so that it writes whole
// lines: rows_to_lds puts 32 of them there (inv: of the scale of the lane's row, for 8 bits), rows_to_memory takes them on.
template <int TO, int ES>
__device__ __forceinline__ void rows_to_lds(const float (&v)[TO][16], int lane, float inv, uint8_t* lds) {
  constexpr int RB = TO * 32 * ES, CH = RB / 16;
  static_assert(RB <= 256, "");
  const int r = lane % 32, h = lane / 32;
#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int byte = (32 * i + 8 * q + 4 * h) * ES;
      uint8_t* to = lds + r * RB + (byte / 16 ^ (r & (CH - 1))) * 16 + byte % 16;
      const float* t = v[i] + 4 * q;
      if (ES == 4)
        *reinterpret_cast<f32x4*>(to) = f32x4{t[0], t[1], t[2], t[3]};
      else if (ES == 2)
        *reinterpret_cast<uint2*>(to) = uint2{pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
      else
        *reinterpret_cast<uint32_t*>(to) = pack_e4m3(t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv);
    }
}

template <int TO, int ES>
__device__ __forceinline__ void rows_to_memory(const MatmulArgs& a, int64_t m_first, int col_first, bool inside, int lane, const uint8_t* lds) {
  constexpr int RB = TO * 32 * ES, CH = RB / 16, PER = 64 / CH;
  const int64_t ldo = ES == 1 ? q8_row_bytes(a.N) : a.ldo;
  const int end = ES == 1 ? (int)q8_row_bytes(a.N) : a.N;
  const int row0 = lane / CH, chunk = lane % CH, col = col_first + chunk * 16 / ES;
  u32x4 w[32 / PER];
#pragma unroll
  for (int p = 0; p < 32 / PER; ++p) {
    const int row = p * PER + row0;
    w[p] = *reinterpret_cast<const u32x4*>(lds + row * RB + (chunk ^ (row & (CH - 1))) * 16);
  }
  const int64_t at = (m_first + row0) * ldo + col;
  if (inside) {
#pragma unroll
    for (int p = 0; p < 32 / PER; ++p) store16<ES>(a.Out, at + p * PER * ldo, 16 / ES, w[p]);
  } else {
#pragma unroll
    for (int p = 0; p < 32 / PER; ++p)
      if (m_first + p * PER + row0 < a.M && col < end) store16<ES>(a.Out, at + p * PER * ldo, end - col, w[p]);
  }
}

// A wave's sums c (bias included; gated: c[TO + i] is what c[i] gates) to Out, JP tiles of 32 rows at a time: one wave a SIMD has nothing to hide the ways
// through LDS behind but another tile.  lds: JP * 32 * 32 TO ES bytes a wave; part: 4 * 32 JP floats.  Called by all waves of the workgroup.  inside: the tile lies within Out;
// last: it holds the last column.
template <int TM, int TN, int ACT, int ES, typename Acc>
__device__ __forceinline__ void store_tile(const MatmulArgs& a, Acc& c, int64_t m0, int n0, bool inside, bool last, int wm, int wn, int lane, uint8_t* lds,
                                           float* part) {
  constexpr bool GATED = ACT == SVDC_ACT_SWIGLU;
  constexpr int TO = GATED ? TN / 2 : TN, JP = TM > 1 && ES < 4 ? 2 : 1;
  constexpr bool SHARED = ES == 1 && TO < 4;        // the two waves of the columns share their scales
  const int h = lane / 32, col_first = n0 + wn * 32 * TO;
  uint8_t* mine = lds + (wn * 2 + wm) * (JP * 32 * 32 * TO * ES);
#pragma unroll
  for (int j0 = 0; j0 < TM; j0 += JP) {
#pragma unroll
    for (int j = 0; j < JP; ++j)
#pragma unroll
      for (int i = 0; i < TN; ++i) hold(c[i][j0 + j]);      // these rows after the ones before, not all in registers at once
    const int64_t m_first = m0 + wm * 32 * TM + 32 * j0;
    float v[JP][TO][16], inv[JP];
#pragma unroll
    for (int j = 0; j < JP; ++j)
#pragma unroll
      for (int i = 0; i < TO; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float z = c[i][j0 + j][e];
          v[j][i][e] = ACT == SVDC_ACT_GELU ? gelu(z) : GATED ? silu(z) * c[TO + i][j0 + j][e] : z;
        }
    if (ES == 1) {
      float top[JP];
#pragma unroll
      for (int j = 0; j < JP; ++j) {
        if (!inside) {
#pragma unroll
          for (int i = 0; i < TO; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (col_first + 32 * i + e / 4 * 8 + 4 * h + e % 4 >= a.N) v[j][i][e] = 0.f;
        }
        float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < TO; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) t[e / 4] = fmaxf(t[e / 4], fabsf(v[j][i][e]));
        const float u = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(u), __float_as_uint(u), false, false);   // the two halves of the wave
        top[j] = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
      }
      if (SHARED) {
        __syncthreads();                   // the maxima of the rows before have been read
#pragma unroll
        for (int j = 0; j < JP; ++j) part[((wn * 2 + wm) * JP + j) * 32 + lane % 32] = top[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < JP; ++j) top[j] = fmaxf(top[j], part[(((wn ^ 1) * 2 + wm) * JP + j) * 32 + lane % 32]);
      }
      const int block = (SHARED ? n0 : col_first) / kScaleBlock, blocks = q8_blocks(a.N), row_bytes = q8_scale_row_bytes(a.N);
#pragma unroll
      for (int j = 0; j < JP; ++j) {
        const int byte = scale_byte(top[j]);
        inv[j] = inverse_scale(byte);
        const int64_t m = m_first + 32 * j + lane;
        if (lane < 32 && m < a.M) {
          uint8_t* to = a.Os + m * row_bytes;
          if (block < blocks && !(SHARED && wn)) to[block] = (uint8_t)byte;
          if (last && wn)
            for (int b = blocks; b < row_bytes; ++b) to[b] = 127;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < JP; ++j) rows_to_lds<TO, ES>(v[j], lane, ES == 1 ? inv[j] : 1.f, mine + j * (32 * 32 * TO * ES));
    asm volatile("" ::: "memory");         // a wave's LDS operations are carried out in order
#pragma unroll
    for (int j = 0; j < JP; ++j) rows_to_memory<TO, ES>(a, m_first + 32 * j, col_first, inside, lane, mine + j * (32 * 32 * TO * ES));
    asm volatile("" ::: "memory");
  }
}

// Values loaded before the last wait for LDS' loads: known here to be there, so that no use of them waits for loads issued since
template <int N>
__device__ __forceinline__ void arrived(int (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

template <int TM, int TN>
struct TileStage {
  __align__(1024) uint8_t b[64 * (TM + TN) * 128];
};

// The tile of workgroup `id`.  Workgroups go round the eight dies in turn; each die gets a run of tiles of its own, in groups of eight rows of tiles, column
// by column, so that the 32 at work on a die at a time share 8 + 4 operands of tiles in its cache.
__device__ __forceinline__ void tile_at(int id, int row_tiles, int column_tiles, int& row, int& column) {
  const int tiles = row_tiles * column_tiles, each = tiles / 8, more = tiles % 8, die = id % 8;
  const int t = die * each + min(die, more) + id / 8;
  const int group = t / (8 * column_tiles), first = group * 8, high = min(8, row_tiles - first), at = t - group * 8 * column_tiles;
  row = uniform(first + at % high);
  column = uniform(at / high);
}

template <int TM, int TN, int ACT, int ES, bool EXACT, int STAGES>
__device__ __forceinline__ void tile_of_product(MatmulArgs a) {
  constexpr bool GATED = ACT == SVDC_ACT_SWIGLU;
  constexpr int BM = 64 * TM, BN = 64 * TN, LOADS = (BM + BN) / 32;
  // A half block is SLOTS instructions long.  Once the second half has been read, at READ, its block's stage is loaded anew: FIRST loads in the rest of the first
  // half, the others in the first LATE slots of the second.  A load takes 16 cycles of its unit, four waves' 64: more than one a slot of 64 cycles
  // hold up the wave, and with it its products (16 loads in 7 slots: 2475 TFLOP/s at 8192 x 8192 x 8192, so dealt out 2617).
  constexpr int SLOTS = TM * TN, READ = SLOTS == 16 ? 10 : SLOTS - 1, FIRST = SLOTS == 16 ? 6 : LOADS / 2, LATE = SLOTS == 16 ? 10 : SLOTS;
  __shared__ TileStage<TM, TN> stage0;
  __shared__ TileStage<TM, TN> stage1;
  __shared__ TileStage<TM, TN> stage2;           // not there with two stages
  __shared__ TileStage<TM, TN> stage3;
  uint8_t* const stages[4] = {stage0.b, stage1.b, STAGES == 4 ? stage2.b : stage0.b, STAGES == 4 ? stage3.b : stage1.b};
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int wm = wave & 1, wn = wave >> 1;
  const int64_t Kp = q8_row_bytes(a.K);
  const int ss = uniform(q8_scale_row_bytes(a.K));
  const int all = q8_blocks(a.K), each = blocks_of_part(all, a.splits), skip = uniform(blockIdx.y * each);      // this part's blocks of columns of A and W
  const int blocks = uniform(min(each, all - skip));
  a.A += (int64_t)skip * 128;
  a.W += (int64_t)skip * 128;
  a.As += skip;
  a.Ws += skip;
  if (ES == 4) a.Out = static_cast<float*>(a.Out) + blockIdx.y * a.M * a.ldo;
  const int columns = GATED ? BN / 2 : BN;                  // of Out
  const int column_tiles = (a.N + columns - 1) / columns;
  const int row_tiles = (int)((a.M + BM - 1) / BM);
  int row_tile, column_tile;
  tile_at(blockIdx.x, row_tiles, column_tiles, row_tile, column_tile);
  const int64_t m0 = (int64_t)row_tile * BM;
  const int n0 = column_tile * columns;

  // row of W behind row i of the tile; rows beyond the last are read as the last one, and what they give is not stored.  Gated: a wave's first 16 TN
  // rows are gates, its others what they multiply
  const auto w_row = [&](int i) {
    if (!GATED) return (int64_t)min(n0 + i, a.N - 1);
    const int w = i / (32 * TN), j = i % (32 * TN), up = j / (16 * TN);
    return (int64_t)min(n0 + w * 16 * TN + j % (16 * TN), a.N - 1) + (up ? a.N : 0);
  };
  const auto a_row = [&](int i) { return min(m0 + i, a.M - 1); };

  // This wave's pieces of 8 rows of a stage: bounds-checked loads from A, the gates and what they multiply, each from the tile's first row on
  const int a_bytes = uniform((int)(min<int64_t>(BM, a.M - m0) * Kp - skip * 128)), w_bytes = uniform((int)(min(columns, a.N - n0) * Kp - skip * 128));
  const int64_t u_first = (GATED ? (int64_t)a.N : 0) + n0;
  const auto A1 = bounded(a.A + m0 * Kp, a_bytes), W1 = bounded(a.W + n0 * Kp, w_bytes), U1 = bounded(a.W + u_first * Kp, w_bytes);
  const auto is_up = [](int j) { return GATED && (j * 32 - BM) % (32 * TN) >= 16 * TN; };
  uint32_t from[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int i = (j * 4 + wave) * 8 + lane / 8, slot = (lane % 8) ^ swizzle(i);
    from[j] = (uint32_t)((j * 32 < BM ? a_row(i) - m0 : w_row(i - BM) - n0 - (is_up(j) ? a.N : 0)) * Kp + slot * 16);
  }
  const auto load = [&](int j, int b, uint8_t* stage, __amdgpu_buffer_rsrc_t A, __amdgpu_buffer_rsrc_t W, __amdgpu_buffer_rsrc_t U) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(j * 32 < BM ? A : is_up(j) ? U : W, stage + (j * 4 + wave) * 1024, 16, from[j], uniform(b * 128), 0, 0);
  };

  const int r = lane % 32, h = lane / 32;
  const int f = swizzle(r);
  const int slot[4] = {((2 * h) ^ f) * 16, ((2 * h + 1) ^ f) * 16, ((4 + 2 * h) ^ f) * 16, ((5 + 2 * h) ^ f) * 16};
  const int a_base = (wm * 32 * TM + r) * 128, w_base = (BM + wn * 32 * TN + r) * 128;

  // scales of four blocks at a time, those of the current block in the lowest byte
  const auto As = bounded(a.As + m0 * ss, uniform((int)min<int64_t>(BM, a.M - m0) * ss - skip)), Ws = bounded(a.Ws, uniform(q8_blocks(GATED ? 2 * a.N : a.N) * ss - skip));
  uint32_t scale_row[TN + TM];
#pragma unroll
  for (int t = 0; t < TN; ++t) scale_row[t] = (uint32_t)(w_row(wn * 32 * TN + t * 32 + r) / kScaleBlock * ss);
#pragma unroll
  for (int t = 0; t < TM; ++t) scale_row[TN + t] = (uint32_t)((a_row(wm * 32 * TM + t * 32 + r) - m0) * ss);
  int sc[TN + TM], next_sc[TN + TM];
  const auto load_scales = [&](int b, int* s) {
#pragma unroll
    for (int t = 0; t < TN + TM; ++t) s[t] = __builtin_amdgcn_raw_buffer_load_b32(t < TN ? Ws : As, scale_row[t], b, 0);
  };

#pragma unroll
  for (int s = 0; s < STAGES; ++s)
    if (s < blocks) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) load(j, s, stages[s], A1, W1, U1);
    }
  // the sums start at the bias: bounds-checked loads, zero beyond the last column and without one
  const uint8_t* const bias_bytes = reinterpret_cast<const uint8_t*>(a.bias);
  const auto bias_z = bounded(bias_bytes, uniform(a.bias ? a.N * 4 : 0)),
             bias_u = bounded(bias_bytes + (GATED ? (int64_t)a.N * 4 : 0), uniform(a.bias ? a.N * 4 : 0));
  f32x16 c[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    f32x16 bias;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int col = n0 + wn * 32 * (GATED ? TN / 2 : TN) + 32 * (GATED ? i % (TN / 2) : i) + e / 4 * 8 + 4 * h + e % 4;
      bias[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(GATED && i >= TN / 2 ? bias_u : bias_z, col * 4, 0, 0));
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) c[i][j] = bias;
  }
  i32x8 x[2][TN + TM];

  load_scales(0, sc);
  // Piece p of 2 (TN + TM) of the operands of a half block, in the order in which they are multiplied
  constexpr int PIECES = 2 * (TN + TM), AT_ONCE = PIECES > 2 * SLOTS ? (PIECES + SLOTS - 1) / SLOTS : 2;
  const auto operand_of = [](int p) { return p / 2 == 0 ? 0 : p / 2 <= TM ? TN + p / 2 - 1 : p / 2 - TM; };
  const auto read = [&](i32x8* y, const uint8_t* stage, int p, int half) {
    const int t = operand_of(p);
    const uint8_t* row = stage + (t < TN ? w_base + t * 4096 : a_base + (t - TN) * 4096);
    const u32x4 v = *reinterpret_cast<const u32x4*>(row + slot[2 * half + p % 2]);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[t][4 * (p % 2) + e] = (int)v[e];
  };
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  arrived(sc);
  __syncthreads();
#pragma unroll
  for (int p = 0; p < PIECES; ++p) read(x[0], stages[0], p, 0);

  int scale_bits = 255;                  // 0 for a block whose scales leave the range of bfloat16: it enters with scales of 0 here, and with its own behind the others
  bool left_out = false;                 // one answer for the wave
  const auto multiply = [&](const i32x8* y, auto&& between) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        between(i * TM + j);
        if (EXACT)
          widened32(c[i][j], y[i], y[TN + j], scale_of(sc[i] & scale_bits), scale_of(sc[TN + j] & scale_bits));
        else
          c[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y[i], y[TN + j], c[i][j], 0, 0, 0, sc[i], 0, sc[TN + j]);
        hold(c[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // Block b lies in `now` with its first half in x[0].  Once all waves have read its second half, block b + STAGES is loaded there; beyond the last one the
  // loads are out of bounds and fetch nothing.
  const auto block = [&](int b, uint8_t* now, uint8_t* then) {
    if (EXACT) {
      bool good = true;
#pragma unroll
      for (int t = 0; t < TN + TM; ++t) good = good && in_range(sc[t] & 255);
      scale_bits = __builtin_amdgcn_ballot_w64(!good) == 0 ? 255 : 0;
      left_out = left_out || scale_bits == 0;
    }
    const int more = b + STAGES < blocks ? -1 : 0;
    const auto A2 = bounded(a.A + m0 * Kp, a_bytes & more), W2 = bounded(a.W + n0 * Kp, w_bytes & more), U2 = bounded(a.W + u_first * Kp, w_bytes & more);
    multiply(x[0], [&](int t) {
#pragma unroll
      for (int p = t * AT_ONCE; p < (t + 1) * AT_ONCE && p < PIECES; ++p) read(x[1], now, p, 1);
      if (t == READ) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t >= READ) {
#pragma unroll
        for (int j = (t - READ) * FIRST / (SLOTS - READ); j < (t - READ + 1) * FIRST / (SLOTS - READ); ++j) load(j, b + STAGES, now, A2, W2, U2);
      }
    });
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((STAGES - 2) * LOADS + FIRST) : "memory");
    multiply(x[1], [&](int t) {
#pragma unroll
      for (int p = t * PIECES / SLOTS; p < (t + 1) * PIECES / SLOTS; ++p) read(x[0], then, p, 0);
      if (t < LATE) {
#pragma unroll
        for (int j = FIRST + t * (LOADS - FIRST) / LATE; j < FIRST + (t + 1) * (LOADS - FIRST) / LATE; ++j) load(j, b + STAGES, now, A2, W2, U2);
      }
    });
#pragma unroll
    for (int t = 0; t < TN + TM; ++t) sc[t] = (int)((uint32_t)sc[t] >> 8);
  };
  int b = 0;
  for (; b + 3 < blocks; b += 4) {
    load_scales(min(b + 4, ss - skip - 4), next_sc);
#pragma unroll
    for (int d = 0; d < 4; ++d) block(b + d, stages[d], stages[(d + 1) % 4]);
    arrived(next_sc);
#pragma unroll
    for (int t = 0; t < TN + TM; ++t) sc[t] = next_sc[t];
  }
  if (b < blocks) {
    block(b, stages[0], stages[1]);
    if (b + 1 < blocks) {
      block(b + 1, stages[1], stages[2]);
      if (b + 2 < blocks) block(b + 2, stages[2], stages[3]);
    }
  }
  if constexpr (EXACT) {
    if (left_out) {
      // the blocks left out, each without scales and then times them, straight from memory: rare, so short rather than fast
      const auto edge = [&](int i) { return kScaleBlock - (a.N + n0 + wn * 16 * TN + 32 * (i - TN / 2)) % kScaleBlock; };   // as in the few rows' kernel
      const auto operand = [&](const uint8_t* row) {
        const u32x4 lo = reinterpret_cast<const u32x4*>(row)[0], hi = reinterpret_cast<const u32x4*>(row)[1];
        return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
      };
      for (int d = 0; d < blocks; ++d) {
        int s[TN + TM];
        bool good = true;
#pragma unroll
        for (int t = 0; t < TN + TM; ++t) {
          s[t] = t < TN ? a.Ws[scale_row[t] + d] : a.As[m0 * ss + scale_row[t] + d];
          good = good && in_range(s[t]);
        }
        if (__builtin_amdgcn_ballot_w64(!good) == 0) continue;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            f32x16 t = {};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int64_t col = d * 128 + half * 64 + h * 32;
              widened32(t, operand(a.W + w_row(wn * 32 * TN + i * 32 + r) * Kp + col), operand(a.A + a_row(wm * 32 * TM + j * 32 + r) * Kp + col), 1.f, 1.f);
            }
            add_scaled(c[i][j], t, GATED && i >= TN / 2 ? Exponents(s[i], s[TN + j], edge(i), 31) : Exponents(s[i], s[TN + j]),
                       [&](int e) { return e / 4 * 8 + 4 * h + e % 4; });
            hold(c[i][j]);
            __builtin_amdgcn_sched_barrier(0);
          }
      }
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0) vmcnt(0)\n\ts_barrier" ::: "memory");
  const bool inside = m0 + BM <= a.M && n0 + columns <= a.N;
  store_tile<TM, TN, ACT, ES>(a, c, m0, n0, inside, column_tile == column_tiles - 1, wm, wn, lane, stage0.b, reinterpret_cast<float*>(stage1.b));
}

// ACT: svdc_act;  ES: bytes of an element of Out;  EXACT: float32 sums;  STAGES: blocks in LDS, 2 or 4.  Part blockIdx.y of a.splits of the columns of A and W
template <int TM, int TN, int ACT, int ES, bool EXACT, int STAGES>
__global__ __launch_bounds__(256) void matmul8_tile_kernel(MatmulArgs a) {
#ifdef __HIP_DEVICE_COMPILE__          // buffer descriptors and accumulation registers mean nothing to the host's pass
  tile_of_product<TM, TN, ACT, ES, EXACT, STAGES>(a);
#endif
}

// The sums of `splits` parts of the columns of A and W, [splits][M][wide] float32, to Out: 16 lanes a block of 128 columns of a row, parts in order.
__global__ __launch_bounds__(256) void matmul8_finish_kernel(MatmulArgs a, const float* parts) {
  const bool gated = a.act == SVDC_ACT_SWIGLU;
  const int wide = gated ? 2 * a.N : a.N, out_blocks = q8_blocks(a.N);
  const int64_t units = a.M * out_blocks, part = a.M * wide;
  const auto add8 = [&](const float* from, int n, float (&v)[8]) {
    for (int s = 0; s < a.splits; ++s, from += part) {
      if (n >= 8) {
        const u32x4_any lo = reinterpret_cast<const u32x4_any*>(from)[0], hi = reinterpret_cast<const u32x4_any*>(from)[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __uint_as_float(lo[e]), v[4 + e] += __uint_as_float(hi[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) v[e] += from[e];
      }
    }
  };
  // whole groups of four units, as the lanes of a wave work on the maxima together
  for (int64_t unit = (int64_t)blockIdx.x * 16 + threadIdx.x / 16; unit < (units + 3) / 4 * 4; unit += (int64_t)gridDim.x * 16) {
    const bool has = unit < units;
    const int64_t row = has ? unit / out_blocks : 0;
    const int block = has ? (int)(unit - row * out_blocks) : 0, col = block * kScaleBlock + threadIdx.x % 16 * 8, n = has ? a.N - col : 0;
    float v[8] = {}, u[8] = {};
    add8(parts + row * wide + col, n, v);
    if (gated) add8(parts + row * wide + a.N + col, n, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = finished(a, col + e, v[e], u[e]);
    if (a.dtype == SVDC_E4M3) {
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
      const int byte = scale_byte(row16_max(top));
      const float inv = inverse_scale(byte);
      if (!has) continue;
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.Out) + row * q8_row_bytes(a.N) + col) =
          uint2{pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), pack_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
      uint8_t* os = a.Os + row * q8_scale_row_bytes(a.N);
      if (threadIdx.x % 16 == 0) {
        os[block] = (uint8_t)byte;
        if (block == out_blocks - 1)
          for (int s = out_blocks; s < q8_scale_row_bytes(a.N); ++s) os[s] = 127;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) {
          if (a.dtype == SVDC_F32)
            static_cast<float*>(a.Out)[row * a.ldo + col + e] = v[e];
          else
            static_cast<bf16_t*>(a.Out)[row * a.ldo + col + e] = (bf16_t)v[e];
        }
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------------------------

template <int TM, int TN, int ACT, int ES, bool EXACT>
void launch_tiles(const MatmulArgs& a, int stages, hipStream_t st) {
  const int columns = ACT == SVDC_ACT_SWIGLU ? 32 * TN : 64 * TN;
  const int64_t tiles = (a.M + 64 * TM - 1) / (64 * TM) * ((a.N + columns - 1) / columns);
  const dim3 grid((unsigned)tiles, a.splits);
  if constexpr (can_be_deep(TM, TN, EXACT))
    if (stages == 4) {
      matmul8_tile_kernel<TM, TN, ACT, ES, EXACT, 4><<<grid, 256, 0, st>>>(a);
      return;
    }
  matmul8_tile_kernel<TM, TN, ACT, ES, EXACT, 2><<<grid, 256, 0, st>>>(a);
}

// Tiles of 64 T rows by 64 tile_width() rows of W
template <int T, int ES>
void launch_tiles(const MatmulArgs& a, int stages, hipStream_t st) {
  constexpr int PLAIN = tile_width(64 * T, false, ES == 1), GATES = tile_width(64 * T, true, ES == 1);
  if (a.act == SVDC_ACT_SWIGLU)
    launch_tiles<T, GATES, SVDC_ACT_SWIGLU, ES, ES == 4>(a, stages, st);
  else if (a.act == SVDC_ACT_GELU)
    launch_tiles<T, PLAIN, SVDC_ACT_GELU, ES, ES == 4>(a, stages, st);
  else
    launch_tiles<T, PLAIN, SVDC_ACT_NONE, ES, ES == 4>(a, stages, st);
}

template <int T>
void launch_tiles(const MatmulArgs& a, int stages, hipStream_t st) {
  if (a.dtype == SVDC_F32)
    launch_tiles<T, 4>(a, stages, st);
  else if (a.dtype == SVDC_BF16)
    launch_tiles<T, 2>(a, stages, st);
  else
    launch_tiles<T, 1>(a, stages, st);
}

template <int TM, int TN, bool EXACT, bool GATED, bool EIGHT>
void launch_shared(const MatmulArgs& a, hipStream_t st) {
  const int64_t tiles = (a.M + 16 * TM - 1) / (16 * TM) * ((a.N + 16 * TN - 1) / (16 * TN));
  matmul8_shared_kernel<TM, TN, EXACT, GATED, EIGHT><<<(unsigned)tiles, kShareWaves * kWave, 0, st>>>(a);
}

template <int TM, bool EXACT>
void launch_shared(const MatmulArgs& a, int columns, hipStream_t st) {
  const bool gated = a.act == SVDC_ACT_SWIGLU;
  if (columns == 16)
    gated ? launch_shared<TM, 1, EXACT, true, false>(a, st) : launch_shared<TM, 1, EXACT, false, false>(a, st);
  else if (columns == 32)
    gated ? launch_shared<TM, 2, EXACT, true, false>(a, st) : launch_shared<TM, 2, EXACT, false, false>(a, st);
  else
    launch_shared<TM, 4, EXACT, false, false>(a, st);
}

void launch_shared(const MatmulArgs& a, const MatmulPlan& plan, hipStream_t st) {
  if (a.dtype == SVDC_F32)
    plan.rows == 16 ? launch_shared<1, true>(a, plan.columns, st) : launch_shared<2, true>(a, plan.columns, st);
  else if (a.dtype == SVDC_BF16)
    plan.rows == 16 ? launch_shared<1, false>(a, plan.columns, st) : launch_shared<2, false>(a, plan.columns, st);
  else
    launch_shared<1, 8, false, false, true>(a, st);
}

int32_t launch_planned(const MatmulPlan& plan, MatmulArgs a, void* workspace, hipStream_t st) {
  a.splits = plan.splits;
  if (plan.rows <= 32) {
    launch_shared(a, plan, st);
  } else if (plan.splits == 1) {
    const bool eight = a.dtype == SVDC_E4M3;
    const int64_t most = rows_of_launch(plan, a.N, a.act == SVDC_ACT_SWIGLU, eight);
    const int64_t out_row = eight ? q8_row_bytes(a.N) : a.ldo * (a.dtype == SVDC_F32 ? 4 : 2);
    for (int64_t left = a.M; left > 0; left -= most) {
      a.M = std::min(left, most);
      if (plan.rows == 256)
        a.dtype == SVDC_BF16 ? launch_tiles<4, 2>(a, plan.stages, st) : launch_tiles<4, 1>(a, plan.stages, st);
      else
        plan.rows == 64 ? launch_tiles<1>(a, plan.stages, st) : launch_tiles<2>(a, plan.stages, st);
      if (hipGetLastError() != hipSuccess) return SVDC_E_HIP;
      a.A += most * q8_row_bytes(a.K);
      a.As += most * q8_scale_row_bytes(a.K);
      a.Out = static_cast<uint8_t*>(a.Out) + most * out_row;
      if (eight) a.Os += most * q8_scale_row_bytes(a.N);
    }
    return SVDC_OK;
  } else {
    MatmulArgs part = a;                       // plain sums of all of W's rows
    part.N = a.act == SVDC_ACT_SWIGLU ? 2 * a.N : a.N;
    part.act = SVDC_ACT_NONE;
    part.bias = nullptr;
    part.Out = workspace;
    part.ldo = part.N;
    a.dtype == SVDC_F32 ? launch_tiles<2, 2, SVDC_ACT_NONE, 4, true>(part, plan.stages, st) : launch_tiles<2, 2, SVDC_ACT_NONE, 4, false>(part, plan.stages, st);
    if (hipGetLastError() != hipSuccess) return SVDC_E_HIP;
    const int64_t groups = (a.M * q8_blocks(a.N) + 15) / 16;
    matmul8_finish_kernel<<<(unsigned)std::min<int64_t>(groups, 1 << 20), 256, 0, st>>>(a, static_cast<const float*>(workspace));
  }
  return launch_status();
}

}  // namespace

size_t matmul8_workspace_bytes(const svdc_matmul8& p) {
  const MatmulPlan plan = matmul8_plan(p, num_compute_units());
  return plan.splits <= 1 ? 0 : (size_t)plan.splits * p.M * wide_of(p) * sizeof(float);
}

int32_t launch_matmul8(const svdc_matmul8& p, const void* A, const void* As, const void* W, const void* Ws, const float* bias, void* Out, void* Os,
                       void* workspace, hipStream_t st) {
  const MatmulArgs a{static_cast<const uint8_t*>(A), static_cast<const uint8_t*>(As), static_cast<const uint8_t*>(W), static_cast<const uint8_t*>(Ws),
                     bias, Out, static_cast<uint8_t*>(Os), p.M, p.ldo, p.N, p.K, p.dtype, p.act, 1};
  return launch_planned(matmul8_plan(p, num_compute_units()), a, workspace, st);
}

}  // namespace svdc
