// Product of matrices in 8 bits with a power-of-two scale for each 128 columns (svdcache_matmul8).
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 columns of 16 rows of W and of 16 rows of A, that is one block of scales of each, and applies the
// scales itself: the sum over blocks is a plain chain of these instructions.  Operand layout per lane l (r = l % 16, g = l / 16):
//     W: 32 bytes of row r,  A: 32 bytes of row r,  result: 4 float32 = z[n = 4 g .. 4 g + 3][m = r]
// The 128 columns may be dealt out to the lanes of a row in any order as long as W and A use the same one; each lane hands over the scale of its own
// row, and as all four lanes of a row lie in one block of scales the order does not matter to the scales either.
//
// The instruction adds the products of 8 consecutive bytes with 13 bits below the largest of them (measured: smaller bits are cut off), then those sums in
// float32.  That is about 4e-5 of a result: nothing beside the rounding of a result to bfloat16 or e4m3, but not float32.  Results in float32 are made with
// bfloat16 instructions, at half the rate: e4m3 values times powers of two are bfloat16 values exactly, and those products are summed with 24 bits.
#include <algorithm>
#include <type_traits>

#include "eight_bit.h"
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
  int N, K, dtype, act;
};

__device__ __forceinline__ f32x4 mfma8(const i32x8& w, const i32x8& a, const f32x4& c, int sw, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 0, 0, 0, sw, 0, sa);
}

__device__ __forceinline__ i32x8 load32(const uint8_t* p) {
  const u32x4 lo = reinterpret_cast<const u32x4*>(p)[0], hi = reinterpret_cast<const u32x4*>(p)[1];
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// 8 e4m3 values times 2^(byte - 127) as bfloat16, exactly
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, int byte) {
  const float s = __uint_as_float((uint32_t)byte << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 128 columns of 16 rows of W and of A; EXACT: with float32 sums
template <bool EXACT>
__device__ __forceinline__ f32x4 product(const i32x8& w, const i32x8& a, f32x4 c, int sw, int sa) {
  if (!EXACT) return mfma8(w, a, c, sw, sa);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[2 * i], w[2 * i + 1], sw), widen8(a[2 * i], a[2 * i + 1], sa), c, 0, 0, 0);
  return c;
}

// x / (1 + exp(-t)), with the hardware's power of two and reciprocal (one step of the last place each): half the instructions of a division
__device__ __forceinline__ float times_sigmoid(float x, float t_log2e) {
  return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-t_log2e));
}
__device__ __forceinline__ float silu(float x) { return times_sigmoid(x, 1.4426950408889634f * x); }
// with t = 2 sqrt(2 / pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu(float x) { return times_sigmoid(x, x * __builtin_fmaf(0.10294324f, x * x, 2.3022082f)); }

// 8 waves: 128 columns of Out for 16 rows, a wave 16 columns of them (and the 16 they gate).
template <bool EXACT>
__global__ __launch_bounds__(512) void matmul8_kernel(MatmulArgs a) {
  __shared__ float part[8][16];
  const int column_tiles = q8_blocks(a.N);
  const int64_t tiles = (a.M + 15) / 16 * column_tiles;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
  const int64_t row_tile = tile / column_tiles;
  const int column_tile = (int)(tile - row_tile * column_tiles);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
  const int64_t Kp = q8_row_bytes(a.K);
  const int blocks = q8_blocks(a.K), ss = q8_scale_row_bytes(a.K);
  const int n0 = column_tile * 128 + wave * 16;
  const int64_t m0 = row_tile * 16;
  const int gated = a.act == SVDC_ACT_SWIGLU;
  // rows beyond the last are read as the last one; what they give is not stored
  const int n = min(n0 + r, a.N - 1);
  const int64_t m = min(m0 + r, a.M - 1);
  const uint8_t* A = a.A + m * Kp + 32 * g;
  const uint8_t* As = a.As + m * ss;
  const uint8_t* W = a.W + n * Kp + 32 * g;
  const uint8_t* Ws = a.Ws + (int64_t)(n / kScaleBlock) * ss;
  const int nu = a.N + n;
  const uint8_t* U = a.W + nu * Kp + 32 * g;
  const uint8_t* Us = a.Ws + (int64_t)(nu / kScaleBlock) * ss;
  f32x4 z = {0.f, 0.f, 0.f, 0.f}, u = z;
  for (int b = 0; b < blocks; ++b) {
    const i32x8 x = load32(A + b * 128);
    z = product<EXACT>(load32(W + b * 128), x, z, Ws[b], As[b]);
    if (gated) u = product<EXACT>(load32(U + b * 128), x, u, Us[b], As[b]);
  }
  float v[4];
  const int nt = n0 + 4 * g;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool in = nt + i < a.N;
    v[i] = z[i] + (a.bias && in ? a.bias[nt + i] : 0.f);
    if (gated) v[i] = silu(v[i]) * (u[i] + (a.bias && in ? a.bias[a.N + nt + i] : 0.f));
    if (a.act == SVDC_ACT_GELU) v[i] = gelu(v[i]);
    if (!in) v[i] = 0.f;
  }
  const int64_t mo = m0 + r;
  if (a.dtype == SVDC_E4M3) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) t = fmaxf(t, fabsf(v[i]));
    t = fmaxf(t, __shfl_xor(t, 16));
    t = fmaxf(t, __shfl_xor(t, 32));
    __syncthreads();                     // the maxima of the tile before have been read
    if (g == 0) part[wave][r] = t;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) t = fmaxf(t, part[w][r]);
    const int byte = scale_byte(t);
    const float inv = inverse_scale(byte);
    if (mo < a.M) {
      *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.Out) + mo * q8_row_bytes(a.N) + nt) =
          pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      uint8_t* os = a.Os + mo * q8_scale_row_bytes(a.N);
      if (wave == 0 && g == 0) os[column_tile] = (uint8_t)byte;
      if (wave == 1 && g == 0 && column_tile == column_tiles - 1)
        for (int s = column_tiles; s < q8_scale_row_bytes(a.N); ++s) os[s] = 127;
    }
  } else if (mo < a.M) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (nt + i < a.N) {
        if (a.dtype == SVDC_F32)
          static_cast<float*>(a.Out)[mo * a.ldo + nt + i] = v[i];
        else
          static_cast<bf16_t*>(a.Out)[mo * a.ldo + nt + i] = (bf16_t)v[i];
      }
  }
  }
}

// ---- tiles ----------------------------------------------------------------------------------------------------------
//
// A workgroup of four waves makes BM = 64 TM rows by BN = 64 TN rows of W; a wave 32 TM by 32 TN of them, with 32 x 32 x 64 instructions (the same rate as
// 16 x 16 x 128, half the operand words).  Two stages of 128 columns of both operands lie in LDS, written by direct loads one block ahead; a wave's operands
// lie in two register sets, one read from LDS while the other is multiplied.  Rows of 128 bytes are eight 16-byte slots; slot s of row r holds columns
// 16 (s ^ swizzle(r)): eight consecutive rows and the rows of one parity of sixteen have different slots of a column, so that reads meet no bank twice.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }   // a value that all lanes hold, as a scalar
__device__ __forceinline__ int swizzle(int row) { return (row & 7) ^ (row >> 3 & 1); }

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <bool EXACT>
__device__ __forceinline__ void product32(f32x16& c, const i32x8& w, const i32x8& a, int sw, int sa) {
  if (!EXACT) {
    c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, c, 0, 0, 0, sw, 0, sa);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w[2 * i], w[2 * i + 1], sw & 255), widen8(a[2 * i], a[2 * i + 1], sa & 255), c, 0, 0, 0);
  }
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

// A wave's finished 32 rows v[i][4 q + e] = Out[row lane % 32][column 32 i + 8 q + 4 (lane / 32) + e] go to memory through its own part of LDS, so that it writes
// whole lines.  inv: of the scale of the lane's row, for 8 bits.
template <int TO, int ES>
__device__ __forceinline__ void store_rows(const MatmulArgs& a, const float (&v)[TO][16], int64_t m_first, int col_first, int lane, float inv, uint8_t* lds) {
  constexpr int RB = TO * 32 * ES, CH = RB / 16, PER = 64 / CH;
  static_assert(RB <= 256, "");
  const int r = lane % 32, h = lane / 32;
  const int64_t ldo = ES == 1 ? q8_row_bytes(a.N) : a.ldo;
  const int end = ES == 1 ? (int)q8_row_bytes(a.N) : a.N;
#pragma unroll
  for (int i = 0; i < TO; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int byte = (32 * i + 8 * q + 4 * h) * ES;
      uint8_t* to = lds + r * RB + (byte / 16 ^ (r & (CH - 1))) * 16 + byte % 16;
      const float *t = v[i] + 4 * q;
      if (ES == 4)
        *reinterpret_cast<f32x4*>(to) = f32x4{t[0], t[1], t[2], t[3]};
      else if (ES == 2)
        *reinterpret_cast<uint2*>(to) = uint2{pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
      else
        *reinterpret_cast<uint32_t*>(to) = pack_e4m3(t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv);
    }
  asm volatile("" ::: "memory");           // a wave's LDS operations are carried out in order
#pragma unroll
  for (int p = 0; p < 32 / PER; ++p) {
    const int row = p * PER + lane / CH, chunk = lane % CH;
    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + row * RB + (chunk ^ (row & (CH - 1))) * 16);
    const int col = col_first + chunk * 16 / ES;
    if (m_first + row < a.M && col < end) store16<ES>(a.Out, (m_first + row) * ldo + col, end - col, w);
  }
  asm volatile("" ::: "memory");
}

// A wave's sums c (bias included; gated: c[TO + i] is what c[i] gates) to Out.  lds: 32 * 32 TO * 4 bytes a wave at most; part: 4 * 32 floats.  Called by all
// waves of the workgroup.  edge: the tile reaches beyond column N.
template <int TM, int TN, int ACT, int ES, typename Acc>
__device__ __forceinline__ void store_tile(const MatmulArgs& a, Acc& c, int64_t m0, int n0, bool edge, int wm, int wn, int lane, uint8_t* lds,
                                           float* part) {
  constexpr bool GATED = ACT == SVDC_ACT_SWIGLU;
  constexpr int TO = GATED ? TN / 2 : TN;
  constexpr bool SHARED = ES == 1 && TO < 4;        // the two waves of the columns share their scales
  const int h = lane / 32, col_first = n0 + wn * 32 * TO;
  uint8_t* mine = lds + (wn * 2 + wm) * (32 * 32 * TO * ES);
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int64_t m_first = m0 + wm * 32 * TM + 32 * j;
#pragma unroll
    for (int i = 0; i < TN; ++i) hold(c[i][j]);      // 32 rows after the other, not all in registers at once
    float v[TO][16];
#pragma unroll
    for (int i = 0; i < TO; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float z = c[i][j][e];
        v[i][e] = ACT == SVDC_ACT_GELU ? gelu(z) : GATED ? silu(z) * c[TO + i][j][e] : z;
      }
    float inv = 1.f;
    if (ES == 1) {
      if (edge) {
#pragma unroll
        for (int i = 0; i < TO; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (col_first + 32 * i + e / 4 * 8 + 4 * h + e % 4 >= a.N) v[i][e] = 0.f;
      }
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < TO; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(v[i][e]));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (SHARED) {
        __syncthreads();                   // the maxima of the rows before have been read
        part[(wn * 2 + wm) * 32 + lane % 32] = top;
        __syncthreads();
        top = fmaxf(top, part[((wn ^ 1) * 2 + wm) * 32 + lane % 32]);
      }
      const int byte = scale_byte(top);
      inv = inverse_scale(byte);
      const int block = (SHARED ? n0 : col_first) / kScaleBlock, blocks = q8_blocks(a.N), row_bytes = q8_scale_row_bytes(a.N);
      if (lane < 32 && m_first + lane < a.M) {
        uint8_t* to = a.Os + (m_first + lane) * row_bytes;
        if (block < blocks && !(SHARED && wn)) to[block] = (uint8_t)byte;
        if (edge && wn)
          for (int b = blocks; b < row_bytes; ++b) to[b] = 127;
      }
    }
    store_rows<TO, ES>(a, v, m_first, col_first, lane, inv, mine);
  }
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

template <int TM, int TN, int ACT, int ES>
__device__ __forceinline__ void tile_of_product(const MatmulArgs& a) {
  constexpr bool EXACT = ES == 4, GATED = ACT == SVDC_ACT_SWIGLU;
  constexpr int BM = 64 * TM, BN = 64 * TN, LOADS = (BM + BN) / 32, READ = TM * TN > 4 ? TN + TM + 1 : TN * TM - 1;
  __shared__ TileStage<TM, TN> stage0;
  __shared__ TileStage<TM, TN> stage1;
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int wm = wave & 1, wn = wave >> 1;
  constexpr bool gated = GATED;
  const int64_t Kp = q8_row_bytes(a.K);
  const int blocks = uniform(q8_blocks(a.K)), ss = uniform(q8_scale_row_bytes(a.K));
  const int columns = gated ? BN / 2 : BN;                  // of Out
  const int column_tiles = (a.N + columns - 1) / columns;
  const int row_tiles = (int)((a.M + BM - 1) / BM);
  int row_tile, column_tile;
  tile_at(blockIdx.x, row_tiles, column_tiles, row_tile, column_tile);
  const int64_t m0 = (int64_t)row_tile * BM;
  const int n0 = column_tile * columns;

  // row of W behind row i of the tile; rows beyond the last are read as the last one, and what they give is not stored.  Gated: a wave's first 16 TN
  // rows are gates, its others what they multiply
  const auto w_row = [&](int i) {
    if (!gated) return (int64_t)min(n0 + i, a.N - 1);
    const int w = i / (32 * TN), j = i % (32 * TN), up = j / (16 * TN);
    return (int64_t)min(n0 + w * 16 * TN + j % (16 * TN), a.N - 1) + (up ? a.N : 0);
  };
  const auto a_row = [&](int i) { return min(m0 + i, a.M - 1); };

  // This wave's pieces of 8 rows of a stage: bounds-checked loads from A, the gates and what they multiply, each from the tile's first row on
  const auto rows_of = [](const uint8_t* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, bytes, 0x00027000); };
  const int a_bytes = uniform((int)(min<int64_t>(BM, a.M - m0) * Kp)), w_bytes = uniform((int)(min(columns, a.N - n0) * Kp));
  const int64_t u_first = (gated ? (int64_t)a.N : 0) + n0;
  const auto A1 = rows_of(a.A + m0 * Kp, a_bytes), W1 = rows_of(a.W + n0 * Kp, w_bytes), U1 = rows_of(a.W + u_first * Kp, w_bytes);
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
  const auto operand = [&](const uint8_t* stage, int t, int half) {       // t < TN: of W, else of A
    const uint8_t* row = stage + (t < TN ? w_base + t * 4096 : a_base + (t - TN) * 4096);
    const u32x4 lo = *reinterpret_cast<const u32x4*>(row + slot[2 * half]), hi = *reinterpret_cast<const u32x4*>(row + slot[2 * half + 1]);
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  // scales of four blocks at a time, those of the current block in the lowest byte
  const auto As = rows_of(a.As + m0 * ss, uniform((int)min<int64_t>(BM, a.M - m0) * ss)), Ws = rows_of(a.Ws, uniform(q8_blocks(gated ? 2 * a.N : a.N) * ss));
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

  // the sums start at the bias: bounds-checked loads, zero beyond the last column and without one
  const uint8_t* const bias_bytes = reinterpret_cast<const uint8_t*>(a.bias);
  const auto bias_z = rows_of(bias_bytes, uniform(a.bias ? a.N * 4 : 0)),
             bias_u = rows_of(bias_bytes + (gated ? (int64_t)a.N * 4 : 0), uniform(a.bias ? a.N * 4 : 0));
  f32x16 c[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    f32x16 bias;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int col = n0 + wn * 32 * (gated ? TN / 2 : TN) + 32 * (gated ? i % (TN / 2) : i) + e / 4 * 8 + 4 * h + e % 4;
      bias[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(gated && i >= TN / 2 ? bias_u : bias_z, col * 4, 0, 0));
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) c[i][j] = bias;
  }
  i32x8 x[2][TN + TM];

  load_scales(0, sc);
  load_scales(min(4, ss - 4), next_sc);
#pragma unroll
  for (int j = 0; j < LOADS; ++j) load(j, 0, stage0.b, A1, W1, U1);
  if (blocks > 1) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) load(j, 1, stage1.b, A1, W1, U1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int t = 0; t < TN + TM; ++t) x[0][t] = operand(stage0.b, t, 0);

  const auto multiply = [&](const i32x8* y, auto&& between) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        between(i * TM + j);
        product32<EXACT>(c[i][j], y[i], y[TN + j], sc[i], sc[TN + j]);
        hold(c[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // Block b lies in `now` with its first half in x[0].  Once all waves have read its second half, block b + 2 is loaded there (beyond the last one the
  // loads are out of bounds and fetch nothing); it has a block and a half's time to arrive.
  const auto block = [&](int b, uint8_t* now, uint8_t* then) {
    const int more = b + 2 < blocks ? -1 : 0;
    const auto A2 = rows_of(a.A + m0 * Kp, a_bytes & more), W2 = rows_of(a.W + n0 * Kp, w_bytes & more), U2 = rows_of(a.W + u_first * Kp, w_bytes & more);
    multiply(x[0], [&](int t) {
      if (t < TN + TM) x[1][t] = operand(now, t, 1);
      if (t == READ) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t >= READ) {
#pragma unroll
        for (int j = (t - READ) * LOADS / (TN * TM - READ); j < (t - READ + 1) * LOADS / (TN * TM - READ); ++j) load(j, b + 2, now, A2, W2, U2);
      }
    });
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LOADS) : "memory");
    multiply(x[1], [&](int t) {
      if (t < TN + TM) x[0][t] = operand(then, t, 0);
    });
    if ((b & 3) == 3) {
#pragma unroll
      for (int t = 0; t < TN + TM; ++t) sc[t] = next_sc[t];
      load_scales(min(b + 5, ss - 4), next_sc);
    } else {
#pragma unroll
      for (int t = 0; t < TN + TM; ++t) sc[t] = (int)((uint32_t)sc[t] >> 8);
    }
  };
  int b = 0;
  for (; b + 1 < blocks; b += 2) {
    block(b, stage0.b, stage1.b);
    block(b + 1, stage1.b, stage0.b);
  }
  if (b < blocks) block(b, stage0.b, stage1.b);
  asm volatile("s_waitcnt lgkmcnt(0) vmcnt(0)\n\ts_barrier" ::: "memory");
  const bool edge = n0 + columns > a.N || column_tile == column_tiles - 1;
  store_tile<TM, TN, ACT, ES>(a, c, m0, n0, edge, wm, wn, lane, stage0.b, reinterpret_cast<float*>(stage1.b));
}

// ACT: svdc_act;  ES: bytes of an element of Out
template <int TM, int TN, int ACT, int ES>
__global__ __launch_bounds__(256) void matmul8_tile_kernel(MatmulArgs a) {
#ifdef __HIP_DEVICE_COMPILE__          // buffer descriptors and accumulation registers mean nothing to the host's pass
  tile_of_product<TM, TN, ACT, ES>(a);
#endif
}

}  // namespace

size_t matmul8_workspace_bytes(const svdc_matmul8&) { return 0; }

namespace {

template <int TM, int TN, int ACT, int ES>
void launch_tiles(const MatmulArgs& a, hipStream_t st) {
  const int columns = ACT == SVDC_ACT_SWIGLU ? 32 * TN : 64 * TN;
  const int64_t tiles = (a.M + 64 * TM - 1) / (64 * TM) * ((a.N + columns - 1) / columns);
  matmul8_tile_kernel<TM, TN, ACT, ES><<<(unsigned)tiles, 256, 0, st>>>(a);
}

template <int TM, int TN, int ES>
void launch_tiles(const MatmulArgs& a, hipStream_t st) {
  if (a.act == SVDC_ACT_SWIGLU)
    launch_tiles<TM, TN, SVDC_ACT_SWIGLU, ES>(a, st);
  else if (a.act == SVDC_ACT_GELU)
    launch_tiles<TM, TN, SVDC_ACT_GELU, ES>(a, st);
  else
    launch_tiles<TM, TN, SVDC_ACT_NONE, ES>(a, st);
}

}  // namespace

int32_t launch_matmul8(const svdc_matmul8& p, const void* A, const void* As, const void* W, const void* Ws, const float* bias, void* Out, void* Os,
                       void*, hipStream_t st) {
  const MatmulArgs a{static_cast<const uint8_t*>(A), static_cast<const uint8_t*>(As), static_cast<const uint8_t*>(W), static_cast<const uint8_t*>(Ws),
                     bias, Out, static_cast<uint8_t*>(Os), p.M, p.ldo, p.N, p.K, p.dtype, p.act};
  if (p.M >= 64) {
    if (p.dtype == SVDC_F32)
      launch_tiles<2, 2, 4>(a, st);
    else if (p.dtype == SVDC_BF16)
      launch_tiles<4, 4, 2>(a, st);
    else
      launch_tiles<4, 4, 1>(a, st);
    return launch_status();
  }
  const int64_t tiles = (p.M + 15) / 16 * q8_blocks(p.N);
  const unsigned grid = (unsigned)std::min<int64_t>(tiles, 1 << 20);
  if (p.dtype == SVDC_F32)
    matmul8_kernel<true><<<grid, 512, 0, st>>>(a);
  else
    matmul8_kernel<false><<<grid, 512, 0, st>>>(a);
  return launch_status();
}

}  // namespace svdc
