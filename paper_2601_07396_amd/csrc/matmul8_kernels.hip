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

__device__ __forceinline__ float gelu(float x) { return x / (1.f + __expf(-1.5957691216057308f * (x + 0.044715f * x * x * x))); }
__device__ __forceinline__ float silu(float x) { return x / (1.f + __expf(-x)); }

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

}  // namespace

size_t matmul8_workspace_bytes(const svdc_matmul8&) { return 0; }

int32_t launch_matmul8(const svdc_matmul8& p, const void* A, const void* As, const void* W, const void* Ws, const float* bias, void* Out, void* Os,
                       void*, hipStream_t st) {
  const MatmulArgs a{static_cast<const uint8_t*>(A), static_cast<const uint8_t*>(As), static_cast<const uint8_t*>(W), static_cast<const uint8_t*>(Ws),
                     bias, Out, static_cast<uint8_t*>(Os), p.M, p.ldo, p.N, p.K, p.dtype, p.act};
  const int64_t tiles = (p.M + 15) / 16 * q8_blocks(p.N);
  const unsigned grid = (unsigned)std::min<int64_t>(tiles, 1 << 20);
  if (p.dtype == SVDC_F32)
    matmul8_kernel<true><<<grid, 512, 0, st>>>(a);
  else
    matmul8_kernel<false><<<grid, 512, 0, st>>>(a);
  return launch_status();
}

}  // namespace svdc
