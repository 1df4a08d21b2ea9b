// Rows into 8 bits: the root-mean-square norm with the residual's addition (svdcache_rms_norm8) and plain quantisation
// (svdcache_quantize8).
//
// Both stream rows once: a lane holds 8 consecutive columns, so the 16 lanes of a DPP row hold the 128 columns that share a
// scale, and the maximum over them is four register moves.  Neither reuses anything but the gain.
#include <algorithm>

#include "eight_bit.h"
#include "svdc_internal.h"

namespace svdc {

namespace {

// 8 consecutive elements as float32, the first `n` of them in range (n may be <= 0 or above 8); zeros beyond.  The pointer is aligned to its elements only.
__device__ __forceinline__ void load8(const bf16_t* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const u32x4_any w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const u32x4_any a = reinterpret_cast<const u32x4_any*>(p)[0], b = reinterpret_cast<const u32x4_any*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void store8(bf16_t* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4_any w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<u32x4_any*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (bf16_t)v[i];
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    u32x4_any a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
    reinterpret_cast<u32x4_any*>(p)[0] = a;
    reinterpret_cast<u32x4_any*>(p)[1] = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

__device__ __forceinline__ float max8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}

// Columns col .. col + 7 of a row in 8 bits; all 16 lanes of a DPP row call it together, for the 128 columns of a block.
__device__ __forceinline__ void store_q8(uint8_t* q_row, uint8_t* scale_row, int D, int col, const float (&v)[8]) {
  const int byte = scale_byte(row16_max(max8(v)));
  const float inv = inverse_scale(byte);
  const int Dp = (int)q8_row_bytes(D);
  if (col < Dp) {
    const uint2 w = {pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                     pack_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
    *reinterpret_cast<uint2*>(q_row + col) = w;
  }
  const int block = col / kScaleBlock;
  if (col % kScaleBlock == 0 && block < q8_scale_row_bytes(D)) scale_row[block] = (uint8_t)(col < Dp ? byte : 127);
}

struct NormArgs {
  const void *X, *F;
  const float* gain;
  void *H, *Y;
  uint8_t *Q, *scales;
  int64_t rows, ldx, ldf, ldh, ldy;
  int D;
  float eps;
};

// Sum over the workgroup's threads, in all of them.
template <int NW>
__device__ __forceinline__ float group_sum(float v, float* part) {
  v = wave_sum(v);
  if (NW == 1) return v;
  const int w = threadIdx.x / kWave;
  __syncthreads();                       // the partial sums of the row before have been read
  if (threadIdx.x % kWave == 0) part[w] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) s += part[i];
  return s;
}

// One workgroup of NW waves takes a row at a time; the row is read twice, the second time out of the caches.
template <typename TX, typename TF, int NW>
__global__ __launch_bounds__(NW* kWave) void rms_norm8_kernel(NormArgs a) {
  __shared__ float part[NW];
  constexpr int kSpan = NW * kWave * 8;
  const int lane8 = threadIdx.x * 8;
  const int Dw = (a.D + 511) / 512 * 512;      // whole blocks of scales, spare bytes included
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* x = static_cast<const TX*>(a.X) + row * a.ldx;
    const TF* f = static_cast<const TF*>(a.F) + row * a.ldf;
    float sum = 0.f;
    for (int c = lane8; c < a.D; c += kSpan) {
      float h[8], t[8];
      load8(x + c, a.D - c, h);
      if (a.F) {
        load8(f + c, a.D - c, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += t[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[i], h[i], sum);
    }
    sum = group_sum<NW>(sum, part);
    const float r = 1.f / sqrtf(sum / (float)a.D + a.eps);
    for (int c = lane8; c < Dw; c += kSpan) {
      float h[8], t[8], y[8];
      load8(x + c, a.D - c, h);
      if (a.F) {
        load8(f + c, a.D - c, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += t[i];
      }
      if (a.H) store8(static_cast<TX*>(a.H) + row * a.ldh + c, a.D - c, h);
      if (a.gain) load8(a.gain + c, a.D - c, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[i] * r * (a.gain ? t[i] : 1.f);
      if (a.D - c < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i >= a.D) y[i] = 0.f;        // not 0 * inf, should the sum be a NaN
      }
      if (a.Y) store8(static_cast<TX*>(a.Y) + row * a.ldy + c, a.D - c, y);
      if (a.Q) store_q8(a.Q + row * q8_row_bytes(a.D), a.scales + row * q8_scale_row_bytes(a.D), a.D, c, y);
    }
  }
}

// One wave takes 512 columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ X, uint8_t* __restrict__ Q, uint8_t* __restrict__ scales, int64_t rows,
                                                            int D, int64_t ldx) {
  const int per_row = (D + 511) / 512;
  const int64_t units = rows * per_row;
  const int lane = threadIdx.x % kWave;
  for (int64_t u = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / per_row;
    const int c = (int)(u - row * per_row) * 512 + lane * 8;
    float v[8];
    load8(X + row * ldx + c, D - c, v);
    store_q8(Q + row * q8_row_bytes(D), scales + row * q8_scale_row_bytes(D), D, c, v);
  }
}

// One workgroup takes 128 x 128 elements: 16 lanes a row, 16 rows at a time.
template <typename T>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const T* __restrict__ X, uint8_t* __restrict__ Q, uint8_t* __restrict__ scales, int64_t rows,
                                                              int D, int64_t ldx) {
  __shared__ float part[16];
  const int nb = q8_blocks(D), ns = q8_scale_row_bytes(D);
  const int64_t blocks = (rows + kScaleBlock - 1) / kScaleBlock * nb;
  const int r = threadIdx.x / 16, i8 = threadIdx.x % 16 * 8;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int64_t br = b / nb;
    const int bc = (int)(b - br * nb), c = bc * kScaleBlock + i8;
    float v[8][8], m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = br * kScaleBlock + 16 * i + r;
      load8(X + row * ldx + c, row < rows ? D - c : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, max8(v[i]));
    m = row16_max(m);
    __syncthreads();                     // the maxima of the block before have been read
    if (threadIdx.x % 16 == 0) part[r] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, part[i]);
    const int byte = scale_byte(m);
    const float inv = inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = br * kScaleBlock + 16 * i + r;
      if (row >= rows) break;
      const uint2 w = {pack_e4m3(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv),
                       pack_e4m3(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv)};
      *reinterpret_cast<uint2*>(Q + row * q8_row_bytes(D) + c) = w;
    }
    if (threadIdx.x == 0) scales[br * ns + bc] = (uint8_t)byte;
    if (bc == nb - 1 && (int)threadIdx.x < ns - nb) scales[br * ns + nb + threadIdx.x] = 127;
  }
}

// workgroups for `units` pieces of work, each a workgroup's turn
unsigned grid_of(int64_t units) { return (unsigned)std::min<int64_t>(units, 1 << 20); }

template <typename TX>
int32_t norm_by_features(const svdc_norm8& p, const NormArgs& a, hipStream_t st) {
  const unsigned grid = grid_of(p.rows);
  if (p.dtype_f == SVDC_F32)
    rms_norm8_kernel<TX, float, 4><<<grid, 4 * kWave, 0, st>>>(a);
  else
    rms_norm8_kernel<TX, bf16_t, 4><<<grid, 4 * kWave, 0, st>>>(a);
  return launch_status();
}

template <typename T>
int32_t quantize(const svdc_quant8& p, const void* X, void* Q, void* scales, hipStream_t st) {
  const T* x = static_cast<const T*>(X);
  uint8_t *q = static_cast<uint8_t*>(Q), *s = static_cast<uint8_t*>(scales);
  if (p.block_rows == 1)
    quantize_rows_kernel<T><<<grid_of((p.rows * ((p.D + 511) / 512) + 3) / 4), 256, 0, st>>>(x, q, s, p.rows, p.D, p.ldx);
  else
    quantize_blocks_kernel<T><<<grid_of((p.rows + 127) / 128 * q8_blocks(p.D)), 256, 0, st>>>(x, q, s, p.rows, p.D, p.ldx);
  return launch_status();
}

}  // namespace

int32_t launch_rms_norm8(const svdc_norm8& p, const void* X, const void* F, const float* gain, void* H, void* Y, void* Q, void* scales,
                         hipStream_t st) {
  const NormArgs a{X, F, gain, H, Y, static_cast<uint8_t*>(Q), static_cast<uint8_t*>(scales), p.rows, p.ldx, p.ldf, p.ldh, p.ldy, p.D, p.eps};
  return p.dtype == SVDC_F32 ? norm_by_features<float>(p, a, st) : norm_by_features<bf16_t>(p, a, st);
}

int32_t launch_quantize8(const svdc_quant8& p, const void* X, void* Q, void* scales, hipStream_t st) {
  return p.dtype == SVDC_F32 ? quantize<float>(p, X, Q, scales, st) : quantize<bf16_t>(p, X, Q, scales, st);
}

}  // namespace svdc
