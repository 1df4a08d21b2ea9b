// Rows into 8 bits: the root-mean-square norm with the residual's addition (svdcache_rms_norm8) and plain quantisation
// (svdcache_quantize8).
//
// Both stream rows once: a lane holds 8 consecutive columns, so the 16 lanes of a DPP row hold the 128 columns that share a
// scale, and the maximum over them is four register moves.  Neither reuses anything but the gain.  Both are bound by memory (a copy of 1 GiB reaches 5.5 TB/s):
//     norm      4608 x 3072 bfloat16 (99 MB) 18.0 us, 5.5 TB/s; 119056 x 3072 float32 with bfloat16 features (4.0 GB) 729 us, 5.5 TB/s; one row 3.0 us, a launch
//     quantise  4608 x 3072 bfloat16 (42 MB) 8.3 us, 5.1 TB/s; 12288 x 3072 in blocks (113 MB) 24.2 us, 4.7 TB/s
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

// Sum over the NW waves of a row, in all of their lanes: four register moves for the 16 lanes of a DPP row, then the four rows, then the waves.
template <int NW>
__device__ __forceinline__ float group_sum(float v, float* part) {
#define SVDC_ROR_ADD(n) \
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + n, 0xf, 0xf, false))
  SVDC_ROR_ADD(8);
  SVDC_ROR_ADD(4);
  SVDC_ROR_ADD(2);
  SVDC_ROR_ADD(1);
#undef SVDC_ROR_ADD
  const auto of = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
  v = (of(0) + of(16)) + (of(32) + of(48));
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

// The norm of rows that fit in registers: NW waves a row, NC chunks of 8 columns a lane, all but the last of them whole.  A wave (or workgroup) takes row after row
// and keeps the gain in registers, where it would be half as many bytes as a row of bfloat16 again.
template <typename TX, typename TF, int NW, int NC>
__global__ __launch_bounds__(256) void rms_norm8_rows_kernel(NormArgs a) {
  __shared__ float part[NW];
  constexpr int kSpan = NW * kWave * 8, ROWS = 4 / NW;       // rows of a workgroup
  const int first = (NW == 1 ? threadIdx.x % kWave : threadIdx.x) * 8;
  const auto left = [&](int k) { return k < NC - 1 ? 8 : a.D - (first + k * kSpan); };
  float gain[NC][8];
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    if (a.gain) {
      load8(a.gain + first + k * kSpan, left(k), gain[k]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) gain[k][i] = left(k) > i ? 1.f : 0.f;
    }
  }
  for (int64_t row = (int64_t)blockIdx.x * ROWS + (NW == 1 ? threadIdx.x / kWave : 0); row < a.rows; row += (int64_t)gridDim.x * ROWS) {
    float h[NC][8];
    const TX* x = static_cast<const TX*>(a.X) + row * a.ldx + first;
#pragma unroll
    for (int k = 0; k < NC; ++k) load8(x + k * kSpan, left(k), h[k]);
    if (a.F) {
      const TF* f = static_cast<const TF*>(a.F) + row * a.ldf + first;
      float t[NC][8];
#pragma unroll
      for (int k = 0; k < NC; ++k) load8(f + k * kSpan, left(k), t[k]);
#pragma unroll
      for (int k = 0; k < NC; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k][i] += t[k][i];
    }
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NC; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[k][i], h[k][i], sum);
    if (a.H) {
      TX* to = static_cast<TX*>(a.H) + row * a.ldh + first;
#pragma unroll
      for (int k = 0; k < NC; ++k) store8(to + k * kSpan, left(k), h[k]);
    }
    sum = group_sum<NW>(sum, part);
    const float r = 1.f / sqrtf(sum / (float)a.D + a.eps);
    uint8_t *q = a.Q + row * q8_row_bytes(a.D), *scales = a.scales + row * q8_scale_row_bytes(a.D);
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[k][i] * r * gain[k][i];
      if (left(k) < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= left(k)) y[i] = 0.f;          // not 0 * inf, should the sum be a NaN
      }
      if (a.Y) store8(static_cast<TX*>(a.Y) + row * a.ldy + first + k * kSpan, left(k), y);
      if (a.Q) store_q8(q, scales, a.D, first + k * kSpan, y);
    }
  }
}

// Longer rows: a workgroup of NW waves takes a row at a time and reads it twice, the second time out of the caches.  4608 x 16384 bfloat16 (528 MB without the second
// read) 133 us, 4.0 TB/s; 300 x 20000 16.1 us; one row of 20000 6.8 us.
template <typename TX, typename TF, int NW>
__global__ __launch_bounds__(NW* kWave) void rms_norm8_long_kernel(NormArgs a) {
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

// One wave takes 512 columns of two rows, so that their loads are in flight together.
constexpr int kRowsPerWave = 2;
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ X, uint8_t* __restrict__ Q, uint8_t* __restrict__ scales, int64_t rows,
                                                            int D, int64_t ldx) {
  const int c = blockIdx.y * 512 + threadIdx.x % kWave * 8;
  for (int64_t row0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * kRowsPerWave; row0 < rows; row0 += (int64_t)gridDim.x * 4 * kRowsPerWave) {
    float v[kRowsPerWave][8];
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) load8(X + (row0 + i) * ldx + c, row0 + i < rows ? D - c : 0, v[i]);
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i)
      if (row0 + i < rows) store_q8(Q + (row0 + i) * q8_row_bytes(D), scales + (row0 + i) * q8_scale_row_bytes(D), D, c, v[i]);
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

template <typename TX, typename TF, int NW>
void norm_rows(const NormArgs& a, int chunks, unsigned grid, hipStream_t st) {
  switch (chunks) {
    case 1: rms_norm8_rows_kernel<TX, TF, NW, 1><<<grid, 256, 0, st>>>(a); break;
    case 2: rms_norm8_rows_kernel<TX, TF, NW, 2><<<grid, 256, 0, st>>>(a); break;
    case 3: rms_norm8_rows_kernel<TX, TF, NW, 3><<<grid, 256, 0, st>>>(a); break;
    case 4: rms_norm8_rows_kernel<TX, TF, NW, 4><<<grid, 256, 0, st>>>(a); break;
    case 5: rms_norm8_rows_kernel<TX, TF, NW, 5><<<grid, 256, 0, st>>>(a); break;
    default: rms_norm8_rows_kernel<TX, TF, NW, 6><<<grid, 256, 0, st>>>(a); break;
  }
}

// A wave a row where there are many rows of few columns (4608 x 1024 bfloat16 7.7 us, with four waves 8.6) or very many rows (119056 x 3072 float32 726 us, with four waves 751);
// else a workgroup of four waves up to 12288 columns (4608 x 3072 bfloat16 17.8 us, with a wave 20.8; one row 3.0, with a wave 4.0); longer rows do not fit in registers.
// Of middling numbers of rows a workgroup takes several, and keeps the gain (4608 rows 17.8 us, a row each 19.3); of many it takes one: they then stream through memory in
// order (119056 rows 726 us, eight workgroups a unit 766).
template <typename TX, typename TF>
void norm(const NormArgs& a, hipStream_t st) {
  const int64_t units = num_compute_units();
  const bool many = a.rows >= 32 * units;
  if (a.rows >= 4 * units && (a.D <= 1024 || (a.D <= 6 * 512 && many)))
    norm_rows<TX, TF, 1>(a, (a.D + 511) / 512, grid_of((a.rows + 3) / 4), st);
  else if (a.D <= 6 * 2048)
    norm_rows<TX, TF, 4>(a, (a.D + 2047) / 2048, grid_of(many ? a.rows : std::min(a.rows, 6 * units)), st);
  else
    rms_norm8_long_kernel<TX, TF, 16><<<grid_of(a.rows), 16 * kWave, 0, st>>>(a);
}

template <typename TX>
int32_t norm_by_features(const svdc_norm8& p, const NormArgs& a, hipStream_t st) {
  p.dtype_f == SVDC_F32 ? norm<TX, float>(a, st) : norm<TX, bf16_t>(a, st);
  return launch_status();
}

template <typename T>
int32_t quantize(const svdc_quant8& p, const void* X, void* Q, void* scales, hipStream_t st) {
  const T* x = static_cast<const T*>(X);
  uint8_t *q = static_cast<uint8_t*>(Q), *s = static_cast<uint8_t*>(scales);
  if (p.block_rows == 1)
    quantize_rows_kernel<T><<<dim3(grid_of((p.rows + 4 * kRowsPerWave - 1) / (4 * kRowsPerWave)), (p.D + 511) / 512), 256, 0, st>>>(x, q, s, p.rows, p.D, p.ldx);
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
