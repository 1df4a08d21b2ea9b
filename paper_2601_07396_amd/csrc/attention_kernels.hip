// softmax(scale Q K^T) V for each head (svdcache_attention).
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup's waves have 32 queries each and share tiles of 32 or 64 keys and their values in LDS.
// Products are made the other way round, so that a lane holds one query's numbers throughout and the softmax needs nothing from other lanes but
// the maximum of its other half of the keys:
//     S^T [keys x queries] = K Q^T     32 x 32 results: lane l holds query l % 32, keys 8 g + 4 (l / 32) + c, g, c = 0 .. 3
//     O^T [columns x queries] = V^T P^T   whose right operand wants from lane l numbers of query l % 32, and which numbers of the summed axis is free as
//                                         long as the left operand has the same: the keys that the lane has.  P goes from one product into the other in registers.
#include <algorithm>

#include "attention_plan.h"
#include "eight_bit.h"
#include "svdc_internal.h"

namespace svdc {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct AttentionArgs {
  const void *Q, *K, *V;
  void* Out;
  const int2 *q_span, *k_span;
  const uint8_t* mask;
  float *sums, *stats;               // of parts: [batch][heads][part][q_rows][width] and [..][2]: maximum (times scale log2 e) and sum
  int64_t q_total, k_total;
  svdc_heads q, k, v, o;
  int batch, heads, share, head_dim, q_rows, k_rows, q_tiles, parts, tiles_of_part;
  float scale;                       // times log2 e
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Rows of sequence b: the span's, as far as it lies within `total` rows, at most `most`
struct Rows {
  int64_t first;
  int count;
  __device__ __forceinline__ Rows(const int2* span, int b, int64_t total, int most) : first(0), count(most) {
    if (span) {
      const int64_t from = max(0, span[b].x), end = min<int64_t>((int64_t)span[b].x + max(0, span[b].y), total);
      first = from;
      count = (int)max<int64_t>(0, min<int64_t>(end - from, most));
      if (!count) first = 0;
    }
  }
};

// v of this lane's number in the lower and in the upper half of the wave
__device__ __forceinline__ float2 both_halves(float v) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(both[0]), __uint_as_float(both[1])};
}
__device__ __forceinline__ float max_of_halves(float v) {
  const float2 both = both_halves(v);
  return fmaxf(both.x, both.y);
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const float2 both = both_halves(v);
  return both.x + both.y;
}

template <typename T, int W>
struct Tile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int KEYS = attention_tile_keys(W, F32), BLOCKS = KEYS / 32;
  static constexpr int CHUNKS = W * (int)sizeof(T) / 16;                                   // of 16 bytes that a row has
  static constexpr int PITCH = CHUNKS <= 8 ? 8 : CHUNKS <= 16 ? 16 : CHUNKS <= 32 ? 32 : 64;  // and that it takes in LDS
  static constexpr int BYTES = KEYS * PITCH * 16;
  // Chunk c of a row lies at c ^ swizzle(row).  Keys are read as 16 bytes of 16 rows at a time, which then lie in different banks; values as 64 bytes of
  // 4 rows, or (float32) 128 bytes of rows r and r + 4.
  __device__ static __forceinline__ int key_swizzle(int row) { return PITCH == 8 ? row >> 1 & 7 : row & 15; }
  __device__ static __forceinline__ int value_swizzle(int row) { return F32 ? (row >> 2 & 1) << 3 : PITCH == 8 ? (row >> 1 & 1) << 2 : (row & 3) << 2; }
};

template <int BYTES>
struct Stage {
  __align__(1024) uint8_t k[BYTES];
  __align__(1024) uint8_t v[BYTES];
};

// Four columns of 16-bit numbers from four rows, transposed: lane i of 16 hands over the address of columns 4 (i % 4) .. + 3 of row i / 4 and gets
// column i of rows 0 .. 3.
__device__ __forceinline__ bf16x4 read_transposed(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(p));
}

// A row's result: 32 columns of lane l's query in v, columns 8 g + 4 (l / 32) + c
template <typename T>
__device__ __forceinline__ void store_columns(T* row, int column, int head_dim, const f32x16& v, int h);
template <>
__device__ __forceinline__ void store_columns<float>(float* row, int column, int head_dim, const f32x16& v, int h) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int c = column + 8 * g + 4 * h;
    if (c + 4 <= head_dim) {
      *reinterpret_cast<f32x4_any*>(row + c) = f32x4_any{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < head_dim) row[c + e] = v[4 * g + e];
    }
  }
}
// the halves of the wave change words, so that each has 8 columns in a row: of group g the lower one, of g + 1 the upper
template <>
__device__ __forceinline__ void store_columns<bf16_t>(bf16_t* row, int column, int head_dim, const f32x16& v, int h) {
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(v[4 * g], v[4 * g + 1]), pack_bf16(v[4 * g + 4], v[4 * g + 5]), false, false),
               y = __builtin_amdgcn_permlane32_swap(pack_bf16(v[4 * g + 2], v[4 * g + 3]), pack_bf16(v[4 * g + 6], v[4 * g + 7]), false, false);
    const uint32_t w[4] = {x[0], y[0], x[1], y[1]};
    const int c = column + 8 * (g + h);
    if (c + 8 <= head_dim) {
      *reinterpret_cast<u32x4_any*>(row + c) = u32x4_any{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < head_dim) reinterpret_cast<uint16_t*>(row)[c + e] = (uint16_t)(w[e / 2] >> 16 * (e % 2));
    }
  }
}

// DIRECT: head_dim, strides and pointers are multiples of 16 bytes, and tiles are loaded straight into LDS.
template <typename T, int W, int WAVES, bool DIRECT>
__device__ __forceinline__ void attend(const AttentionArgs& a) {
  using G = Tile<T, W>;
  constexpr int KEYS = G::KEYS, BLOCKS = G::BLOCKS, PITCH = G::PITCH, E = 16 / (int)sizeof(T);
  constexpr int STAGES = !DIRECT || WAVES == 4 || 6 * G::BYTES > (96 << 10) ? 2 : 3;
  constexpr int LOADS = KEYS * PITCH / (64 * WAVES);          // of each operand, a wave and tile
  static_assert(LOADS * 64 * WAVES == KEYS * PITCH, "");
  __shared__ Stage<G::BYTES> stage0;
  __shared__ Stage<G::BYTES> stage1;
  __shared__ Stage<G::BYTES> stage2;                          // not there with two stages
  Stage<G::BYTES>* const stages[3] = {&stage0, &stage1, STAGES == 3 ? &stage2 : &stage0};

  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
  // Workgroups go round the eight dies in turn; each die gets a run of them, so that the ones at work on it at a time share keys in its cache.
  int id;
  {
    const int all = gridDim.x, each = all / 8, more = all % 8, die = blockIdx.x % 8;
    id = uniform(die * each + min(die, more) + blockIdx.x / 8);
  }
  const int q_tile = id % a.q_tiles, part = id / a.q_tiles % a.parts, head = id / (a.q_tiles * a.parts) % a.heads, b = id / (a.q_tiles * a.parts * a.heads);
  const Rows queries(a.q_span, b, a.q_total, a.q_rows), keys(a.k_span, b, a.k_total, a.k_rows);
  const int q0 = q_tile * 32 * WAVES;
  if (q0 >= queries.count) return;
  const int mine = q0 + 32 * wave + r;                        // this lane's query
  const bool there = mine < queries.count;
  const int k_count = uniform(keys.count);
  const int from = uniform(part * a.tiles_of_part), to = uniform(min(from + a.tiles_of_part, (k_count + KEYS - 1) / KEYS));

  const T* K = static_cast<const T*>(a.K) + ((a.k_span ? 0 : b * a.k.seq) + keys.first * a.k.row + (head / a.share) * a.k.head);
  const T* V = static_cast<const T*>(a.V) + ((a.k_span ? 0 : b * a.v.seq) + keys.first * a.v.row + (head / a.share) * a.v.head);
  const uint8_t* mask = a.mask ? a.mask + (a.k_span ? keys.first : (int64_t)b * a.k_rows) : nullptr;

  // ---- tiles of keys and values ----
  const int k_row = uniform((int)(a.k.row * sizeof(T))), v_row = uniform((int)(a.v.row * sizeof(T)));
  const int row_bytes = a.head_dim * (int)sizeof(T);
  uint32_t k_from[LOADS], v_from[LOADS];
  u32x4 kept_k[DIRECT ? 1 : LOADS], kept_v[DIRECT ? 1 : LOADS];
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int slot = (n * WAVES + wave) * 64 + lane, row = slot / PITCH, c = slot % PITCH;
    const int kc = (c ^ G::key_swizzle(row)) * 16, vc = (c ^ G::value_swizzle(row)) * 16;
    k_from[n] = kc < row_bytes ? (uint32_t)(row * k_row + kc) : 0x80000000u;      // out of bounds
    v_from[n] = vc < row_bytes ? (uint32_t)(row * v_row + vc) : 0x80000000u;
  }
  // Direct loads are bounds-checked: rows behind the last key are none of memory.
  const auto fetch = [&](int tile, Stage<G::BYTES>& stage) {
    const int rows = uniform(tile < to ? min(KEYS, k_count - tile * KEYS) : 0);
    const auto Kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(K + (int64_t)tile * KEYS * a.k.row), 0, rows ? (rows - 1) * k_row + row_bytes : 0, 0x00027000);
    const auto Vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(V + (int64_t)tile * KEYS * a.v.row), 0, rows ? (rows - 1) * v_row + row_bytes : 0, 0x00027000);
#pragma unroll
    for (int n = 0; n < LOADS; ++n) __builtin_amdgcn_raw_ptr_buffer_load_lds(Kb, stage.k + (n * WAVES + wave) * 1024, 16, k_from[n], 0, 0, 0);
#pragma unroll
    for (int n = 0; n < LOADS; ++n) __builtin_amdgcn_raw_ptr_buffer_load_lds(Vb, stage.v + (n * WAVES + wave) * 1024, 16, v_from[n], 0, 0, 0);
  };
  // The same through registers, at any alignment and width.
  const auto chunk_of = [&](const T* rows, int64_t row_stride, int row, int c, int count) {
    u32x4 w = {};
    const int column = c * E;
    if (row < count && column < a.head_dim) {
      const T* p = rows + row * row_stride + column;
      if (column + E <= a.head_dim) {
        w = *reinterpret_cast<const u32x4_any*>(p);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (column + e < a.head_dim) {
            if (sizeof(T) == 4)
              w[e] = reinterpret_cast<const uint32_t*>(p)[e];
            else
              w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << 16 * (e % 2);
          }
      }
    }
    return w;
  };
  const auto take = [&](int tile) {
    const int count = tile < to ? k_count - tile * KEYS : 0;
#pragma unroll
    for (int n = 0; n < LOADS && !DIRECT; ++n) {
      const int slot = (n * WAVES + wave) * 64 + lane, row = slot / PITCH, c = slot % PITCH;
      kept_k[n] = chunk_of(K + (int64_t)tile * KEYS * a.k.row, a.k.row, row, c ^ G::key_swizzle(row), count);
      kept_v[n] = chunk_of(V + (int64_t)tile * KEYS * a.v.row, a.v.row, row, c ^ G::value_swizzle(row), count);
    }
  };
  const auto put = [&](Stage<G::BYTES>& stage) {
#pragma unroll
    for (int n = 0; n < LOADS && !DIRECT; ++n) {
      const int slot = (n * WAVES + wave) * 64 + lane;
      *reinterpret_cast<u32x4*>(stage.k + slot * 16) = kept_k[n];
      *reinterpret_cast<u32x4*>(stage.v + slot * 16) = kept_v[n];
    }
  };
  // Which keys of a tile take part, a bit each
  const auto present = [&](int tile) -> uint64_t {
    const int count = k_count - tile * KEYS;
    const uint64_t all = KEYS == 64 ? ~0ull : 0xffffffffull;
    if (!mask) return count >= KEYS ? all : (1ull << count) - 1;
    const bool in = lane < min(KEYS, count) && mask[(int64_t)tile * KEYS + lane];
    return __builtin_amdgcn_ballot_w64(in);
  };

  if (DIRECT && row_bytes != PITCH * 16) {
    // columns behind the last one are multiplied by zeros: they hold numbers
    uint32_t* const z[3] = {reinterpret_cast<uint32_t*>(stages[0]), reinterpret_cast<uint32_t*>(stages[1]), reinterpret_cast<uint32_t*>(stages[2])};
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      for (int i = threadIdx.x; i < (int)sizeof(Stage<G::BYTES>) / 16; i += 64 * WAVES) reinterpret_cast<u32x4*>(z[s])[i] = u32x4{};
    __syncthreads();
  }
  if (DIRECT) {
    fetch(from, *stages[0]);
    if (STAGES == 3) fetch(from + 1, *stages[1]);
  } else {
    take(from);
    put(*stages[0]);
  }

  // ---- queries, as right operands ----
  constexpr int STEPS = W / (2 * E);                          // 16 bytes of a row for each half of the wave
  u32x4 q[STEPS];
  {
    const T* Q = static_cast<const T*>(a.Q) + ((a.q_span ? 0 : b * a.q.seq) + (queries.first + (there ? mine : 0)) * a.q.row + head * a.q.head);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = chunk_of(Q, 0, 0, 2 * s + h, 1);
  }

  f32x16 o[W / 32] = {};
  float top = -INFINITY, top_scaled = 0.f, sum = 0.f;
  // addresses in a tile: of this lane's 16 bytes of keys, and of what it reads of values
  const int key_at = r * PITCH * 16, key_sw = G::key_swizzle(r);
  int value_at[W / 32];
#pragma unroll
  for (int d = 0; d < W / 32; ++d) {
    if (G::F32) {
      value_at[d] = 4 * h * PITCH * 16 + ((8 * d + r / 4) ^ G::value_swizzle(4 * h)) * 16 + r % 4 * 4;
    } else {
      const int i = lane % 16, row = 4 * h + i / 4;
      value_at[d] = row * PITCH * 16 + ((4 * d + 2 * (lane / 16 & 1) + (i % 4) / 2) ^ G::value_swizzle(row)) * 16 + i % 2 * 8;
    }
  }

  const auto step = [&](int tile, Stage<G::BYTES>& now, Stage<G::BYTES>& next) {
    if (DIRECT)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * 2 * LOADS) : "memory");
    else
      __syncthreads();
    const uint64_t keep = present(tile);
    if (DIRECT)
      fetch(tile + STAGES - 1, next);
    else
      take(tile + 1);
    const bool whole = keep == (KEYS == 64 ? ~0ull : 0xffffffffull);
    if (keep) {
      if (!whole) {
        // values of keys left out count as zeros: a probability of zero does not make nothing of a NaN
        for (int i = threadIdx.x; i < KEYS * PITCH; i += 64 * WAVES)
          if (!(keep >> i / PITCH & 1)) reinterpret_cast<u32x4*>(now.v)[i] = u32x4{};
        __syncthreads();
      }
      f32x16 s[BLOCKS] = {};
#pragma unroll
      for (int x = 0; x < STEPS; ++x)
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(now.k + key_at + 32 * t * PITCH * 16 + ((2 * x + h) ^ key_sw) * 16);
          if (G::F32) {
#pragma unroll
            for (int c = 0; c < 4; ++c) s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[c]), __uint_as_float(q[x][c]), s[t], 0, 0, 0);
          } else {
            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[x]), s[t], 0, 0, 0);
          }
        }
      if (!whole) {
#pragma unroll
        for (int t = 0; t < BLOCKS; ++t) {
          const uint32_t bits = (uint32_t)(keep >> 32 * t) >> 4 * h;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(bits >> (8 * (i / 4) + i % 4) & 1)) s[t][i] = -INFINITY;
        }
      }
      float high = s[0][0];
#pragma unroll
      for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) high = fmaxf(high, s[t][i]);
      high = max_of_halves(high);
      // The maximum that is subtracted may be any number near the true one: it follows only where probabilities would pass 2^8
      if (__builtin_amdgcn_ballot_w64(high * a.scale > top_scaled + 8.f || (top == -INFINITY && high > -INFINITY))) {
        const float next_top = fmaxf(top, high);
        const float less = next_top == top ? 1.f : __builtin_amdgcn_exp2f((top - next_top) * a.scale);
        sum *= less;
#pragma unroll
        for (int d = 0; d < W / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= less;
        top = next_top;
        top_scaled = top == -INFINITY ? 0.f : top * a.scale;
      }
#pragma unroll
      for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.scale, -top_scaled));
          sum += s[t][i];
        }
#pragma unroll
      for (int t = 0; t < BLOCKS; ++t) {
        if (G::F32) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < W / 32; ++d) {
              const float v = *reinterpret_cast<const float*>(now.v + value_at[d] + (32 * t + 8 * (i / 4) + i % 4) * PITCH * 16);
              o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[t][i], o[d], 0, 0, 0);
            }
        } else {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            u32x4 p;
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = pack_bf16(s[t][8 * x + 2 * i], s[t][8 * x + 2 * i + 1]);
#pragma unroll
            for (int d = 0; d < W / 32; ++d) {
              const uint8_t* at = now.v + value_at[d] + (32 * t + 16 * x) * PITCH * 16;
              const bf16x4 lo = read_transposed(at), hi = read_transposed(at + 8 * PITCH * 16);
              const bf16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p), o[d], 0, 0, 0);
            }
          }
        }
      }
    }
    if (!DIRECT) put(next);
  };
  for (int tile = from; tile < to; tile += STAGES) {
    step(tile, *stages[0], *stages[STAGES - 1]);
    if (tile + 1 < to) step(tile + 1, *stages[1], *stages[0]);
    if (STAGES == 3 && tile + 2 < to) step(tile + 2, *stages[2], *stages[1]);
  }
  if (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing lands in LDS behind the workgroup's end

  sum = sum_of_halves(sum);
  if (!there) return;
  if (a.parts > 1) {
    const int64_t at = (((int64_t)b * a.heads + head) * a.parts + part) * a.q_rows + mine;
    if (h == 0) {
      a.stats[2 * at] = sum == 0.f ? -INFINITY : top_scaled;   // a sum that is no number counts
      a.stats[2 * at + 1] = sum;
    }
#pragma unroll
    for (int d = 0; d < W / 32; ++d) store_columns<float>(a.sums + at * W, 32 * d, W, o[d], h);
    return;
  }
  const float share = sum == 0.f ? 0.f : 1.f / sum;
  T* Out = static_cast<T*>(a.Out) + ((a.q_span ? 0 : b * a.o.seq) + (queries.first + mine) * a.o.row + head * a.o.head);
#pragma unroll
  for (int d = 0; d < W / 32; ++d) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] *= share;
    store_columns<T>(Out, 32 * d, a.head_dim, o[d], h);
  }
}

template <typename T, int W, int WAVES, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : 1) void attention_kernel(AttentionArgs a) {
#ifdef __HIP_DEVICE_COMPILE__          // buffer descriptors mean nothing to the host's pass
  attend<T, W, WAVES, DIRECT>(a);
#endif
}

// Joins the parts of the keys, a wave for each query and head: lane l's columns are l, l + 64, ...
template <typename T, int W>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  const int lane = threadIdx.x % kWave;
  const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;                 // (batch, head, row)
  const int row = (int)(id % a.q_rows), head = (int)(id / a.q_rows % a.heads), b = (int)(id / ((int64_t)a.q_rows * a.heads));
  if (b >= a.batch) return;
  const Rows queries(a.q_span, b, a.q_total, a.q_rows);
  if (row >= queries.count) return;
  const int64_t first = ((int64_t)b * a.heads + head) * a.parts * a.q_rows + row;
  float top = -INFINITY, sum = 0.f;                            // of part `lane`
  if (lane < a.parts) {
    const float2 s = reinterpret_cast<const float2*>(a.stats)[first + (int64_t)lane * a.q_rows];
    top = s.x, sum = s.y;
  }
  float high = top;
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) high = fmaxf(high, __shfl_xor(high, i));
  const float weight = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - high);
  const float total = wave_sum(top == -INFINITY ? 0.f : weight * sum);
  constexpr int EACH = (W + 63) / 64;
  float o[EACH] = {};
  for (int p = 0; p < a.parts; ++p) {
    const float w = __shfl(weight, p);
    if (w == 0.f) continue;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (64 * e + lane < W) o[e] = __builtin_fmaf(w, a.sums[(first + (int64_t)p * a.q_rows) * W + 64 * e + lane], o[e]);
  }
  const float share = total == 0.f ? 0.f : 1.f / total;
  T* Out = static_cast<T*>(a.Out) + ((a.q_span ? 0 : b * a.o.seq) + (queries.first + row) * a.o.row + head * a.o.head);
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (64 * e + lane < a.head_dim) st_elem(Out, 64 * e + lane, o[e] * share);
}

template <typename T, int W>
void attention_of(const AttentionArgs& a, const AttentionPlan& plan, bool direct, hipStream_t st) {
  const unsigned grid = (unsigned)((int64_t)a.batch * a.heads * a.q_tiles * plan.parts);
  if (plan.waves == 8) {
    if constexpr (W <= 128) direct ? attention_kernel<T, W, 8, true><<<grid, 512, 0, st>>>(a) : attention_kernel<T, W, 8, false><<<grid, 512, 0, st>>>(a);
  } else {
    direct ? attention_kernel<T, W, 4, true><<<grid, 256, 0, st>>>(a) : attention_kernel<T, W, 4, false><<<grid, 256, 0, st>>>(a);
  }
  if (plan.parts > 1) attention_join_kernel<T, W><<<(unsigned)(((int64_t)a.batch * a.heads * a.q_rows + 3) / 4), 256, 0, st>>>(a);
}

template <typename T>
void attention_by_width(const AttentionArgs& a, const AttentionPlan& plan, bool direct, hipStream_t st) {
  switch (attention_width(a.head_dim)) {
    case 64: attention_of<T, 64>(a, plan, direct, st); break;
    case 96: attention_of<T, 96>(a, plan, direct, st); break;
    case 128: attention_of<T, 128>(a, plan, direct, st); break;
    default: attention_of<T, 256>(a, plan, direct, st); break;
  }
}

// bytes of the parts' sums, a multiple of 256, and of their statistics
size_t sums_bytes(const svdc_attention& p, const AttentionPlan& plan) {
  return (size_t)p.batch * p.heads * plan.parts * p.q_rows * attention_width(p.head_dim) * sizeof(float);
}
size_t stats_bytes(const svdc_attention& p, const AttentionPlan& plan) { return (size_t)p.batch * p.heads * plan.parts * p.q_rows * 2 * sizeof(float); }

}  // namespace

size_t attention_workspace_bytes(const svdc_attention& p) {
  const AttentionPlan plan = attention_plan(p, num_compute_units());
  return plan.parts > 1 ? sums_bytes(p, plan) + stats_bytes(p, plan) : 0;
}

int32_t launch_attention(const svdc_attention& p, const void* Q, const void* K, const void* V, const int32_t* q_span, const int32_t* k_span,
                         const uint8_t* key_mask, void* Out, void* workspace, hipStream_t st) {
  const AttentionPlan plan = attention_plan(p, num_compute_units());
  const int64_t unit = p.dtype == SVDC_F32 ? 4 : 8;
  const auto sixteen = [&](const void* x, const svdc_heads& s, bool spans) {
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && s.row % unit == 0 && s.head % unit == 0 && (spans || s.seq % unit == 0);
  };
  const bool direct = p.head_dim % unit == 0 && sixteen(K, p.k, k_span) && sixteen(V, p.v, k_span);
  const AttentionArgs a{Q, K, V, Out, reinterpret_cast<const int2*>(q_span), reinterpret_cast<const int2*>(k_span), key_mask,
                        static_cast<float*>(workspace), reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + (plan.parts > 1 ? sums_bytes(p, plan) : 0)),
                        p.q_total, p.k_total, p.q, p.k, p.v, p.o, (int)p.batch, p.heads, p.heads / p.kv_heads, p.head_dim, (int)p.q_rows, (int)p.k_rows,
                        (int)((p.q_rows + 32 * plan.waves - 1) / (32 * plan.waves)), plan.parts, plan.tiles_of_part, p.scale * 1.4426950408889634f};
  p.dtype == SVDC_F32 ? attention_by_width<float>(a, plan, direct, st) : attention_by_width<bf16_t>(a, plan, direct, st);
  return launch_status();
}

}  // namespace svdc
