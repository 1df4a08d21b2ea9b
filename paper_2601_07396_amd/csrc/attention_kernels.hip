// softmax(scale Q K^T) V for each head (svdcache_attention).
//
// One pass over the keys with a running shift and sum of the softmax.  A workgroup's four waves have 32 queries each and share tiles of 32 or 64 keys and their values in LDS, loaded
// one tile ahead.  Products are made the other way round, so that a lane holds one query's numbers throughout and the softmax needs nothing from other lanes:
//     S^T [keys x queries] = K Q^T     32 x 32 results: lane l holds query l % 32, keys 8 g + 4 (l / 32) + c, g, c = 0 .. 3
//     O^T [columns x queries] = V^T P^T   whose right operand wants from lane l numbers of query l % 32, and which numbers of the summed axis is free as
//                                         long as the left operand has the same: the keys that the lane has.  P goes from one product into the other in registers.
// P = 2^(scale log2(e) S - shift) is rounded to bfloat16 for bfloat16 tensors (the matrix cores' other operand, V, is that too): each probability by at most 2^-8 of itself, a result by
// 2^-8 sum p |v|, more than its own rounding where values cancel.  Its sums are made of the rounded numbers, so that what rounding moves the probabilities by on the whole drops out.
// On random numbers the distance to 64 bits is 1.7e-3 of the result, of which rounding it alone makes 1.6e-3.
//
// What bounds it: the matrix cores, and the clock, which the card lowers under this load.  4608 x 4608, 24 heads of 128, bfloat16: 242 us, 1080 TFLOP/s; while every
// compute unit has two workgroups its matrix cores are 84 % busy, at 1.7 GHz; over the whole call 59 % at 1.86 GHz.  A large bfloat16 matrix product reaches 1410 TFLOP/s on
// the card.  29764 x 29764, 3 heads: 1.20 ms, 1135 TFLOP/s.  float32 products go at a sixteenth of the rate: 4608 x 4608, 24 heads, 1.84 ms, 142 TFLOP/s of 154.  Few rows are bound by
// memory: 64 queries over 119056 keys of 24 heads 270 us, 5.4 TB/s.  Forms that were slower: eight waves of 32 queries with four stages, half of them half a step behind (255 us; 47 %
// busy, one barrier for eight waves); the maximum of each tile before its exponentials (271 us); sums by additions beside the exponentials (they cost a sixth of that phase).
#include <algorithm>
#include <type_traits>

#include "attention_plan.h"
#include "eight_bit.h"
#include "svdc_internal.h"

namespace svdc {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// of lambdas: what is not inlined would keep their captures, the sums, in memory
#define INLINE __attribute__((always_inline))

struct AttentionArgs {
  const void *Q, *K, *V;
  void* Out;
  const int2 *q_span, *k_span;
  const uint8_t* mask;
  float *sums, *stats, *large;       // of parts: [unit][part][query][width]; [..][2]: what was subtracted from the exponents, and their powers' sum; [..]: where that is large, its product
  int64_t q_total, k_total;
  svdc_heads q, k, v, o;
  int kv_heads, share, head_dim, q_rows, k_rows, q_tiles, whole, units, parts, tiles_of_part;
  float scale;                       // times log2 e
};

// what all lanes hold, as a scalar
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename T>
__device__ __forceinline__ T* uniform(T* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<T*>((uint64_t)(uint32_t)uniform((int)(u >> 32)) << 32 | (uint32_t)uniform((int)u));
}

// A unit of work: a tile of the queries of all heads that share a head of keys, one head's rows behind the other's.  Workgroups go round the eight dies in turn, so with eight heads of
// keys side by side, then the next queries of these, a die has a head at a time, whose keys its workgroups share in the die's cache; and packed sequences of different lengths are
// spread over all dies (5 sequences of 0 to 1301 rows, 16 float32 heads: 186 us; with a run of units for each die 415 us, which for equal lengths takes as long).
struct Unit {
  static constexpr int HEADS_AT_ONCE = 8;
  int b, kv_head, q_tile;
  __device__ __forceinline__ Unit(const AttentionArgs& a, int id) {
    b = uniform(id / (a.q_tiles * a.kv_heads));
    id -= b * a.q_tiles * a.kv_heads;
    const int first = id / (a.q_tiles * HEADS_AT_ONCE) * HEADS_AT_ONCE, side = min(HEADS_AT_ONCE, a.kv_heads - first);
    id -= first * a.q_tiles;
    kv_head = uniform(first + id % side);
    q_tile = uniform(id / side);
  }
};
// Query i of a unit: its row of the sequence and its head, and where it lies in a tensor from the sequence's first row on
struct Query {
  int row, head;
  bool there;
  __device__ __forceinline__ Query(const AttentionArgs& a, const Unit& u, int i, int count) {
    const int at = u.q_tile * kTileQueries + i;
    if (a.share == 1) {                    // without a division
      row = at, head = u.kv_head, there = row < count;
    } else {
      const int of_share = at / a.q_rows;
      row = at - of_share * a.q_rows;
      head = u.kv_head * a.share + of_share;
      there = of_share < a.share && row < count;
    }
  }
  __device__ __forceinline__ int64_t at(const svdc_heads& s, int64_t first) const { return (first + row) * s.row + head * s.head; }
};

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

constexpr int WAVES = kTileQueries / 32;                       // of a workgroup
constexpr float SLACK = 6.f, LARGE = 65536.f;                  // of what is subtracted from the exponents: how far above the maximum it begins, and from where on it is coarse

template <int BYTES>
struct Lds {
  __align__(1024) uint8_t b[BYTES];
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
template <typename T, int W, bool DIRECT, bool MASKED>
__device__ __forceinline__ void attend(const AttentionArgs& a) {
  using G = Tile<T, W>;
  constexpr int KEYS = G::KEYS, BLOCKS = G::BLOCKS, PITCH = G::PITCH, E = 16 / (int)sizeof(T);
  constexpr int LOADS = KEYS * PITCH / (64 * WAVES);          // of each operand, a wave and tile
  constexpr uint64_t ALL = KEYS == 64 ? ~0ull : 0xffffffffull;
  static_assert(LOADS * 64 * WAVES == KEYS * PITCH, "");
  __shared__ Lds<G::BYTES> columns0, columns1, keys0, keys1;  // two stages of values and of keys

  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane % 32, h = lane / 32;
  // The first `whole` workgroups have a unit each, the others a part of the keys of one of the rest.
  const bool split = blockIdx.x >= (unsigned)a.whole;
  const int at = blockIdx.x - (split ? a.whole : 0), rest = a.units - a.whole;
  const int part = uniform(split ? at / rest : 0), unit = uniform(split ? a.whole + at % rest : at);
  const Unit u(a, unit);
  const int b = u.b, kv_head = u.kv_head;
  const Rows queries(a.q_span, b, a.q_total, a.q_rows), keys(a.k_span, b, a.k_total, a.k_rows);
  {
    // nothing to do where all of the tile's queries are behind the sequence's end
    const int row = a.share == 1 ? u.q_tile * kTileQueries : u.q_tile * kTileQueries % a.q_rows;
    if (queries.count == 0 || (row >= queries.count && (a.share == 1 || row + kTileQueries <= a.q_rows))) return;
  }
  const int k_count = uniform(keys.count);
  const int from = uniform(part * a.tiles_of_part), to = uniform(min(split ? from + a.tiles_of_part : INT32_MAX, (k_count + KEYS - 1) / KEYS));

  const T* K = uniform(static_cast<const T*>(a.K) + ((a.k_span ? 0 : b * a.k.seq) + keys.first * a.k.row + kv_head * a.k.head));
  const T* V = uniform(static_cast<const T*>(a.V) + ((a.k_span ? 0 : b * a.v.seq) + keys.first * a.v.row + kv_head * a.v.head));

  // ---- tiles of keys and values ----
  const int k_row = uniform((int)(a.k.row * sizeof(T))), v_row = uniform((int)(a.v.row * sizeof(T)));
  const int row_bytes = a.head_dim * (int)sizeof(T);
  uint32_t k_from[LOADS], v_from[LOADS];
  u32x4 kept[DIRECT ? 1 : LOADS];
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int slot = (n * WAVES + wave) * 64 + lane, row = slot / PITCH, c = slot % PITCH;
    const int kc = (c ^ G::key_swizzle(row)) * 16, vc = (c ^ G::value_swizzle(row)) * 16;
    k_from[n] = kc < row_bytes ? (uint32_t)(row * k_row + kc) : 0x80000000u;      // out of bounds
    v_from[n] = vc < row_bytes ? (uint32_t)(row * v_row + vc) : 0x80000000u;
  }
  // Which keys of a tile take part, a bit each.  The mask's bytes are loaded a step before they are looked at.
  const auto mask = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(MASKED ? uniform(a.mask + (a.k_span ? keys.first : (int64_t)b * a.k_rows)) : nullptr), 0,
                                                      MASKED ? k_count : 0, 0x00027000);
  const auto mask_byte = [&](int tile) INLINE -> int {               // none behind the last key
    return MASKED ? __builtin_amdgcn_raw_buffer_load_b8(mask, lane < KEYS ? tile * KEYS + lane : -1, 0, 0) : 0;
  };
  const auto present = [&](int tile, int byte) INLINE -> uint64_t {
    if (MASKED) return __builtin_amdgcn_ballot_w64(byte != 0);
    const int count = k_count - tile * KEYS;
    return count >= KEYS ? ALL : (1ull << max(0, count)) - 1;
  };
  // Direct loads are bounds-checked, and give zeros for rows behind the last key and, by an address out of bounds, for keys left out: a probability of zero
  // would not make nothing of a NaN.
  const auto tile_of = [&](const T* rows, int64_t stride, int bytes, int tile) INLINE {
    const int count = tile < to ? min(KEYS, k_count - tile * KEYS) : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(rows + (int64_t)tile * KEYS * stride), 0, uniform(count ? (count - 1) * bytes + row_bytes : 0), 0x00027000);
  };
  const auto fetch = [&](__amdgpu_buffer_rsrc_t tile, uint32_t at, int n, uint64_t keep, uint8_t* stage) INLINE {
    if (MASKED && !(keep >> ((n * WAVES + wave) * 64 + lane) / PITCH & 1)) at = 0x80000000u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, stage + (n * WAVES + wave) * 1024, 16, at, 0, 0, 0);
  };
  const auto fetch_keys = [&](int tile, uint64_t keep, uint8_t* stage) INLINE {
    const auto from_here = tile_of(K, a.k.row, k_row, tile);
#pragma unroll
    for (int n = 0; n < LOADS; ++n) fetch(from_here, k_from[n], n, keep, stage);
  };
  const auto fetch_values = [&](int tile, uint64_t keep, uint8_t* stage) INLINE {
    const auto from_here = tile_of(V, a.v.row, v_row, tile);
#pragma unroll
    for (int n = 0; n < LOADS; ++n) fetch(from_here, v_from[n], n, keep, stage);
  };
  // The same through registers, at any alignment and width.
  // Heads of 16 bytes or more without branches, so that many loads are on their way: the chunk over a head's end is read as the head's last 16 bytes, and moved down when it is put
  // to use.
  const auto load_chunk = [&](const T* rows, int64_t row_stride, int row, int c, bool present) INLINE {
    u32x4 w = {};
    const int column = c * E;
    present = present && column < a.head_dim;
    if (a.head_dim >= E) {
      w = *reinterpret_cast<const u32x4_any*>(rows + (present ? row * row_stride + min(column, a.head_dim - E) : 0));
    } else if (present) {
      const T* p = rows + row * row_stride + column;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (column + e < a.head_dim) {
          if (sizeof(T) == 4)
            w[e] = reinterpret_cast<const uint32_t*>(p)[e];
          else
            w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << 16 * (e % 2);
        }
    }
    return w;
  };
  const auto chunk_of = [&](u32x4 w, int c, bool present) INLINE {
    const int over = a.head_dim >= E ? max(0, c * E + E - a.head_dim) : 0, bits = over * (int)sizeof(T) * 8;      // of columns behind the last one
    const uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
    const uint64_t down_lo = bits >= 64 ? hi >> (bits & 63) : lo >> bits | (bits ? hi << (64 - bits) : 0), down_hi = bits >= 64 ? 0 : hi >> bits;
    present = present && c * E < a.head_dim;
    return present ? u32x4{(uint32_t)down_lo, (uint32_t)(down_lo >> 32), (uint32_t)down_hi, (uint32_t)(down_hi >> 32)} : u32x4{};
  };
  const auto take = [&](const T* rows, int64_t stride, int tile, uint64_t keep, auto&& swizzle) INLINE {
#pragma unroll
    for (int n = 0; n < LOADS; ++n) kept[n] = u32x4{};
    if (tile >= to) return;                                    // the first row of a tile that is there can be read
#pragma unroll
    for (int n = 0; n < LOADS; ++n) {
      const int slot = (n * WAVES + wave) * 64 + lane, row = slot / PITCH, c = slot % PITCH;
      kept[n] = load_chunk(rows + (int64_t)tile * KEYS * stride, stride, row, c ^ swizzle(row), keep >> row & 1);
    }
  };
  const auto put = [&](uint8_t* stage, uint64_t keep, auto&& swizzle) INLINE {
#pragma unroll
    for (int n = 0; n < LOADS; ++n) {
      const int slot = (n * WAVES + wave) * 64 + lane, row = slot / PITCH, c = slot % PITCH;
      *reinterpret_cast<u32x4*>(stage + slot * 16) = chunk_of(kept[n], c ^ swizzle(row), keep >> row & 1);
    }
  };
  const auto take_keys = [&](int tile, uint64_t keep) INLINE { take(K, a.k.row, tile, keep, G::key_swizzle); };
  const auto take_values = [&](int tile, uint64_t keep) INLINE { take(V, a.v.row, tile, keep, G::value_swizzle); };
  const auto put_keys = [&](uint8_t* stage, uint64_t keep) INLINE { put(stage, keep, G::key_swizzle); };
  const auto put_values = [&](uint8_t* stage, uint64_t keep) INLINE { put(stage, keep, G::value_swizzle); };
  // The last tile lies in stage 0.
  const int steps = max(0, to - from - 1), first = uniform(steps % 2);
  const auto keys_at = [&](int i) INLINE -> uint8_t* { return i % 2 ? keys1.b : keys0.b; };
  const auto values_at = [&](int i) INLINE -> uint8_t* { return i % 2 ? columns1.b : columns0.b; };
  uint64_t keep[4];                                           // of this step's tile and the next ones
  int byte = 0;
  if (from < to) {
    int bytes[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) bytes[i] = mask_byte(from + i);
    byte = mask_byte(from + 3);
#pragma unroll
    for (int i = 0; i < 3; ++i) keep[i] = present(from + i, bytes[i]);
    if (DIRECT) {
      fetch_keys(from, keep[0], keys_at(first));
      fetch_keys(from + 1, keep[1], keys_at(first + 1));
      fetch_values(from, keep[0], values_at(first));
    } else {
      take_keys(from, keep[0]), put_keys(keys_at(first), keep[0]);
      take_keys(from + 1, keep[1]), put_keys(keys_at(first + 1), keep[1]);
      take_values(from, keep[0]), put_values(values_at(first), keep[0]);
    }
  }

  // ---- queries, as right operands ----
  constexpr int STEPS = W / (2 * E);                          // 16 bytes of a row for each half of the wave
  u32x4 q[STEPS];
  bool idle;                                                  // a wave without queries
  {
    const Query mine(a, u, 32 * wave + r, queries.count);
    idle = __builtin_amdgcn_ballot_w64(mine.there) == 0;
    const T* Q = static_cast<const T*>(a.Q) + ((a.q_span ? 0 : b * a.q.seq) + (mine.there ? mine.at(a.q, queries.first) : queries.first * a.q.row));
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bool present = mine.there && (2 * s + h) * 16 < row_bytes;
      if (DIRECT)
        q[s] = *reinterpret_cast<const u32x4*>(Q + (present ? (2 * s + h) * E : 0));
      else
        q[s] = load_chunk(Q, 0, 0, 2 * s + h, mine.there);
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bool present = mine.there && (2 * s + h) * 16 < row_bytes;
      if (DIRECT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) q[s][e] = present ? q[s][e] : 0u;
      } else {
        q[s] = chunk_of(q[s], 2 * s + h, mine.there);
      }
    }
  }

  f32x16 o[W / 32] = {};
  f32x16 s0[BLOCKS], s1[BLOCKS];                              // products of this tile's keys and of the next one's, in turns
  u32x4 p[2 * BLOCKS];                                        // probabilities of this tile: 2^(product scale log2 e - shift), in bfloat16
  f32x16 exact_p[BLOCKS];                                     // or in float32
  // Their sums.  bfloat16: made by a 16 x 16 product, for which lanes 16 g .. 16 g + 15 are columns 0 .. 15 with eight numbers of the summed axis each.  Ones in row 0 for even g,
  // which hold queries 0 .. 15, and in row 1 for odd g, which hold queries 16 .. 31: lane n's sums[0] is query n's, sums[1] query 16 + n's.
  float shift = -INFINITY, sum = 0.f;
  uint64_t coarse = 0;                                        // lanes whose shift is large, and kept as the product that it lies SLACK above
  f32x4 sums = {};
  int lost = 0;
  const uint32_t one_here = lane % 16 == lane / 16 % 2 ? 0x3f803f80u : 0u;
  const u32x4 ones = {one_here, one_here, one_here, one_here};
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

  // The products of a step are dealt out over the softmax's other work, so that both units are busy: `between(n, all)` does the n-th of `all` shares of it behind the n-th
  // product.
  constexpr int AHEAD = !G::F32 || W < 128 ? 3 : W == 128 ? 2 : 1;                    // operands are read from LDS so many products ahead, as many as there are registers for
  constexpr int KEY_PRODUCTS = STEPS * BLOCKS, VALUE_PRODUCTS = G::F32 ? 16 * BLOCKS : 2 * BLOCKS * (W / 32);
  u32x4 k[AHEAD + 1];
  bf16x8 v[AHEAD + 1];
  const auto read_key = [&](const uint8_t* stage, int n) INLINE {
    k[n % (AHEAD + 1)] = *reinterpret_cast<const u32x4*>(stage + key_at + 32 * (n % BLOCKS) * PITCH * 16 + ((2 * (n / BLOCKS) + h) ^ key_sw) * 16);
  };
  const auto read_value = [&](const uint8_t* stage, int n) INLINE {
    constexpr int D = W / 32;
    const uint8_t* at = stage + value_at[n % D] + 16 * (n / D) * PITCH * 16;
    if (!G::F32) v[n % (AHEAD + 1)] = __builtin_shufflevector(read_transposed(at), read_transposed(at + 8 * PITCH * 16), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto first_keys = [&](const uint8_t* stage) INLINE {
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) read_key(stage, n);
  };
  const auto first_values = [&](const uint8_t* stage) INLINE {
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) read_value(stage, n);
  };
  const auto multiply_keys = [&](f32x16 (&s)[BLOCKS], const uint8_t* stage, auto&& between) INLINE {
    constexpr int N = KEY_PRODUCTS;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (n + AHEAD < N) read_key(stage, n + AHEAD);
      const int x = n / BLOCKS, t = n % BLOCKS;
      const u32x4 w = k[n % (AHEAD + 1)];
      f32x16 c = {};
      if (x) c = s[t];
      if (G::F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(w[e]), __uint_as_float(q[x][e]), c, 0, 0, 0);
      } else {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, q[x]), c, 0, 0, 0);
      }
      s[t] = c;
      between(n, N);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto multiply_values = [&](const uint8_t* stage) INLINE {
    constexpr int D = W / 32, N = VALUE_PRODUCTS;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (G::F32) {
        const int t = n / 16, i = n % 16;
        sum += exact_p[t][i];
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const float v = *reinterpret_cast<const float*>(stage + value_at[d] + (32 * t + 8 * (i / 4) + i % 4) * PITCH * 16);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, exact_p[t][i], o[d], 0, 0, 0);
        }
      } else {
        if (n + AHEAD < N) read_value(stage, n + AHEAD);
        if (n % D == 0) sums = mfma16(ones, p[n / D], sums);
        o[n % D] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[n % (AHEAD + 1)], __builtin_bit_cast(bf16x8, p[n / D]), o[n % D], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // Probabilities of this tile.  A pair of them comes into being over three shares of the work, so that nothing waits for what was begun just before: exponents, powers, and
  // what the product takes.  `over` gathers the exponents' highest bit, which numbers from 2 on have (and what is no number).
  constexpr int PAIRS = 8 * BLOCKS;
  uint32_t over;
  float x[2][2];                                              // exponents and powers on their way
  const auto exponents = [&](const f32x16 (&s)[BLOCKS], float off, float by, int m) INLINE {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      x[m % 2][e] = __builtin_fmaf(s[m / 8][2 * (m % 8) + e] - off, a.scale, -by);
      asm volatile("" : "+v"(x[m % 2][e]));                    // here, and not where the compiler would move it
    }
  };
  float y[2][2];
  const auto powers = [&](int m) INLINE {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      y[m % 2][e] = __builtin_amdgcn_exp2f(x[m % 2][e]);
      asm volatile("" : "+v"(y[m % 2][e]));
    }
  };
  const auto operands = [&](int m) INLINE {
    if (m == 0) over = 0;
    if (G::F32) {
      exact_p[m / 8][2 * (m % 8)] = y[m % 2][0], exact_p[m / 8][2 * (m % 8) + 1] = y[m % 2][1];
      over |= __float_as_uint(y[m % 2][0]) | __float_as_uint(y[m % 2][1]);
    } else {
      uint32_t w = pack_bf16(y[m % 2][0], y[m % 2][1]);
      asm volatile("" : "+v"(w));
      p[m / 4][m % 4] = w;
      over |= w;
    }
  };
  // the n-th of `all` shares, and what is left behind the last one
  const auto probabilities = [&](const f32x16 (&s)[BLOCKS], float off, float by, int n, int all) INLINE {
#pragma unroll
    for (int m = n * PAIRS / all; m < (n + 1) * PAIRS / all; ++m) {
      if (m == 0) exponents(s, off, by, 0);
      if (m >= 1) operands(m - 1);
      powers(m);
      if (m + 1 < PAIRS) exponents(s, off, by, m + 1);
      if (m + 1 == PAIRS) operands(m);
    }
  };
  const auto leave_out = [&](f32x16 (&s)[BLOCKS], uint64_t keep) INLINE {
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t) {
      const uint32_t bits = (uint32_t)(keep >> 32 * t) >> 4 * h;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(bits >> (8 * (i / 4) + i % 4) & 1)) s[t][i] = -INFINITY;
    }
  };
  // What is subtracted from the exponents may be any number not far from the maximum: it stays until a probability passes 2, then follows to SLACK above the maximum, and the
  // tile's probabilities are made again.  -infinity until there is a key: then everything passes.
  // Below 2^16 the roundings of a shift move an exponent by 2^-7 at most.  From there on (coarse) they would in the end pass SLACK, or the shift float32: the exponents are made of the
  // products' distances from the largest one, which are exact for equal products, and every tile's probabilities are made again.  (coarse is a mask in scalar registers, and the shift holds
  // that product, because the masked float32 kernel of 128 columns has no vector register left.)
  const auto follow = [&](const f32x16 (&s)[BLOCKS]) INLINE {
    constexpr uint32_t TOP = G::F32 ? 0x40000000u : 0x40004000u;
    // (where sums and operands do not fit the registers, what is likely decides what lies in scratch: 12 float32 heads of 256 columns, 4608 x 4608, 2.94 and 3.02 ms)
    const bool near = (__builtin_amdgcn_ballot_w64((over & TOP) != 0) | coarse) == 0;
    if (G::F32 && W > 128 ? __builtin_expect(near, 1) : near) return;
    float high = -INFINITY;
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) high = fmaxf(high, s[t][i]);
    const float product = max_of_halves(high);
    high = product * a.scale;
    const float before = shift;
    // 2 and what rounds to it is well above: behind this, only what is no number still passes
    bool up = !(high - shift < 0.5f), large = up && product != -INFINITY && !(fabsf(high + SLACK) < LARGE);
    if (up) shift = high + SLACK;
    float less = !up ? 1.f : before == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(before - shift), by = shift == -INFINITY ? 0.f : shift;
    float off = 0.f;
    if (__builtin_expect((coarse | __builtin_amdgcn_ballot_w64(large)) != 0, 0)) {
      const bool was_large = coarse >> lane & 1;
      if (was_large) {
        up = !((product - before) * a.scale < SLACK + 0.5f);
        large = !up || !(fabsf(high + SLACK) < LARGE);
        shift = !up ? before : large ? product : high + SLACK;
        less = !up ? 1.f : __builtin_amdgcn_exp2f(large ? (before - product) * a.scale : before * a.scale + SLACK - shift);
      } else if (large) {
        shift = product;
      }
      coarse = __builtin_amdgcn_ballot_w64(large);
      by = large ? SLACK : shift == -INFINITY ? 0.f : shift;
      off = large ? shift : 0.f;
    }
    sum *= less;
    sums[0] *= less;
    sums[1] *= __shfl(less, lane % 16 + 16);
#pragma unroll
    for (int d = 0; d < W / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= less;
#pragma unroll
    for (int n = 0; n < 8; ++n) probabilities(s, off, by, n, 8);
    if (!G::F32 && (over & TOP)) {                             // no number: not into a column that another query's sum comes from, but into the result
      lost = 1;
#pragma unroll
      for (int i = 0; i < 2 * BLOCKS; ++i) p[i] = u32x4{};
    }
  };
  const auto nothing = [](int, int) INLINE {};
  // Begins a step: all waves have what they asked for in the last one, and are done with what they read in it.
  const auto begin = [&]() INLINE {
    if (DIRECT)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else
      __syncthreads();
  };

  if (DIRECT && idle) {
    // a wave without queries loads its share of the tiles
    if (from < to) begin();
    for (int tile = from; tile + 1 < to; ++tile) {
      begin();
      keep[3] = present(tile + 3, byte);
      byte = mask_byte(tile + 4);
      fetch_values(tile + 1, keep[1], values_at(first + tile - from + 1));
      fetch_keys(tile + 2, keep[2], keys_at(first + tile - from));
#pragma unroll
      for (int i = 0; i < 3; ++i) keep[i] = keep[i + 1];
    }
    if (from < to) begin();
    return;
  }
  if (from < to) {
    begin();
    first_keys(keys_at(first));
    multiply_keys(s0, keys_at(first), nothing);
    if (keep[0] != ALL) leave_out(s0, keep[0]);
    // Tile by tile: its probabilities beside the products of the next one's keys, then its products with the values.  The stages of its keys and of the values of the tile before
    // are free and loaded anew, a load here and there: at once they would hold up the wave.
    const auto step = [&](int tile, uint8_t* keys_now, const uint8_t* keys_next, const uint8_t* values_now, uint8_t* values_next, f32x16 (&s)[BLOCKS],
                          f32x16 (&s_next)[BLOCKS]) INLINE {
      begin();
      first_keys(keys_next);
      keep[3] = present(tile + 3, byte);
      byte = mask_byte(tile + 4);
      const auto keys_tile = tile_of(K, a.k.row, k_row, tile + 2), values_tile = tile_of(V, a.v.row, v_row, tile + 1);
      if (!DIRECT) take_keys(tile + 2, keep[2]);
      multiply_keys(s_next, keys_next, [&](int n, int all) INLINE {
        probabilities(s, 0.f, shift, n, all);
#pragma unroll
        for (int j = n * 2 * LOADS / all; DIRECT && j < (n + 1) * 2 * LOADS / all; ++j) {
          if (j < LOADS)
            fetch(values_tile, v_from[j % LOADS], j % LOADS, keep[1], values_next);
          else
            fetch(keys_tile, k_from[j % LOADS], j % LOADS, keep[2], keys_now);
        }
      });
      first_values(values_now);
      follow(s);
      if (!DIRECT) put_keys(keys_now, keep[2]), take_values(tile + 1, keep[1]);
      if (keep[1] != ALL) leave_out(s_next, keep[1]);
      multiply_values(values_now);
      if (!DIRECT) put_values(values_next, keep[1]);
#pragma unroll
      for (int i = 0; i < 3; ++i) keep[i] = keep[i + 1];
    };
    int tile = from;
    if (first) {
      step(tile++, keys1.b, keys0.b, columns1.b, columns0.b, s0, s1);
#pragma unroll
      for (int t = 0; t < BLOCKS; ++t) s0[t] = s1[t];
    }
    while (tile + 1 < to) {
      step(tile++, keys0.b, keys1.b, columns0.b, columns1.b, s0, s1);
      step(tile++, keys1.b, keys0.b, columns1.b, columns0.b, s1, s0);
    }
    begin();
#pragma unroll
    for (int n = 0; n < 8; ++n) probabilities(s0, 0.f, shift, n, 8);
    follow(s0);
    first_values(columns0.b);
    multiply_values(columns0.b);
  }

  if (G::F32) {
    sum = sum_of_halves(sum);
  } else {
    const float x = __shfl(sums[0], lane % 16), y = __shfl(sums[1], lane % 16);
    sum = lost | __shfl_xor(lost, 32) ? NAN : lane & 16 ? y : x;
  }
  int own = 32 * wave + r;
  asm volatile("" : "+v"(own));                                // made anew, not kept in registers all along
  const Query mine(a, u, own, queries.count);
  if (!mine.there) return;
  if (split) {
    const int64_t at = ((int64_t)(unit - a.whole) * a.parts + part) * kTileQueries + 32 * wave + r;
    if (h == 0) {
      const float top = fmaxf(coarse >> lane & 1 ? __builtin_fmaf(shift, a.scale, SLACK) : shift, -3.4e38f);
      a.stats[2 * at] = sum == 0.f ? -INFINITY : top;          // a sum that is no number counts
      a.stats[2 * at + 1] = sum;
      if (!(fabsf(top) < LARGE)) a.large[at] = shift;
    }
#pragma unroll
    for (int d = 0; d < W / 32; ++d) store_columns<float>(a.sums + at * W, 32 * d, W, o[d], h);
    return;
  }
  const float share = sum == 0.f ? 0.f : 1.f / sum;
  T* Out = static_cast<T*>(a.Out) + ((a.q_span ? 0 : b * a.o.seq) + mine.at(a.o, queries.first));
#pragma unroll
  for (int d = 0; d < W / 32; ++d) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] *= share;
    store_columns<T>(Out, 32 * d, a.head_dim, o[d], h);
  }
}

template <typename T, int W, bool DIRECT, bool MASKED>
__global__ __launch_bounds__(64 * WAVES, W <= 128 && DIRECT ? 2 : 1) void attention_kernel(AttentionArgs a) {
#ifdef __HIP_DEVICE_COMPILE__          // buffer descriptors mean nothing to the host's pass
  attend<T, W, DIRECT, MASKED>(a);
#endif
}

__device__ __forceinline__ float max_of_wave(float v) {
#pragma unroll
  for (int e = 32; e > 0; e >>= 1) v = fmaxf(v, __shfl_xor(v, e));
  return v;
}

// Joins the parts of the keys, a wave for each query of the units that were split: lane l's columns are l, l + 64, ...
template <typename T, int W>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  const int lane = threadIdx.x % kWave;
  const int id = uniform(blockIdx.x * 4 + threadIdx.x / kWave), n = id / kTileQueries, i = id % kTileQueries;
  const Unit u(a, a.whole + n);
  const Rows queries(a.q_span, u.b, a.q_total, a.q_rows);
  const Query mine(a, u, i, queries.count);
  if (!mine.there) return;
  const int64_t first = (int64_t)n * a.parts * kTileQueries + i;
  constexpr int EACH = (W + 63) / 64, AT_ONCE = 8 / EACH;       // loads in flight
  const float* from = a.sums + first * W + lane;
  float x[AT_ONCE][EACH];
  const auto load = [&](int p0) INLINE {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (64 * e + lane < W) x[i][e] = from[(int64_t)min(p0 + i, a.parts - 1) * kTileQueries * W + 64 * e];
  };
  float top = -INFINITY, sum = 0.f;                            // of part `lane`
  if (lane < a.parts) {
    const float2 s = reinterpret_cast<const float2*>(a.stats)[first + lane * kTileQueries];
    top = s.x, sum = s.y;
  }
  load(0);
  float distance = top - max_of_wave(top);
  const bool large = top != -INFINITY && !(fabsf(top) < LARGE);
  if (__builtin_amdgcn_ballot_w64(large)) {                    // their own differences are too coarse, or none
    const float product = large ? a.large[first + lane * kTileQueries] : (top - SLACK) / a.scale;
    distance = (product - max_of_wave(product)) * a.scale;
  }
  const float weight = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(distance);
  const float total = wave_sum(top == -INFINITY ? 0.f : weight * sum);
  float o[EACH] = {};
  for (int p0 = 0; p0 < a.parts; p0 += AT_ONCE) {
    if (p0) load(p0);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const float w = __shfl(weight, (p0 + i) % kWave);        // 0 for a part without keys, whose sums are zeros, and where float32 ends: times a NaN still NaN
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (64 * e + lane < W && p0 + i < a.parts) o[e] = __builtin_fmaf(w, x[i][e], o[e]);
    }
  }
  const float share = total == 0.f ? 0.f : 1.f / total;
  T* Out = static_cast<T*>(a.Out) + ((a.q_span ? 0 : u.b * a.o.seq) + mine.at(a.o, queries.first));
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (64 * e + lane < a.head_dim) st_elem(Out, 64 * e + lane, o[e] * share);
}

template <typename T, int W, bool DIRECT>
void attention_masked(const AttentionArgs& a, unsigned grid, hipStream_t st) {
  a.mask ? attention_kernel<T, W, DIRECT, true><<<grid, 64 * WAVES, 0, st>>>(a) : attention_kernel<T, W, DIRECT, false><<<grid, 64 * WAVES, 0, st>>>(a);
}

template <typename T, int W>
void attention_of(const AttentionArgs& a, bool direct, hipStream_t st) {
  const int rest = a.units - a.whole;
  const unsigned grid = (unsigned)(a.whole + rest * a.parts);
  direct ? attention_masked<T, W, true>(a, grid, st) : attention_masked<T, W, false>(a, grid, st);
  if (rest) attention_join_kernel<T, W><<<rest * (kTileQueries / 4), 256, 0, st>>>(a);
}

template <typename T>
void attention_by_width(const AttentionArgs& a, bool direct, hipStream_t st) {
  switch (attention_width(a.head_dim)) {
    case 64: attention_of<T, 64>(a, direct, st); break;
    case 96: attention_of<T, 96>(a, direct, st); break;
    case 128: attention_of<T, 128>(a, direct, st); break;
    default: attention_of<T, 256>(a, direct, st); break;
  }
}

// Queries of all parts: a multiple of 128.  Their sums, their statistics and their large shifts' products lie one behind the other.
size_t part_queries(const AttentionPlan& plan) { return (size_t)(plan.units - plan.whole) * plan.parts * kTileQueries; }

}  // namespace

size_t attention_workspace_bytes(const svdc_attention& p) {
  const AttentionPlan plan = attention_plan(p, num_compute_units());
  return part_queries(plan) * (attention_width(p.head_dim) + 3) * sizeof(float);
}

int32_t launch_attention(const svdc_attention& p, const void* Q, const void* K, const void* V, const int32_t* q_span, const int32_t* k_span,
                         const uint8_t* key_mask, void* Out, void* workspace, hipStream_t st) {
  const AttentionPlan plan = attention_plan(p, num_compute_units());
  const int64_t unit = p.dtype == SVDC_F32 ? 4 : 8;
  const auto sixteen = [&](const void* x, const svdc_heads& s, bool spans) {
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && s.row % unit == 0 && s.head % unit == 0 && (spans || s.seq % unit == 0);
  };
  const bool direct = p.head_dim % unit == 0 && sixteen(Q, p.q, q_span) && sixteen(K, p.k, k_span) && sixteen(V, p.v, k_span);
  float* const stats = static_cast<float*>(workspace) + part_queries(plan) * attention_width(p.head_dim);
  const AttentionArgs a{Q, K, V, Out, reinterpret_cast<const int2*>(q_span), reinterpret_cast<const int2*>(k_span), key_mask,
                        static_cast<float*>(workspace), stats, stats + 2 * part_queries(plan),
                        p.q_total, p.k_total, p.q, p.k, p.v, p.o, p.kv_heads, p.heads / p.kv_heads, p.head_dim, (int)p.q_rows, (int)p.k_rows,
                        plan.q_tiles, plan.whole, plan.units, plan.parts, plan.tiles_of_part, p.scale * 1.4426950408889634f};
  p.dtype == SVDC_F32 ? attention_by_width<float>(a, direct, st) : attention_by_width<bf16_t>(a, direct, st);
  return launch_status();
}

}  // namespace svdc
