// Heads of queries and keys on their way into the attention: angles of a rotation with several position axes (svdcache_rotary_table), norm and
// rotation of each head in one pass (svdcache_norm_rotate).
//
// Both stream their rows once and reuse next to nothing.
#include <algorithm>

#include "eight_bit.h"
#include "svdc_internal.h"

namespace svdc {

namespace {

constexpr int kMaxPairs = 128;

// ---- angles -----------------------------------------------------------------------------------------------------------

struct RotaryArgs {
  const void* pos;
  float* table;
  int64_t rows, ld;
  int axes, pairs;
  int first[SVDC_MAX_AXES + 1];       // pair at which an axis begins
  double theta[SVDC_MAX_AXES];
};

// cos and sin of 2 pi t.  t is reduced to an eighth of a turn around the next quarter in 64 bits, where nothing is lost; what is left has
// 2^-28 of a turn of rounding as a float32.
__device__ __forceinline__ float2 turn(double t) {
  const double quarter = rint(4.0 * t);
  const float x = (float)(t - 0.25 * quarter);
  float s, c;
  sincospif(2.f * x, &s, &c);
  const int q = (int)(quarter - 4.0 * floor(0.25 * quarter));
  const float2 half = q & 1 ? float2{-s, c} : float2{c, s};
  return q & 2 ? float2{-half.x, -half.y} : half;
}

// A workgroup makes the frequencies of all pairs once, in turns, and then takes rows in turn.
template <typename T>
__global__ __launch_bounds__(256) void rotary_table_kernel(RotaryArgs a) {
  __shared__ double turns[kMaxPairs];
  __shared__ int axis_of[kMaxPairs];
  for (int j = threadIdx.x; j < a.pairs; j += 256) {
    int axis = 0;
#pragma unroll
    for (int k = 1; k < SVDC_MAX_AXES; ++k)
      if (k < a.axes && j >= a.first[k]) axis = k;
    const int i = j - a.first[axis], n = a.first[axis + 1] - a.first[axis];
    turns[j] = pow(a.theta[axis], -(double)i / n) * 0.15915494309189533577;   // 1 / (2 pi)
    axis_of[j] = axis;
  }
  __syncthreads();
  const T* pos = static_cast<const T*>(a.pos);
  const int rows_at_once = 256 / a.pairs, r = threadIdx.x / a.pairs, j = threadIdx.x % a.pairs;
  if (r >= rows_at_once) return;
  const double step = turns[j];
  const int axis = axis_of[j];
  for (int64_t row = (int64_t)blockIdx.x * rows_at_once + r; row < a.rows; row += (int64_t)gridDim.x * rows_at_once)
    reinterpret_cast<float2*>(a.table)[row * a.pairs + j] = turn((double)pos[row * a.ld + axis] * step);
}

// ---- norm and rotation ------------------------------------------------------------------------------------------------

struct HeadsArgs {
  const void *q, *k, *v;
  void *qo, *ko, *vo;
  const float *gain_q, *gain_k, *table;
  int64_t all_rows, table_seq;
  svdc_heads sq, sk, sv, sqo, sko, svo;
  int rows, heads, kv_heads, head_dim, norm, pairs;
  float eps;
};

// How the columns of a head lie in its lanes: 8 to a lane, as four pairs.  Anywhere: pairs lane, lane + G, ..., column by column.  The others want
// head_dim in eights and turned pairs in fours, and load whole words: four pairs of neighbours are 8 columns in a row, of halves twice 4.
enum Columns { kAnywhere, kNeighbours, kHalves };

// Pair `j` of all (turned ones first, then what is left by twos) -> its columns; `to` may be beyond the last column
__device__ __forceinline__ void columns_of(int j, int pairs, bool halves, int& from, int& to) {
  const bool split = halves && j < pairs;
  from = split ? j : 2 * j;
  to = split ? pairs + j : 2 * j + 1;
}

__device__ __forceinline__ float bits_of(const float* p) { return *p; }
__device__ __forceinline__ float bits_of(const bf16_t* p) { return (float)*p; }

// four columns in a row, at any alignment of an element
__device__ __forceinline__ void load4(const bf16_t* p, float* v) {
  typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
  const u32x2_any w = *reinterpret_cast<const u32x2_any*>(p);
  v[0] = bf16_lo(w[0]), v[1] = bf16_hi(w[0]), v[2] = bf16_lo(w[1]), v[3] = bf16_hi(w[1]);
}
__device__ __forceinline__ void load4(const float* p, float* v) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  const f32x4_any w = *reinterpret_cast<const f32x4_any*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = w[i];
}
__device__ __forceinline__ void load8(const bf16_t* p, float* v) {
  const u32x4_any w = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
}
__device__ __forceinline__ void load8(const float* p, float* v) { load4(p, v), load4(p + 4, v + 4); }
__device__ __forceinline__ void store4(bf16_t* p, const float* v) {
  typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
  *reinterpret_cast<u32x2_any*>(p) = u32x2_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const float* v) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float* v) {
  *reinterpret_cast<u32x4_any*>(p) = u32x4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* p, const float* v) { store4(p, v), store4(p + 4, v + 4); }

// A lane's columns of a head, v[2 t] and v[2 t + 1] the columns of its t-th pair
template <int G, Columns C>
struct Lane {
  int first;                // kNeighbours: its 8 columns; kHalves: its first four of either half, or its 8 columns behind them
  int pairs, head_dim;
  bool halves, split, there;

  __device__ __forceinline__ Lane(const HeadsArgs& a, int lane, bool halves) : pairs(a.pairs), head_dim(a.head_dim), halves(halves) {
    first = C == kAnywhere ? lane : 8 * lane;
    there = C == kAnywhere || first < head_dim;
    split = C == kHalves && 4 * lane < pairs;
    if (split) first = 4 * lane;
  }
  // what `f` makes of (pair t, its columns in v's order): for the tables and gains
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      int j, from, to;
      if (C == kAnywhere) {
        j = first + t * G;
        columns_of(j, pairs, halves, from, to);
      } else if (C == kHalves && split) {
        j = from = first + t, to = pairs + from;
      } else {
        j = first / 2 + t, from = first + 2 * t, to = from + 1;
      }
      f(t, j, from, to);
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* p, float (&v)[8]) const {
    if (C == kAnywhere) {
      each([&](int t, int, int from, int to) {
        v[2 * t] = from < head_dim ? bits_of(p + from) : 0.f;
        v[2 * t + 1] = to < head_dim ? bits_of(p + to) : 0.f;
      });
    } else if (!there) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else if (C == kHalves && split) {
      float lo[4], hi[4];
      load4(p + first, lo);
      load4(p + pairs + first, hi);
#pragma unroll
      for (int t = 0; t < 4; ++t) v[2 * t] = lo[t], v[2 * t + 1] = hi[t];
    } else {
      load8(p + first, v);
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* p, const float (&v)[8]) const {
    if (C == kAnywhere) {
      each([&](int t, int, int from, int to) {
        if (from < head_dim) st_elem(p, from, v[2 * t]);
        if (to < head_dim) st_elem(p, to, v[2 * t + 1]);
      });
    } else if (!there) {
    } else if (C == kHalves && split) {
      const float lo[4] = {v[0], v[2], v[4], v[6]}, hi[4] = {v[1], v[3], v[5], v[7]};
      store4(p + first, lo);
      store4(p + pairs + first, hi);
    } else {
      store8(p + first, v);
    }
  }
};

// sum over G lanes in a row, G a power of two up to 32, in all of them
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#define SVDC_DPP_ADD(control) v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), control, 0xf, 0xf, false))
  if (G >= 2) SVDC_DPP_ADD(0xb1);    // quad_perm 1 0 3 2
  if (G >= 4) SVDC_DPP_ADD(0x4e);    // quad_perm 2 3 0 1
  if (G >= 8) SVDC_DPP_ADD(0x141);   // eight lanes mirrored: the other quad
  if (G >= 16) SVDC_DPP_ADD(0x140);  // sixteen lanes mirrored: the other eight
#undef SVDC_DPP_ADD
  if (G >= 32) v += __shfl_xor(v, 16, 32);
  return v;
}

// A workgroup takes a row at a time: G lanes a head, 64 / G heads a wave, the four waves the heads of Q, K and V in turn, AT_ONCE turns of loads in flight.
// The gains stay in registers.
template <typename TI, typename TO, int G, Columns C>
__global__ __launch_bounds__(256) void norm_rotate_kernel(HeadsArgs a, int layout) {
  constexpr int EACH = kWave / G, AT_ONCE = 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), in_wave = threadIdx.x % kWave, mine = in_wave / G;
  const Lane<G, C> lane(a, in_wave % G, layout == SVDC_PAIRS_HALVES);
  const int turns_q = a.q ? (a.heads + EACH - 1) / EACH : 0, turns_k = a.k ? (a.kv_heads + EACH - 1) / EACH : 0,
            turns = turns_q + turns_k + (a.v ? (a.kv_heads + EACH - 1) / EACH : 0);
  float gain[2][8];
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const float* g = a.norm ? (part ? a.gain_k : a.gain_q) : nullptr;
    lane.each([&](int t, int, int from, int to) {
      gain[part][2 * t] = g && from < a.head_dim ? g[from] : 1.f;
      gain[part][2 * t + 1] = g && to < a.head_dim ? g[to] : 1.f;
    });
  }
  bool turned[4];                 // what is not stays as it is, infinities beside it or not
  lane.each([&](int t, int j, int, int) { turned[t] = j < a.pairs; });
  const float share = 1.f / (float)a.head_dim;
  for (int64_t at = blockIdx.x; at < a.all_rows; at += gridDim.x) {
    const int b = __builtin_amdgcn_readfirstlane((uint32_t)at / (uint32_t)a.rows), row = (int)at - b * a.rows;
    float2 turn_by[4];
    {
      const float2* table = reinterpret_cast<const float2*>(a.table) + (b * a.table_seq + (int64_t)row * a.pairs);
      lane.each([&](int t, int j, int, int) { turn_by[t] = turned[t] ? table[j] : float2{1.f, 0.f}; });
    }
    for (int turn0 = wave; turn0 < turns; turn0 += 4 * AT_ONCE) {
      float v[AT_ONCE][8];
      // part and head of a turn, the first of its heads; none beyond the last
      const auto head_of = [&](int i, int& part, int& first) {
        int turn = turn0 + 4 * i;
        part = turn < turns_q ? 0 : turn < turns_q + turns_k ? 1 : 2;
        turn -= part == 0 ? 0 : part == 1 ? turns_q : turns_q + turns_k;
        first = turn * EACH;
        const int head = first + mine;
        return turn0 + 4 * i < turns && head < (part ? a.kv_heads : a.heads) ? head : -1;
      };
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        int part, first;
        const int head = head_of(i, part, first);
        const svdc_heads& s = part == 0 ? a.sq : part == 1 ? a.sk : a.sv;
        const TI* p = static_cast<const TI*>(part == 0 ? a.q : part == 1 ? a.k : a.v) + (b * s.seq + row * s.row + first * s.head) + mine * s.head;
        if (head >= 0) {
          lane.load(p, v[i]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        int part, first;
        const int head = head_of(i, part, first);
        if (part < 2) {                                        // the same for all lanes
          if (a.norm) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(v[i][e], v[i][e], sum);
            const float inv = 1.f / sqrtf(__builtin_fmaf(group_sum<G>(sum), share, a.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * inv * (part ? gain[1][e] : gain[0][e]);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float x = v[i][2 * t], y = v[i][2 * t + 1];
            if (turned[t]) {
              v[i][2 * t] = __builtin_fmaf(x, turn_by[t].x, -(y * turn_by[t].y));
              v[i][2 * t + 1] = __builtin_fmaf(x, turn_by[t].y, y * turn_by[t].x);
            }
          }
        }
        const svdc_heads& s = part == 0 ? a.sqo : part == 1 ? a.sko : a.svo;
        TO* p = static_cast<TO*>(part == 0 ? a.qo : part == 1 ? a.ko : a.vo) + (b * s.seq + row * s.row + first * s.head) + mine * s.head;
        if (head >= 0) lane.store(p, v[i]);
      }
    }
  }
}

// Workgroups for rows in turn: six to a compute unit keep it busy and read the gains seldom.
template <typename TI, typename TO, int G>
void norm_rotate_in(const HeadsArgs& a, int layout, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(a.all_rows, 6 * num_compute_units());
  if (a.head_dim % 8 || a.pairs % 4)
    norm_rotate_kernel<TI, TO, G, kAnywhere><<<grid, 256, 0, st>>>(a, layout);
  else if (layout == SVDC_PAIRS_HALVES && a.pairs)
    norm_rotate_kernel<TI, TO, G, kHalves><<<grid, 256, 0, st>>>(a, layout);
  else
    norm_rotate_kernel<TI, TO, G, kNeighbours><<<grid, 256, 0, st>>>(a, layout);
}

template <typename TI, typename TO>
void norm_rotate(const HeadsArgs& a, int layout, hipStream_t st) {
  if (a.head_dim <= 8)
    norm_rotate_in<TI, TO, 1>(a, layout, st);
  else if (a.head_dim <= 32)
    norm_rotate_in<TI, TO, 4>(a, layout, st);
  else if (a.head_dim <= 64)
    norm_rotate_in<TI, TO, 8>(a, layout, st);
  else if (a.head_dim <= 128)
    norm_rotate_in<TI, TO, 16>(a, layout, st);
  else
    norm_rotate_in<TI, TO, 32>(a, layout, st);
}

}  // namespace

int32_t launch_rotary_table(const svdc_rotary& p, const void* pos, float* table, hipStream_t st) {
  RotaryArgs a{pos, table, p.rows, p.ld, p.axes, 0, {}, {}};
  for (int k = 0; k < p.axes; ++k) {
    a.first[k] = a.pairs;
    a.pairs += p.dims[k] / 2;
    a.first[k + 1] = a.pairs;
    a.theta[k] = p.theta[k];
  }
  const int64_t turns = (p.rows + 256 / a.pairs - 1) / (256 / a.pairs);
  const unsigned grid = (unsigned)std::min<int64_t>(turns, 8 * num_compute_units());
  if (p.whole)
    rotary_table_kernel<int32_t><<<grid, 256, 0, st>>>(a);
  else
    rotary_table_kernel<float><<<grid, 256, 0, st>>>(a);
  return launch_status();
}

int32_t launch_norm_rotate(const svdc_norm_rotate& p, const void* Q, const void* K, const void* V, const float* gain_q, const float* gain_k,
                           const float* table, void* Qo, void* Ko, void* Vo, hipStream_t st) {
  const HeadsArgs a{Q,   K,   V,   Qo,   Ko,   Vo,   gain_q,      gain_k,  table,      p.batch * p.rows, p.table_seq, p.q,
                    p.k, p.v, p.qo, p.ko, p.vo, (int)p.rows, p.heads, p.kv_heads, p.head_dim,       p.norm,      p.pairs,
                    p.eps};
  if (p.dtype == SVDC_F32)
    p.dtype_out == SVDC_F32 ? norm_rotate<float, float>(a, p.layout, st) : norm_rotate<float, bf16_t>(a, p.layout, st);
  else
    p.dtype_out == SVDC_F32 ? norm_rotate<bf16_t, float>(a, p.layout, st) : norm_rotate<bf16_t, bf16_t>(a, p.layout, st);
  return launch_status();
}

}  // namespace svdc
