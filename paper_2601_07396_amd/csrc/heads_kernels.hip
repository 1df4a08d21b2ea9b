// Heads of queries and keys on their way into the attention: angles of a rotation with several position axes (svdcache_rotary_table), norm and
// rotation of each head in one pass (svdcache_norm_rotate).
//
// Both stream their rows once and reuse next to nothing.  Norm and rotation are bound by memory (a copy of 1 GiB reaches 5.2 TB/s):
//     4608 rows, 24 + 24 heads of 128, bfloat16 (116 MB) 25.7 us, 4.5 TB/s, 21.9 of it in the kernel; 4 x 4096 rows, float32 into bfloat16 with values (908 MB) 172 us, 5.3 TB/s
//     odd heads: 3 x 1001 rows, 16 + 8 heads of 72, 27 pairs of halves, float32 (42 MB) 12.7 us; one row 4.1 us, a launch
// The angles: 119056 x 64 pairs (62 MB) 16-17 us, 3.8 TB/s; 4608 x 64 4.1 us.  Of 17.2 us the stores alone, 8 bytes a lane, take 13.7 (4.5 TB/s), the powers in 64 bits that every
// workgroup begins with 2.7, and reduction and series beside the stores 1.4 (each left out in turn).
#include <algorithm>
#include <cmath>

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
  double theta[SVDC_MAX_AXES], log_theta[SVDC_MAX_AXES];      // by the number of the axis' pairs
};

// cos and sin of 2 pi t.  t is reduced to an eighth of a turn around the next quarter in 64 bits, where nothing is lost; what is left, 2^-28 of a turn off as a
// float32, goes into the first terms of the two Taylor series: at pi / 4 the next ones are 2^-29 (sine) and 2^-33 (cosine).
__device__ __forceinline__ float2 turn(double t) {
  const double whole = t - rint(t), quarter = rint(4.0 * whole);
  const float x = (float)__builtin_fma(quarter, -0.25, whole) * 6.2831853f, y = x * x;
  const float s = x * __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 2.7557319e-6f, -1.984127e-4f), 8.3333333e-3f), -0.16666667f), 1.f);
  const float c = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const int q = (int)quarter;
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
    // What rounding the exponent left out, (-i - e n) / n, counts ln(theta) times: theta^(e + r) = theta^e (1 + r ln(theta)).
    const double e = -(double)i / n;
    float left = (float)(__builtin_fma(-e, n, -i) * a.log_theta[axis]);
    asm volatile("" : "+v"(left));                            // one register across the power, where all are in use
    const double power = pow(a.theta[axis], e);
    turns[j] = __builtin_fma(power, left, power) * 0.15915494309189533577;   // 1 / (2 pi)
    axis_of[j] = axis;
  }
  __syncthreads();
  const T* pos = static_cast<const T*>(a.pos);
  const int rows_at_once = 256 / a.pairs, r = threadIdx.x / a.pairs, j = threadIdx.x % a.pairs;
  if (r >= rows_at_once) return;
  const double step = turns[j];
  const int axis = axis_of[j];
  const int64_t stride = (int64_t)gridDim.x * rows_at_once;
  const T* from = pos + axis;
  float2* to = reinterpret_cast<float2*>(a.table) + j;
  int64_t row = (int64_t)blockIdx.x * rows_at_once + r;
  for (; row + 3 * stride < a.rows; row += 4 * stride) {
    T x[4];                                 // four rows' positions in flight
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = from[(row + i * stride) * a.ld];
#pragma unroll
    for (int i = 0; i < 4; ++i) to[(row + i * stride) * a.pairs] = turn((double)x[i] * step);
  }
  for (; row < a.rows; row += stride) to[row * a.pairs] = turn((double)from[row * a.ld] * step);
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

// How the columns of a head lie in its lanes: 8 to a lane, as four pairs.  Neighbours and halves want head_dim in eights and turned pairs in fours, and load whole words: four pairs
// of neighbours are 8 columns in a row, of halves twice 4.  Odd ones are at home anywhere: pairs lane, lane + G, ..., a pair or a column at a time.
enum Columns { kNeighbours, kHalves, kOddNeighbours, kOddHalves };
constexpr bool odd_columns(Columns c) { return c == kOddNeighbours || c == kOddHalves; }

// Pair `j` of all (turned ones first, then what is left by twos) -> its columns; `to` may be beyond the last column
__device__ __forceinline__ void columns_of(int j, int pairs, bool halves, int& from, int& to) {
  const bool split = halves && j < pairs;
  from = split ? j : 2 * j;
  to = split ? pairs + j : 2 * j + 1;
}

// four or eight columns in a row as they lie in memory, at any alignment of an element
template <int N>
__device__ __forceinline__ void load_words(const void* p, uint32_t* w) {
  typedef uint32_t words __attribute__((ext_vector_type(N), aligned(2)));
  const words x = *static_cast<const words*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = x[i];
}
template <int N>
__device__ __forceinline__ void store_words(void* p, const uint32_t* w) {
  typedef uint32_t words __attribute__((ext_vector_type(N), aligned(2)));
  words x;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = w[i];
  *static_cast<words*>(p) = x;
}

// A lane's columns of a head, in the end v[2 t] and v[2 t + 1] the columns of its t-th pair
template <int G, Columns C>
struct Lane {
  int first;                // kNeighbours: its 8 columns; kHalves: its first four of either half, or its 8 columns behind them
  int pairs, head_dim;
  bool split, there;

  __device__ __forceinline__ Lane(const HeadsArgs& a, int lane) : pairs(a.pairs), head_dim(a.head_dim) {
    first = odd_columns(C) ? lane : 8 * lane;
    there = odd_columns(C) || first < head_dim;
    split = C == kHalves && 4 * lane < pairs;
    if (split) first = 4 * lane;
  }
  // f(t, which of all pairs, its columns) for each of the lane's pairs
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      int j, from, to;
      if (odd_columns(C)) {
        j = first + t * G;
        columns_of(j, pairs, C == kOddHalves, from, to);
      } else if (C == kHalves && split) {
        j = from = first + t, to = pairs + from;
      } else {
        j = first / 2 + t, from = first + 2 * t, to = from + 1;
      }
      f(t, j, from, to);
    }
  }
  // What lies in memory stays as it is until it is worked on: half the registers for bfloat16.
  template <typename T>
  static constexpr int words = odd_columns(C) ? 8 : 2 * (int)sizeof(T);
  template <typename T>
  __device__ __forceinline__ void load(const T* p, bool present, uint32_t (&w)[words<T>]) const {
    constexpr int N = words<T>;
    if (odd_columns(C)) {
      each([&](int t, int, int from, int to) {
        if (C == kOddNeighbours && to < head_dim) {                 // two columns in a row
          uint32_t both[2] = {};
          if (present) load_words<(int)sizeof(T) / 2>(p + from, both);
          w[2 * t] = sizeof(T) == 4 ? both[0] : both[0] << 16;
          w[2 * t + 1] = sizeof(T) == 4 ? both[1] : both[0] & 0xffff0000u;
        } else {
          w[2 * t] = __float_as_uint(present && from < head_dim ? ld_elem(p, from) : 0.f);
          w[2 * t + 1] = __float_as_uint(present && to < head_dim ? ld_elem(p, to) : 0.f);
        }
      });
    } else if (!(present && there)) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = 0;
    } else if (C == kHalves && split) {
      load_words<N / 2>(p + first, w);
      load_words<N / 2>(p + pairs + first, w + N / 2);
    } else {
      load_words<4>(p + first, w);
      if (N == 8) load_words<4>(reinterpret_cast<const uint32_t*>(p + first) + 4, w + N / 2);
    }
  }
  template <typename T>
  __device__ __forceinline__ void unpack(const uint32_t (&w)[words<T>], float (&v)[8]) const {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = odd_columns(C) || sizeof(T) == 4 ? __uint_as_float(w[i % words<T>]) : i % 2 ? bf16_hi(w[i / 2 % words<T>]) : bf16_lo(w[i / 2 % words<T>]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool apart = C == kHalves && split;
      v[2 * t] = apart ? x[t] : x[2 * t];
      v[2 * t + 1] = apart ? x[4 + t] : x[2 * t + 1];
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* p, const float (&v)[8]) const {
    if (odd_columns(C)) {
      each([&](int t, int, int from, int to) {
        if (C == kOddNeighbours && to < head_dim) {
          const uint32_t both[2] = {sizeof(T) == 4 ? __float_as_uint(v[2 * t]) : pack_bf16(v[2 * t], v[2 * t + 1]), __float_as_uint(v[2 * t + 1])};
          store_words<(int)sizeof(T) / 2>(p + from, both);
        } else {
          if (from < head_dim) st_elem(p, from, v[2 * t]);
          if (to < head_dim) st_elem(p, to, v[2 * t + 1]);
        }
      });
      return;
    }
    if (!there) return;
    constexpr int N = 2 * (int)sizeof(T);
    const bool apart = C == kHalves && split;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = apart ? v[2 * (i % 4) + i / 4] : v[i];
    uint32_t w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(x[i % 8]) : pack_bf16(x[2 * i % 8], x[(2 * i + 1) % 8]);
    if (apart) {
      store_words<N / 2>(p + first, w);
      store_words<N / 2>(p + pairs + first, w + N / 2);
    } else {
      store_words<4>(p + first, w);
      if (N == 8) store_words<4>(reinterpret_cast<uint32_t*>(p + first) + 4, w + N / 2);
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

// One of the three tensors.  A wave takes a row, G lanes a head, 64 / G heads at a time, AT_ONCE times that in flight, or as many rows of fewer heads; the table's part and the gain
// stay in registers.
template <typename TI, typename TO, int G, Columns C>
__device__ __forceinline__ void rows_of_heads(const HeadsArgs& a, const void* in, void* out, const svdc_heads& si, const svdc_heads& so, int heads, const float* gains, bool norm,
                                              bool rotate) {
  constexpr int EACH = kWave / G, AT_ONCE = odd_columns(C) || C == kHalves ? 2 : G == 32 && sizeof(TI) == 4 ? 4 : 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), in_wave = threadIdx.x % kWave, mine = in_wave / G;
  const Lane<G, C> lane(a, in_wave % G);
  float gain[8];
  bool turned[4];                 // what is not stays as it is, infinities beside it or not
  lane.each([&](int t, int j, int from, int to) {
    gain[2 * t] = gains && from < a.head_dim ? gains[from] : 1.f;
    gain[2 * t + 1] = gains && to < a.head_dim ? gains[to] : 1.f;
    turned[t] = rotate && j < a.pairs;
  });
  const float share = 1.f / (float)a.head_dim;
  const int rows_at_once = heads < EACH ? EACH / heads : 1, row_mine = heads < EACH ? mine / heads : 0, head_mine = heads < EACH ? mine % heads : mine;
  const int64_t lane_in = head_mine * si.head, lane_out = head_mine * so.head;
  for (int64_t at0 = ((int64_t)blockIdx.x * 4 + wave) * rows_at_once; at0 < a.all_rows; at0 += (int64_t)gridDim.x * 4 * rows_at_once) {
    const bool here = row_mine < rows_at_once && at0 + row_mine < a.all_rows;
    const int at = (int)(here ? at0 + row_mine : at0), b = a.all_rows == a.rows ? 0 : (int)((uint32_t)at / (uint32_t)a.rows), row = at - b * a.rows;
    const TI* from = static_cast<const TI*>(in) + (b * si.seq + row * si.row) + lane_in;
    TO* to = static_cast<TO*>(out) + (b * so.seq + row * so.row) + lane_out;
    float2 turn_by[4];
    const float2* table = reinterpret_cast<const float2*>(a.table) + (b * a.table_seq + (int64_t)row * a.pairs);
    lane.each([&](int t, int j, int, int) { turn_by[t] = turned[t] ? table[j] : float2{1.f, 0.f}; });
    for (int head0 = 0; head0 < heads; head0 += AT_ONCE * EACH) {
      uint32_t w[AT_ONCE][Lane<G, C>::template words<TI>];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int head = head0 + i * EACH;
        if (head < heads) lane.load(from + head * si.head, here && head + head_mine < heads, w[i]);
      }
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int head = head0 + i * EACH;
        if (head >= heads) break;                              // for all lanes
        float v[8];
        lane.template unpack<TI>(w[i], v);
        if (norm) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(v[e], v[e], sum);
          const float mean = __builtin_fmaf(group_sum<G>(sum), share, a.eps);
          const float inv = __builtin_amdgcn_rsqf(mean < 1.17549435e-38f ? 1.17549435e-38f : mean);   // no number stays none
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = v[e] * inv * gain[e];
        }
        if (rotate) {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float x = v[2 * t], y = v[2 * t + 1];
            if (turned[t]) {
              v[2 * t] = __builtin_fmaf(x, turn_by[t].x, -(y * turn_by[t].y));
              v[2 * t + 1] = __builtin_fmaf(x, turn_by[t].y, y * turn_by[t].x);
            }
          }
        }
        if (here && head + head_mine < heads) lane.store(to + head * so.head, v);
      }
    }
  }
}

// blockIdx.y: which of the tensors that are there
template <typename TI, typename TO, int G, Columns C>
__global__ __launch_bounds__(256, odd_columns(C) ? 3 : 4) void norm_rotate_kernel(HeadsArgs a) {
  int part = blockIdx.y;
  if (!a.q) ++part;
  if (!a.k && part >= 1) ++part;
  const bool q = part == 0, k = part == 1;
  rows_of_heads<TI, TO, G, C>(a, q ? a.q : k ? a.k : a.v, q ? a.qo : k ? a.ko : a.vo, q ? a.sq : k ? a.sk : a.sv, q ? a.sqo : k ? a.sko : a.svo, q ? a.heads : a.kv_heads,
                              !a.norm ? nullptr : q ? a.gain_q : k ? a.gain_k : nullptr, a.norm && part < 2, a.pairs > 0 && part < 2);
}

template <typename TI, typename TO, int G>
void norm_rotate_in(const HeadsArgs& a, int layout, hipStream_t st) {
  const auto waves = [&](int heads) { return (a.all_rows * std::min(heads, kWave / G) + kWave / G - 1) / (kWave / G); };      // about
  const int64_t most = std::max(a.q ? waves(a.heads) : 0, a.k || a.v ? waves(a.kv_heads) : 0);
  const dim3 grid((unsigned)std::min<int64_t>((most + 3) / 4, 1 << 20), (a.q != nullptr) + (a.k != nullptr) + (a.v != nullptr));
  const bool halves = layout == SVDC_PAIRS_HALVES && a.pairs, odd = a.head_dim % 8 || a.pairs % 4;
  if (odd)
    halves ? norm_rotate_kernel<TI, TO, G, kOddHalves><<<grid, 256, 0, st>>>(a) : norm_rotate_kernel<TI, TO, G, kOddNeighbours><<<grid, 256, 0, st>>>(a);
  else
    halves ? norm_rotate_kernel<TI, TO, G, kHalves><<<grid, 256, 0, st>>>(a) : norm_rotate_kernel<TI, TO, G, kNeighbours><<<grid, 256, 0, st>>>(a);
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
  RotaryArgs a{pos, table, p.rows, p.ld, p.axes, 0, {}, {}, {}};
  for (int k = 0; k < p.axes; ++k) {
    a.first[k] = a.pairs;
    a.pairs += p.dims[k] / 2;
    a.first[k + 1] = a.pairs;
    a.theta[k] = p.theta[k];
    a.log_theta[k] = std::log(p.theta[k]) / (p.dims[k] / 2);
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
