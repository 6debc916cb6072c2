// The InnerProduct layer in 8-bit integers, and its gradients from activations kept in 8 bits (include/mi355i8.h).
//
// Forward: sum_i c[n][i] v[o][i] by the integer matrix instructions, exact in 32 bits in any order; then s_n t_o, bias, ReLU, one rounding.
// Gradients: the scale of a row is on the side of dz in both,
//   dw[o][i] = sum_n (dz[n][o] s_n) c[n][i]      dx[n][i] = sum_o (dz[n][o] t_o) v[o][i]
// so the codes go into the bf16 matrix instructions as they are (whole numbers up to 127 are bf16's) and dz times the scale as terms that make it
// up: a bf16 dz and a scale of 8 bits have products of 16, two terms; others are rounded to fp32's 24, three terms.
#include <hip/hip_runtime.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "device_utils.h"
#include "elements.h"
#include "internal.h"
#include "mi355i8.h"
#include "wave_ops.h"

struct i8_desc {
  i8_params_t p;
  int64_t row;             // bytes of a row of codes
  int32_t fwd;             // FwdForm
  int32_t filter_tile, filter_splits, filter_per;  // backward filter: tile (rows and columns), workgroups that share a sum, steps of each
  int32_t data_tile, data_splits, data_per;        // backward data
  int32_t waves;           // of the forward pass by rows
  int32_t token;           // few rows are brought to 8 bits by the workgroups that multiply them
  size_t ws_bytes;
  char names[192];
};

namespace mi355conv {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kRowUnit = 128;          // bytes that a row of codes is a multiple of
constexpr int kMostInputs = 133120;    // 127^2 times this fits 32 bits
constexpr int kUnits = 256;            // compute units
constexpr int64_t kMaxElems = (int64_t)1 << 30;
constexpr int kMostBlocks = 1 << 21;   // of up to 1024 threads: a launch has fewer than 2^32

enum FwdForm { kRows, kTile64By4, kTile64By2, kTile128By2, kTile128, kTile256 };  // by: groups of waves that share the sums

// ---- rows to 8 bits ----

// The smallest number of 8 significant bits whose 127-fold reaches most, at least 2^-126; NaN where most is not finite.  The quotient is
// rounded to nearest: cut to 8 bits it is that number or the one below (127 times 8 bits are exact).
__device__ __forceinline__ float scale_for(float most) {
  if (!(most < INFINITY)) return NAN;
  const uint32_t down = __builtin_bit_cast(uint32_t, most / 127.f) & 0xffff0000u;
  const float lo = __builtin_bit_cast(float, down);
  return fmaxf(127.f * lo >= most ? lo : __builtin_bit_cast(float, down + 0x10000u), 0x1p-126f);
}

// The whole number nearest x / s, the even one of two.  x times the rounded reciprocal is within 2^-15 of the quotient; x - q s is exact in fp32
// (a multiple of the smaller one's last bit, not more than s), and says which side of a half x is on.
__device__ __forceinline__ int code_of(float x, float s, float inverse) {
  float q = rintf(x * inverse);
  const float left = fmaf(-q, s, x), twice = 2.f * fabsf(left);
  if (twice > s || (twice == s && ((int)q & 1))) q += copysignf(1.f, left);
  return (int)q;
}

// A vector's codes, four a word.  x / s plus 1.5 2^23 has the whole number in its last byte, and is one off at most, where x is as far from it as
// half a step or farther: hardly ever, and then all are looked at closely.
template <class E>
__device__ __forceinline__ void codes_of(const u32x4& vec, float s, float inverse, uint32_t (&w)[E::VEC / 4]) {
  float x[E::VEC], most = 0.f;
  uint32_t c[E::VEC];
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) {
    x[i] = E::get(vec, i);
    const float placed = fmaf(x[i], inverse, 0x1.8p23f), q = placed - 0x1.8p23f;
    c[i] = __builtin_bit_cast(uint32_t, placed);
    most = fmaxf(most, fabsf(fmaf(-q, s, x[i])));
  }
  if (!(most < 0.5f * s)) {
#pragma unroll
    for (int i = 0; i < E::VEC; ++i) c[i] = (uint32_t)code_of(x[i], s, inverse);
  }
#pragma unroll
  for (int i = 0; i < E::VEC / 4; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x04000c0cu);
    w[i] = s < INFINITY ? lo | hi : 0u;
  }
}

// The largest magnitude of a thread's vectors, as bits: of both halves of a word side by side where an element is 16 bits.  NaN is above infinity.
template <int DTYPE>
struct Most {
  typedef unsigned short Pair __attribute__((ext_vector_type(2)));
  uint32_t most = 0;

  __device__ __forceinline__ void look(const u32x4& vec) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t word = vec[i];
      if constexpr (DTYPE == MI355_F32)
        most = max(most, word & 0x7fffffffu);
      else
        most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Pair, most), __builtin_bit_cast(Pair, word & 0x7fff7fffu)));
    }
  }

  __device__ __forceinline__ uint32_t magnitude() const {  // fp32's bits
    if constexpr (DTYPE == MI355_F32) return most;
    const u32x4 both = {most, 0, 0, 0};
    return max(__builtin_bit_cast(uint32_t, Elem<DTYPE>::get(both, 0)), __builtin_bit_cast(uint32_t, Elem<DTYPE>::get(both, 1)));
  }
};

// THREADS threads for a row: its largest magnitude, then the codes, from registers for up to NV vectors a thread, read again beyond.  Bound by
// memory: 8192 x 4096 bf16 23 us, 4.4 TB/s.  THREADS 64: a wave for each row, four in a workgroup.  (A wave and 8 vectors a thread there: 32 us.)
template <int DTYPE, int THREADS, int NV>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void i8_quantise_kernel(const void* __restrict__ x, int8_t* __restrict__ codes, float* __restrict__ scales, int rows,
                                                          int k, int64_t row_bytes) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  constexpr int VEC = E::VEC;
  __shared__ uint32_t most_of[16];
  const int tid = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int step = THREADS == 64 ? gridDim.x * 4 : gridDim.x;
  const int vectors = (int)(row_bytes / VEC);
  for (int64_t r = THREADS == 64 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x; r < rows; r += step) {
    const T* const from = static_cast<const T*>(x) + r * k;
    auto load = [&](int v) {
      const int at = v * VEC;
      if (at + VEC <= k) return load_vec<E>(from + at);
      float f[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = at + i < k ? E::to_float(from[at + i]) : 0.f;
      return E::pack(f);
    };
    Most<DTYPE> seen;
    u32x4 held[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      held[j] = u32x4{0, 0, 0, 0};
      if (j * THREADS + tid < vectors) held[j] = load(j * THREADS + tid);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) seen.look(held[j]);
    for (int v = NV * THREADS + tid; v < vectors; v += THREADS) seen.look(load(v));
    uint32_t most = (uint32_t)wave_reduce((int)seen.magnitude(), 0, [](int a, int b) { return max(a, b); });
    if constexpr (THREADS > 64) {
      __syncthreads();
      if (lane == 0) most_of[wave] = most;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) most = max(most, most_of[w]);
    }
    const float s = scale_for(__builtin_bit_cast(float, most)), inverse = 1.f / s;
    if (tid == 0) scales[r] = s;
    int8_t* const to = codes + r * row_bytes;
    auto put = [&](const u32x4& vec, int v) {
      uint32_t w[VEC / 4];
      codes_of<E>(vec, s, inverse, w);
      if constexpr (VEC == 8)
        *reinterpret_cast<uint2*>(to + (int64_t)v * 8) = make_uint2(w[0], w[1]);
      else
        *reinterpret_cast<uint32_t*>(to + (int64_t)v * 4) = w[0];
    };
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * THREADS + tid < vectors) put(held[j], j * THREADS + tid);
    for (int v = NV * THREADS + tid; v < vectors; v += THREADS) put(load(v), v);
  }
}

template <int DTYPE>
int launch_quantise(const void* x, int8_t* codes, float* scales, int rows, int k, int64_t row, hipStream_t stream) {
  const int64_t vectors = row / Elem<DTYPE>::VEC;
  if (vectors <= 64 * 4)
    hipLaunchKernelGGL((i8_quantise_kernel<DTYPE, 64, 4>), dim3((uint32_t)std::min<int64_t>(((int64_t)rows + 3) / 4, kMostBlocks)), dim3(256), 0, stream, x, codes, scales, rows, k, row);
  else if (vectors > 256 * 4 && rows <= 2 * kUnits)  // (48 x 9216 fp32: 256 threads 7.6 us, 1024 4.8)
    hipLaunchKernelGGL((i8_quantise_kernel<DTYPE, 1024, 4>), dim3(rows), dim3(1024), 0, stream, x, codes, scales, rows, k, row);
  else
    hipLaunchKernelGGL((i8_quantise_kernel<DTYPE, 256, 4>), dim3(std::min(rows, kMostBlocks)), dim3(256), 0, stream, x, codes, scales, rows, k, row);
  return (int)hipGetLastError();
}

int quantise(const i8_desc* d, const void* x, int8_t* codes, float* scales, int rows, hipStream_t stream) {
  switch (d->p.dtype) {
    case MI355_F32: return launch_quantise<MI355_F32>(x, codes, scales, rows, d->p.k, d->row, stream);
    case MI355_F16: return launch_quantise<MI355_F16>(x, codes, scales, rows, d->p.k, d->row, stream);
    default: return launch_quantise<MI355_BF16>(x, codes, scales, rows, d->p.k, d->row, stream);
  }
}

// ---- forward ----

struct FwdArgs {
  const int8_t *codes, *w_codes;
  const float *scale, *w_scale;
  const void* bias;
  void* y;
  int64_t row;
  int32_t m, o, relu;
};

// One result: the scales one after the other, as their product may leave fp32 where the result does not; so would the sum's, below 2^31, with
// a scale of 2^97 and more, which therefore comes last.  (Scales are 2^-126 at least: nothing falls below fp32's normal numbers on the way.)
__device__ __forceinline__ float finish(int sum, float s, float t, float bias, int relu) {
  const bool large = s >= 0x1p96f;
  const float z = fmaf((float)sum * (large ? t : s), large ? s : t, bias);
  return relu ? (z > 0.f ? z : 0.f) : z;
}

// What the waves of a workgroup have found for 16 MT rows and 16 outputs, [waves][MT * 256] in `parts`, into the results.
template <class E, int MT>
__device__ __forceinline__ void join_waves(const FwdArgs& a, const int* parts, int waves, int o0, const float* scale) {
  for (int i = threadIdx.x; i < MT * 256; i += blockDim.x) {
    // (consecutive threads: consecutive outputs of a row)
    const int t = i >> 8, n = 16 * t + (i >> 4 & 15), out = o0 + (i & 15);
    if (n >= a.m || out >= a.o) continue;
    const int at = t * 256 + (i & 3) * 64 + ((i & 15) >> 2) * 16 + (i >> 4 & 15);
    int sum = 0;
#pragma unroll 4
    for (int p = 0; p < waves; ++p) sum += parts[p * MT * 256 + at];
    const float bias = a.bias ? E::to_float(static_cast<const typename E::T*>(a.bias)[out]) : 0.f;
    static_cast<typename E::T*>(a.y)[(int64_t)n * a.o + out] = E::from_float(finish(sum, scale[n], a.w_scale[out], bias, a.relu));
  }
}

// Up to 16 MT rows by 16 outputs in a workgroup, whose waves take the inputs in turn, 128 at a time, and add up through shared memory: nothing is used by two
// waves, and operands come from memory as the instructions take them, 16 inputs of a row or an output a lane, those of AHEAD turns at a time.
// Bound by the L2 caches, from which every workgroup reads all its rows' codes: 32 x 4096 -> 4096 9 us (and 4 to bring the rows to 8 bits), 17 MB of memory
// and 50 of L2.
template <int DTYPE, int MT>
__global__ __launch_bounds__(1024) void i8_rows_kernel(FwdArgs a) {
  typedef Elem<DTYPE> E;
  constexpr int AHEAD = MT == 1 ? 4 : 2;
  extern __shared__ int parts[];  // [waves][MT * 256]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int blocks = (int)(a.row / kRowUnit), tiles = (a.o + 15) / 16;
  for (int64_t item = blockIdx.x; item < tiles; item += gridDim.x) {
    const int o0 = (int)item * 16;
    const int8_t* const w = a.w_codes + (int64_t)min(o0 + (lane & 15), a.o - 1) * a.row + 16 * (lane >> 4);
    const int8_t* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = a.codes + (int64_t)min(16 * t + (lane & 15), a.m - 1) * a.row + 16 * (lane >> 4);
    i32x4 acc[MT] = {};
    auto turn = [&](int b0, auto count) {
      constexpr int N = decltype(count)::value;
      i32x4 wv[N][2], xv[N][MT][2];
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = (b0 + i * waves) * kRowUnit + 64 * h;
          wv[i][h] = *reinterpret_cast<const i32x4*>(w + at);
#pragma unroll
          for (int t = 0; t < MT; ++t) xv[i][t][h] = *reinterpret_cast<const i32x4*>(x[t] + at);
        }
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[i][h], xv[i][t][h], acc[t], 0, 0, 0);
    };
    int b = wave;
    for (; b + (AHEAD - 1) * waves < blocks; b += AHEAD * waves) turn(b, std::integral_constant<int, AHEAD>());
    if (AHEAD == 4 && b + waves < blocks) {
      turn(b, std::integral_constant<int, 2>());
      b += 2 * waves;
    }
    if (b < blocks) turn(b, std::integral_constant<int, 1>());
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) parts[(wave * MT + t) * 256 + r * 64 + lane] = acc[t][r];  // output 4 (lane / 16) + r, row lane % 16
    __syncthreads();
    join_waves<E, MT>(a, parts, waves, o0, a.scale);
  }
}

// Few rows that are not yet in 8 bits: every workgroup makes them so for itself, while its weights are on their way, and the first one leaves them for the
// caller.  Rows of codes in shared memory; a wave keeps up to kTokenAhead turns of weights in registers.  1 x 4096 -> 4096 6 us, of which memory would
// take 3.3.
constexpr int kTokenRows = 4, kTokenBytes = 32768, kTokenAhead = 4;

template <int DTYPE>
__global__ __launch_bounds__(1024) void i8_token_kernel(FwdArgs a, const void* __restrict__ x, int8_t* __restrict__ codes, float* __restrict__ scales, int k) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  constexpr int VEC = E::VEC;
  extern __shared__ __attribute__((aligned(16))) int8_t rows[];  // [m][row], then [waves][256] of sums
  __shared__ uint32_t most_of[kTokenRows][16];
  __shared__ float scale[kTokenRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int blocks = (int)(a.row / kRowUnit), row = (int)a.row, vectors = row / VEC;
  int o0 = blockIdx.x * 16;
  const int8_t* w;
  i32x4 wv[kTokenAhead][2] = {};
  auto ask = [&]() {
    w = a.w_codes + (int64_t)min(o0 + (lane & 15), a.o - 1) * a.row + 16 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < kTokenAhead; ++i)
      if (wave + i * waves < blocks) {
#pragma unroll
        for (int h = 0; h < 2; ++h) wv[i][h] = *reinterpret_cast<const i32x4*>(w + (wave + i * waves) * kRowUnit + 64 * h);
      }
  };
  ask();
  auto load = [&](int n, int v) {
    const T* const from = static_cast<const T*>(x) + (int64_t)n * k;
    const int at = v * VEC;
    if (at + VEC <= k) return load_vec<E>(from + at);
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = at + i < k ? E::to_float(from[at + i]) : 0.f;
    return E::pack(f);
  };
  for (int n = 0; n < a.m; ++n) {
    Most<DTYPE> seen;
    for (int v = tid; v < vectors; v += blockDim.x) seen.look(load(n, v));
    const uint32_t most = (uint32_t)wave_reduce((int)seen.magnitude(), 0, [](int p, int q) { return max(p, q); });
    if (lane == 0) most_of[n][wave] = most;
  }
  __syncthreads();
  for (int n = 0; n < a.m; ++n) {
    uint32_t most = 0;
    for (int p = 0; p < waves; ++p) most = max(most, most_of[n][p]);
    const float s = scale_for(__builtin_bit_cast(float, most)), inverse = 1.f / s;
    if (tid == 0) {
      scale[n] = s;
      if (blockIdx.x == 0) scales[n] = s;
    }
    for (int v = tid; v < vectors; v += blockDim.x) {
      uint32_t w[VEC / 4];
      codes_of<E>(load(n, v), s, inverse, w);
#pragma unroll
      for (int i = 0; i < VEC / 4; ++i) {
        reinterpret_cast<uint32_t*>(rows + n * row)[v * (VEC / 4) + i] = w[i];
        if (blockIdx.x == 0) reinterpret_cast<uint32_t*>(codes + (int64_t)n * row)[v * (VEC / 4) + i] = w[i];
      }
    }
  }
  __syncthreads();
  const int8_t* const mine = rows + min(lane & 15, a.m - 1) * row + 16 * (lane >> 4);
  int* const parts = reinterpret_cast<int*>(rows + a.m * row);
  for (;;) {
    i32x4 acc = {0, 0, 0, 0};
    auto multiply = [&](int b, const i32x4(&v)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[h], *reinterpret_cast<const i32x4*>(mine + b * kRowUnit + 64 * h), acc, 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kTokenAhead; ++i)
      if (wave + i * waves < blocks) multiply(wave + i * waves, wv[i]);
    for (int b = wave + kTokenAhead * waves; b < blocks; b += waves) {
      i32x4 v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) v[h] = *reinterpret_cast<const i32x4*>(w + b * kRowUnit + 64 * h);
      multiply(b, v);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) parts[wave * 256 + r * 64 + lane] = acc[r];
    __syncthreads();
    join_waves<E, 1>(a, parts, waves, o0, scale);
    if ((int64_t)o0 + (int64_t)gridDim.x * 16 >= a.o) break;
    o0 += gridDim.x * 16;
    ask();
    __syncthreads();
  }
}

typedef const __attribute__((address_space(1))) uint32_t* GlobalPtr;
typedef __attribute__((address_space(3))) uint32_t* LdsPtr;

template <class E>
__device__ __forceinline__ void store_four(typename E::T* at, const float (&v)[4]) {
  if constexpr (E::VEC == 4) {
    store_vec<E>(at, E::pack(v));
  } else {
    struct __attribute__((packed, aligned(2))) Four {
      u32x2 v;
    };
    const u32x4 w = E::pack({v[0], v[1], v[2], v[3], 0.f, 0.f, 0.f, 0.f});
    reinterpret_cast<Four*>(at)->v = u32x2{w[0], w[1]};
  }
}

// Tiles in the order in which the compute units of an XCD, which share an L2, take them: eight rows of tiles by all columns.
__device__ __forceinline__ void tile_place(int tiles_m, int tiles_n, int& tm, int& tn) {
  const int id = (int)xcd_contiguous_block_id(), band = 8 * tiles_n, first = id / band * 8, high = min(8, tiles_m - first);
  tm = first + id % band % high;
  tn = id % band / high;
}

// Of 64 neighbouring columns, the one that stands at place p of shared memory: lane l of the instructions then holds columns 4 l .. 4 l + 3 in four of
// its tiles, and stores them together.
__device__ __forceinline__ int column_at(int p) { return (p & ~63) + 4 * (p & 15) + (p >> 4 & 3); }

// WM x WN waves, each 64 rows of x by 16 NT outputs.  128 inputs at a time go straight into shared memory, one step ahead, as rows of 8 pieces of 16
// bytes whose order is turned from row to row, so that neither side meets a bank twice.  Bound by the matrix units, 51 % busy: 8192 x 4096 -> 4096 130 us,
// 2.1 POP/s; of few tiles by what a group of waves waits for in each step, 48 x 9216 -> 4096 20 us by four groups, 64 workgroups on 256 units.  (Three or four buffers: no change where
// there are few tiles, 60 against 44 us for 3000 x 4096 -> 2000, as a compute unit then holds one workgroup.)
// DEPTH: groups of such waves in a workgroup that take the steps in turn, each with shared memory of its own, and add up in the end: where there are few tiles a
// compute unit has more than a wave for each of its matrix units.
template <int DTYPE, int WM, int WN, int NT, int DEPTH = 1>
__global__ __launch_bounds__(WM * WN * DEPTH * 64, DEPTH > 1 ? 1 : 2) void i8_tile_kernel(FwdArgs a) {
  typedef Elem<DTYPE> E;
  constexpr int THREADS = WM * WN * 64, BM = WM * 64, BN = WN * NT * 16, ROWS = BM + BN, LOADS = ROWS * 8 / THREADS;
  __shared__ __attribute__((aligned(16))) int8_t lds[2 * DEPTH][ROWS * kRowUnit];
  const int lane = threadIdx.x & 63, tid = (int)threadIdx.x % THREADS, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int part = DEPTH > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS) : 0;
  int tm, tn;
  tile_place((a.m + BM - 1) / BM, (a.o + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, o0 = tn * BN, steps = (int)(a.row / kRowUnit);
  const int8_t* from[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int at = j * THREADS + tid, r = at >> 3, piece = (at & 7) ^ (r & 7);
    from[j] = (r < BM ? a.codes + (int64_t)min(m0 + r, a.m - 1) * a.row : a.w_codes + (int64_t)min(o0 + column_at(r - BM), a.o - 1) * a.row) + 16 * piece;
  }
  auto load = [&](int step, int buffer) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(from[j] + (int64_t)step * kRowUnit), (LdsPtr)&lds[2 * part + buffer][(j * THREADS + wave * 64) * 16], 16, 0, 0);
  };
  i32x4 acc[4][NT] = {};
  if (part < steps) load(part, 0);
  for (int s = part, buffer = 0; s - part < steps; s += DEPTH, buffer ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's pieces are in shared memory
    __syncthreads();                     // everybody's are, and nobody reads the other buffer any more
    if (s + DEPTH < steps) load(s + DEPTH, buffer ^ 1);
    if (DEPTH > 1 && s >= steps) continue;
    const int8_t* const base = lds[2 * part + buffer];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x4 x[4], w[NT];
      const int piece = 4 * h + (lane >> 4);
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = *reinterpret_cast<const i32x4*>(base + (wm * 64 + t * 16 + (lane & 15)) * kRowUnit + 16 * (piece ^ (lane & 7)));
#pragma unroll
      for (int t = 0; t < NT; ++t)
        w[t] = *reinterpret_cast<const i32x4*>(base + (BM + wn * NT * 16 + t * 16 + (lane & 15)) * kRowUnit + 16 * (piece ^ (lane & 7)));
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[t][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], w[u], acc[t][u], 0, 0, 0);
    }
  }
  if constexpr (DEPTH > 1) {  // each group adds up some of the rows
    static_assert(4 % DEPTH == 0 && WM * WN * 4 * NT * 1024 <= 2 * ROWS * kRowUnit, "");
    i32x4* const sums = reinterpret_cast<i32x4*>(lds);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < NT; ++u) sums[(((part * WM * WN + wave) * 4 + t) * NT + u) * 64 + lane] = acc[t][u];
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t / (4 / DEPTH) == part) {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          acc[t][u] = sums[((wave * 4 + t) * NT + u) * 64 + lane];
#pragma unroll
          for (int p = 1; p < DEPTH; ++p) acc[t][u] += sums[(((p * WM * WN + wave) * 4 + t) * NT + u) * 64 + lane];
        }
      }
  }
#pragma unroll
  for (int g = 0; g < NT / 4; ++g) {
    const int out = o0 + wn * NT * 16 + g * 64 + 4 * (lane & 15);
    if (out >= a.o) continue;
    float t[4], bias[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = min(out + q, a.o - 1);
      t[q] = a.w_scale[at];
      bias[q] = a.bias ? E::to_float(static_cast<const typename E::T*>(a.bias)[at]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = m0 + wm * 64 + i * 16 + 4 * (lane >> 4) + r;
        if (n >= a.m || (DEPTH > 1 && i / (4 / DEPTH) != part)) continue;
        const float s = a.scale[n];
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = finish(acc[i][4 * g + q][r], s, t[q], bias[q], a.relu);
        typename E::T* const to = static_cast<typename E::T*>(a.y) + (int64_t)n * a.o + out;
        if (out + 4 <= a.o) {
          store_four<E>(to, v);
        } else {
          for (int q = 0; q < a.o - out; ++q) to[q] = E::from_float(v[q]);
        }
      }
  }
}

template <int DTYPE>
int launch_forward(const i8_desc* d, const FwdArgs& a, const void* x, int8_t* codes, float* scales, hipStream_t stream) {
  const int m = d->p.m, o = d->p.num_output;
  if (x && d->token) {
    hipLaunchKernelGGL(i8_token_kernel<DTYPE>, dim3(std::min((o + 15) / 16, kMostBlocks)), dim3(64 * d->waves), (size_t)(m * d->row + d->waves * 1024), stream, a, x, codes, scales, d->p.k);
    return (int)hipGetLastError();
  }
  if (x) {
    const int e = launch_quantise<DTYPE>(x, codes, scales, m, d->p.k, d->row, stream);
    if (e) return e;
  }
  const auto tiles = [&](int tile) { return dim3((uint32_t)((int64_t)((m + tile - 1) / tile) * ((o + tile - 1) / tile))); };
  if (d->fwd == kTile256) {
    hipLaunchKernelGGL((i8_tile_kernel<DTYPE, 4, 2, 8>), tiles(256), dim3(512), 0, stream, a);
  } else if (d->fwd == kTile128) {
    hipLaunchKernelGGL((i8_tile_kernel<DTYPE, 2, 2, 4>), tiles(128), dim3(256), 0, stream, a);
  } else if (d->fwd == kTile128By2) {
    hipLaunchKernelGGL((i8_tile_kernel<DTYPE, 2, 2, 4, 2>), tiles(128), dim3(512), 0, stream, a);
  } else if (d->fwd == kTile64By4) {
    hipLaunchKernelGGL((i8_tile_kernel<DTYPE, 1, 1, 4, 4>), tiles(64), dim3(256), 0, stream, a);
  } else if (d->fwd == kTile64By2) {
    hipLaunchKernelGGL((i8_tile_kernel<DTYPE, 1, 1, 4, 2>), tiles(64), dim3(128), 0, stream, a);
  } else {
    const int mt = m > 16 ? 2 : 1;
    const dim3 grid((uint32_t)std::min((o + 15) / 16, kMostBlocks)), block(64 * d->waves);
    const size_t lds = (size_t)d->waves * mt * 1024;  // at most 32 KB
    if (mt == 1)
      hipLaunchKernelGGL((i8_rows_kernel<DTYPE, 1>), grid, block, lds, stream, a);
    else
      hipLaunchKernelGGL((i8_rows_kernel<DTYPE, 2>), grid, block, lds, stream, a);
  }
  return (int)hipGetLastError();
}

// ---- gradients ----

struct BwdArgs {
  const int8_t* codes;  // [reduction][row]
  const float* scale;   // [reduction]
  const void* dz;       // [n][o]
  void* out;            // filter: dw; data: dx
  float* db;            // filter, may be null
  float* parts;         // splits > 1: [splits][rows][k], then [splits][o] of db
  float* db_parts;
  int64_t row;
  int32_t n, o, k;
  int32_t per;          // steps of a split
  float beta;
};

constexpr int step_of(int tile) { return tile == 64 ? 64 : 32; }  // terms of the sums that a step takes

// Values as bf16 terms, two at a time: the rounded value, what is left of it rounded, and so on.
template <int TERMS>
__device__ __forceinline__ void pair_terms(float a, float b, uint32_t (&w)[TERMS]) {
  typedef __bf16 Pair __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    w[t] = __builtin_bit_cast(uint32_t, Pair{(__bf16)a, (__bf16)b});
    if (t + 1 < TERMS) {
      a -= __builtin_bit_cast(float, w[t] << 16);
      b -= __builtin_bit_cast(float, w[t] & 0xffff0000u);
    }
  }
}

// TILE rows of the result (filter: outputs, data: rows of x) by TILE inputs.  Both factors are made into bf16 operands on the way from memory to
// shared memory, where the 8 terms of the sum that a lane of the matrix instructions takes lie together.  Half of the waves do it for dz, half for
// the codes: a lane takes 8 terms of four neighbouring rows or columns, so that turning them costs nothing beside the conversion.  The next step's values
// are asked for before the instructions on this one's first term and converted after them: a compute unit's matrix and vector units are then
// both busy, with waves that are at different places.
// Every load is in range and none waits for a branch: the last terms of a sum that are fewer than 8 come as the last 8, with zeros for those that the
// groups before hold, and the last outputs that are fewer than four as the last four, each to its own place.  SLOW: sums or rows too short
// for that, one by one.
// Waves of 16 MT rows by 16 NT inputs.  Bound by matrix and vector units together, 53 and 41 % busy: dw of 8192 x 4096 -> 4096 bf16 438 us, 1.26 PFLOP/s
// in two terms; dx 435.  (A higher priority during the matrix instructions: dw fp32 1408 against 1148 us.)
template <int DTYPE, bool FILTER, int TILE, bool SLOW>
__global__ __launch_bounds__(TILE == 256 ? 512 : 256, 2) void i8_gradient_kernel(BwdArgs a) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  constexpr int THREADS = TILE == 256 ? 512 : 256, HALF = THREADS / 2, WN = TILE == 64 ? 1 : 2, MT = TILE == 64 ? 1 : 4, NT = TILE / (16 * WN);
  constexpr int TERMS = DTYPE == MI355_BF16 ? 2 : 3, STEP = step_of(TILE), GROUPS = STEP / 8;
  // pieces of 16 bytes: [term][group of 8 terms of the sum][place], and the same of the codes; a lane's place is its number modulo 16 in every
  // access, so that the lanes that go together, eight of two neighbouring sixteens, meet no bank twice
  constexpr int GROUP = TILE + 16, TERM = GROUPS * GROUP, BUFFER = (TERMS + 1) * TERM;
  __shared__ __attribute__((aligned(16))) u32x4 lds[2][BUFFER];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
  const int rows = FILTER ? a.o : a.n, depth = FILTER ? a.n : a.o;
  int tm, tn;
  tile_place((rows + TILE - 1) / TILE, (a.k + TILE - 1) / TILE, tm, tn);
  const int r0 = tm * TILE, i0 = tn * TILE;
  const int first = blockIdx.y * a.per, steps = min(a.per, (depth + STEP - 1) / STEP - first);
  const bool sum_bias = FILTER && a.db && tn == 0;

  const bool of_dz = wave < HALF / 64;
  const int half = of_dz ? tid : tid - HALF, p = half % (TILE / 4);  // four rows or columns 4 p ..
  const int g = TILE == 256 ? __builtin_amdgcn_readfirstlane(half / (TILE / 4)) : half / (TILE / 4);  // group: a wave's
  // the place of a row or column: of 64 neighbours, 4 l + q stands at 16 q + l
  auto place_of = [](int i) { return (i & ~63) + (i & 3) * 16 + (i >> 2 & 15); };
  const int col = (int)min((int64_t)i0 + 4 * p, a.row - 4);
  const int out = SLOW ? r0 + 4 * p : min(r0 + 4 * p, rows - 4);  // filter
  int places[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) places[q] = !FILTER || !of_dz ? place_of(4 * p + q) : out + q >= r0 ? place_of(out + q - r0) : TILE;  // (another tile's: nobody reads it)
  // the first term of a group's 8 in a step, and how many of them are not the group's
  auto first_of = [&](int step, int group, int& skip) {
    const int d0 = (first + step) * STEP + 8 * group, from = max(0, min(d0, depth - 8));
    skip = d0 - from;
    return from;
  };
  constexpr int DATA_ROWS = TILE * GROUPS / HALF;  // data: 8 terms of rows data_row and on, HALF / GROUPS apart
  const int data_group = (half >> 4) % GROUPS, data_row = (half & 15) + (half >> 4) / GROUPS * 16;
  constexpr int WORDS = DTYPE == MI355_F32 ? 4 : 2;
  typedef typename std::conditional<DTYPE == MI355_F32, u32x4, u32x2>::type Four;
  struct __attribute__((packed, aligned(sizeof(T)))) FourMem {
    Four v;
  };
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  f32x4 acc[MT][NT] = {};

  struct Filter {
    Four z[8];
  };
  struct Data {
    u32x4 z[DATA_ROWS][DTYPE == MI355_F32 ? 2 : 1];
  };
  struct Way {  // what is on its way
    typename std::conditional<FILTER, Filter, Data>::type raw;
    float s[8];
    uint32_t c[8];
    int skip;
  };

  auto load_codes = [&](Way& way, int step) {
    const int from = first_of(step, g, way.skip);
    const int8_t* const at = a.codes + (int64_t)from * a.row + col;
#pragma unroll
    for (int j = 0; j < 8; ++j) way.c[j] = *reinterpret_cast<const uint32_t*>(at + (int64_t)(SLOW ? min(j, depth - 1 - from) : j) * a.row);
  };
  auto load_dz = [&](Way& way, int step) {
    const int from = first_of(step, FILTER ? g : data_group, way.skip);
#pragma unroll
    for (int j = 0; j < 8; ++j) way.s[j] = a.scale[SLOW ? min(from + j, depth - 1) : from + j];
    if constexpr (FILTER) {
      const T* const z = static_cast<const T*>(a.dz) + (int64_t)from * a.o + (SLOW ? 0 : out);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (SLOW) {
          const T* const row = z + (int64_t)min(j, depth - 1 - from) * a.o;
          float f[E::VEC];
#pragma unroll
          for (int q = 0; q < E::VEC; ++q) f[q] = q < 4 ? E::to_float(row[min(out + q, a.o - 1)]) : 0.f;
          const u32x4 v = E::pack(f);
#pragma unroll
          for (int w = 0; w < WORDS; ++w) way.raw.z[j][w] = v[w];
        } else {
          way.raw.z[j] = reinterpret_cast<const FourMem*>(z + (int64_t)j * a.o)->v;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < DATA_ROWS; ++i) {
        const T* const z = static_cast<const T*>(a.dz) + (int64_t)min(r0 + data_row + i * (HALF / GROUPS), rows - 1) * a.o + from;
        if constexpr (SLOW) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = E::to_float(z[min(j, depth - 1 - from)]);
          if constexpr (DTYPE == MI355_F32) {
            way.raw.z[i][0] = E::pack({f[0], f[1], f[2], f[3]});
            way.raw.z[i][1] = E::pack({f[4], f[5], f[6], f[7]});
          } else {
            way.raw.z[i][0] = E::pack(f);
          }
        } else {
          way.raw.z[i][0] = load_vec<E>(z);
          if constexpr (DTYPE == MI355_F32) way.raw.z[i][1] = load_vec<E>(z + 4);
        }
      }
    }
  };
  auto put_codes = [&](const Way& way, u32x4* buffer) {
    u32x4* const to = buffer + TERMS * TERM + g * GROUP;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t two[1];
        pair_terms<1>((float)(int8_t)(way.c[2 * j] >> 8 * q), (float)(int8_t)(way.c[2 * j + 1] >> 8 * q), two);
        w[j] = two[0];
      }
      to[places[q]] = w;
    }
  };
  // The 8 terms' dz, zeros for those that are not the group's, whatever they hold.
  auto keep_own = [&](const Way& way, float (&v)[8]) {
    if (way.skip > 0 || SLOW) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j >= way.skip && j < depth ? v[j] : 0.f;
    }
  };
  auto terms_of = [&](const Way& way, float (&v)[8], u32x4 (&w)[TERMS]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= way.s[j];
    keep_own(way, v);  // (their scales may be NaN)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t two[TERMS];
      pair_terms<TERMS>(v[2 * j], v[2 * j + 1], two);
#pragma unroll
      for (int t = 0; t < TERMS; ++t) w[t][j] = two[t];
    }
  };
  auto put_dz = [&](const Way& way, u32x4* buffer) {
    if constexpr (FILTER) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          u32x4 z = {};
#pragma unroll
          for (int i = 0; i < WORDS; ++i) z[i] = way.raw.z[j][i];
          v[j] = E::get(z, q);
        }
        if (sum_bias) {
          keep_own(way, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) bias[q] += v[j];
        }
        u32x4 w[TERMS];
        terms_of(way, v, w);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) buffer[t * TERM + g * GROUP + places[q]] = w[t];
      }
    } else {
#pragma unroll
      for (int i = 0; i < DATA_ROWS; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = E::get(way.raw.z[i][j / E::VEC], j % E::VEC);
        u32x4 w[TERMS];
        terms_of(way, v, w);
        const int row = data_row + i * (HALF / GROUPS);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) buffer[t * TERM + data_group * GROUP + row] = w[t];
      }
    }
  };

  // Both kinds of waves take the same steps, and meet at the same barriers.
  auto products = [&](int step, auto&& between) {
#pragma unroll
    for (int part = 0; part < STEP / 32; ++part) {
      const u32x4* const A = lds[step & 1] + (4 * part + (lane >> 4)) * GROUP + wm * MT * 16 + (lane & 15);
      const u32x4* const B = lds[step & 1] + TERMS * TERM + (4 * part + (lane >> 4)) * GROUP + wn * NT * 16 + (lane & 15);
      bf16x8 w[NT];
#pragma unroll
      for (int u = 0; u < NT; ++u) w[u] = __builtin_bit_cast(bf16x8, B[u * 16]);
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        bf16x8 x[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = __builtin_bit_cast(bf16x8, A[t * TERM + 16 * i]);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int u = 0; u < NT; ++u) acc[i][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], w[u], acc[i][u], 0, 0, 0);
        if (part + 1 == STEP / 32 && t + 2 == TERMS) {
          __builtin_amdgcn_sched_barrier(0);
          between();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    __syncthreads();
  };
  auto work = [&](auto&& load, auto&& put) {
    if constexpr (TILE == 256) {
      Way way;
      load(way, 0);
      put(way, lds[0]);
      __syncthreads();
      for (int step = 0; step < steps; ++step) {
        const bool more = step + 1 < steps;
        if (more) load(way, step + 1);
        __builtin_amdgcn_sched_barrier(0);
        products(step, [&]() {
          if (more) put(way, lds[(step + 1) & 1]);
        });
      }
    } else {
      // The small tile's registers hold two steps: few workgroups and short sums leave a step's loads no time otherwise.  (Loads beyond the last
      // step are the last one's again.)
      Way one, two;
      load(one, 0);
      put(one, lds[0]);
      load(one, min(1, steps - 1));
      __syncthreads();
      for (int step = 0; step < steps; step += 2) {
        load(two, min(step + 2, steps - 1));
        __builtin_amdgcn_sched_barrier(0);
        products(step, [&]() {
          if (step + 1 < steps) put(one, lds[1]);
        });
        if (step + 1 == steps) break;
        load(one, min(step + 3, steps - 1));
        __builtin_amdgcn_sched_barrier(0);
        products(step + 1, [&]() {
          if (step + 2 < steps) put(two, lds[0]);
        });
      }
    }
  };
  if (steps > 0) {
    if (of_dz)
      work(load_dz, put_dz);
    else
      work(load_codes, put_codes);
  }

  const bool split = gridDim.y > 1;
  if (sum_bias) {  // the groups' sums of each output
    float* const sums = reinterpret_cast<float*>(lds);
    if (of_dz) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (out + q >= r0 && out + q < r0 + TILE) sums[g * TILE + out + q - r0] = bias[q];
    }
    __syncthreads();
    if (tid < TILE && r0 + tid < a.o) {
      float v = sums[tid];
#pragma unroll
      for (int i = 1; i < GROUPS; ++i) v += sums[i * TILE + tid];
      if (split)
        a.db_parts[(int64_t)blockIdx.y * a.o + r0 + tid] = v;
      else
        a.db[r0 + tid] = a.beta == 0.f ? v : a.db[r0 + tid] + v;
    }
  }
#pragma unroll
  for (int h = 0; h < NT / 4; ++h) {
    const int at = i0 + wn * NT * 16 + h * 64 + 4 * (lane & 15);
    if (at >= a.k) continue;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int in_tile = 4 * (lane >> 4) + r, tile = wm * MT + i;  // of 16 rows; filter: as the places go
        const int to_row = r0 + (FILTER ? (tile >> 2) * 64 + 4 * in_tile + (tile & 3) : 16 * tile + in_tile);
        if (to_row >= rows) continue;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = acc[i][4 * h + q][r];
        const int64_t place = (int64_t)to_row * a.k + at;
        const int count = min(4, a.k - at);
        if (split || FILTER) {
          typedef Elem<MI355_F32> F;
          float* const to = split ? a.parts + (int64_t)blockIdx.y * rows * a.k + place : static_cast<float*>(a.out) + place;
          const bool add = !split && a.beta != 0.f;
          if (count == 4) {
            if (add) {
              const u32x4 old = load_vec<F>(to);
#pragma unroll
              for (int q = 0; q < 4; ++q) v[q] += F::get(old, q);
            }
            store_vec<F>(to, F::pack(v));
          } else {
            for (int q = 0; q < count; ++q) to[q] = add ? to[q] + v[q] : v[q];
          }
        } else {
          T* const to = static_cast<T*>(a.out) + place;
          if (count == 4) {
            store_four<E>(to, v);
          } else {
            for (int q = 0; q < count; ++q) to[q] = E::from_float(v[q]);
          }
        }
      }
  }
}

// The splits' sums in one, four elements a thread; beta as the kernels take it.
template <class E>
__device__ __forceinline__ void join_four(const float* parts, typename E::T* out, int64_t count, int splits, float beta, int64_t i) {
  typedef Elem<MI355_F32> F;
  float v[4];
  if (i + 4 <= count) {
    u32x4 w = load_vec<F>(parts + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = F::get(w, q);
#pragma unroll 4
    for (int s = 1; s < splits; ++s) {
      w = load_vec<F>(parts + s * count + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += F::get(w, q);
    }
    if (beta != 0.f) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += E::to_float(out[i + q]);
    }
    store_four<E>(out + i, v);
  } else {
    for (int64_t j = i; j < count; ++j) {
      float sum = parts[j];
      for (int s = 1; s < splits; ++s) sum += parts[s * count + j];
      out[j] = E::from_float(beta != 0.f ? E::to_float(out[j]) + sum : sum);
    }
  }
}

// Of the result, and by the last workgroups of the bias gradient (bias_count 0: none).  Bound by memory: 777 x 1111 of six parts 5 us.
template <class E>
__global__ __launch_bounds__(256) void i8_join_kernel(const float* __restrict__ parts, typename E::T* __restrict__ out, int64_t count, const float* __restrict__ bias_parts,
                                                      float* __restrict__ bias_out, int64_t bias_count, int splits, float beta, int blocks) {
  if ((int)blockIdx.x >= blocks) {
    const int64_t i = ((int64_t)(blockIdx.x - blocks) * 256 + threadIdx.x) * 4;
    if (i < bias_count) join_four<Elem<MI355_F32>>(bias_parts, bias_out, bias_count, splits, beta, i);
    return;
  }
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < count; i += (int64_t)blocks * 1024) join_four<E>(parts, out, count, splits, beta, i);
}

// Whether a gradient's sums or rows are too short for loads of 8 terms of four outputs.
bool slow(int64_t rows, int64_t depth, bool filter) { return depth < 8 || (filter && rows < 4); }

template <int DTYPE, bool FILTER>
int launch_gradient(const BwdArgs& a, int tile, int splits, hipStream_t stream) {
  const int rows = FILTER ? a.o : a.n;
  const dim3 grid((uint32_t)(((int64_t)rows + tile - 1) / tile * (((int64_t)a.k + tile - 1) / tile)), splits);
  if (slow(rows, FILTER ? a.n : a.o, FILTER))
    hipLaunchKernelGGL((i8_gradient_kernel<DTYPE, FILTER, 128, true>), grid, dim3(256), 0, stream, a);
  else if (tile == 256) {
    if constexpr (FILTER || DTYPE != MI355_F32)
      hipLaunchKernelGGL((i8_gradient_kernel<DTYPE, FILTER, 256, false>), grid, dim3(512), 0, stream, a);
    else
      return (int)hipErrorInvalidDeviceFunction;  // not built: plan_gradient never asks for it
  } else if (tile == 64)
    hipLaunchKernelGGL((i8_gradient_kernel<DTYPE, FILTER, 64, false>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((i8_gradient_kernel<DTYPE, FILTER, 128, false>), grid, dim3(256), 0, stream, a);
  const int e = (int)hipGetLastError();
  if (e || splits == 1) return e;
  typedef typename std::conditional<FILTER, Elem<MI355_F32>, Elem<DTYPE>>::type Out;
  const int64_t count = (int64_t)rows * a.k, bias_count = FILTER && a.db ? a.o : 0;
  const int blocks = (int)std::min<int64_t>((count + 1023) / 1024, 1 << 20), bias_blocks = (int)((bias_count + 1023) / 1024);
  hipLaunchKernelGGL(i8_join_kernel<Out>, dim3(blocks + bias_blocks), dim3(256), 0, stream, a.parts, static_cast<typename Out::T*>(a.out), count, a.db_parts, a.db,
                     bias_count, splits, a.beta, blocks);
  return (int)hipGetLastError();
}

template <bool FILTER>
int gradient(const i8_desc* d, const BwdArgs& a, hipStream_t stream) {
  const int tile = FILTER ? d->filter_tile : d->data_tile, splits = FILTER ? d->filter_splits : d->data_splits;
  switch (d->p.dtype) {
    case MI355_F32: return launch_gradient<MI355_F32, FILTER>(a, tile, splits, stream);
    case MI355_F16: return launch_gradient<MI355_F16, FILTER>(a, tile, splits, stream);
    default: return launch_gradient<MI355_BF16, FILTER>(a, tile, splits, stream);
  }
}

__global__ __launch_bounds__(256) void i8_clear_kernel(float* to, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) to[i] = 0.f;
}

int clear(float* to, int64_t count, hipStream_t stream) {
  hipLaunchKernelGGL(i8_clear_kernel, dim3((uint32_t)std::min<int64_t>((count + 255) / 256, 1 << 16)), dim3(256), 0, stream, to, count);
  return (int)hipGetLastError();
}

int64_t tiles_of(int64_t rows, int64_t columns, int tile) { return (rows + tile - 1) / tile * ((columns + tile - 1) / tile); }

// The forward pass.  A few rows by themselves (16 x 4096 -> 8192 14.3 us, in tiles 14.8, -> 16384 21.7, 18.7; 32 x 4096 -> 4096 13.1, 14.8, -> 6000 18.3, 14.9); more of them
// share weights better in tiles; where there are few tiles, small ones whose sums several groups of waves share:
// a step of 128 inputs takes 0.7 us in a group, whatever its tile is, as every group waits for its own reads of shared memory (us, rows, 64 by 4, 64 by 2,
// 128 by 2, 128, 256: 64 x 4096 -> 4096 17.7, 15.5, 18.2; 64 x 4096 -> 16384 43.7, 20.2, 19.8; 300 rows -, -, 19.6, 25.0, 28.5; 512 rows
// -, 26.1, 21.5, 26.1, 29.5; 700 rows -, -, 33.5, 26.4, 29.9; 1024 rows -, 46, 35.4, 28.9, 32.0, 60; 1300 rows -, -, 48.8, 47.9, 38.9, 61.7).  From then on a tile of 256
// has a compute unit to itself, of 128 half of one, and a round of the former takes 1.5 times as long (2048 rows 45.6, with 256 64.8; 2500 rows 64.2, 65.9;
// 4096 rows 85.3, 75.0; 6000 rows 128, 132).
int32_t plan_forward(int64_t m, int64_t o) {
  if (m <= kTokenRows || (m <= 32 && (m > 16 ? 2 : 1) * o <= 8192)) return kRows;
  if (tiles_of(m, o, 64) <= kUnits) return kTile64By4;
  if (tiles_of(m, o, 64) <= 2 * kUnits) return kTile64By2;
  if (tiles_of(m, o, 128) <= kUnits) return kTile128By2;
  const int64_t large = (tiles_of(m, o, 256) + kUnits - 1) / kUnits, medium = (tiles_of(m, o, 128) + 2 * kUnits - 1) / (2 * kUnits);  // rounds
  return 3 * large < 2 * medium ? kTile256 : kTile128;
}

// The tile of a gradient, and the workgroups that share a sum.  A tile of 256 has a compute unit to itself, of 128 half of one; a round of the former takes
// 1.4 times as long as one of the latter where dz is two terms, 1.6 to 2.0 where it is three, 2.5 for dx in fp32, whose kernel of 256 was built only to
// measure it (and is never taken: a tile of 256 is four of 128 at most, so that there are at least half as many rounds of them) (us, 256 and 128: dw of 8192 x 4096 -> 4096 bf16 460, 674, fp16 738, 949, fp32 1146, 1145; dx of the same 434, 606; 759, 877; 1177, 944; dw of
// 8192 x 4096 -> 2048 bf16, half a round, 436, 356).  Where a tile of 128 leaves half of the units without work, 64: dx of 100 x 999 <- 333 fp32 10.1, with
// 128 16.4; of 512 x 333 <- 150 fp32 6.7, 11.8; dw of 2000 x 512 -> 512 bf16 17.0, 18.4, of 1999 x 1111 -> 777 fp16 40.3, 38.1 (the one of these that the rule
// makes 5 % slower); of 1000 x 2000 -> 1000 bf16, 128 tiles of
// 128, 29.7, 30.6; of 64 x 4096 -> 4096 bf16 32.8, 22.0.
void plan_gradient(int64_t rows, int64_t k, int64_t depth, int dtype, bool filter, int32_t& tile, int32_t& splits, int32_t& per) {
  const int64_t large = (tiles_of(rows, k, 256) + kUnits - 1) / kUnits, medium = (tiles_of(rows, k, 128) + 2 * kUnits - 1) / (2 * kUnits);  // rounds
  const double round = dtype == MI355_BF16 ? 1.43 : filter || dtype == MI355_F16 ? 1.85 : 2.3;
  tile = slow(rows, depth, filter) ? 128 : tiles_of(rows, k, 128) < kUnits / 2 ? 64 : round * large < medium ? 256 : 128;
  const int64_t step = step_of(tile), steps = std::max<int64_t>(1, (depth + step - 1) / step);
  const int64_t tiles = std::max<int64_t>(1, tiles_of(rows, k, tile)), places = tile == 256 ? 1 : 2 * kUnits;
  splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(places / tiles, steps / (tiles <= kUnits / 2 ? 4 : 8)), 64));
  per = (int32_t)((steps + splits - 1) / splits);
  splits = (int32_t)((steps + per - 1) / per);
}

bool workspace_missing(const i8_desc* d, const void* ws, size_t bytes, int& status) {
  if (!d->ws_bytes) return false;
  status = !ws || bytes < d->ws_bytes ? CONV_EWORKSPACE : ((uintptr_t)ws & 15u) ? CONV_EINVAL : CONV_OK;
  return status != CONV_OK;
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int i8_desc_create(i8_desc_t** out, const i8_params_t* pp) {
  if (!out || !pp) return CONV_EINVAL;
  const i8_params_t p = *pp;
  if (p.m < 0 || p.k < 1 || p.num_output < 1 || (p.dtype != MI355_F32 && p.dtype != MI355_F16 && p.dtype != MI355_BF16)) return CONV_EINVAL;
  if ((p.bias_term != 0 && p.bias_term != 1) || (p.relu != 0 && p.relu != 1)) return CONV_EINVAL;
  const int64_t M = p.m, K = p.k, O = p.num_output;
  if (K > kMostInputs || M * K >= kMaxElems || O * K >= kMaxElems || M * O >= kMaxElems) return CONV_ESHAPE;
  i8_desc* d = new (std::nothrow) i8_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->p = p;
  d->row = (K + kRowUnit - 1) / kRowUnit * kRowUnit;
  d->fwd = plan_forward(M, O);
  d->waves = (int32_t)std::max<int64_t>(1, std::min<int64_t>(tiles_of(M, O, 16) > 4 * kUnits ? 4 : 16, d->row / kRowUnit));
  d->token = d->fwd == kRows && M <= kTokenRows && M * d->row <= kTokenBytes;
  plan_gradient(O, K, M, p.dtype, true, d->filter_tile, d->filter_splits, d->filter_per);
  plan_gradient(M, K, O, p.dtype, false, d->data_tile, d->data_splits, d->data_per);
  if (M > 0) {
    if (d->filter_splits > 1) d->ws_bytes = (size_t)d->filter_splits * (O * K + O) * 4;
    if (d->data_splits > 1) d->ws_bytes = std::max(d->ws_bytes, (size_t)d->data_splits * M * K * 4);
  }
  char fwd[48];
  if (d->fwd == kRows)
    snprintf(fwd, sizeof(fwd), "%si8_rows[m%d](W=%d)", d->token ? "i8_token/" : "", p.m > 16 ? 32 : 16, d->waves);
  else
    snprintf(fwd, sizeof(fwd), "i8_tile[%s]", d->fwd == kTile256 ? "256" : d->fwd == kTile128 ? "128" : d->fwd == kTile128By2 ? "128,by2" : d->fwd == kTile64By2 ? "64,by2" : "64,by4");
  snprintf(d->names, sizeof(d->names), "fwd=%s;bwd_filter=i8_gradient[%d%s](S=%d);bwd_data=i8_gradient[%d%s](S=%d)", fwd, d->filter_tile, slow(O, M, true) ? ",slow" : "",
           d->filter_splits, d->data_tile, slow(M, O, false) ? ",slow" : "", d->data_splits);
  *out = d;
  return CONV_OK;
}

int i8_desc_destroy(i8_desc_t* d) {
  if (!d) return CONV_EINVAL;
  delete d;
  return CONV_OK;
}

int i8_desc_workspace_bytes(const i8_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = d->ws_bytes;
  return CONV_OK;
}

int i8_desc_row_bytes(const i8_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = (size_t)d->row;
  return CONV_OK;
}

const char* i8_desc_kernel_names(const i8_desc_t* d) { return d ? d->names : ""; }

int i8_pack(const i8_desc_t* d, const void* w, int8_t* w_codes, float* w_scale, void* hip_stream) {
  if (!d || !w || !w_codes || !w_scale || misaligned(w_codes)) return CONV_EINVAL;
  const int e = quantise(d, w, w_codes, w_scale, d->p.num_output, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int i8_quantise(const i8_desc_t* d, const void* x, int8_t* codes, float* scale, void* hip_stream) {
  if (!d) return CONV_EINVAL;
  if (d->p.m == 0) return CONV_OK;
  if (!x || !codes || !scale || misaligned(codes)) return CONV_EINVAL;
  const int e = quantise(d, x, codes, scale, d->p.m, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int i8_forward(const i8_desc_t* d, const void* x, const int8_t* w_codes, const float* w_scale, const void* bias, void* y,
               int8_t* codes, float* scale, void* ws, size_t ws_bytes, void* hip_stream) {
  (void)ws, (void)ws_bytes;
  if (!d || !w_codes || !w_scale || misaligned(w_codes) || (d->p.bias_term != 0) != (bias != nullptr)) return CONV_EINVAL;
  if (d->p.m == 0) return CONV_OK;
  if (!y || !codes || !scale || misaligned(codes)) return CONV_EINVAL;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const FwdArgs a = {codes, w_codes, scale, w_scale, bias, y, d->row, d->p.m, d->p.num_output, d->p.relu};
  const int e = d->p.dtype == MI355_F32   ? launch_forward<MI355_F32>(d, a, x, codes, scale, stream)
                : d->p.dtype == MI355_F16 ? launch_forward<MI355_F16>(d, a, x, codes, scale, stream)
                                          : launch_forward<MI355_BF16>(d, a, x, codes, scale, stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int i8_backward_filter(const i8_desc_t* d, const int8_t* codes, const float* scale, const void* dz, float* dw, float* db, float beta,
                       void* ws, size_t ws_bytes, void* hip_stream) {
  if (!d || !dw || (db && !d->p.bias_term) || (beta != 0.f && beta != 1.f)) return CONV_EINVAL;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int64_t O = d->p.num_output, K = d->p.k;
  if (d->p.m == 0) {
    if (beta != 0.f) return CONV_OK;
    int e = clear(dw, O * K, stream);
    if (!e && db) e = clear(db, O, stream);
    return e ? record_hip_error(e) : CONV_OK;
  }
  int status = CONV_OK;
  if (!codes || !scale || !dz || misaligned(codes)) return CONV_EINVAL;
  if (workspace_missing(d, ws, ws_bytes, status)) return status;
  float* const parts = static_cast<float*>(ws);
  const BwdArgs a = {codes, scale, dz, dw, db, parts, parts + d->filter_splits * O * K, d->row, d->p.m, d->p.num_output, d->p.k, d->filter_per, beta};
  const int e = gradient<true>(d, a, stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int i8_backward_data(const i8_desc_t* d, const int8_t* w_codes, const float* w_scale, const void* dz, void* dx, void* ws,
                     size_t ws_bytes, void* hip_stream) {
  if (!d || !w_codes || !w_scale || misaligned(w_codes)) return CONV_EINVAL;
  if (d->p.m == 0) return CONV_OK;
  int status = CONV_OK;
  if (!dz || !dx) return CONV_EINVAL;
  if (workspace_missing(d, ws, ws_bytes, status)) return status;
  const BwdArgs a = {w_codes, w_scale, dz, dx, nullptr, static_cast<float*>(ws), nullptr, d->row, d->p.m, d->p.num_output, d->p.k, d->data_per, 0.f};
  const int e = gradient<false>(d, a, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
