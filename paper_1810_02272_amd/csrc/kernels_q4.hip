// The InnerProduct layer's forward pass on 4-bit weights with group scales (include/mi355q4.h).
//
// The weights' values are exact in bf16 and fp16, and so are their products with x in fp32: the matrix instructions take them as they
// are, a group's sum comes out of them in fp32, and one multiply-add by the group's scale adds it to the output's.
// fp32 x is three bf16 terms that make it up exactly.
//
// Packed weights, for the 16x16x32 instructions with x as the left operand (16 rows) and w as the right one (16 outputs):
//   codes [tile of 16 outputs][block of 128 inputs][lane][4 words]: lane l, word d holds the codes of output l % 16,
//         inputs 32 d + 8 (l / 16) .. + 7, the first in the lowest four bits: a wave's 1 KB is one load
//   scales [tile][block][output][128 / group]
// with zeros beyond num_output and k.
#include <hip/hip_runtime.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "device_utils.h"
#include "elements.h"
#include "internal.h"
#include "mi355q4.h"

struct q4_desc {
  q4_params_t p;
  int32_t tiles, blocks;  // of 16 outputs and 128 inputs
  int32_t nt, waves;      // tiles of a workgroup, its waves
  int32_t prepared;       // fp32 x is laid out as operands before
  int32_t splits, per_split;  // workgroups that share the inputs of an output, blocks of each
  size_t ws_bytes;
  char names[96];
};

namespace mi355conv {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 16, kBlockK = 128;
constexpr int kUnits = 256;  // compute units
constexpr int64_t kMaxElems = (int64_t)1 << 30;
constexpr int64_t kMostBlocks = 1 << 22;  // of 256 threads: a launch has fewer than 2^32

struct Q4Args {
  const void* x;
  const u32x4* codes;
  const uint16_t* scales;
  const void* bias;
  void* y;
  u32x4* terms;  // fp32: x as operands (x_terms_kernel)
  float* parts;  // splits > 1: [splits][m][o]
  int32_t m, k, o, tiles, blocks;
  int32_t splits, per_split;
  int32_t relu;
};

// One thread for each of a block's 64 vectors of codes, and the first ones for its scales.  WORDS: rows of codes start on words, as
// they do where k is a multiple of 8; byte by byte, 4096 x 128256 took 545 us.
template <bool WORDS>
__global__ __launch_bounds__(256) void q4_pack_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales,
                                                      u32x4* __restrict__ to, uint16_t* __restrict__ to_scales, int k, int o, int blocks,
                                                      int64_t vectors, int group) {
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < vectors; v += (int64_t)gridDim.x * 256) {
    const int lane = (int)(v & 63);
    const int64_t tb = v >> 6;
    const int tile = (int)(tb / blocks), block = (int)(tb % blocks);
    const int row = tile * kTile + (lane & 15), stride = (k + 1) / 2;
    u32x4 w = {0, 0, 0, 0};
    if (row < o) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int at = block * kBlockK + 32 * d + 8 * (lane >> 4);
        if constexpr (WORDS) {
          if (at < k) w[d] = *reinterpret_cast<const uint32_t*>(codes + (int64_t)row * stride + at / 2);
          continue;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int i = at + 2 * b;
          if (i < k) {
            uint32_t c = codes[(int64_t)row * stride + i / 2];
            if (i + 1 >= k) c &= 15u;
            w[d] |= c << (8 * b);
          }
        }
      }
    }
    to[v] = w;
    const int per = kBlockK / group, groups = (k + group - 1) / group;
    if (lane < 16) {
      for (int g = 0; g < per; ++g) {
        const int at = block * per + g;
        to_scales[(tb * kTile + lane) * per + g] = row < o && at < groups ? scales[(int64_t)row * groups + at] : 0;
      }
    }
  }
}

template <int DTYPE>
struct Operand;  // what the matrix instructions take for x and w: TERMS of them for x

template <>
struct Operand<MI355_BF16> {
  typedef bf16x8 V;
  static constexpr int TERMS = 1;
  static __device__ __forceinline__ V weights(uint32_t c) {
    const u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 3))};
    return __builtin_bit_cast(V, r);
  }
  static __device__ __forceinline__ f32x4 mma(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

template <>
struct Operand<MI355_F16> {
  typedef f16x8 V;
  static constexpr int TERMS = 1;
  static __device__ __forceinline__ V weights(uint32_t c) {
    const u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 3))};
    return __builtin_bit_cast(V, r);
  }
  static __device__ __forceinline__ f32x4 mma(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

template <>
struct Operand<MI355_F32> : Operand<MI355_BF16> {
  static constexpr int TERMS = 3;
};

// An fp32 value's terms: its leading 8 bits, the next 8, the last 8, each cut off and so exact, but for bits below 2^-133, bf16's last.  What is
// not finite is the first term's.
__device__ __forceinline__ void three_terms(float x, uint32_t (&t)[3]) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  if ((u & 0x7F800000u) == 0x7F800000u) {
    t[0] = (u & 0x7FFFFFu) ? 0x7FC0u : u >> 16;
    t[1] = t[2] = 0;
    return;
  }
  t[0] = u >> 16;
  const float r1 = x - __builtin_bit_cast(float, u & 0xffff0000u);
  const uint32_t v = __builtin_bit_cast(uint32_t, r1);
  t[1] = v >> 16;
  const float r2 = r1 - __builtin_bit_cast(float, v & 0xffff0000u);
  t[2] = __builtin_bit_cast(uint32_t, r2) >> 16;
}

// Eight consecutive values of x as operands.
template <int DTYPE>
__device__ __forceinline__ void load_operand(const typename Elem<DTYPE>::T* p, typename Operand<DTYPE>::V (&v)[Operand<DTYPE>::TERMS]) {
  typedef Elem<DTYPE> E;
  typedef typename Operand<DTYPE>::V V;
  if constexpr (DTYPE == MI355_F32) {
    const u32x4 h[2] = {load_vec<E>(p), load_vec<E>(p + 4)};
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a[3], b[3];
      three_terms(E::get(h[i >> 1], 2 * i & 3), a);
      three_terms(E::get(h[i >> 1], (2 * i & 3) + 1), b);
#pragma unroll
      for (int t = 0; t < 3; ++t) w[t][i] = a[t] | b[t] << 16;
    }
#pragma unroll
    for (int t = 0; t < 3; ++t) v[t] = __builtin_bit_cast(V, w[t]);
  } else {
    v[0] = __builtin_bit_cast(V, load_vec<E>(p));
  }
}

// Row i of a tile of 16 rows of x is row row_place(i) of the instruction's left operand: its results then stand in register i / 4 of the
// lanes 16 (i % 4) .. + 15, and up to four rows take one register.
__device__ __forceinline__ int place_row(int place) { return (place & 3) * 4 + (place >> 2); }

// fp32 x as operands: [tile of 16 rows][32 inputs][term][lane], zeros beyond m and k.  One thread for each lane of the three terms.
__global__ __launch_bounds__(256) void x_terms_kernel(const float* __restrict__ x, u32x4* __restrict__ to, int m, int k, int steps, int64_t lanes) {
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < lanes; v += (int64_t)gridDim.x * 256) {
    const int lane = (int)(v & 63);
    const int64_t ts = v >> 6;
    const int step = (int)(ts % steps);
    const int64_t row = ts / steps * 16 + place_row(lane & 15);
    const int at = 32 * step + 8 * (lane >> 4);
    float f[8];
    const float* const p = x + row * k + at;
    if (row < m && at + 8 <= k) {
      const u32x4 a = load_vec<Elem<MI355_F32>>(p), b = load_vec<Elem<MI355_F32>>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = Elem<MI355_F32>::get(a, i);
        f[4 + i] = Elem<MI355_F32>::get(b, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = row < m && at + i < k ? p[i] : 0.f;
    }
    bf16x8 w[3];
    load_operand<MI355_F32>(f, w);
#pragma unroll
    for (int t = 0; t < 3; ++t) to[(ts * 3 + t) * 64 + lane] = __builtin_bit_cast(u32x4, w[t]);
  }
}

template <int PER>
__device__ __forceinline__ void load_scales(const uint16_t* at, float (&scale)[PER]) {
  uint32_t w[2] = {0, 0};
  if constexpr (PER == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(at);
    w[0] = u.x, w[1] = u.y;
  } else if constexpr (PER == 2) {
    w[0] = *reinterpret_cast<const uint32_t*>(at);
  } else {
    w[0] = *at;
  }
#pragma unroll
  for (int g = 0; g < PER; ++g) scale[g] = __builtin_bit_cast(float, g & 1 ? w[g >> 1] & 0xffff0000u : w[g >> 1] << 16);
}

// Waves of a workgroup.  Up to 16 for one tile of rows; the accumulators of more take the registers of 8.
template <int MT>
constexpr int kMostWaves = MT == 1 ? 16 : 8;

// MT times 16 rows of x by NT tiles of 16 outputs in a workgroup, which goes on to the next 16 MT rows where there are more: batches of more than
// 64 rows read the codes again for each 64, and no more workgroups share them (4096 -> 4096 bf16: 65 rows 21.5 us,
// 128 25.7, 512 84, 2048 316).  Its waves take the blocks of inputs in turn, each on its own, and
// add up through shared memory at the end: nothing of x is used by two waves.  REGS: result registers that hold rows.  STREAM: the codes
// go around the last-level cache.
// PREPARED: x comes as operands (x_terms_kernel).
template <int DTYPE, int MT, int NT, int REGS, int GROUP, bool STREAM, bool PREPARED>
__global__ __launch_bounds__(kMostWaves<MT> * 64) void q4_kernel(Q4Args a) {
  typedef Operand<DTYPE> Op;
  typedef Elem<DTYPE> E;
  typedef typename Op::V V;
  constexpr int PER = kBlockK / GROUP, TERMS = Op::TERMS;
  extern __shared__ float parts[];  // [waves][NT * REGS * 64]
  constexpr int SLOT = NT * REGS * 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int quarter = lane >> 4;
  const int groups = (a.tiles + NT - 1) / NT;
  const int begin = blockIdx.y * a.per_split, end = min(begin + a.per_split, a.blocks);
  for (int tile0 = blockIdx.x * NT; tile0 < groups * NT; tile0 += gridDim.x * NT) {
    for (int m0 = 0; m0 < a.m; m0 += 16 * MT) {
      f32x4 acc[MT][NT] = {};
      const typename E::T* rows[MT];
      int from[MT];  // fp32: the lane whose operand is read, the tile's first row's where there is no row
#pragma unroll
      for (int t = 0; t < MT; ++t) from[t] = m0 + 16 * t + place_row(lane & 15) < a.m ? lane : lane & 48;
      if constexpr (!PREPARED) {
#pragma unroll
        for (int t = 0; t < MT; ++t)  // (rows beyond m: the last one's values again, for results that nobody stores)
          rows[t] = static_cast<const typename E::T*>(a.x) + (int64_t)min(m0 + 16 * t + place_row(lane & 15), a.m - 1) * a.k + 8 * quarter;
      }
      // A block's codes and scales; its operands of inputs 32 d and on (GUARDED: zeros beyond k); their products.
      auto load_codes = [&](int b, u32x4(&w)[NT], float(&scale)[NT][PER]) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int64_t tb = (int64_t)min(tile0 + n, a.tiles - 1) * a.blocks + b;
          if constexpr (STREAM)
            w[n] = __builtin_nontemporal_load(&a.codes[tb * 64 + lane]);
          else
            w[n] = a.codes[tb * 64 + lane];
          load_scales<PER>(a.scales + (tb * kTile + (lane & 15)) * PER, scale[n]);
        }
      };
      auto load_x = [&](int b, int d, V(&x)[MT][TERMS], auto guarded) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          if constexpr (PREPARED) {
#pragma unroll
            for (int i = 0; i < TERMS; ++i)
              x[t][i] = __builtin_bit_cast(V, a.terms[(((int64_t)(m0 / 16 + t) * a.blocks * 4 + b * 4 + d) * TERMS + i) * 64 + from[t]]);
          } else {
            const int at = b * kBlockK + 32 * d, left = decltype(guarded)::value ? a.k - at - 8 * quarter : 8;
            if (left >= 8) {
              load_operand<DTYPE>(rows[t] + at, x[t]);
            } else {
              // (loads of the last input in the place of those beyond it: none waits for a branch)
              typename E::T f[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) f[i] = rows[t][min(at + i, a.k - 1 - 8 * quarter)];
#pragma unroll
              for (int i = 0; i < 8; ++i) f[i] = i < left ? f[i] : (typename E::T)0.f;
              load_operand<DTYPE>(f, x[t]);
            }
          }
        }
      };
      f32x4 sum[MT][NT];
      auto multiply = [&](int d, const u32x4(&w)[NT], const float(&scale)[NT][PER], const V(&x)[MT][TERMS]) {
        V wv[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) wv[n] = Op::weights(w[n][d]);
        // (term by term: an instruction that adds to the one before it would wait for it)
#pragma unroll
        for (int i = 0; i < TERMS; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < MT; ++t)
              sum[t][n] = Op::mma(x[t][i], wv[n], i == 0 && d * 32 % GROUP == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sum[t][n]);
        if ((d + 1) * 32 % GROUP == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int r = 0; r < REGS; ++r) acc[t][n][r] = fmaf(sum[t][n][r], scale[n][d * 32 / GROUP], acc[t][n][r]);
        }
      };
      u32x4 w[NT];
      float scale[NT][PER];
      const int full = PREPARED ? end : min(end, a.k / kBlockK);
      int b = begin + wave;
      if constexpr (MT == 2 || MT == 3) {
        // Two waves on a SIMD do not hide a load: operands are asked for two steps ahead, codes one block ahead.  (64 rows leave no
        // registers for that.  64 x 4096 -> 8000: 20.8 us without, 23.4 with; 48 x 12000 -> 500: 18.8 without, 15.9 with.  As it is, the
        // kernels of 64 rows in 16 bits keep 304 bytes a lane in scratch memory with groups of 32 and 96 with groups of 64, none with 128,
        // 20.9 and 18.4 us; those of 48 rows 36 with groups of 32, in fp32 20 with groups of 128.)
        if (b < full) {
          V x[2][MT][TERMS];
          load_codes(b, w, scale);
          load_x(b, 0, x[0], std::false_type());
          load_x(b, 1, x[1], std::false_type());
          for (; b < full; b += waves) {
            const int next = b + waves < full ? b + waves : b;  // (the last one's again)
            u32x4 next_w[NT];
            float next_scale[NT][PER];
            multiply(0, w, scale, x[0]);
            load_x(b, 2, x[0], std::false_type());
            __builtin_amdgcn_sched_barrier(0);
            multiply(1, w, scale, x[1]);
            load_x(b, 3, x[1], std::false_type());
            load_codes(next, next_w, next_scale);
            __builtin_amdgcn_sched_barrier(0);
            multiply(2, w, scale, x[0]);
            load_x(next, 0, x[0], std::false_type());
            __builtin_amdgcn_sched_barrier(0);
            multiply(3, w, scale, x[1]);
            load_x(next, 1, x[1], std::false_type());
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              w[n] = next_w[n];
#pragma unroll
              for (int g = 0; g < PER; ++g) scale[n][g] = next_scale[n][g];
            }
          }
        }
      } else {
        for (; b < full; b += waves) {
          load_codes(b, w, scale);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            V x[MT][TERMS];
            load_x(b, d, x, std::false_type());
            multiply(d, w, scale, x);
          }
        }
      }
      if (!PREPARED && b < end) {
        load_codes(b, w, scale);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          V x[MT][TERMS] = {};
          if (b * kBlockK + 32 * d < a.k) load_x(b, d, x, std::true_type());
          multiply(d, w, scale, x);
        }
      }

#pragma unroll
      for (int t = 0; t < MT; ++t) {
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < REGS; ++r) parts[wave * SLOT + (n * REGS + r) * 64 + lane] = acc[t][n][r];
        __syncthreads();
        for (int i = threadIdx.x; i < SLOT; i += blockDim.x) {
          float v = parts[i];
#pragma unroll 4
          for (int p = 1; p < waves; ++p) v += parts[p * SLOT + i];
          const int nr = i >> 6, out = (tile0 + nr / REGS) * kTile + (i & 15), row = m0 + 16 * t + 4 * (nr % REGS) + (i >> 4 & 3);
          if (out >= a.o || row >= a.m) continue;
          const int64_t at = (int64_t)row * a.o + out;
          if (a.splits > 1) {
            a.parts[(int64_t)blockIdx.y * a.m * a.o + at] = v;
          } else {
            if (a.bias) v += E::to_float(static_cast<const typename E::T*>(a.bias)[out]);
            if (a.relu) v = v > 0.f ? v : 0.f;
            static_cast<typename E::T*>(a.y)[at] = E::from_float(v);
          }
        }
      }
    }
  }
}

// The splits' sums in one: a workgroup for 256 outputs of a row.
template <int DTYPE>
__global__ __launch_bounds__(256) void q4_join_kernel(Q4Args a) {
  typedef Elem<DTYPE> E;
  const int out = blockIdx.x * 256 + threadIdx.x;
  if (out >= a.o) return;
  const int64_t count = (int64_t)a.m * a.o;
  const float bias = a.bias ? E::to_float(static_cast<const typename E::T*>(a.bias)[out]) : 0.f;
  for (int row = blockIdx.y; row < a.m; row += gridDim.y) {
    const int64_t i = (int64_t)row * a.o + out;
    float v = a.parts[i];
#pragma unroll 4
    for (int s = 1; s < a.splits; ++s) v += a.parts[s * count + i];
    v += bias;
    if (a.relu) v = v > 0.f ? v : 0.f;
    static_cast<typename E::T*>(a.y)[i] = E::from_float(v);
  }
}

int m_tiles(const q4_desc* d) { return std::max(1, std::min((d->p.m + 15) / 16, 4)); }

size_t terms_bytes(const q4_desc* d) {
  const size_t tiles = ((size_t)d->p.m + 15) / 16, per = m_tiles(d);
  return (tiles + per - 1) / per * per * d->blocks * 4 * 3 * 1024;
}

size_t codes_bytes(const q4_desc* d) { return (size_t)d->tiles * d->blocks * 1024; }

size_t packed_bytes(const q4_desc* d) { return codes_bytes(d) + (size_t)d->tiles * d->blocks * kTile * (kBlockK / d->p.group) * 2; }

template <int DTYPE, int MT, int NT, int REGS, bool STREAM = false, bool PREPARED = DTYPE == MI355_F32>
void launch_group(const q4_desc* d, const Q4Args& a, hipStream_t stream) {
  const int groups = (d->tiles + NT - 1) / NT;
  const dim3 grid(std::min(groups, 1 << 22), d->splits), block(64 * d->waves);
  const size_t lds = (size_t)d->waves * NT * REGS * 256;  // at most 64 KB
  switch (d->p.group) {
    case 32: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, NT, REGS, 32, STREAM, PREPARED>), grid, block, lds, stream, a); break;
    case 64: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, NT, REGS, 64, STREAM, PREPARED>), grid, block, lds, stream, a); break;
    default: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, NT, REGS, 128, STREAM, PREPARED>), grid, block, lds, stream, a);
  }
}

// Codes of weights that the last-level cache (256 MB) does not hold from call to call go around it.  us through it and around it, one row of 4096
// bf16: weights that it does not hold at the call, as after other layers' work, 60.7 and 56.1 (282 MB packed), 64.1 and 59.0 (254), 50.1
// and 45.3 (226); the same weights call after call 70.9 and 65.3 (330), 53.9 and 56.1 (282), 46.2 and 58.2 (254), 35.6 and 45.0 (226): from
// 256 MB on what they lose is less and less, and what they gain is not.  (Batches of more than 16 rows are not bound by the codes.)
bool streams(const q4_desc* d) { return d->p.m <= 16 && packed_bytes(d) > (size_t)256 << 20; }

// Tiles of a workgroup for up to four rows and many outputs.  4096 x 128256: bf16 2 tiles 58.7 us, 4 65.7; fp32, whose operands are three
// times as many loads, 95.4 and 67.6.
template <int DTYPE>
constexpr int kManyTiles = DTYPE == MI355_F32 ? 4 : 2;

template <int DTYPE>
int launch_forward(const q4_desc* d, const Q4Args& a, hipStream_t stream) {
  if (d->prepared) {
    const int64_t lanes = (int64_t)(terms_bytes(d) / 48);
    hipLaunchKernelGGL(x_terms_kernel, dim3((uint32_t)std::min((lanes + 255) / 256, kMostBlocks)), dim3(256), 0, stream, static_cast<const float*>(a.x), a.terms, a.m, a.k,
                       d->blocks * 4, lanes);
    const int e = (int)hipGetLastError();
    if (e) return e;
  }
  const bool stream_codes = streams(d);
  switch (m_tiles(d)) {
    case 1:
      if (d->p.m <= 4) {
        if (d->nt == 1)
          d->prepared ? launch_group<DTYPE, 1, 1, 1>(d, a, stream) : launch_group<DTYPE, 1, 1, 1, false, false>(d, a, stream);
        else
          stream_codes ? launch_group<DTYPE, 1, kManyTiles<DTYPE>, 1, true>(d, a, stream) : launch_group<DTYPE, 1, kManyTiles<DTYPE>, 1>(d, a, stream);
      } else if (d->nt == 1) {
        d->prepared ? launch_group<DTYPE, 1, 1, 4>(d, a, stream) : launch_group<DTYPE, 1, 1, 4, false, false>(d, a, stream);
      } else if (d->nt == 2) {
        d->prepared ? launch_group<DTYPE, 1, 2, 4>(d, a, stream) : launch_group<DTYPE, 1, 2, 4, false, false>(d, a, stream);
      } else {
        stream_codes ? launch_group<DTYPE, 1, 4, 4, true>(d, a, stream) : launch_group<DTYPE, 1, 4, 4>(d, a, stream);
      }
      break;
    case 2: launch_group<DTYPE, 2, 4, 4>(d, a, stream); break;
    case 3: launch_group<DTYPE, 3, 4, 4>(d, a, stream); break;
    default: launch_group<DTYPE, 4, 4, 4>(d, a, stream);
  }
  int e = (int)hipGetLastError();
  if (e || d->splits == 1) return e;
  hipLaunchKernelGGL(q4_join_kernel<DTYPE>, dim3((d->p.num_output + 255) / 256, std::min(d->p.m, 65535)), dim3(256), 0, stream, a);
  return (int)hipGetLastError();
}

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int q4_desc_create(q4_desc_t** out, const q4_params_t* pp) {
  if (!out || !pp) return CONV_EINVAL;
  const q4_params_t p = *pp;
  if (p.m < 0 || p.k < 1 || p.num_output < 1 || (p.dtype != MI355_F32 && p.dtype != MI355_F16 && p.dtype != MI355_BF16)) return CONV_EINVAL;
  if ((p.group != 32 && p.group != 64 && p.group != 128) || (p.bias_term != 0 && p.bias_term != 1) || (p.relu != 0 && p.relu != 1))
    return CONV_EINVAL;
  const int64_t M = p.m, K = p.k, O = p.num_output;
  if (M * K >= kMaxElems || O * K >= kMaxElems || M * O >= kMaxElems) return CONV_ESHAPE;
  q4_desc* d = new (std::nothrow) q4_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->p = p;
  d->tiles = (p.num_output + kTile - 1) / kTile;
  d->blocks = (p.k + kBlockK - 1) / kBlockK;
  const int mt = m_tiles(d);
  // Tiles of a workgroup: a load of x serves them all, but where there are few of them they are workgroups of their own.  One row,
  // 4096 x 4096 (256 tiles): 1 tile 5.1 us, 2 tiles 7.0; 4096 x 128256 (8016): 74.4 and 62.3.  16 rows, 4096 x 20000 (1250): 2 tiles 16.7 us,
  // 4 16.2; 4096 x 30000: 23.2 and 19.1; 4096 x 128256: 103 and 64.
  const bool wide = p.dtype == MI355_F32;  // (1 x 4096 -> 30000 fp32, 1875 tiles: 1 tile 35.5 us, 4 24.4)
  d->nt = mt > 1                                       ? 4
          : p.m > 4                                    ? (d->tiles <= kUnits ? 1 : d->tiles < 4 * kUnits ? 2 : 4)
          : d->tiles < (wide ? 4 : 8) * kUnits         ? 1
          : wide                                       ? kManyTiles<MI355_F32>
                                                       : kManyTiles<MI355_BF16>;
  const int groups = (d->tiles + d->nt - 1) / d->nt;
  // Waves: as many as there may be where a compute unit has one workgroup, four where it has several (8 rows, 4096 x 100000: 4 waves
  // 58 us, 8 waves 64; 16 rows, 4096 x 4096: 4 waves 12.9, 8 8.9, 16 8.1); at least two blocks for each then.
  d->waves = groups > kUnits ? 4 : mt > 1 || p.m <= 4 ? 8 : 16;
  d->splits = 1;
  d->per_split = d->blocks;
  if (mt > 1) {  // 48 rows, 9216 x 4096: 1 part 40.8 us, 2 27.7, 4 22.1; 64 rows, 4096 x 8000, 125 groups: 1 part 24.6, 2 20.5, 4 27.5
    const int splits = std::max(1, std::min(kUnits / groups, d->blocks / d->waves));
    d->per_split = (d->blocks + splits - 1) / splits;
    d->splits = (d->blocks + d->per_split - 1) / d->per_split;
  }
  d->waves = std::max(1, std::min(d->waves, groups > kUnits ? (d->per_split + 1) / 2 : d->per_split));
  // fp32 x is cut into its terms once, by a launch of its own, but where little is cut: 4 x 76 -> 104 5.4 us, prepared 7.8; 5 x 2251 -> 45 9.0 and
  // 8.7, 1 x 4096 -> 4096 12.3 and 10.5.
  d->prepared = p.dtype == MI355_F32 && (d->nt == 4 || groups > kUnits || d->blocks > 8);
  if (p.m > 0) {
    if (d->prepared) d->ws_bytes += terms_bytes(d);
    if (d->splits > 1) d->ws_bytes += (size_t)d->splits * p.m * p.num_output * 4;
  }
  snprintf(d->names, sizeof(d->names), "fwd=%sq4[m%d,n%d%s%s](S=%d,W=%d)", d->prepared ? "terms+" : "", 16 * mt, 16 * d->nt, p.m <= 4 ? ",r1" : "", streams(d) && d->nt > (p.m <= 4 ? 1 : 2) ? ",stream" : "", d->splits, d->waves);
  *out = d;
  return CONV_OK;
}

int q4_desc_destroy(q4_desc_t* d) {
  if (!d) return CONV_EINVAL;
  delete d;
  return CONV_OK;
}

int q4_desc_workspace_bytes(const q4_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = d->ws_bytes;
  return CONV_OK;
}

int q4_desc_packed_bytes(const q4_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = packed_bytes(d);
  return CONV_OK;
}

const char* q4_desc_kernel_names(const q4_desc_t* d) { return d ? d->names : ""; }

int q4_pack(const q4_desc_t* d, const uint8_t* codes, const uint16_t* scales, void* packed, void* hip_stream) {
  if (!d || !codes || !scales || !packed || ((uintptr_t)packed & 15u)) return CONV_EINVAL;
  const int64_t vectors = (int64_t)d->tiles * d->blocks * 64;
  const bool words = d->p.k % 8 == 0 && ((uintptr_t)codes & 3u) == 0;
  hipLaunchKernelGGL(words ? q4_pack_kernel<true> : q4_pack_kernel<false>, dim3((uint32_t)std::min((vectors + 255) / 256, kMostBlocks)), dim3(256), 0, (hipStream_t)hip_stream, codes, scales,
                     static_cast<u32x4*>(packed), reinterpret_cast<uint16_t*>(static_cast<char*>(packed) + codes_bytes(d)), d->p.k, d->p.num_output,
                     d->blocks, vectors, d->p.group);
  const int e = (int)hipGetLastError();
  return e ? record_hip_error(e) : CONV_OK;
}

int q4_forward(const q4_desc_t* d, const void* x, const void* packed, const void* bias, void* y, void* ws, size_t ws_bytes,
               void* hip_stream) {
  if (!d || !packed || ((uintptr_t)packed & 15u)) return CONV_EINVAL;
  if ((d->p.bias_term != 0) != (bias != nullptr)) return CONV_EINVAL;
  if (d->p.m == 0) return CONV_OK;
  if (!x || !y) return CONV_EINVAL;
  if (d->ws_bytes && (!ws || ws_bytes < d->ws_bytes)) return CONV_EWORKSPACE;
  if (d->ws_bytes && ((uintptr_t)ws & 15u)) return CONV_EINVAL;
  Q4Args a = {};
  a.x = x;
  a.codes = static_cast<const u32x4*>(packed);
  a.scales = reinterpret_cast<const uint16_t*>(static_cast<const char*>(packed) + codes_bytes(d));
  a.bias = bias;
  a.y = y;
  a.m = d->p.m;
  a.k = d->p.k;
  a.o = d->p.num_output;
  a.tiles = d->tiles;
  a.blocks = d->blocks;
  a.relu = d->p.relu;
  a.splits = d->splits;
  a.per_split = d->per_split;
  char* const space = static_cast<char*>(ws);
  a.terms = reinterpret_cast<u32x4*>(space);
  a.parts = reinterpret_cast<float*>(space + (d->prepared ? terms_bytes(d) : 0));
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int e = d->p.dtype == MI355_F32   ? launch_forward<MI355_F32>(d, a, stream)
                : d->p.dtype == MI355_F16 ? launch_forward<MI355_F16>(d, a, stream)
                                          : launch_forward<MI355_BF16>(d, a, stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
