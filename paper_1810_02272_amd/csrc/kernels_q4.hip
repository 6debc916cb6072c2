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

#include "device_utils.h"
#include "elements.h"
#include "internal.h"
#include "mi355q4.h"

struct q4_desc {
  q4_params_t p;
  int32_t tiles, blocks;  // of 16 outputs and 128 inputs
  size_t ws_bytes;
  char names[96];
};

namespace mi355conv {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 16, kBlockK = 128;
constexpr int64_t kMaxElems = (int64_t)1 << 30;

struct Q4Args {
  const void* x;
  const u32x4* codes;
  const uint16_t* scales;
  const void* bias;
  void* y;
  int32_t m, k, o, tiles, blocks;
  int32_t relu;
};

// One thread for each of a block's 64 vectors of codes, and the first ones for its scales.
__global__ __launch_bounds__(256) void q4_pack_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales,
                                                      u32x4* __restrict__ to, uint16_t* __restrict__ to_scales, int k, int o, int blocks,
                                                      int64_t vectors, int group) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v >= vectors) return;
  const int lane = (int)(v & 63);
  const int64_t tb = v >> 6;
  const int tile = (int)(tb / blocks), block = (int)(tb % blocks);
  const int row = tile * kTile + (lane & 15), stride = (k + 1) / 2;
  u32x4 w = {0, 0, 0, 0};
  if (row < o) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int at = block * kBlockK + 32 * d + 8 * (lane >> 4);
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

template <int DTYPE>
struct Operand;  // what the matrix instructions take for x and w: TERMS of them for x

template <>
struct Operand<MI355_BF16> {
  typedef bf16x8 V;
  static constexpr int TERMS = 1;
  static __device__ __forceinline__ V weights(uint32_t c) {
    V r;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 1);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, 1.f, 3);
    r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = d[0], r[5] = d[1], r[6] = e[0], r[7] = e[1];
    return r;
  }
  static __device__ __forceinline__ f32x4 mma(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

template <>
struct Operand<MI355_F16> {
  typedef f16x8 V;
  static constexpr int TERMS = 1;
  static __device__ __forceinline__ V weights(uint32_t c) {
    V r;
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 1);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.f, 3);
    r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = d[0], r[5] = d[1], r[6] = e[0], r[7] = e[1];
    return r;
  }
  static __device__ __forceinline__ f32x4 mma(V a, V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

template <>
struct Operand<MI355_F32> : Operand<MI355_BF16> {
  static constexpr int TERMS = 3;
};

// An fp32 value's terms: its leading 8 bits, the next 8, the last 8, each cut off and so exact.  What is not finite is the first term's.
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

// Eight consecutive inputs of a row of x from input `at` on, as operands; zeros beyond k.
template <int DTYPE>
__device__ __forceinline__ void load_x(const void* x, int64_t row, int at, int k, typename Operand<DTYPE>::V (&v)[Operand<DTYPE>::TERMS]) {
  typedef Elem<DTYPE> E;
  typedef typename Operand<DTYPE>::V V;
  const typename E::T* const p = static_cast<const typename E::T*>(x) + row * k + at;
  if constexpr (DTYPE == MI355_F32) {
    float f[8];
    if (at + 8 <= k) {
      const u32x4 a = load_vec<E>(p), b = load_vec<E>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = E::get(a, i);
        f[4 + i] = E::get(b, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = at + i < k ? p[i] : 0.f;
    }
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a[3], b[3];
      three_terms(f[2 * i], a);
      three_terms(f[2 * i + 1], b);
#pragma unroll
      for (int t = 0; t < 3; ++t) w[t][i] = a[t] | b[t] << 16;
    }
#pragma unroll
    for (int t = 0; t < 3; ++t) v[t] = __builtin_bit_cast(V, u32x4{w[t][0], w[t][1], w[t][2], w[t][3]});
  } else {
    if (at + 8 <= k) {
      v[0] = __builtin_bit_cast(V, load_vec<E>(p));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[0][i] = at + i < k ? p[i] : (typename E::T)0.f;
    }
  }
}

// MT times 16 rows of x by a tile of 16 outputs in a workgroup, whose waves take the blocks of inputs in turn.
template <int DTYPE, int MT, int GROUP>
__global__ __launch_bounds__(256) void q4_kernel(Q4Args a) {
  typedef Operand<DTYPE> Op;
  typedef Elem<DTYPE> E;
  constexpr int PER = kBlockK / GROUP;
  __shared__ f32x4 parts[4][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x;
  for (int m0 = blockIdx.y * 64; m0 < a.m; m0 += gridDim.y * 64) {
    f32x4 acc[MT] = {};
    for (int b = wave; b < a.blocks; b += 4) {
      const int64_t tb = (int64_t)tile * a.blocks + b;
      const u32x4 w = a.codes[tb * 64 + lane];
      float scale[PER];
#pragma unroll
      for (int g = 0; g < PER; ++g) scale[g] = __builtin_bit_cast(float, (uint32_t)a.scales[(tb * kTile + (lane & 15)) * PER + g] << 16);
      f32x4 sum[MT] = {};
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const typename Op::V wv = Op::weights(w[d]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int row = m0 + 16 * t + (lane & 15);
          typename Op::V x[Op::TERMS] = {};
          const int at = b * kBlockK + 32 * d + 8 * (lane >> 4);
          if (row < a.m && at < a.k) load_x<DTYPE>(a.x, row, at, a.k, x);
#pragma unroll
          for (int i = 0; i < Op::TERMS; ++i) sum[t] = Op::mma(x[i], wv, sum[t]);
          if ((d + 1) * 32 % GROUP == 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(sum[t][r], scale[d * 32 / GROUP], acc[t][r]);
            sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) parts[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < MT; t += 4) {
      const f32x4 z = (parts[0][t][lane] + parts[1][t][lane]) + (parts[2][t][lane] + parts[3][t][lane]);
      const int out = tile * kTile + (lane & 15);
      if (out < a.o) {
        const float bias = a.bias ? E::to_float(static_cast<const typename E::T*>(a.bias)[out]) : 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = m0 + 16 * t + 4 * (lane >> 4) + r;
          float v = z[r] + bias;
          if (a.relu) v = v > 0.f ? v : 0.f;
          if (row < a.m) static_cast<typename E::T*>(a.y)[(int64_t)row * a.o + out] = E::from_float(v);
        }
      }
    }
    __syncthreads();
  }
}

template <int DTYPE, int MT>
void launch_group(const Q4Args& a, int group, hipStream_t stream) {
  const dim3 grid(a.tiles, std::min((a.m + 63) / 64, 65535)), block(256);
  switch (group) {
    case 32: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, 32>), grid, block, 0, stream, a); break;
    case 64: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, 64>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((q4_kernel<DTYPE, MT, 128>), grid, block, 0, stream, a);
  }
}

template <int DTYPE>
void launch_rows(const Q4Args& a, int group, hipStream_t stream) {
  switch (std::min((a.m + 15) / 16, 4)) {
    case 1: launch_group<DTYPE, 1>(a, group, stream); break;
    case 2: launch_group<DTYPE, 2>(a, group, stream); break;
    case 3: launch_group<DTYPE, 3>(a, group, stream); break;
    default: launch_group<DTYPE, 4>(a, group, stream);
  }
}

size_t codes_bytes(const q4_desc* d) { return (size_t)d->tiles * d->blocks * 1024; }

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
  snprintf(d->names, sizeof(d->names), "fwd=q4[m%d]", std::min((p.m + 15) / 16, 4) * 16);
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
  *bytes = codes_bytes(d) + (size_t)d->tiles * d->blocks * kTile * (kBlockK / d->p.group) * 2;
  return CONV_OK;
}

const char* q4_desc_kernel_names(const q4_desc_t* d) { return d ? d->names : ""; }

int q4_pack(const q4_desc_t* d, const uint8_t* codes, const uint16_t* scales, void* packed, void* hip_stream) {
  if (!d || !codes || !scales || !packed || ((uintptr_t)packed & 15u)) return CONV_EINVAL;
  const int64_t vectors = (int64_t)d->tiles * d->blocks * 64;
  hipLaunchKernelGGL(q4_pack_kernel, dim3((uint32_t)((vectors + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream, codes, scales,
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
  switch (d->p.dtype) {
    case MI355_F32: launch_rows<MI355_F32>(a, d->p.group, (hipStream_t)hip_stream); break;
    case MI355_F16: launch_rows<MI355_F16>(a, d->p.group, (hipStream_t)hip_stream); break;
    default: launch_rows<MI355_BF16>(a, d->p.group, (hipStream_t)hip_stream);
  }
  const int e = (int)hipGetLastError();
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
