// The norm over many tensors and clipping by it (include/mi355gn.h): a pass that sums squares, and one that multiplies.
//
// Bound by memory: every gradient is read twice and written once (in place and unclipped: read once).  The factor needs all squares
// first, so what the second pass reads again comes from memory but for what the last-level cache (256 MB) still holds; it
// walks the gradients from their end, where that is.
// The squares are summed in fp64, whose multiply-add runs at fp32's rate on this chip: no square of an fp32 value overflows or
// vanishes in it.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "device_utils.h"
#include "elements.h"
#include "internal.h"
#include "mi355gn.h"

struct gn_desc {
  int32_t tensors;
  int64_t* counts;
  int32_t* dtypes;
  int64_t bytes;
  size_t ws_bytes;
  char names[64];
};

namespace mi355conv {

namespace {

constexpr int kSegments = 96;      // of one launch: their table is a kernel argument
constexpr int kMaxTensors = 1 << 18;
constexpr int kThreads = 256;
constexpr int kBlocks = 2048;      // eight workgroups on each compute unit: partial sums of a call, one a workgroup
constexpr int kMaxLaunches = (kMaxTensors + kSegments - 1) / kSegments;

// Tensors of a type that follow each other in memory.
struct Segment {
  const void* in;
  void* out;
  int64_t count;
  int32_t dtype;
  int32_t chunk0;  // chunks of the launch before this segment
};

struct GnArgs {
  Segment seg[kSegments];
  int32_t segments, chunks;
  int32_t chunk_bytes;
  int32_t parts;       // partial sums of the whole call
  int32_t part0;       // of this launch's first workgroup
  int32_t last;        // the launch that writes the norm
  double limit;
  double* sums;
  float* norm;
};

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// The workgroup's sum, in every thread.
__device__ __forceinline__ double block_add(double v, double (&lds)[kThreads / 64]) {
  v = wave_add(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  __syncthreads();
  return v;
}

// Which segment a chunk belongs to: the last one that starts at or before it.
__device__ __forceinline__ int segment_of(const GnArgs& a, int chunk) {
  int lo = 0, hi = a.segments - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seg[mid].chunk0 <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// f(element values of a vector, how many) over the elements [from, to) of a segment.
template <int DTYPE>
__device__ __forceinline__ double sum_range(const void* base, int64_t from, int64_t to) {
  typedef Elem<DTYPE> E;
  const typename E::T* const p = static_cast<const typename E::T*>(base) + from;
  const int n = (int)(to - from), full = n / E::VEC;
  double acc[2] = {0., 0.};
#pragma unroll 4
  for (int v = threadIdx.x; v < full; v += kThreads) {
    const u32x4 r = load_vec<E>(p + v * E::VEC);
#pragma unroll
    for (int i = 0; i < E::VEC; ++i) {
      const double x = (double)E::get(r, i);
      acc[i & 1] = fma(x, x, acc[i & 1]);
    }
  }
  for (int i = full * E::VEC + threadIdx.x; i < n; i += kThreads) {
    const double x = (double)E::to_float(p[i]);
    acc[0] = fma(x, x, acc[0]);
  }
  return acc[0] + acc[1];
}

struct __attribute__((packed, aligned(8))) Pair64Mem {
  double v[2];
};

template <>
__device__ __forceinline__ double sum_range<MI355_F64>(const void* base, int64_t from, int64_t to) {
  const double* const p = static_cast<const double*>(base) + from;
  const int n = (int)(to - from), full = n / 2;
  double acc[2] = {0., 0.};
#pragma unroll 4
  for (int v = threadIdx.x; v < full; v += kThreads) {
    const Pair64Mem r = *reinterpret_cast<const Pair64Mem*>(p + 2 * v);
    acc[0] = fma(r.v[0], r.v[0], acc[0]);
    acc[1] = fma(r.v[1], r.v[1], acc[1]);
  }
  if ((n & 1) && threadIdx.x == 0) acc[0] = fma(p[n - 1], p[n - 1], acc[0]);
  return acc[0] + acc[1];
}

template <int DTYPE>
__device__ __forceinline__ void scale_range(const void* base, void* out, int64_t from, int64_t to, double factor) {
  typedef Elem<DTYPE> E;
  const typename E::T* const p = static_cast<const typename E::T*>(base) + from;
  typename E::T* const q = static_cast<typename E::T*>(out) + from;
  const int n = (int)(to - from), full = n / E::VEC;
  const float f = (float)factor;
#pragma unroll 4
  for (int v = threadIdx.x; v < full; v += kThreads) {
    const u32x4 r = load_vec<E>(p + v * E::VEC);
    float x[E::VEC];
#pragma unroll
    for (int i = 0; i < E::VEC; ++i) x[i] = E::get(r, i) * f;
    store_vec<E>(q + v * E::VEC, E::pack(x));
  }
  for (int i = full * E::VEC + threadIdx.x; i < n; i += kThreads) q[i] = E::from_float(E::to_float(p[i]) * f);
}

template <>
__device__ __forceinline__ void scale_range<MI355_F64>(const void* base, void* out, int64_t from, int64_t to, double factor) {
  const double* const p = static_cast<const double*>(base) + from;
  double* const q = static_cast<double*>(out) + from;
  const int n = (int)(to - from), full = n / 2;
#pragma unroll 4
  for (int v = threadIdx.x; v < full; v += kThreads) {
    Pair64Mem r = *reinterpret_cast<const Pair64Mem*>(p + 2 * v);
    r.v[0] *= factor;
    r.v[1] *= factor;
    *reinterpret_cast<Pair64Mem*>(q + 2 * v) = r;
  }
  if ((n & 1) && threadIdx.x == 0) q[n - 1] = p[n - 1] * factor;
}

__device__ __forceinline__ int elem_bytes(int dtype) { return dtype == MI355_F64 ? 8 : dtype == MI355_F32 ? 4 : 2; }

__global__ __launch_bounds__(kThreads) void gn_sum_kernel(const GnArgs a) {
  __shared__ double lds[kThreads / 64];
  double sum = 0.;
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Segment& s = a.seg[segment_of(a, c)];
    const int64_t per = a.chunk_bytes / elem_bytes(s.dtype), from = (int64_t)(c - s.chunk0) * per;
    const int64_t to = from + per < s.count ? from + per : s.count;
    switch (s.dtype) {
      case MI355_F32: sum += sum_range<MI355_F32>(s.in, from, to); break;
      case MI355_F16: sum += sum_range<MI355_F16>(s.in, from, to); break;
      case MI355_BF16: sum += sum_range<MI355_BF16>(s.in, from, to); break;
      default: sum += sum_range<MI355_F64>(s.in, from, to);
    }
  }
  sum = block_add(sum, lds);
  if (threadIdx.x == 0) a.sums[a.part0 + blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void gn_scale_kernel(const GnArgs a) {
  __shared__ double lds[kThreads / 64];
  double sum = 0.;
  for (int i = threadIdx.x; i < a.parts; i += kThreads) sum += a.sums[i];
  const double norm = sqrt(block_add(sum, lds));
  if (a.last && a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const double factor = norm > a.limit ? a.limit / norm : 1.;
  for (int c0 = blockIdx.x; c0 < a.chunks; c0 += gridDim.x) {
    const int c = a.chunks - 1 - c0;
    const Segment& s = a.seg[segment_of(a, c)];
    if (factor == 1. && s.in == s.out) continue;
    const int64_t per = a.chunk_bytes / elem_bytes(s.dtype), from = (int64_t)(c - s.chunk0) * per;
    const int64_t to = from + per < s.count ? from + per : s.count;
    switch (s.dtype) {
      case MI355_F32: scale_range<MI355_F32>(s.in, s.out, from, to, factor); break;
      case MI355_F16: scale_range<MI355_F16>(s.in, s.out, from, to, factor); break;
      case MI355_BF16: scale_range<MI355_BF16>(s.in, s.out, from, to, factor); break;
      default: scale_range<MI355_F64>(s.in, s.out, from, to, factor);
    }
  }
}

// The tensors in runs of those that follow each other, from tensor i on: the table of one launch.  Returns the next launch's first.
int next_launch(const gn_desc* d, const void* const* grads, void* const* outs, int i, int chunk_bytes, GnArgs& a) {
  a.segments = a.chunks = 0;
  for (; i < d->tensors; ++i) {
    const int64_t n = d->counts[i];
    if (n == 0) continue;
    const int size = dtype_bytes(d->dtypes[i]);
    Segment* const s = a.segments ? &a.seg[a.segments - 1] : nullptr;
    if (s && s->dtype == d->dtypes[i] && static_cast<const char*>(s->in) + s->count * size == grads[i] &&
        static_cast<char*>(s->out) + s->count * size == outs[i]) {
      s->count += n;
      continue;
    }
    if (a.segments == kSegments) break;
    a.seg[a.segments++] = Segment{grads[i], outs[i], n, d->dtypes[i], 0};
  }
  for (int k = 0; k < a.segments; ++k) {
    Segment& s = a.seg[k];
    s.chunk0 = a.chunks;
    const int64_t per = chunk_bytes / dtype_bytes(s.dtype);
    a.chunks += (int32_t)((s.count + per - 1) / per);
  }
  return i;
}

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int gn_desc_create(gn_desc_t** out, const gn_params_t* p) {
  if (!out || !p || p->tensors < 0 || (p->tensors > 0 && (!p->counts || !p->dtypes))) return CONV_EINVAL;
  if (p->tensors > kMaxTensors) return CONV_ESHAPE;
  int64_t total = 0, bytes = 0;
  for (int i = 0; i < p->tensors; ++i) {
    if (p->counts[i] < 0 || p->dtypes[i] < MI355_F32 || p->dtypes[i] > MI355_F64) return CONV_EINVAL;
    if (p->counts[i] >= (int64_t)1 << 40 || (total += p->counts[i]) >= (int64_t)1 << 40) return CONV_ESHAPE;
    bytes += p->counts[i] * dtype_bytes(p->dtypes[i]);
  }
  gn_desc* d = new (std::nothrow) gn_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->tensors = p->tensors;
  d->bytes = bytes;
  if (p->tensors > 0) {
    d->counts = new (std::nothrow) int64_t[p->tensors];
    d->dtypes = new (std::nothrow) int32_t[p->tensors];
    if (!d->counts || !d->dtypes) {
      gn_desc_destroy(d);
      return CONV_EINVAL;
    }
    std::copy(p->counts, p->counts + p->tensors, d->counts);
    std::copy(p->dtypes, p->dtypes + p->tensors, d->dtypes);
  }
  d->ws_bytes = (size_t)(kBlocks + kMaxLaunches) * sizeof(double);
  snprintf(d->names, sizeof(d->names), "clip=gn_sum+gn_scale(T=%d)", d->tensors);
  *out = d;
  return CONV_OK;
}

int gn_desc_destroy(gn_desc_t* d) {
  if (!d) return CONV_EINVAL;
  delete[] d->counts;
  delete[] d->dtypes;
  delete d;
  return CONV_OK;
}

int gn_desc_workspace_bytes(const gn_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = d->ws_bytes;
  return CONV_OK;
}

const char* gn_desc_kernel_names(const gn_desc_t* d) { return d ? d->names : ""; }

int gn_clip(const gn_desc_t* d, const void* const* grads, double limit, void* const* outs, float* norm, void* ws, size_t ws_bytes,
            void* hip_stream) {
  if (!d || !(limit >= 0.) || (d->tensors > 0 && (!grads || !outs))) return CONV_EINVAL;
  for (int i = 0; i < d->tensors; ++i)
    if (d->counts[i] > 0 && (!grads[i] || !outs[i])) return CONV_EINVAL;
  if (!ws || ws_bytes < d->ws_bytes) return CONV_EWORKSPACE;
  if ((uintptr_t)ws & 15u) return CONV_EINVAL;
  const hipStream_t stream = (hipStream_t)hip_stream;
  GnArgs a = {};
  // A chunk is what a workgroup takes at a time: large ones where there is enough for every workgroup.
  a.chunk_bytes = (int32_t)std::min<int64_t>(std::max<int64_t>(d->bytes / kBlocks / 4096 * 4096, 4096), 64 << 10);
  while (d->bytes / a.chunk_bytes >= 1 << 30) a.chunk_bytes *= 2;
  a.limit = limit;
  a.sums = static_cast<double*>(ws);
  a.norm = norm;
  int launches = 0;
  for (int i = 0; i < d->tensors || launches == 0; ++launches) {
    GnArgs t = a;
    i = next_launch(d, grads, outs, i, a.chunk_bytes, t);
  }
  const int most = std::max(1, kBlocks / launches);
  a.parts = 0;
  for (int i = 0, k = 0; k < launches; ++k) {
    i = next_launch(d, grads, outs, i, a.chunk_bytes, a);
    a.part0 = a.parts;
    const int blocks = std::max(1, std::min(a.chunks, most));
    a.parts += blocks;
    hipLaunchKernelGGL(gn_sum_kernel, dim3(blocks), dim3(kThreads), 0, stream, a);
    const int e = (int)hipGetLastError();
    if (e) return record_hip_error(e);
  }
  for (int i = 0, k = 0; k < launches; ++k) {
    i = next_launch(d, grads, outs, i, a.chunk_bytes, a);
    a.last = k == launches - 1;
    hipLaunchKernelGGL(gn_scale_kernel, dim3(std::max(1, std::min(a.chunks, kBlocks))), dim3(kThreads), 0, stream, a);
    const int e = (int)hipGetLastError();
    if (e) return record_hip_error(e);
  }
  return CONV_OK;
}

}  // extern "C"
