// The norm over many tensors and clipping by it (include/mi355gn.h): a pass that sums squares, and one that multiplies.
//
// Bound by memory: every gradient is read twice and written once (in place and unclipped: read once).  The factor needs all squares
// first, so what the second pass reads again comes from memory but for what the last-level cache (256 MB) still holds; a launch of
// it (up to 96 runs of tensors) walks its gradients from their end, where that is.  Several launches go from the first on, as those of
// the first pass do; what is in the cache is then the last ones', and waits there, as the others' reads and writes go around it.  242
// tensors of their own memory, 708 MB clipped: 325.5 us, as views of one buffer 314.7 (one state's buffers call after call).
// The squares are summed in fp64, whose multiply-add runs at fp32's rate on this chip: no square of an fp32 value overflows or
// vanishes in it.  Those of fp64 values may: the large and the small ones have sums of their own, of squares of scaled values (Squares).
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
#include "wave_ops.h"

struct gn_desc {
  int32_t tensors;
  int32_t ranges;  // sums of squares that there are: 3 with fp64 tensors, 1 without
  int64_t* counts;
  int32_t* dtypes;
  int64_t bytes;
  size_t ws_bytes;
  char names[64];
};

namespace mi355conv {

namespace {

// Of one launch: their table is a kernel argument, 3 KB of them; a short one where all fit that (a flat buffer for each type).
constexpr int kSegments = 96, kFewSegments = 8;
constexpr int kMaxTensors = 1 << 18;
constexpr int kThreads = 256;
constexpr int kChunk = 16 << 10;   // bytes that a workgroup takes at a time: four vectors a thread
constexpr int kSumBlocks = 4096, kScaleBlocks = 16384;
constexpr int kMaxLaunches = (kMaxTensors + kSegments - 1) / kSegments;
constexpr int kMostParts = kSumBlocks + kMaxLaunches;
// Up to this many partial sums each workgroup of the second pass adds them up for itself; beyond, a kernel in between does.
constexpr int kFewParts = 512;
// Of gradients that the last-level cache (256 MB) does not hold, the first pass reads around it all but this much at the end,
// where the second pass begins, or which it leaves alone until then.
constexpr int64_t kCacheBytes = (int64_t)256 << 20, kKeptBytes = (int64_t)192 << 20;

// Tensors of a type that follow each other in memory.
struct Segment {
  const void* in;
  void* out;
  int64_t count;
  int32_t dtype;
  int32_t chunk0;  // chunks of the launch before this segment
};

struct GnCall {
  int32_t segments, chunks;
  int32_t kept;        // chunks of this launch from this one on are read through the cache; chunks: all are
  int32_t parts;       // partial sums of the whole call
  int32_t part0;       // of this launch's first workgroup
  int32_t last;        // the launch that writes the norm
  int32_t ranges;
  double limit;
  double* sums;        // [ranges][kMostParts], then the factor where parts > kFewParts
  float* norm;
};

template <int SEGMENTS>
struct GnArgs : GnCall {
  Segment seg[SEGMENTS];
};

struct NormArgs {
  int32_t parts, ranges;
  double limit;
  double* sums;
  float* norm;
};

// The workgroup's sum, in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double (&lds)[THREADS / 64]) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
  return v;
}

// Sums of squares: of values from kLow to kHigh, of the smaller ones as x / kScale, of the larger ones as x kScale.  No square in them overflows
// or loses bits that count, nor do sums of 2^40: they stay between 2^-960 and 2^1000.
struct Squares {
  double mid, low, high;
};

constexpr double kLow = 0x1p-480, kHigh = 0x1p480, kScale = 0x1p-600;

__device__ __forceinline__ void add_square(Squares& s, double x) {
  const double size = fabs(x);
  if (size >= kHigh) {
    x *= kScale;
    s.high = fma(x, x, s.high);
  } else if (size < kLow) {
    x *= 1. / kScale;
    s.low = fma(x, x, s.low);
  } else {  // (NaN too)
    s.mid = fma(x, x, s.mid);
  }
}

__device__ __forceinline__ double norm_of(const Squares& s) {
  if (s.high > 0.) return sqrt(s.high + s.mid * kScale * kScale) * (1. / kScale);
  if (s.mid != 0.) return sqrt(s.mid + s.low * kScale * kScale);
  return sqrt(s.low) * kScale;
}

// The norm of all parts, by a workgroup.
template <int THREADS>
__device__ __forceinline__ double norm_of_parts(const double* sums, int parts, int ranges, double (&lds)[THREADS / 64]) {
  double total[3] = {0., 0., 0.};
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    if (r >= ranges) break;
    double sum = 0.;
    for (int i = threadIdx.x; i < parts; i += THREADS) sum += sums[r * kMostParts + i];
    if (r > 0) __syncthreads();
    total[r] = block_sum<THREADS>(sum, lds);
  }
  return norm_of(Squares{total[0], total[1], total[2]});
}

__device__ __forceinline__ double factor_of(double norm, double limit) { return norm > limit ? limit / norm : 1.; }

// Which segment a chunk belongs to: the last one that starts at or before it.
template <class Args>
__device__ __forceinline__ int segment_of(const Args& a, int chunk) {
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

// Both passes take a chunk, kChunk bytes or what is left of a segment, as four vectors a thread, all loaded before the first is used,
// and its last elements one by one.
template <int DTYPE, bool STREAM, class Vec, class One>
__device__ __forceinline__ void each(const Segment& s, int64_t from, Vec&& vec, One&& one) {
  typedef Elem<DTYPE> E;
  constexpr int VEC = E::VEC, PER = kChunk / 16 / kThreads;
  const typename E::T* const p = static_cast<const typename E::T*>(s.in) + from;
  const int64_t left = s.count - from;
  const int n = left < kChunk / 16 * VEC ? (int)left : kChunk / 16 * VEC, full = n / VEC;
  u32x4 r[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int v = j * kThreads + (int)threadIdx.x;
    if (v < full) r[j] = get_vec<E, STREAM>(p + v * VEC);
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int v = j * kThreads + (int)threadIdx.x;
    if (v < full) vec(r[j], from + v * VEC);
  }
  const int i = full * VEC + (int)threadIdx.x;
  if (i < n) one(p[i], from + i);
}

template <int DTYPE, bool STREAM>
__device__ __forceinline__ void sum_chunk(const Segment& s, int64_t from, Squares& sum) {
  typedef Elem<DTYPE> E;
  double acc[2] = {0., 0.};
  uint32_t any = 0;  // fp64: bits of the values but for their signs
  each<DTYPE, STREAM>(
      s, from,
      [&](const u32x4& r, int64_t) {
#pragma unroll
        for (int i = 0; i < E::VEC; ++i) {
          const double x = (double)E::get(r, i);
          acc[i & 1] = fma(x, x, acc[i & 1]);
        }
        if constexpr (DTYPE == MI355_F64) any |= r[0] | r[2] | (r[1] | r[3]) << 1;
      },
      [&](typename E::T v, int64_t) {
        const double x = (double)E::to_float(v);
        acc[0] = fma(x, x, acc[0]);
        any |= v != (typename E::T)0.f ? 1u : 0u;
      });
  const double squares = acc[0] + acc[1];
  if constexpr (DTYPE == MI355_F64) {
    // Of a thread's nine values at most, none overflowed then, and what vanished is below 2^-119 of the rest.  Otherwise, and but for zeros,
    // one by one.  (Each value looked at first: 1.25 GB clipped in 624 us, 583 so.  As much of zeros, looked at one by one: 753 us, 580 so.)
    if (any != 0 && !(squares >= 0x1p-900 && squares <= 0x1p960)) {
      each<DTYPE, false>(
          s, from,
          [&](const u32x4& r, int64_t) {
#pragma unroll
            for (int i = 0; i < E::VEC; ++i) add_square(sum, E::get(r, i));
          },
          [&](double v, int64_t) { add_square(sum, v); });
      return;
    }
  }
  sum.mid += squares;
}

// A factor in fp64, or in fp32, whose normal numbers do not reach as far down: below them it is a number of all 24 bits times a power of
// two, applied one after the other (3e38 clipped to 1 came out 5e-6 off by a subnormal factor, 1e25 to 1e-20 as zeros).
template <typename F>
struct Factor {
  F f;
  __device__ __forceinline__ explicit Factor(double factor) : f(factor) {}
  __device__ __forceinline__ F times(F x) const { return x * f; }
};

template <>
struct Factor<float> {
  float f;
  int e = 0;  // (an instruction a value that is not seen beside the memory's time)
  __device__ __forceinline__ explicit Factor(double factor) { f = (float)(factor < (double)FLT_MIN ? frexp(factor, &e) : factor); }
  __device__ __forceinline__ float times(float x) const { return ldexpf(x * f, e); }
};

template <int DTYPE, bool STREAM_IN, bool STREAM_OUT>
__device__ __forceinline__ void scale_chunk(const Segment& s, int64_t from, double factor) {
  typedef Elem<DTYPE> E;
  typedef decltype(E::get(u32x4(), 0)) F;  // fp64 for fp64, fp32 for the others
  typename E::T* const q = static_cast<typename E::T*>(s.out);
  const Factor<F> f(factor);
  each<DTYPE, STREAM_IN>(
      s, from,
      [&](const u32x4& r, int64_t at) {
        F x[E::VEC];
#pragma unroll
        for (int i = 0; i < E::VEC; ++i) x[i] = f.times(E::get(r, i));
        put_vec<E, STREAM_OUT>(q + at, E::pack(x));
      },
      [&](typename E::T v, int64_t at) { q[at] = E::from_float(f.times(E::to_float(v))); });
}

__device__ __forceinline__ int elem_shift(int dtype) { return dtype == MI355_F64 ? 3 : dtype == MI355_F32 ? 2 : 1; }

template <bool STREAM, bool WIDE>
__device__ __forceinline__ void sum_any(const Segment& s, int64_t from, Squares& sum) {
  switch (s.dtype) {
    case MI355_F32: sum_chunk<MI355_F32, STREAM>(s, from, sum); break;
    case MI355_F16: sum_chunk<MI355_F16, STREAM>(s, from, sum); break;
    case MI355_BF16: sum_chunk<MI355_BF16, STREAM>(s, from, sum); break;
    default:
      if constexpr (WIDE) sum_chunk<MI355_F64, STREAM>(s, from, sum);
  }
}

template <bool STREAM_IN, bool STREAM_OUT>
__device__ __forceinline__ void scale_any(const Segment& s, int64_t from, double factor) {
  switch (s.dtype) {
    case MI355_F32: scale_chunk<MI355_F32, STREAM_IN, STREAM_OUT>(s, from, factor); break;
    case MI355_F16: scale_chunk<MI355_F16, STREAM_IN, STREAM_OUT>(s, from, factor); break;
    case MI355_BF16: scale_chunk<MI355_BF16, STREAM_IN, STREAM_OUT>(s, from, factor); break;
    default: scale_chunk<MI355_F64, STREAM_IN, STREAM_OUT>(s, from, factor);
  }
}

// WIDE: with fp64 tensors.  (The sums that they need take registers, of which calls without them make more waves: 144 MB of fp32 and bf16
// clipped in 77.0 us with them, 73.5 without; 298 MB of fp64 in 145 us by five waves on a SIMD, 140 by six.)
template <int SEGMENTS, bool STREAM, bool WIDE>
__global__ __launch_bounds__(kThreads, 6) void gn_sum_kernel(const GnArgs<SEGMENTS> a) {
  __shared__ double lds[kThreads / 64];
  Squares sum = {0., 0., 0.};
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const Segment& s = a.seg[segment_of(a, c)];
    const int64_t from = (int64_t)(c - s.chunk0) * (kChunk >> elem_shift(s.dtype));
    if (STREAM && c < a.kept)
      sum_any<true, WIDE>(s, from, sum);
    else
      sum_any<false, WIDE>(s, from, sum);
  }
  double* const to = a.sums + a.part0 + blockIdx.x;
  const double mid = block_sum<kThreads>(sum.mid, lds);
  if (threadIdx.x == 0) to[0] = mid;
  if constexpr (!WIDE) return;
  __syncthreads();
  const double low = block_sum<kThreads>(sum.low, lds);
  __syncthreads();
  const double high = block_sum<kThreads>(sum.high, lds);
  if (threadIdx.x == 0) {
    to[kMostParts] = low;
    to[2 * kMostParts] = high;
  }
}

// The norm and the factor of many partial sums.
__global__ __launch_bounds__(1024) void gn_norm_kernel(const NormArgs a) {
  __shared__ double lds[16];
  const double norm = norm_of_parts<1024>(a.sums, a.parts, a.ranges, lds);
  if (threadIdx.x == 0) {
    if (a.norm) *a.norm = (float)norm;
    a.sums[a.ranges * kMostParts] = factor_of(norm, a.limit);
  }
}

template <int SEGMENTS, bool STREAM_IN, bool STREAM_OUT>
__global__ __launch_bounds__(kThreads) void gn_scale_kernel(const GnArgs<SEGMENTS> a) {
  __shared__ double lds[kThreads / 64];
  double factor;
  if (a.parts > kFewParts) {
    factor = a.sums[a.ranges * kMostParts];
  } else {
    const double norm = norm_of_parts<kThreads>(a.sums, a.parts, a.ranges, lds);
    if (a.last && a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
    factor = factor_of(norm, a.limit);
  }
  for (int c0 = blockIdx.x; c0 < a.chunks; c0 += gridDim.x) {
    const int c = a.chunks - 1 - c0;
    const Segment& s = a.seg[segment_of(a, c)];
    if (factor == 1. && s.in == s.out) continue;
    const int64_t from = (int64_t)(c - s.chunk0) * (kChunk >> elem_shift(s.dtype));
    if (STREAM_IN && c < a.kept)
      scale_any<true, STREAM_OUT>(s, from, factor);
    else
      scale_any<false, STREAM_OUT>(s, from, factor);
  }
}

// The tensors in runs of those that follow each other, from tensor i on: the table of one launch.  Returns the next launch's first.
// (A run goes on where its type's last tensor ended, whatever other types stand between.)
int next_launch(const gn_desc* d, const void* const* grads, void* const* outs, int i, GnArgs<kSegments>& a) {
  a.segments = a.chunks = 0;
  Segment* open[4] = {};
  for (; i < d->tensors; ++i) {
    const int64_t n = d->counts[i];
    if (n == 0) continue;
    const int size = dtype_bytes(d->dtypes[i]);
    Segment* const s = open[d->dtypes[i]];
    if (s && static_cast<const char*>(s->in) + s->count * size == grads[i] && static_cast<char*>(s->out) + s->count * size == outs[i]) {
      s->count += n;
      continue;
    }
    if (a.segments == kSegments) break;
    a.seg[a.segments] = Segment{grads[i], outs[i], n, d->dtypes[i], 0};
    open[d->dtypes[i]] = &a.seg[a.segments++];
  }
  for (int k = 0; k < a.segments; ++k) {
    Segment& s = a.seg[k];
    s.chunk0 = a.chunks;
    const int64_t per = kChunk / dtype_bytes(s.dtype);
    a.chunks += (int32_t)((s.count + per - 1) / per);
  }
  return i;
}

GnArgs<kFewSegments> few(const GnArgs<kSegments>& a) {
  GnArgs<kFewSegments> t;
  static_cast<GnCall&>(t) = a;
  std::copy(a.seg, a.seg + kFewSegments, t.seg);
  return t;
}

template <bool STREAM, bool WIDE>
void launch_sum(const GnArgs<kSegments>& a, int blocks, hipStream_t stream) {
  if (a.segments <= kFewSegments)
    hipLaunchKernelGGL((gn_sum_kernel<kFewSegments, STREAM, WIDE>), dim3(blocks), dim3(kThreads), 0, stream, few(a));
  else
    hipLaunchKernelGGL((gn_sum_kernel<kSegments, STREAM, WIDE>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

template <bool STREAM_IN, bool STREAM_OUT>
void launch_scale(const GnArgs<kSegments>& a, int blocks, hipStream_t stream) {
  if (a.segments <= kFewSegments)
    hipLaunchKernelGGL((gn_scale_kernel<kFewSegments, STREAM_IN, STREAM_OUT>), dim3(blocks), dim3(kThreads), 0, stream, few(a));
  else
    hipLaunchKernelGGL((gn_scale_kernel<kSegments, STREAM_IN, STREAM_OUT>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

int run_clip(const gn_desc* d, const void* const* grads, void* const* outs, GnArgs<kSegments>& a, hipStream_t stream) {
  int launches = 0;
  int64_t chunks = 0, out_bytes = 0;  // of the outputs in other memory
  for (int i = 0; i < d->tensors || launches == 0; ++launches) {
    i = next_launch(d, grads, outs, i, a);
    chunks += a.chunks;
    for (int k = 0; k < a.segments; ++k)
      if (a.seg[k].in != a.seg[k].out) out_bytes += a.seg[k].count * dtype_bytes(a.seg[k].dtype);
  }
  const bool stream_in = d->bytes > kCacheBytes, stream_out = d->bytes + out_bytes > kCacheBytes;
  const int64_t kept = chunks - (stream_in ? kKeptBytes / kChunk : chunks);  // of all chunks, those from here on
  const int most = std::max(1, kSumBlocks / launches);
  int64_t before = 0;
  a.parts = 0;
  for (int i = 0, k = 0; k < launches; ++k) {
    if (launches > 1) i = next_launch(d, grads, outs, i, a);
    a.kept = (int32_t)std::max<int64_t>(0, std::min<int64_t>(kept - before, a.chunks));
    before += a.chunks;
    a.part0 = a.parts;
    const int blocks = std::max(1, std::min(a.chunks, most));
    a.parts += blocks;
    if (a.ranges > 1)
      stream_in ? launch_sum<true, true>(a, blocks, stream) : launch_sum<false, true>(a, blocks, stream);
    else
      stream_in ? launch_sum<true, false>(a, blocks, stream) : launch_sum<false, false>(a, blocks, stream);
    const int e = (int)hipGetLastError();
    if (e) return e;
  }
  if (a.parts > kFewParts) {
    const NormArgs n = {a.parts, a.ranges, a.limit, a.sums, a.norm};
    hipLaunchKernelGGL(gn_norm_kernel, dim3(1), dim3(1024), 0, stream, n);
    const int e = (int)hipGetLastError();
    if (e) return e;
  }
  before = 0;
  for (int i = 0, k = 0; k < launches; ++k) {
    if (launches > 1) i = next_launch(d, grads, outs, i, a);
    a.kept = (int32_t)std::max<int64_t>(0, std::min<int64_t>(kept - before, a.chunks));
    before += a.chunks;
    a.last = k == launches - 1;
    const int blocks = std::max(1, std::min(a.chunks, kScaleBlocks));
    stream_in ? launch_scale<true, true>(a, blocks, stream) : stream_out ? launch_scale<false, true>(a, blocks, stream) : launch_scale<false, false>(a, blocks, stream);
    const int e = (int)hipGetLastError();
    if (e) return e;
  }
  return 0;
}

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int gn_desc_create(gn_desc_t** out, const gn_params_t* p) {
  if (!out || !p || p->tensors < 0 || (p->tensors > 0 && (!p->counts || !p->dtypes))) return CONV_EINVAL;
  if (p->tensors > kMaxTensors) return CONV_ESHAPE;
  int64_t total = 0, bytes = 0;
  int ranges = 1;
  for (int i = 0; i < p->tensors; ++i) {
    if (p->counts[i] < 0 || p->dtypes[i] < MI355_F32 || p->dtypes[i] > MI355_F64) return CONV_EINVAL;
    if (p->counts[i] >= (int64_t)1 << 40 || (total += p->counts[i]) >= (int64_t)1 << 40) return CONV_ESHAPE;
    bytes += p->counts[i] * dtype_bytes(p->dtypes[i]);
    if (p->dtypes[i] == MI355_F64) ranges = 3;
  }
  gn_desc* d = new (std::nothrow) gn_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->tensors = p->tensors;
  d->bytes = bytes;
  d->ranges = ranges;
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
  d->ws_bytes = (size_t)(ranges * kMostParts + 1) * sizeof(double);
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
  GnArgs<kSegments> a = {};
  a.limit = limit;
  a.ranges = d->ranges;
  a.sums = static_cast<double*>(ws);
  a.norm = norm;
  const int e = run_clip(d, grads, outs, a, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
