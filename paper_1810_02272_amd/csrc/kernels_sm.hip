// Drawing tokens under a temperature, top-k, top-p and min-p from given uniform numbers (include/mi355sm.h).
//
// A first launch reads the rows once, in segments, and leaves each segment's maximum and sum of weights.  Where there is no limit the second one
// finds the segment that the uniform number falls on, and the token in it.
// What is kept under limits is what a cut keeps, x > value or x = value and index <= last, and what min-p keeps: top-k and top-p only move the
// cut.  The second launch puts the logits near the maximum in a list, in the order of their indices; the cut's place in it is found by a histogram of the
// distances below the maximum, finer ones of a bin that holds many, and an exact order of the few of the last bin; the token by the
// sums of the list's weights.  Where the list does not hold what is kept, the same runs over the row itself.  (The histogram's weights are rounded to
// whole numbers; where the weights' own sums do not end in the bin that it picks, the cut is found by those.)
// Rows of a single segment take one launch, from shared memory.
//
// Weights are 64 bits wide: with 128256 tokens borders lie 2^-17 of the whole apart, and a uniform number falls within fp32's error of one in
// every hundredth row.  exp(scale (x - m)) = 2^(n / 64) 2^(r / 64) with n a whole number and |r| <= 1/2: the 64 roots of 2 and a polynomial.
#include <float.h>
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "device_utils.h"
#include "elements.h"
#include "internal.h"
#include "mi355sm.h"
#include "rows.h"
#include "wave_ops.h"

struct sm_desc {
  sm_params_t p;
  int32_t held;      // a row is held by a team: one launch
  int32_t segments;  // of a row
  int32_t chunks;    // of a segment
  int32_t shift;     // weights as whole numbers: 2^shift, so that a row's sum stays below 2^62
  size_t ws_bytes;
  char names[64];
};

namespace mi355conv {

namespace {

// What the first launch leaves of a segment: its largest logit (infinity if there is a NaN or an infinity), and the sum of weights relative to it.
struct Part {
  float most, unused;
  double sum;
};

struct SmArgs {
  const void* logits;
  int64_t stride;
  const float *u, *scale, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logp;
  Part* parts;  // [rows][segments]
  float* tops;  // [rows][segments][kTops]: maxima of a segment's groups of threads
  int32_t rows, vocab, segments, chunks, shift;
};

constexpr int kBins = 1024;     // of a histogram
constexpr int kSorted = 1024;   // logits that are put in order
constexpr int kList = 12288;    // logits near the maximum that a long row's list holds
constexpr int kGroups = 16;     // of vectors, whose sums stand side by side
constexpr int kTops = 4;        // groups of lanes of a segment
constexpr int kChunkVecs = 4;   // vectors of a lane of the first launch, and of a thread that holds a row's share
constexpr int kMostSegments = 256;
constexpr int kUnits = 256;     // compute units
constexpr int kAhead = 8;        // vectors that a thread asks for at a time
constexpr float kFew = 256.f;    // logits that are ranked for little; where a few weigh most, a share of the row does not show them
constexpr float kNear = 8.f;    // nats below the maximum that the list holds: weights from 3e-4 on

// 2^(i / 64), computed to 60 digits and rounded.
constexpr int kRootCount = 64, kRootBits = 6;
__device__ const double kRoots[kRootCount] = {
    1.0, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284,
    1.0442737824274138, 1.0556451783605572, 1.0671404006768237, 1.0787607977571199,
    1.0905077326652577, 1.102382583307841, 1.1143867425958924, 1.1265216186082418,
    1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812,
    1.189207115002721, 1.202156731452703, 1.215247359980469, 1.22848053610687,
    1.241857812073484, 1.255380757024691, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.339667524053303,
    1.3542555469368927, 1.3690024229745905, 1.383909881963832, 1.3989796725383112,
    1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647,
    1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384,
    1.5422108254079407, 1.559004400237837, 1.5759808451078865, 1.593142151342267,
    1.6104903319492543, 1.6280274218573478, 1.645755478153965, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.718619298122478, 1.7373338352737062,
    1.7562521603732995, 1.7753764925265212, 1.7947090750031072, 1.8142521755003989,
    1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656,
    1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.978456026387951,
};

// In shared memory with i 2^14 taken out of the upper word: adding (64 n + i) 2^14 to it gives 2^(n + i / 64).  (512 of them, and a term less: the lanes'
// reads meet in the banks, 110 us for 1024 x 128256; 32, and a term more: 106.)
__device__ __forceinline__ void fill_roots(double* root, int tid) {
  if (tid < kRootCount) root[tid] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, kRoots[tid]) - ((uint64_t)tid << (20 - kRootBits + 32)));
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int wave_scan(int v) {  // the sum of the lanes up to this one
  v += dpp_move<0x111, 0xF>(0, v);
  v += dpp_move<0x112, 0xF>(0, v);
  v += dpp_move<0x114, 0xF>(0, v);
  v += dpp_move<0x118, 0xF>(0, v);
  v += dpp_move<0x142, 0xA>(0, v);
  return v + dpp_move<0x143, 0xC>(0, v);
}

__device__ __forceinline__ double wave_scan(double v) {
  v += dpp_move<0x111, 0xF>(0., v);
  v += dpp_move<0x112, 0xF>(0., v);
  v += dpp_move<0x114, 0xF>(0., v);
  v += dpp_move<0x118, 0xF>(0., v);
  v += dpp_move<0x142, 0xA>(0., v);
  return v + dpp_move<0x143, 0xC>(0., v);
}

__device__ __forceinline__ uint64_t move_words(uint64_t v, int which) {
  const double d = __builtin_bit_cast(double, v);
  const double r = which == 0   ? dpp_move<0x111, 0xF>(0., d)
                   : which == 1 ? dpp_move<0x112, 0xF>(0., d)
                   : which == 2 ? dpp_move<0x114, 0xF>(0., d)
                   : which == 3 ? dpp_move<0x118, 0xF>(0., d)
                   : which == 4 ? dpp_move<0x142, 0xA>(0., d)
                                : dpp_move<0x143, 0xC>(0., d);
  return __builtin_bit_cast(uint64_t, r);
}

__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  v += move_words(v, 0);
  v += move_words(v, 1);
  v += move_words(v, 2);
  v += move_words(v, 3);
  v += move_words(v, 4);
  return v + move_words(v, 5);
}

// exp of the difference to the row's or segment's largest logit: 2^((64 n + i + r) / 64), |r| <= 1/2.  The number 1.5 2^52 brings 64 n + i
// into the lower word; the polynomial's next term is below 2^-44.5.  What is below 2^-995 counts as 0: from 2^-1022 on the power would run out of its
// exponent.
struct Exponential {
  const double* root;  // in shared memory
  double top, c;
  float low;    // the smallest number that is at most 690 nats below the largest logit; rounded up where a step of that one may be many nats
  bool steep;   // `low` itself weighs something beside 1, so that it cannot stand for what is below it

  __device__ __forceinline__ void set(float largest, float scale) {
    top = largest;
    c = (double)scale * (kRootCount * 1.44269504088896340736);
    const float span = 690.f * __builtin_amdgcn_rcpf(scale);
    low = largest - span;  // within a sixteenth of a nat, where neither number has more than 2^20 of them
    steep = fabsf(largest) * scale >= 0x1p20f;
    if (steep) {
      const double border = (double)largest - (double)span;
      const float near = (float)border;
      const int bits = __builtin_bit_cast(int, near);
      low = fmaxf((double)near < border ? __builtin_bit_cast(float, bits < 0 ? bits - 1 : bits + 1) : near, -FLT_MAX);
      steep = !((largest - low) * scale >= 600.f);
    }
  }

  static constexpr double kWhole = 0x1.8p52;

  // The weights of N logits, none of which is below `low`, as a power of 2 and a factor, and added to a sum one after the other.  Their steps go side by side, so that a wave waits
  // once for N entries.  Ten operations in 64 bits a logit take most of the time.  (One of them is the difference, which makes the largest one's weight
  // 1 exactly, and so sums of equal ones exact.)
  template <int N, class F>
  __device__ __forceinline__ void terms(const float (&x)[N], F&& f) const {
    constexpr double L = 0.69314718055994530942 / kRootCount;
    double r[N], entry[N];
    uint32_t at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double d = (double)x[i] - top, placed = fma(d, c, kWhole);
      r[i] = fma(d, c, kWhole - placed);
      at[i] = (uint32_t)__builtin_bit_cast(uint64_t, placed);
      entry[i] = root[at[i] & (kRootCount - 1)];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u32x2 words = __builtin_bit_cast(u32x2, entry[i]);
      words[1] += at[i] << (20 - kRootBits);
      double p = fma(L * L * L * L / 24, r[i], L * L * L / 6);
      p = fma(fma(fma(p, r[i], L * L / 2), r[i], L), r[i], 1.);
      f(i, __builtin_bit_cast(double, words), p);
    }
  }

  template <int N>
  __device__ __forceinline__ double add(double sum, const float (&x)[N]) const {
    terms(x, [&](int, double power, double rest) { sum = fma(power, rest, sum); });
    return sum;
  }

  // Those of any logits.
  template <int N>
  __device__ __forceinline__ void of(const float (&x)[N], double (&w)[N]) const {
    float held[N];
#pragma unroll
    for (int i = 0; i < N; ++i) held[i] = __builtin_amdgcn_fmed3f(x[i], low, FLT_MAX);
    terms(held, [&](int i, double power, double rest) { w[i] = x[i] >= low ? power * rest : 0.; });
  }

  __device__ __forceinline__ double near(float x) const { return add<1>(0., {x}); }

  __device__ __forceinline__ double operator()(float x) const { return x >= low ? near(x) : 0.; }
};

template <int THREADS>
struct Shared {
  static constexpr int WAVES = THREADS / 64;
  double root[kRootCount];
  double sum[WAVES];
  float most[WAVES];
};

// Over the team, in the same order every time.
template <int THREADS>
__device__ __forceinline__ double team_sum(Shared<THREADS>& lds, double v) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_sum(v);
  __syncthreads();
  if (lane == 0) lds.sum[wave] = v;
  __syncthreads();
  double all = lds.sum[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) all += lds.sum[w];
  return all;
}

template <int THREADS>
__device__ __forceinline__ float team_most(Shared<THREADS>& lds, float most) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  most = wave_most(most);
  __syncthreads();
  if (lane == 0) lds.most[wave] = most;
  __syncthreads();
  most = lds.most[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) most = fmaxf(most, lds.most[w]);
  return most;
}

__device__ __forceinline__ bool scale_is_good(float scale) { return scale >= 0x1p-60f && scale <= 0x1p60f; }

// Vectors of a row [from, from + THREADS kChunkVecs), thread by thread.
template <class E, int THREADS>
__device__ __forceinline__ void load_chunk(const typename E::T* row, int from, int nv, int n, int tid, u32x4 (&x)[kChunkVecs]) {
#pragma unroll
  for (int j = 0; j < kChunkVecs; ++j) {
    const int v = from + j * THREADS + tid;
    x[j] = v < nv ? row_vec<E>(row, v, n) : lowest_vec<E>();
  }
}

// The largest one; infinity if there is one or a NaN.
template <class E>
__device__ __forceinline__ float chunk_most(const u32x4 (&x)[kChunkVecs]) {
  float most = -INFINITY;
#pragma unroll
  for (int j = 0; j < kChunkVecs; ++j)
#pragma unroll
    for (int i = 0; i < E::VEC; ++i) most = __builtin_elementwise_maximum(most, E::get(x[j], i));  // NaN if there is one
  return most < INFINITY ? most : INFINITY;
}

template <class E>
__device__ __forceinline__ double chunk_sum(const u32x4 (&x)[kChunkVecs], const Exponential& weight) {
  double s = 0.;
  if (weight.steep) {  // (hardly ever: by a loop, so that the usual way keeps its registers)
    u32x4 left[kChunkVecs];
#pragma unroll
    for (int j = 0; j < kChunkVecs; ++j) left[j] = x[j];
#pragma unroll 1
    for (int i = 0; i < kChunkVecs * E::VEC / 4; ++i) {
      const float logit[4] = {E::get(left[0], 0), E::get(left[0], 1), E::get(left[0], 2), E::get(left[0], 3)};
      double w[4];
      weight.of(logit, w);
      s += (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
      for (int j = 0; j < kChunkVecs; ++j) {
        const u32x4 next = left[min(j + 1, kChunkVecs - 1)];
        left[j] = E::VEC == 4 ? next : u32x4{left[j][2], left[j][3], next[0], next[1]};
      }
    }
    return s;
  }
#pragma unroll
  for (int j = 0; j < kChunkVecs; ++j) {
#pragma unroll
    for (int h = 0; h < E::VEC; h += 4) {
      float logit[4];  // (`low`, e^-600 or less, in the place of less: nothing beside 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) logit[i] = __builtin_amdgcn_fmed3f(E::get(x[j], h + i), weight.low, FLT_MAX);
      s = weight.add(s, logit);
      __builtin_amdgcn_sched_barrier(0);  // (vectors side by side would take more registers than there are)
    }
  }
  return s;
}

// The first launch: a wave for each segment, which knows no other and waits for none; the next one's vectors are on their way while it works.
// Bound by the weights' arithmetic, ten operations of 64 bits a logit: 1024 x 128256 bf16 91 us (vector units 91 % busy), 2.9 TB/s of the 5.1 that
// a copy reaches; 64 rows 7.5 us.  (Five workgroups a compute unit by fewer registers: 100 against 94 us.)
template <int DTYPE>
__global__ __launch_bounds__(256) void sm_sums_kernel(SmArgs a) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  __shared__ double root[kRootCount];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  fill_roots(root, threadIdx.x);
  __syncthreads();
  const int n = a.vocab, nv = (n + E::VEC - 1) / E::VEC, total = gridDim.x * 4, per = a.chunks * 64 * kChunkVecs;
  const int step_r = total / a.segments, step_s = total % a.segments;
  const int first = blockIdx.x * 4 + wave;
  int r = first / a.segments, segment = first % a.segments;
  u32x4 x[kChunkVecs];
  float scale = 1.f;
  auto load = [&](int row, int from) {
#pragma unroll
    for (int j = 0; j < kChunkVecs; ++j) x[j] = begin_row_vec<E>(static_cast<const T*>(a.logits) + (int64_t)row * a.stride, from + j * 64 + lane, nv, n);
  };
  auto load_first = [&]() {
    if (r >= a.rows) return;
    load(r, segment * per);
    if (a.scale) scale = a.scale[r];
  };
  load_first();
  while (r < a.rows) {
    const int64_t it = (int64_t)r * a.segments + segment;
    const float used = scale_is_good(scale) ? scale : 1.f;  // (of a bad one the next launch makes what it is)
    Exponential weight = {root};
    float most = -INFINITY, mine = -INFINITY;
    double sum = 0.;
    for (int c = 0; c < a.chunks; ++c) {
      const int from = segment * per + c * 64 * kChunkVecs;
      if (c > 0) load(r, from);
      u32x4 now[kChunkVecs];
#pragma unroll
      for (int j = 0; j < kChunkVecs; ++j) now[j] = x[j];
      if ((from + 64 * kChunkVecs) * E::VEC > n) {
#pragma unroll
        for (int j = 0; j < kChunkVecs; ++j) now[j] = end_row_vec<E>(now[j], from + j * 64 + lane, nv, n);
      }
      const float here = chunk_most<E>(now), all = wave_most(here);
      mine = fmaxf(mine, here);
      if (all > most) {
        weight.set(all, used);
        if (most > -INFINITY && all < INFINITY) sum *= weight(most);
        most = all;
      }
      if (c + 1 == a.chunks) {
        r += step_r;
        segment += step_s;
        if (segment >= a.segments) {
          segment -= a.segments;
          ++r;
        }
        load_first();
      }
      if (fabsf(most) < INFINITY) sum += chunk_sum<E>(now, weight);
    }
    const float top = group_most<16>(mine);
    if ((lane & 15) == 0) a.tops[it * kTops + lane / 16] = top;
    sum = wave_sum(sum);
    if (lane == 0) a.parts[it] = Part{most, 0.f, sum};
  }
}

struct Cut {
  float value;
  int last;  // an index of the row, or a place in the list
};

template <bool HELD>
constexpr int kListed = HELD ? 2048 : kList;  // (rows that a team holds are few passes away)

template <int THREADS, bool LIMITED, bool HELD>
struct RowLds : Shared<THREADS> {
  static constexpr int WAVES = THREADS / 64;
  u32x4 held[HELD ? 256 * kChunkVecs : 1];  // rows of one segment
  double part[kGroups][WAVES];
  double segment[HELD ? 1 : kMostSegments];
  uint64_t sorted[LIMITED ? kSorted : 1];
  uint64_t weights[LIMITED ? kBins : 1];
  int count[LIMITED ? kBins : 1];
  float value[LIMITED ? kListed<HELD> : 1];  // the list: logits near the maximum and their indices, in the order of these, in a part for each wave
  int index[LIMITED ? kListed<HELD> : 1];
  uint64_t whole[WAVES];
  int number[WAVES];
  uint32_t places;
  int found, before, inside;
};

template <int DTYPE, int THREADS, bool LIMITED, bool HELD>
struct Team {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  typedef RowLds<THREADS, LIMITED, HELD> Lds;
  static constexpr int VEC = E::VEC, WAVES = THREADS / 64, SHARE = kListed<HELD> / WAVES;  // of the list, for each wave

  // (a function's own shared memory: a reference kept in the team would make every access a generic one)
  static __device__ __forceinline__ Lds& memory() {
    __shared__ Lds lds;
    return lds;
  }

  const T* row;
  int n, nv, tid, lane, wave, shift;
  float m, scale;  // the maximum
  Exponential weight;
  Cut cut;
  bool parts_ready;
  int part_end[WAVES];  // of the list's parts, one after the other
  int listed;           // in this wave's part

  __device__ __forceinline__ u32x4 vec(int v) const {
    if constexpr (HELD) return v < nv ? memory().held[v] : lowest_vec<E>();
    return long_row_vec<E>(row, v, nv, n);
  }

  __device__ __forceinline__ bool keeps(float x, int at) const { return (x > cut.value) | ((x == cut.value) & (at <= cut.last)); }

  __device__ __forceinline__ float distance(float x) const { return fminf((m - x) * scale, FLT_MAX); }

  // Where the i-th of the list stands.
  __device__ __forceinline__ int place_of(int i) const {
    int place = i;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w) place += i >= part_end[w] ? SHARE - (part_end[w] - (w ? part_end[w - 1] : 0)) : 0;
    return place;
  }

  // f(logit, index, weight) for the elements of a vector, in order, four at a time; without weights (0 in their place) where they are not asked for.
  template <bool WEIGHT, class F>
  __device__ __forceinline__ void elements(u32x4 x, int v, F&& f) const {
    const Slot<E> at = slot_of<E>(v, n);
    constexpr int WORDS = 16 / VEC;  // of four elements
#pragma unroll 1
    for (int h = 0; h < VEC; h += 4) {
      float logit[4];
      double w[4] = {0., 0., 0., 0.};
#pragma unroll
      for (int i = 0; i < 4; ++i) logit[i] = E::get(x, i);
      if constexpr (WEIGHT) weight.of(logit, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) f(logit[i], at.base + h + i, w[i]);
      if constexpr (WORDS == 2) x = u32x4{x[2], x[3], x[0], x[1]};
    }
  }

  // The same for turns [j0, j1) of the team over the vectors [from, to), -inf beyond, with after(turn) behind each.
  template <bool WEIGHT, class F, class After>
  __device__ __forceinline__ void turns(int from, int to, int j0, int j1, F&& f, After&& after) const {
    constexpr int AHEAD = !LIMITED ? 1 : HELD ? 4 : kAhead;
    for (int j = j0; j < j1; j += AHEAD) {
      u32x4 x[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int v = from + (j + i) * THREADS + tid;
        x[i] = vec(v < to ? v : nv);
      }
#pragma unroll 1
      for (int i = 0; i < min(AHEAD, j1 - j); ++i) {
        elements<WEIGHT>(x[0], from + (j + i) * THREADS + tid, f);
        after(j + i);
#pragma unroll
        for (int o = 0; o + 1 < AHEAD; ++o) x[o] = x[o + 1];
      }
    }
  }

  // For the whole row (LIST: what the list holds, with places for indices, whose order is the same; each wave its part), by all threads; -inf in the place of
  // what is not there.
  template <bool LIST, bool WEIGHT, class F, class After>
  __device__ __forceinline__ void each(F&& f, After&& after) const {
    if constexpr (LIST) {
      const int first = wave * SHARE, end = first + listed;
#pragma unroll 1
      for (int i0 = first + lane; i0 - lane < end; i0 += 256) {
        float logit[4];
        double w[4] = {0., 0., 0., 0.};
#pragma unroll
        for (int i = 0; i < 4; ++i) logit[i] = i0 + i * 64 < end ? memory().value[i0 + i * 64] : -INFINITY;
        if constexpr (WEIGHT) weight.of(logit, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) f(logit[i], i0 + i * 64, w[i]);
      }
    } else {
      turns<WEIGHT>(0, nv, 0, (nv + THREADS - 1) / THREADS, f, after);
    }
  }
  template <bool LIST, bool WEIGHT, class F>
  __device__ __forceinline__ void each(F&& f) const {
    each<LIST, WEIGHT>(f, [](int) {});
  }

  // Turns that are added up together, so that a sum over `length` of them is known in at most kGroups parts.
  static __device__ __forceinline__ int group_of(int length) { return length <= 4 ? 1 : max(4, (length + kGroups - 1) / kGroups); }

  // Sums of(...) over the turns of a group, each wave's into memory().part.
  struct GroupSum {
    double s = 0.;
    int g = 0, in = 0;
  };
  __device__ __forceinline__ void group_after(GroupSum& sums, int per, bool last) const {
    if (++sums.in < per && !last) return;
    const double s = wave_sum(sums.s);
    if (lane == 0) memory().part[sums.g][wave] = s;
    sums.s = 0.;
    sums.in = 0;
    ++sums.g;
  }

  // The groups' sums stand in the lanes: the first group with which they pass `target`, or the last one of any weight; target becomes what is left of
  // it before that group.
  static __device__ __forceinline__ int pick(double s, int groups, double& target) {
    double sum = 0., before = 0.;
    int chosen = 0;
    for (int g = 0; g < groups; ++g) {
      const double part = read_lane(s, g);
      if (part > 0.) {
        chosen = g;
        before = sum;
        sum += part;
        if (sum > target) break;
      }
    }
    target -= before;
    return chosen;
  }

  // The same by a scan over 64 lanes.
  static __device__ __forceinline__ int pick_lane(double mine, double& target) {
    const double up_to = wave_scan(mine);
    const uint64_t some = __ballot(mine > 0.), passed = __ballot(mine > 0. && up_to > target);
    const int chosen = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some | 1);
    target -= read_lane(up_to - mine, chosen);
    return chosen;
  }

  // The index of the first logit of the vectors [from, to) with which the sum of of(logit, index, weight) passes the target: u times the whole
  // (FRACTION), or as given.  ready: the first round's parts stand in memory().part.
  template <bool FRACTION, bool WEIGHT, class W>
  __device__ __forceinline__ int locate(int from, int to, double target, W&& of, double& whole, bool ready = false) {
    int j0 = 0, j1 = (to - from + THREADS - 1) / THREADS, place = 0;
    bool first = FRACTION;
    for (;;) {
      const int length = j1 - j0, per = group_of(length), groups = (length + per - 1) / per;
      __syncthreads();
      if (!ready) {
        GroupSum sums;
        turns<WEIGHT>(from, to, j0, j1, [&](float x, int at, double w) { sums.s += of(x, at, w); }, [&](int j) { group_after(sums, per, j + 1 == j1); });
        __syncthreads();
      }
      ready = false;
      double s = 0.;
      if (lane < groups)
        for (int w = 0; w < WAVES; ++w) s += memory().part[lane][w];
      if (first) {
        whole = wave_sum(s);
        target *= whole;
        first = false;
      }
      const int g = pick(s, groups, target);
      j0 += g * per;
      j1 = min(j0 + per, j1);
      if (per == 1) {
        place = pick(lane < WAVES ? memory().part[g][lane] : 0., WAVES, target);
        break;
      }
    }
    if (wave == place) {
      const int v = from + j0 * THREADS + tid;
      const u32x4 mine = vec(v < to ? v : nv);
      double here = 0.;
      elements<WEIGHT>(mine, v, [&](float x, int at, double w) { here += of(x, at, w); });
      const int at_lane = pick_lane(here, target);
      if (lane == at_lane) {
        double sum = 0.;
        int index = 0;
        bool done = false;
        elements<WEIGHT>(mine, v, [&](float x, int at, double weight_of) {
          const double w = of(x, at, weight_of);
          sum += w;
          if (w > 0. && !done) {
            index = at;
            done = sum > target;
          }
        });
        memory().found = index;
      }
    }
    __syncthreads();
    return memory().found;
  }

  // memory().sorted in descending order: by a wave where they are few, which counts those above each.
  __device__ __forceinline__ void sort(int entries) {
    __syncthreads();
    if (entries <= 64) {
      if (wave == 0) {
        const uint64_t mine = lane < entries ? memory().sorted[lane] : 0;
        int rank = 0;
        for (int o = 0; o < entries; ++o) rank += read_lane(mine, o) > mine ? 1 : 0;
        wave_sync();
        if (lane < entries) memory().sorted[rank] = mine;
      }
      __syncthreads();
      return;
    }
    int size = 128;
    while (size < entries) size *= 2;
    for (int i = entries + tid; i < size; i += THREADS) memory().sorted[i] = 0;
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        __syncthreads();
        for (int i = tid; i < size / 2; i += THREADS) {
          const int a = 2 * i - (i & (j - 1)), b = a + j;
          const uint64_t x = memory().sorted[a], y = memory().sorted[b];
          if ((x < y) == ((a & k) == 0)) {
            memory().sorted[a] = y;
            memory().sorted[b] = x;
          }
        }
      }
    __syncthreads();
  }

  // The first bin with which the counts (WEIGHT: the weights) reach the target, counted from `carry` on: its number, or -1 (`surely`: the last bin that
  // holds any); memory().before and memory().inside are the count before it and its own.  The carries go on to the end of the bins.
  template <bool WEIGHT>
  __device__ __forceinline__ int find_bin(uint64_t target, uint64_t& carry, int& count_carry, bool surely) {
    constexpr int PER = kBins / THREADS;
    __syncthreads();
    int counts[PER], count = 0;
    uint64_t values[PER], value = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      counts[i] = memory().count[tid * PER + i];
      values[i] = WEIGHT ? memory().weights[tid * PER + i] : (uint64_t)counts[i];
      count += counts[i];
      value += values[i];
    }
    const int count_to = wave_scan(count);
    const uint64_t value_to = wave_scan(value);
    if (lane == 63) {
      memory().number[wave] = count_to;
      memory().whole[wave] = value_to;
    }
    if (tid == 0) {
      memory().found = INT_MAX;
      memory().places = 0;
    }
    __syncthreads();
    int count_before = count_carry, count_all = count_carry;
    uint64_t before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) {
        count_before += memory().number[w];
        before += memory().whole[w];
      }
      count_all += memory().number[w];
      all += memory().whole[w];
    }
    if (surely && all < target) target = all;  // (a rounding)
    count_before += count_to - count;
    before += value_to - value;
    int mine = INT_MAX, mine_before = 0, mine_count = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      before += values[i];
      if (mine == INT_MAX && counts[i] > 0 && before >= target) {
        mine = tid * PER + i;
        mine_before = count_before;
        mine_count = counts[i];
      }
      count_before += counts[i];
    }
    if (mine != INT_MAX) atomicMin(&memory().found, mine);
    __syncthreads();
    const int found = memory().found;
    if (mine == found && mine != INT_MAX) {
      memory().before = mine_before;
      memory().inside = mine_count;
    }
    __syncthreads();
    carry = all;
    count_carry = count_all;
    return found == INT_MAX ? -1 : found;
  }

  __device__ __forceinline__ void clear_bins() {
    __syncthreads();
    for (int i = tid; i < kBins; i += THREADS) {
      memory().count[i] = 0;
      memory().weights[i] = 0;
    }
    __syncthreads();
  }

  __device__ __forceinline__ uint64_t fixed(double w) const { return (uint64_t)rint(ldexp(w, shift)); }

  // The same of a weight, up to 1: 2^shift of it are at most 2^50, which 2^52 rounds and shows as a whole number.
  template <bool WEIGHT>
  __device__ __forceinline__ void count_in(int b, double w) {
    atomicAdd(&memory().count[b], 1);
    if (WEIGHT) {
      const double placed = fma(w, __builtin_bit_cast(double, (uint64_t)(1023 + shift) << 52), 0x1p52);
      atomicAdd((unsigned long long*)&memory().weights[b], (unsigned long long)(__builtin_bit_cast(uint64_t, placed) & 0xFFFFFFFFFFFFFull));
    }
  }

  // Moves the cut to where the counts (WEIGHT: the weights) of what it keeps reach the target, in descending order.  LIST: none is below `least`.
  // [bracket.x, bracket.y]: distances between which it is likely to be (bracket.y = 0: not known).  False where the counts do not reach it, or whole numbers
  // of weights pick a bin that the weights' own sums do not end in: then the cut is as it was, and halve() finds it.
  // PARTS: the sums of the weights from q on of what it then keeps are left for locate(), if parts_ready says so.
  template <bool WEIGHT, bool LIST, bool PARTS = false>
  __device__ __forceinline__ bool find_cut(double target, float least, float2 bracket, double q = 0.) {
    // histograms by distance: of the bracket, then near the maximum, then beyond; d of (from, to]
    float end = LIST ? distance(least) : FLT_MAX;
    parts_ready = false;
    float from = -1.f, to = -1.f, start = 0.f, per = 0.f;
    double above_sum = 0.;
    int bin = -1, count_carry = 0;
    uint64_t carry = 0;
    for (int phase = bracket.y > 0.f ? 0 : 1; phase < 3 && bin < 0; ++phase) {
      from = phase == 0 ? bracket.x : phase == 1 ? -1.f : kNear;
      to = phase == 0 ? bracket.y : phase == 1 ? fminf(kNear, end) : end;
      if (phase == 2) {
        if (!LIST) to = end = distance(least_finite());
        if (end <= kNear) break;
      }
      start = fmaxf(from, 0.f);
      per = to > start ? fminf(kBins / (to - start), FLT_MAX) : 0.f;
      clear_bins();
      double sum = 0.;
      int count = 0;
      each<LIST, WEIGHT>([&](float logit, int at, double w) {
        // (one branch: conditions side by side cost less)
        const float d = distance(logit);
        const bool in = (d <= to) & (logit > -INFINITY) & keeps(logit, at), above = in & !(d > from);
        count += above ? 1 : 0;
        sum += above ? w : 0.;
        if (in & (d > from)) count_in<WEIGHT>(min((int)((d - start) * per), kBins - 1), w);
      });
      above_sum = 0.;
      count_carry = 0;
      carry = 0;
      if (from >= 0.f) {
        count_carry = (int)team_sum<THREADS>(memory(), (double)count);
        if (WEIGHT) above_sum = team_sum<THREADS>(memory(), sum);
        carry = WEIGHT ? fixed(above_sum) : (uint64_t)count_carry;
      }
      if (carry < (WEIGHT ? fixed(target) : (uint64_t)target) || from < 0.f)
        bin = find_bin<WEIGHT>(WEIGHT ? fixed(target) : (uint64_t)target, carry, count_carry, false);
    }
    if (bin < 0) return false;
    bool by_key = false;
    uint32_t high = 0, low = 0;  // by key: bins of (high - key) >> bits
    int bits = 0, above = memory().before, inside = memory().inside;
    for (;;) {
      // what the bin holds: to be sorted if it is few; their range; the weight above them
      float most = -INFINITY, least_in = INFINITY;
      double sum = 0.;
      GroupSum sums;
      const int length = (nv + THREADS - 1) / THREADS, per_group = group_of(length);
      each<LIST, WEIGHT || PARTS>([&](float logit, int at, double w) {
        const bool in = (logit > -INFINITY) & keeps(logit, at);
        int side;  // below 0: above the bin
        if (by_key) {
          const uint32_t key = order_key(logit);
          side = (int)((high - min(max(key, low), high)) >> bits) - bin;
          side = key > high ? -1 : key < low ? 1 : side;
        } else {
          const float d = distance(logit);
          side = min((int)((__builtin_amdgcn_fmed3f(d, start, to) - start) * per), kBins - 1) - bin;
          side = d <= from ? -1 : d > to ? 1 : side;
        }
        const bool above = in & (side < 0);
        if (WEIGHT) sum += above ? w : 0.;
        if (PARTS) sums.s += above & (w >= q) ? w : 0.;
        if (in & (side == 0)) {
          most = fmaxf(most, logit);
          least_in = fminf(least_in, logit);
          if (inside <= kSorted) {
            const uint32_t place = atomicAdd(&memory().places, 1u);
            if (place < (uint32_t)kSorted) memory().sorted[place] = entry_of(logit, at);
          }
        }
      }, [&](int j) {
        if (PARTS) group_after(sums, per_group, j + 1 == length);
      });
      if constexpr (WEIGHT) {
        sum = team_sum<THREADS>(memory(), sum);
        if (sum >= target && sum > 0.) return false;  // what is above the bin reaches it
      }
      if (inside <= kSorted) {
        sort(inside);
        int place = (int)target - above - 1;
        if constexpr (WEIGHT) {
          place = sorted_place(inside, sum, target);
          if (place < 0) return false;
        }
        place = max(0, min(place, inside - 1));
        const uint64_t entry = memory().sorted[place];
        cut.value = key_value((uint32_t)(entry >> 32));
        cut.last = (int)(0xFFFFFFFFu - (uint32_t)entry);
        if constexpr (PARTS) {
          add_sorted(place + 1, per_group, q);
          parts_ready = true;
        }
        return true;
      }
      most = team_most<THREADS>(memory(), most);
      least_in = -team_most<THREADS>(memory(), -least_in);
      if (most == least_in) {  // equal ones: by their indices
        double order = target - above;
        if constexpr (WEIGHT) {
          order = fmax(ceil((target - sum) / weight(most)), 1.);
          if (order > (double)inside) return false;
        }
        const Cut kept = cut;
        cut.last = nth_equal<LIST>(most, (int)order);
        cut.value = most;
        if (most == kept.value) cut.last = min(cut.last, kept.last);
        return true;
      }
      by_key = true;
      high = order_key(most);
      low = order_key(least_in);
      bits = max(0, 32 - __builtin_clz(high - low) - 10);
      clear_bins();
      each<LIST, WEIGHT>([&](float logit, int at, double w) {
        const uint32_t key = order_key(logit);
        if ((key <= high) & (key >= low) & keeps(logit, at)) count_in<WEIGHT>((int)((high - key) >> bits), w);
      });
      uint64_t before = WEIGHT ? 0 : (uint64_t)above;
      int count_before = above;
      bin = find_bin<WEIGHT>(WEIGHT ? fixed(fmax(target - sum, 0.)) : (uint64_t)target, before, count_before, true);
      if (bin < 0) return false;
      above = memory().before;
      inside = memory().inside;
    }
  }

  // Moves the cut to where the weights of what it keeps reach the target, in descending order, by the sums of the weights alone: a pass for each bit of
  // the logits' order.  For the rows where find_cut's whole numbers are not enough: equal logits are rounded alike, and those of a row of millions that
  // weigh little each may all be rounded to nothing.  (Hardly ever: 1.2 ms for a row of 128256, 13 for a million.)
  template <bool LIST>
  __device__ __forceinline__ void halve(double target) {
    uint32_t high = order_key(m), low = order_key(-FLT_MAX);  // the sum from `low` on reaches the target, the one above `high` does not
    double above = 0.;                                        // the latter
    while (low < high) {
      const uint32_t middle = high - (high - low) / 2;
      double sum = 0.;
      each<LIST, false>([&](float logit, int at, double) {
        const uint32_t key = order_key(logit);
        if ((key >= middle) & (key <= high) & keeps(logit, at)) sum += weight(logit);
      });
      sum = above + team_sum<THREADS>(memory(), sum);
      if (sum >= target) {
        low = middle;
      } else {
        above = sum;
        high = middle - 1;
      }
    }
    const float value = key_value(high);
    int count = 0;
    each<LIST, false>([&](float logit, int at, double) { count += (logit == value) & keeps(logit, at) ? 1 : 0; });
    const double equal = team_sum<THREADS>(memory(), (double)count);
    const Cut kept = cut;
    int last = INT_MAX;
    if (equal > 0.) last = nth_equal<LIST>(value, (int)fmin(fmax(ceil((target - above) / weight(value)), 1.), equal));
    cut = Cut{value, value == kept.value ? min(last, kept.last) : last};
    parts_ready = false;
  }

  // The weights from q on of the first of memory().sorted to the parts of their groups and waves, in their order.
  __device__ __forceinline__ void add_sorted(int entries, int per, double q) {
    double* const weights = reinterpret_cast<double*>(memory().weights);
    for (int i = tid; i < entries; i += THREADS) {
      const uint64_t entry = memory().sorted[i];
      const double w = weight(key_value((uint32_t)(entry >> 32)));
      const int v = (int)(0xFFFFFFFFu - (uint32_t)entry) / VEC, turn = v / THREADS;
      weights[i] = w >= q ? w : 0.;
      memory().count[i] = turn / per * WAVES + (v - turn * THREADS) / 64;
    }
    __syncthreads();
    if (tid < kGroups * WAVES) {
      double s = 0.;
      for (int i = 0; i < entries; ++i) s += memory().count[i] == tid ? weights[i] : 0.;
      if (s > 0.) memory().part[tid / WAVES][tid % WAVES] += s;
    }
    __syncthreads();
  }

  // The index of the order-th (from 1) of the logits that equal x, all of which the cut keeps.
  template <bool LIST>
  __device__ __forceinline__ int nth_equal(float x, int order) {
    if constexpr (LIST) {  // places, part by part
      int mine = 0;
      for (int i = lane; i - lane < listed; i += 64) mine += (int)__builtin_popcountll(__ballot(i < listed && memory().value[wave * SHARE + i] == x));
      __syncthreads();
      if (lane == 0) memory().number[wave] = mine;
      __syncthreads();
      for (int w = 0; w < wave; ++w) order -= memory().number[w];
      if (order >= 1 && order <= mine) {
        for (int i = lane; i - lane < listed; i += 64) {
          const bool equal = i < listed && memory().value[wave * SHARE + i] == x;
          const uint64_t mask = __ballot(equal);
          if (equal && (int)__builtin_popcountll(mask & ((2ull << lane) - 1)) == order) memory().found = wave * SHARE + i;
          order -= (int)__builtin_popcountll(mask);
        }
      }
      __syncthreads();
      return memory().found;
    } else {
      double whole;
      return locate<false, false>(0, nv, order - 0.5, [&](float logit, int at, double) { return (logit == x) & keeps(logit, at) ? 1. : 0.; }, whole);
    }
  }

  // The first place of memory().sorted with which the weights reach the target, counted from `sum` on; -1 where there is none.
  __device__ __forceinline__ int sorted_place(int entries, double sum, double target) {
    if (entries <= 64) {
      const double w = lane < entries ? weight(key_value((uint32_t)(memory().sorted[lane] >> 32))) : 0.;
      const uint64_t reached = __ballot(lane < entries && sum + wave_scan(w) >= target);
      return reached ? __builtin_ctzll(reached) : -1;
    }
    constexpr int PER = kSorted / THREADS;
    double w[PER], mine = 0.;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      w[i] = at < entries ? weight(key_value((uint32_t)(memory().sorted[at] >> 32))) : 0.;
      mine += w[i];
    }
    const double to = wave_scan(mine);
    if (tid == 0) memory().found = INT_MAX;
    if (lane == 63) memory().sum[wave] = to;
    __syncthreads();
#pragma unroll
    for (int o = 0; o < WAVES; ++o)
      if (o < wave) sum += memory().sum[o];
    sum += to - mine;
    bool done = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      sum += w[i];
      if (!done && tid * PER + i < entries && sum >= target) {
        atomicMin(&memory().found, tid * PER + i);
        done = true;
      }
    }
    __syncthreads();
    return memory().found == INT_MAX ? -1 : memory().found;
  }

  // Those of a wave's vectors from v on into its part of the list, which holds `mine` already; how many it then holds, more than SHARE if that is too many.
  __device__ __forceinline__ int list_vec(u32x4 x, int v, float bound, int mine) const {
    if (v + 64 >= nv) {  // where the row ends
      if constexpr (HELD)
        x = v + lane < nv ? x : lowest_vec<E>();
      else
        x = end_row_vec<E>(x, v + lane, nv, n);
    }
    uint32_t own = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) own |= E::get(x, i) >= bound ? 1u << i : 0u;
    if (__ballot(own != 0) == 0) return mine;
    const int count = __builtin_popcount(own), up_to = wave_scan(count), all = read_lane(up_to, 63);
    if (mine + all > SHARE) return SHARE + 1;
    int place = wave * SHARE + mine + up_to - count;
    const int at = slot_of<E>(v + lane, n).base;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (own >> i & 1) {
        memory().value[place] = E::get(x, i);
        memory().index[place] = at + i;
        ++place;
      }
    return mine + all;
  }

  // Logits from `bound` on into the list, in the order of their indices: each wave takes a part of the row and fills a part of the list.  The number of them, or -1 where a wave found more than its part holds.
  __device__ __forceinline__ int fill_list(float bound) {
    const int per = ((nv + WAVES - 1) / WAVES + 63) / 64 * 64, to = min(nv, (wave + 1) * per);
    int mine = 0;
    __syncthreads();
    constexpr int AHEAD = HELD ? 4 : 8;
    for (int v0 = wave * per; v0 < to && mine <= SHARE; v0 += AHEAD * 64) {
      u32x4 x[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int v = v0 + j * 64 + lane;
        if constexpr (HELD)
          x[j] = memory().held[min(v, nv - 1)];
        else
          x[j] = begin_row_vec<E>(row, v, nv, n);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (v0 + j * 64 < to && mine <= SHARE) mine = list_vec(x[j], v0 + j * 64, bound, mine);
    }
    if (lane == 0) memory().number[wave] = mine;
    listed = min(mine, SHARE);
    __syncthreads();
    int all = 0;
    bool over = false;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int count = __builtin_amdgcn_readfirstlane(memory().number[w]);
      over |= count > SHARE;
      all += count;
      part_end[w] = all;
    }
    return over ? -1 : all;
  }

  // Where the k-th logit, or (k = 0) the place up to which the weights reach p of `all`, is likely to lie: distances that are likely before and
  // after it, from every so many-th vector, and in `likely` about how many logits lie up to the second.  Weights beyond a place are those of
  // many small ones, which a share of the row shows well.
  __device__ __forceinline__ float2 estimate(int k, double p, double all, int& likely) {
    constexpr float kPer = kBins / 32.f;  // 32 nats
    const int stride = max(1, nv / THREADS), v = tid * stride;
    const float share = (float)nv / (float)min(THREADS, (nv + stride - 1) / stride);
    clear_bins();
    if (v < nv)
      elements<false>(vec(v), v, [&](float logit, int, double) {
        if (logit > -INFINITY) atomicAdd(&memory().count[(int)fminf(distance(logit) * kPer, kBins - 1.f)], 1);
      });
    __syncthreads();
    // the last bin first: what lies beyond a bin
    constexpr int PER = kBins / THREADS;
    float value[PER], mine = 0.f;
    int counts[PER], count = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int bin = kBins - 1 - (tid * PER + i);
      counts[i] = memory().count[bin];
      value[i] = (float)counts[i] * __expf(-(float)bin / kPer);
      mine += value[i];
      count += counts[i];
    }
    const int count_to = wave_scan(count);
    const double value_to = wave_scan((double)mine);
    if (lane == 63) {
      memory().number[wave] = count_to;
      memory().sum[wave] = value_to;
    }
    if (tid == 0) {
      memory().before = kBins;
      memory().found = 0;
      memory().inside = 0;
    }
    __syncthreads();
    int beyond = count_to - count, total = 0;
    double weight_beyond = value_to - mine;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) {
        beyond += memory().number[w];
        weight_beyond += memory().sum[w];
      }
      total += memory().number[w];
    }
    // the first bin up to which there is surely not enough left out, the last one up to which there surely is
    const double left = all * (1. - p) / share;
    int low = kBins, high = 0, high_count = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int bin = kBins - 1 - (tid * PER + i), up_to = total - beyond;  // logits up to this bin's end
      const bool enough = (k > 0 ? up_to * share >= 1.4f * k + 8.f * share : weight_beyond <= 0.7 * left) && up_to * share >= kFew;
      const bool short_of = k > 0 ? up_to * share < 0.7f * k - 8.f * share : weight_beyond > 1.4 * left;
      if (!short_of) low = bin;
      if (!enough && high == 0) {
        high = bin + 1;
        high_count = up_to;
      }
      beyond += counts[i];
      weight_beyond += value[i];
    }
    if (low < kBins) atomicMin(&memory().before, low);
    if (high > 0) atomicMax(&memory().found, high);
    __syncthreads();
    if (high > 0 && high == memory().found) memory().inside = high_count;
    const int a = memory().before, b = memory().found + 1;
    __syncthreads();
    likely = (int)fminf(memory().inside * share, 1e9f);
    return make_float2(a / kPer, b / kPer);
  }

  __device__ __forceinline__ float least_finite() const {
    float least = INFINITY;
    each<false, false>([&](float logit, int, double) { least = logit > -INFINITY ? fminf(least, logit) : least; });
    return -team_most<THREADS>(memory(), -least);
  }

  // The sum of the weights that the cut keeps.
  template <bool LIST>
  __device__ __forceinline__ double kept_sum() {
    double sum = 0.;
    each<LIST, true>([&](float logit, int at, double w) {
      sum += keeps(logit, at) ? w : 0.;
    });
    return team_sum<THREADS>(memory(), sum);
  }

  // The place in the list of the token.
  __device__ __forceinline__ int locate_in_list(double u, double q, double& whole) {
    // each lane a run of its wave's part
    const int first = wave * SHARE, per = (listed + 63) / 64, from = first + min(lane * per, listed), to = first + min((lane + 1) * per, listed);
    auto of = [&](int i, double w) { return (w >= q) & keeps(memory().value[i], i) ? w : 0.; };
    double mine = 0.;
    for (int i = from; i < to; i += 4) {
      float x[4];
      double w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = memory().value[min(i + j, to - 1)];
      weight.of(x, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) mine += i + j < to ? of(i + j, w[j]) : 0.;
    }
    const double sum = wave_sum(mine);
    __syncthreads();
    if (lane == 0) memory().part[0][wave] = sum;
    __syncthreads();
    const double s = lane < WAVES ? memory().part[0][lane] : 0.;
    whole = wave_sum(s);
    double target = u * whole;
    const int place = pick(s, WAVES, target);
    if (wave == place) {
      const int at_lane = pick_lane(mine, target);
      if (lane == at_lane) {
        double reached = 0.;
        int chosen = from;
        for (int i = from; i < to; ++i) {
          const double w = of(i, weight(memory().value[i]));
          reached += w;
          if (w > 0.) {
            chosen = i;
            if (reached > target) break;
          }
        }
        memory().found = chosen;
      }
    }
    __syncthreads();
    return memory().found;
  }

  // The list's place of the token, where the list has at most one logit for each thread and k of them, or all that min-p keeps, or what top-p
  // needs: each thread ranks its own by counting those above it; weights in that order give the number of them that the limits keep.
  // all: the weight that top-p goes by, where top-k has no part in it.  -1 where the list does not hold what is kept.
  __device__ __forceinline__ int rank_and_locate(double u, int k, double p, double q, double all, bool complete, int entries, double& whole) {
    const bool mine = tid < entries;
    const float x = mine ? memory().value[place_of(tid)] : -INFINITY;
    const uint64_t key = mine ? entry_of(x, tid) : 0;
    const double w = mine ? weight(x) : 0.;
    uint64_t* const keys = memory().sorted;
    double* const ordered = reinterpret_cast<double*>(memory().weights);
    keys[tid] = key;
    __syncthreads();
    int rank = 0;
    if (wave * 64 < entries) {
#pragma unroll 4
      for (int o = 0; o < entries; ++o) rank += keys[o] > key ? 1 : 0;
    }
    if (mine)
      ordered[rank] = w;
    else
      ordered[tid] = 0.;
    __syncthreads();
    // every wave the same: a run of the order for each lane
    constexpr int PER = THREADS / 64;
    double run[PER], sum = 0.;
    int kept_q = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = lane * PER + i;
      run[i] = at < entries ? ordered[at] : 0.;
      if (k > 0 && at >= k) run[i] = 0.;
      sum += run[i];
      kept_q += (int)__builtin_popcountll(__ballot(at < entries && run[i] >= q));
    }
    const double up_to = wave_scan(sum), held = read_lane(up_to, 63);
    int kept = k > 0 ? min(k, entries) : entries;
    if (p < 1.) {
      const double target = fmax((k > 0 ? held : all) * p, 0.);
      if (target > held && !complete) return -1;
      double reached = up_to - sum;
      int before = 0;  // those before the one that reaches it
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        reached += run[i];
        before += (int)__builtin_popcountll(__ballot(lane * PER + i < entries && reached < target));
      }
      kept = min(kept, before + 1);
    }
    if (q > 0.) kept = min(kept, kept_q);
    const double part = mine && rank < kept ? w : 0., part_to = wave_scan(part);
    if (lane == 63) memory().part[0][wave] = part_to;
    __syncthreads();
    const double s = lane < WAVES ? memory().part[0][lane] : 0.;
    whole = wave_sum(s);
    double target = u * whole;
    const int place = pick(s, WAVES, target);
    if (wave == place) {
      const int at_lane = pick_lane(part, target);
      if (lane == at_lane) memory().found = tid;
    }
    __syncthreads();
    return memory().found;
  }

  // A bound that at least k logits reach, from the maxima of `groups` groups: the leading 16 bits of the k-th largest one, where every lane takes
  // the larger ones of four shares of them.
  __device__ __forceinline__ float bound_of(const float* tops, int groups, int k) {
    if (min(groups, 256) < k) return -INFINITY;
    uint32_t keys[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float most = -INFINITY;
      for (int g = i * 64 + lane; g < groups; g += 256) most = fmaxf(most, tops[g]);
      keys[i] = order_key(most);
    }
    uint32_t bound = 0;
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t with = bound | 1u << bit;
      int count = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) count += (int)__builtin_popcountll(__ballot(keys[i] >= with));
      if (count >= k) bound = with;
    }
    return bound <= 0x007FFFFFu ? -INFINITY : key_value(bound);  // (the key of -inf and the unused ones below it)
  }
};

// The second launch (HELD: the only one, of rows of one segment): a team for each row.  Without limits a segment's logits are all that it reads: 1024 x
// 128256 bf16 11 us.  With limits it is bound by the chain of passes over the row and the list that one compute unit makes, 1 x 32000 14 us, 64 x 128256
// 22 us of which the list takes 9 to 15; one row that keeps thousands of 50257 30 to 41 us, one whose list does not hold what is kept 73.  Held rows:
// 1 x 8192 8 us without limits, 22 with top-k 50 and top-p 0.9.
// (Teams of 1024 threads: registers spill, 20 against 13 us for 1 x 32000.)
template <int DTYPE, int THREADS, bool LIMITED, bool HELD>
__global__ __launch_bounds__(THREADS) void sm_row_kernel(SmArgs a) {
  typedef Elem<DTYPE> E;
  typedef Team<DTYPE, THREADS, LIMITED, HELD> Rows;
  typename Rows::Lds& lds = Rows::memory();
  const int tid = threadIdx.x;
  fill_roots(lds.root, tid);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int r = (int)row;
    Rows t;
    t.tid = tid;
    t.lane = tid & 63;
    t.wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    t.row = static_cast<const typename E::T*>(a.logits) + (int64_t)r * a.stride;
    t.n = a.vocab;
    t.nv = (a.vocab + E::VEC - 1) / E::VEC;
    t.shift = a.shift;
    const float scale = a.scale ? a.scale[r] : 1.f, u = a.u[r];
    const float p = LIMITED && a.top_p ? a.top_p[r] : 1.f, q = LIMITED && a.min_p ? a.min_p[r] : 0.f;
    const int k = LIMITED && a.top_k ? a.top_k[r] : 0;
    const bool bad = !scale_is_good(scale) || !(u >= 0.f && u <= 1.f) || p != p || q != q;
    const Part* const parts = a.parts + (int64_t)r * a.segments;

    __syncthreads();  // the row before this one
    float most = -INFINITY;
    u32x4 x[kChunkVecs];
    Part part = {-INFINITY, 0.f, 0.};
    if constexpr (HELD) {
      load_chunk<E, 256>(t.row, 0, t.nv, t.n, tid, x);
#pragma unroll
      for (int j = 0; j < kChunkVecs; ++j) lds.held[j * 256 + tid] = x[j];
      most = chunk_most<E>(x);
    } else if (tid < a.segments) {
      part = parts[tid];
      most = part.most;
    }
    if (bad) most = INFINITY;
    most = team_most<THREADS>(lds, most);
    if (!(fabsf(most) < INFINITY)) {
      if (tid == 0) {
        a.token[r] = -1;
        if (a.logp) a.logp[r] = most < 0.f ? -INFINITY : NAN;
      }
      continue;
    }
    t.m = most;
    t.scale = scale;
    t.weight.root = lds.root;
    t.weight.set(most, scale);
    t.cut = Cut{-INFINITY, INT_MAX};
    double whole = 0.;
    int token = -1;

    if constexpr (LIMITED) {
      const double least_weight = fmin((double)q, 1.);
      const bool by_count = k > 0 && k < t.n, by_weight = p < 1.f;
      double all = 0.;
      if (by_weight && !by_count) {
        if constexpr (HELD)
          all = team_sum<THREADS>(lds, chunk_sum<E>(x, t.weight));
        else
          all = team_sum<THREADS>(lds, tid < a.segments ? part.sum * t.weight(part.most) : 0.);
      }
      // what the list has to hold: k logits, or what makes up p of the weight, or all that min-p keeps
      float bound = -FLT_MAX;
      float2 bracket = {0.f, 0.f};
      int likely = 0;
      if (by_count || by_weight) {
        if (by_count && !HELD) bound = fmaxf(bound, t.bound_of(a.tops + (int64_t)r * a.segments * kTops, a.segments * kTops, k));
        if (!by_count && q > 0.f && all <= (double)q * kListed<HELD>) {
          // what min-p keeps is few: each of them has a share q of the weight or more
        } else if (bound == -FLT_MAX) {
          bracket = t.estimate(by_count ? k : 0, (double)p, all, likely);
          bound = most - bracket.y / scale;
        }
      }
      bool complete = !by_count && !by_weight;  // all that min-p keeps
      if (q > 0.f) {
        const float low = most + (logf(fminf(q, 1.f)) * 1.00001f - 1e-5f) / scale;  // (below the border, whatever the roundings)
        const float lower = low - fabsf(low) * 1e-6f;
        if (complete || (lower >= bound && !(by_count && by_weight))) {  // (the weight of k logits is that of all of them)
          complete = true;
          likely = 0;
          bound = lower;
        }
      }
      bound = fminf(fmaxf(bound, -FLT_MAX), most);
      int entries = -1;
      if ((by_count || by_weight || q > 0.f) && likely <= kListed<HELD>) entries = t.fill_list(bound);
      if (entries >= 0 && entries <= THREADS && (!by_count || k <= entries || (complete && !by_weight)) && (by_count || by_weight || complete)) {
        const int place = t.rank_and_locate((double)u, by_count ? k : 0, (double)p, least_weight, all, complete, entries, whole);
        if (place >= 0) token = lds.index[t.place_of(place)];
      } else if (entries >= 0) {
        bool enough = by_count || by_weight || complete;
        const float lowest = bound;
        if (by_count) {
          if (k < entries)
            enough = t.template find_cut<false, true>((double)k, lowest, make_float2(0.f, 0.f));
          else
            enough = k == entries || complete;
        }
        if (enough && by_weight) {
          const double kept = t.template kept_sum<true>(), target = fmax((by_count ? kept : all) * (double)p, 0.);
          if (by_count && k > entries)
            enough = false;  // (the weight of k logits is not known)
          else if (target > kept)
            enough = complete;
          else if (!t.template find_cut<true, true>(target, lowest, make_float2(0.f, 0.f)))
            t.template halve<true>(target);
        }
        if (enough)
          token = lds.index[t.locate_in_list((double)u, least_weight, whole)];
        else
          t.cut = Cut{-INFINITY, INT_MAX};
      }
      if (token < 0) {
        if (by_count) {
          if (by_weight)
            t.template find_cut<false, false>((double)k, 0.f, bracket);
          else
            t.template find_cut<false, false, true>((double)k, 0.f, bracket, least_weight);
        }
        if (by_weight) {
          const double target = fmax((by_count ? t.template kept_sum<false>() : all) * (double)p, 0.);
          if (!t.template find_cut<true, false, true>(target, 0.f, by_count ? make_float2(0.f, 0.f) : bracket, least_weight)) t.template halve<false>(target);
        }
        token = t.template locate<true, true>(
            0, t.nv, (double)u, [&](float logit, int at, double w) { return (w >= least_weight) & t.keeps(logit, at) ? w : 0.; }, whole,
            (by_count || by_weight) && t.parts_ready);
      }
    } else {
      auto plain = [](float, int, double w) { return w; };
      if constexpr (HELD) {
        token = t.template locate<true, true>(0, t.nv, (double)u, plain, whole);
      } else {
        if (tid < kMostSegments) lds.segment[tid] = tid < a.segments ? part.sum * t.weight(part.most) : 0.;
        __syncthreads();
        double four[4], mine = 0.;  // of four segments
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          four[i] = lds.segment[4 * t.lane + i];
          mine += four[i];
        }
        whole = wave_sum(mine);
        double target = (double)u * whole;
        const int lane = t.pick_lane(mine, target);
        double before = 0., sum = 0.;
        int chosen = 0;
        bool done = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double s = read_lane(four[i], lane);
          if (s > 0. && !done) {
            chosen = i;
            before = sum;
            sum += s;
            done = sum > target;
          }
        }
        const int per = a.chunks * 64 * kChunkVecs, from = (4 * lane + chosen) * per;
        double ignored;
        token = t.template locate<false, true>(from, min(from + per, t.nv), target - before, plain, ignored);
      }
    }
    if (tid == 0) {
      a.token[r] = token;
      if (a.logp) a.logp[r] = (float)log(t.weight(E::to_float(t.row[token])) / whole);
    }
  }
}

template <int DTYPE, bool LIMITED>
int launch_rows(const sm_desc* d, const SmArgs& a, hipStream_t stream) {
  const dim3 grid(std::min(a.rows, 1 << 20));
  if (d->held) {
    hipLaunchKernelGGL((sm_row_kernel<DTYPE, 256, LIMITED, true>), grid, dim3(256), 0, stream, a);
    return (int)hipGetLastError();
  }
  hipLaunchKernelGGL(sm_sums_kernel<DTYPE>, dim3((uint32_t)std::min<int64_t>(((int64_t)a.rows * a.segments + 3) / 4, kUnits * 4)), dim3(256), 0, stream, a);
  const int e = (int)hipGetLastError();
  if (e) return e;
  hipLaunchKernelGGL((sm_row_kernel<DTYPE, LIMITED ? 512 : 256, LIMITED, false>), grid, dim3(LIMITED ? 512 : 256), 0, stream, a);
  return (int)hipGetLastError();
}

template <int DTYPE>
int launch(const sm_desc* d, const SmArgs& a, hipStream_t stream) {
  return a.top_k || a.top_p || a.min_p ? launch_rows<DTYPE, true>(d, a, stream) : launch_rows<DTYPE, false>(d, a, stream);
}

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int sm_desc_create(sm_desc_t** out, const sm_params_t* pp) {
  if (!out || !pp) return CONV_EINVAL;
  const sm_params_t p = *pp;
  if (p.rows < 0 || p.vocab < 1 || (p.dtype != MI355_F32 && p.dtype != MI355_F16 && p.dtype != MI355_BF16)) return CONV_EINVAL;
  if (p.vocab >= 1 << 30) return CONV_ESHAPE;
  sm_desc* d = new (std::nothrow) sm_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->p = p;
  const int64_t chunk = 64 * kChunkVecs * 16 / dtype_bytes(p.dtype), chunks = (p.vocab + chunk - 1) / chunk;  // of logits
  d->chunks = (int32_t)((chunks + kMostSegments - 1) / kMostSegments);
  d->segments = (int32_t)((chunks + d->chunks - 1) / d->chunks);
  d->held = chunks <= 4;
  int bits = 0;
  while (((int64_t)1 << bits) < p.vocab) ++bits;
  d->shift = std::min(50, 61 - bits);
  if (!d->held) d->ws_bytes = (size_t)p.rows * d->segments * (sizeof(Part) + kTops * sizeof(float));
  snprintf(d->names, sizeof(d->names), d->held ? "sample=sm_row" : "sample=sm_sums+sm_row");
  *out = d;
  return CONV_OK;
}

int sm_desc_destroy(sm_desc_t* d) {
  if (!d) return CONV_EINVAL;
  delete d;
  return CONV_OK;
}

int sm_desc_workspace_bytes(const sm_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = d->ws_bytes;
  return CONV_OK;
}

const char* sm_desc_kernel_names(const sm_desc_t* d) { return d ? d->names : ""; }

int sm_sample(const sm_desc_t* d, const void* logits, int64_t stride, const float* u, const float* scale, const int32_t* top_k,
              const float* top_p, const float* min_p, int32_t* token, float* logp, void* ws, size_t ws_bytes, void* hip_stream) {
  if (!d) return CONV_EINVAL;
  if (d->p.rows == 0) return CONV_OK;
  if (!logits || !u || !token || (d->p.rows > 1 && stride < d->p.vocab)) return CONV_EINVAL;
  if (d->ws_bytes && (!ws || ws_bytes < d->ws_bytes)) return CONV_EWORKSPACE;
  if (d->ws_bytes && ((uintptr_t)ws & 15u)) return CONV_EINVAL;
  Part* const parts = static_cast<Part*>(ws);
  const SmArgs a = {logits, stride, u, scale, top_p, min_p, top_k, token, logp, parts, reinterpret_cast<float*>(parts + (size_t)d->p.rows * d->segments),
                    d->p.rows, d->p.vocab, d->segments, d->chunks, d->shift};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int e = d->p.dtype == MI355_F32   ? launch<MI355_F32>(d, a, stream)
                : d->p.dtype == MI355_F16 ? launch<MI355_F16>(d, a, stream)
                                          : launch<MI355_BF16>(d, a, stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
