// Log probabilities of given tokens over a large vocabulary, with the entropy, the most likely alternatives and the gradient
// of a loss on them (include/mi355lp.h).
//
// With c = scale log2(e) and any reference M, every quantity of a row follows from t_i = c x_i - M:
//   s = sum 2^t_i      s2 = sum 2^t_i t_i      log2 p_i = t_i - log2 s      H = ln 2 (log2 s - s2 / s)
//   d_logits_i = 2^t_i (A + B t_i) + [i = token] w scale,   B = -u scale ln 2 / s,   A = scale (-w - u (H - ln 2 log2 s)) / s
// so one pass finds s and s2 beside a running maximum, and a second one writes the gradient.  M is the maximum's own c x: the same
// number enters every t_i, so that its rounding cancels.
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
#include "mi355lp.h"
#include "wave_ops.h"

struct lp_desc {
  lp_params_t p;
  float c;          // scale log2(e)
  int32_t form;     // of the passes that see a whole row (Form)
  int32_t splits;   // parts of a row in different workgroups (1: none)
  int32_t seg;      // logits of a part
  size_t ws_bytes;
  char names[160];
};

namespace mi355conv {

namespace {

constexpr int kMaxTop = 64;
constexpr float kLn2 = 0.693147180559945309f;

struct LpArgs {
  const void* logits;
  int64_t stride;
  const int32_t* token;
  const float *d_logp, *d_entropy;
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_token;
  void* d_logits;
  int64_t d_stride;
  float4* parts;      // [rows][splits]: maximum, s, s2
  uint64_t* cand;     // [rows][splits][top]: the alternatives of a part
  int32_t rows, vocab, top, splits, seg;
  float scale, c;
};

// What a row's passes share.
struct RowStat {
  float M, c;      // t = c x - M
  float log2s, H;  // log2 s, entropy in nats
  float step;      // nats per unit of t
};

__device__ __forceinline__ float exp2_fast(float t) { return __builtin_amdgcn_exp2f(t); }  // 0 below 2^-126

// t for a product with 2^t, which is 0 where this cuts off: -inf must not meet a 0.
__device__ __forceinline__ float finite(float t) { return fmaxf(t, -200.f); }

// M is c x of a maximum, rounded to fp32: t there is the rounding, at most 32 up to 2^30.  Maxima below that range (large finite masks
// throughout) take its end for M, and leave sums of 0; beyond() takes care of those that are a row's.
constexpr float kMostReference = 0x1p30f;

__device__ __forceinline__ float reference(float m, float c) { return fminf(fmaxf(m * c, -kMostReference), kMostReference); }

// Whether a row's maximum is beyond that range.  Different values are then so far apart (2^-24 of c m, 64, at least) that p is shared by
// those equal to the maximum, and t may be P (x - m) with a power of two P for c: P m is exact, and so is the difference.
__device__ __forceinline__ bool beyond(float m, float c) { return !(fabsf(m * c) <= kMostReference) && m != -INFINITY; }

__device__ __forceinline__ float power_for(float m, float c) { return ldexpf(1.f, min(ilogbf(c) + 1, 126 - ilogbf(m))); }

struct Sums {
  float m, s, s2;
};

// Adds what another part of the row has found: relative to that part's own maximum m_t.  A part that lies beyond the range in a row that
// does not is 2^-64 of it at most (beyond), and its sums may be relative to another number than the range's end: nothing of it is added.
__device__ __forceinline__ void add_part(Sums& a, float M, bool over, float c, float m_t, float s_t, float s2_t) {
  const float d = reference(m_t, c) - M;
  const float f = over ? (m_t == a.m ? 1.f : 0.f) : m_t * c < -kMostReference ? 0.f : exp2_fast(d);
  a.s += f * s_t;
  a.s2 += f == 0.f ? 0.f : over ? s2_t : f * (s2_t + d * s_t);
}

__device__ __forceinline__ RowStat finish(const Sums& a, float c, float scale) {
  RowStat r;
  const bool over = beyond(a.m, c);
  r.c = over ? power_for(a.m, c) : c;
  r.step = over ? scale / r.c : kLn2;
  r.M = a.m == -INFINITY ? 0.f : a.m * r.c;
  if (a.m == -INFINITY && a.s == 0.f) {  // nothing but -inf
    r.log2s = INFINITY;
    r.H = 0.f;
  } else {
    r.log2s = log2f(a.s);
    r.H = kLn2 * (r.log2s - a.s2 / a.s);
  }
  return r;
}

// The natural logarithm of the probability of a logit.
__device__ __forceinline__ float log_prob(const RowStat& r, float x, float scale) {
  const float t = fmaf(x, r.c, -r.M);
  if (t == -INFINITY && x != -INFINITY) return x * scale - r.M / r.c * scale - kLn2 * r.log2s;  // c x is out of range, scale x may not be
  return fmaf(r.step, t, -kLn2 * r.log2s);
}

template <bool ENT>
__device__ __forceinline__ void put_stats(float* to, const RowStat& r) {
  store_vec<Elem<MI355_F32>>(to, Elem<MI355_F32>::pack({r.M, r.log2s, ENT ? r.H : NAN, r.c}));  // (without s2, H is not one)
}

struct GradScale {
  float A, B, at_token;
};

__device__ __forceinline__ GradScale grad_scale(const RowStat& r, float w, float u, float scale) {
  const float inv = exp2f(-r.log2s) * scale;
  GradScale g;
  g.B = -u * kLn2 * inv;
  g.A = inv * (-w - u * (r.log2s < INFINITY ? r.H - kLn2 * r.log2s : 0.f));
  if (r.log2s == INFINITY) g.A = g.B = 0.f;
  g.at_token = w * scale;
  return g;
}

// The wave's lanes' sums in one, in every lane.
__device__ __forceinline__ Sums wave_merge(float m, float s, float s2, float c) {
  Sums a = {wave_most(m), 0.f, 0.f};
  add_part(a, reference(a.m, c), beyond(a.m, c), c, m, s, s2);
  a.s = wave_sum(a.s);
  a.s2 = wave_sum(a.s2);
  return a;
}

// Logits in the order of the alternatives, as unsigned numbers: -0 is 0, NaN the greatest.  With the index below it, each once.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFEu;
  const uint32_t u = x == 0.f ? 0u : __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

__device__ __forceinline__ uint64_t entry_of(float x, int index) { return (uint64_t)order_key(x) << 32 | (0xFFFFFFFFu - (uint32_t)index); }

// ---- a row in the registers of a team of THREADS threads ----
// Vector v of a row holds its elements v VEC and on.  A partial one at the end, the tail, is thread 0's: it is loaded so that it ends
// with the row, and what an earlier vector holds as well is taken out (-inf): every access is inside the row.
template <class E>
struct Slot {
  int base;  // of element 0, negative in rows shorter than a vector
  int lo;    // elements from here on are this vector's
};

template <class E>
__device__ __forceinline__ Slot<E> slot_of(int v, int n) {
  const int b = v * E::VEC, over = b + E::VEC - n;
  return over <= 0 ? Slot<E>{b, 0} : Slot<E>{b - over, over};
}

template <class E>
__device__ __forceinline__ u32x4 lowest_vec() {
  return u32x4{E::kLowest, E::kLowest, E::kLowest, E::kLowest};
}

template <class E>
__device__ __forceinline__ u32x4 without_first(const u32x4& v, int lo) {
  u32x4 r = v;
  constexpr int PER = E::VEC / 4;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (PER == 1) {
      if (w < lo) r[w] = E::kLowest;
    } else {
      if (2 * w < lo) r[w] = (r[w] & 0xffff0000u) | (E::kLowest & 0xffffu);
      if (2 * w + 1 < lo) r[w] = (r[w] & 0xffffu) | (E::kLowest & 0xffff0000u);
    }
  }
  return r;
}

// Vector v (v VEC < n), wherever it lies.
template <class E, bool STREAM = false>
__device__ __forceinline__ u32x4 row_vec(const typename E::T* row, int v, int n) {
  const Slot<E> at = slot_of<E>(v, n);
  if (at.base >= 0) {
    const u32x4 r = get_vec<E, STREAM>(row + at.base);
    return at.lo ? without_first<E>(r, at.lo) : r;
  }
  float x[E::VEC];
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) x[i] = i >= at.lo ? E::to_float(row[at.base + i]) : -INFINITY;
  return E::pack(x);
}

template <class E, bool STREAM>
__device__ __forceinline__ void store_row_vec(typename E::T* row, int v, int n, const float (&x)[E::VEC]) {
  const Slot<E> at = slot_of<E>(v, n);
  if (at.lo == 0) {
    put_vec<E, STREAM>(row + at.base, E::pack(x));
    return;
  }
#pragma unroll
  for (int i = 0; i < E::VEC; ++i)
    if (i >= at.lo) row[at.base + i] = E::from_float(x[i]);
}

// One vector into a thread's sums.
template <class E, bool ENT>
__device__ __forceinline__ void add_vec(const u32x4& r, float c, float& m, float& M, float& s, float& s2) {
  float x[E::VEC];
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) x[i] = E::get(r, i);
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) most = fmaxf(most, x[i]);
  if (most > m) {
    const float to = reference(most, c), d = M - to, f = m == -INFINITY ? 0.f : exp2_fast(d);
    if (ENT) s2 = f == 0.f ? s * 0.f : f * (s2 + d * s);  // (NaN stays)
    s *= f;
    M = to;
    m = most;
  }
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) {
    const float t = fmaf(x[i], c, -M), e = exp2_fast(t);
    s += e;
    if (ENT) s2 = fmaf(e, finite(t), s2);
  }
}

template <bool ENT>
__device__ __forceinline__ float grad_of(float logit, const RowStat& st, const GradScale& g) {
  const float t = fmaf(logit, st.c, -st.M), e = exp2_fast(t);
  return e * (ENT ? fmaf(g.B, finite(t), g.A) : g.A);
}

template <class E, bool ENT>
__device__ __forceinline__ void grad_vec(const u32x4& r, const RowStat& st, const GradScale& g, float (&x)[E::VEC]) {
#pragma unroll
  for (int i = 0; i < E::VEC; ++i) x[i] = grad_of<ENT>(E::get(r, i), st, g);
}

// Keeps the compiler from carrying what one pass computed from the vectors (unpacked logits, lane masks) to the next one: it would
// take several times the registers that the vectors themselves do.
template <int NV>
__device__ __forceinline__ void forget(u32x4 (&r)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(r[j]));
}

__device__ __forceinline__ int forget(int uniform) {
  uniform = __builtin_amdgcn_readfirstlane(uniform);
  asm volatile("" : "+s"(uniform));
  return uniform;
}

// Keeps the scheduler from working on many vectors side by side, which takes more registers than there are.
__device__ __forceinline__ void one_by_one() { __builtin_amdgcn_sched_barrier(0); }

// f(vector, its number) for the thread's vectors of a row that are not among the NV in registers, four loads at a time.
template <class E, int THREADS, int NV, class F>
__device__ __forceinline__ void beyond_registers(const typename E::T* row, int full, int tid, F&& f) {
  for (int v0 = NV * THREADS; v0 < full; v0 += 4 * THREADS) {
    u32x4 r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int v = v0 + j * THREADS + tid;
      if (v < full) r[j] = load_vec<E>(row + (int64_t)v * E::VEC);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int v = v0 + j * THREADS + tid;
      if (v < full) f(r[j], v);
      one_by_one();
    }
  }
}

__device__ __forceinline__ int forget_lane(int per_lane) {
  asm volatile("" : "+v"(per_lane));
  return per_lane;
}

template <int THREADS>
__device__ __forceinline__ void team_sync() {
  if constexpr (THREADS == 64)
    wave_sync();
  else
    __syncthreads();
}

// Vectors that hold a candidate for a team's alternatives.  Where there are more, the alternatives are found one by one.
template <int THREADS>
constexpr int kHits = THREADS == 64 ? 64 : 256;

template <int THREADS>
struct TeamLds {
  u32x4 hit[kHits<THREADS>];
  uint64_t cand[kHits<THREADS> * 8];
  float4 sums[THREADS / 64];
  int hit_at[kHits<THREADS>];
  uint32_t group_top[64];
  float bound, at_token;
  uint32_t hits;
  uint64_t best[THREADS / 64];
};

// The greatest number that at least `top` of the wave's keys reach, its lower 16 bits cut off: a bound from below all the same.
__device__ __forceinline__ uint32_t top_bound(uint32_t key, int top) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t with = bound | 1u << bit;
    if (__builtin_popcountll(__ballot(key >= with)) >= top) bound = with;
  }
  return bound;
}

// A wave ranks `count` different entries by counting those above each.  Of more than 64 (short rows, that no bound has been found for) it
// first keeps those that pass a bound from 64 shares of them.
template <class Out>
__device__ __forceinline__ void rank_entries(uint64_t* cand, int count, int top, int lane, Out&& out) {
  if (count > 64) {
    uint32_t most = 0;
    for (int i = lane; i < count; i += 64) most = max(most, (uint32_t)(cand[i] >> 32));
    const uint32_t bound = top_bound(most, top);
    int kept = 0;
    for (int i0 = 0; i0 < count; i0 += 64) {
      const uint64_t mine = cand[min(i0 + lane, count - 1)];
      const bool pass = i0 + lane < count && (uint32_t)(mine >> 32) >= bound;
      const uint64_t mask = __ballot(pass);
      wave_sync();
      if (pass) cand[kept + __builtin_popcountll(mask & ((1ull << lane) - 1))] = mine;
      wave_sync();
      kept += (int)__builtin_popcountll(mask);
    }
    count = kept;
  }
  if (count <= 64) {
    const uint64_t mine = lane < count ? cand[lane] : 0;
    int rank = 0;
#pragma unroll 4
    for (int o = 0; o < count; ++o) rank += read_lane(mine, o) > mine ? 1 : 0;
    if (lane < count && rank < top) out(rank, mine);
  } else {
    for (int i = lane; i < count; i += 64) {
      const uint64_t mine = cand[i];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < count; ++o) rank += cand[o] > mine ? 1 : 0;
      if (rank < top) out(rank, mine);
    }
  }
}

// The `top` greatest entries of the row part [first, first + n), out(rank, entry) for each; 0 stands for none.
// The top-th greatest of 64 groups' maxima bounds the top-th greatest logit from below, so few others pass it: of 128256 normal
// logits, 24 for 20.  The vectors that hold one are put aside, and one wave ranks the logits in them that pass by counting those above
// each.  Where too many vectors do (equal logits, all but a few banned), each place is found by a pass over the row.
// m: the thread's maximum; odd: whether it has met a NaN, which no maximum shows.
template <class E, int THREADS, int NV, class Out>
__device__ __forceinline__ void team_top(TeamLds<THREADS>& lds, const u32x4 (&r)[NV], const u32x4& tail, const typename E::T* row, int first,
                                         int n, int top, float m, bool odd, int tid, Out&& out) {
  constexpr int VEC = E::VEC, GROUP = THREADS / 64;
  const int nv = (n + VEC - 1) / VEC, full = n / VEC, lane = tid & 63;
  const float gm = group_most<GROUP>(m);
  if (tid % GROUP == 0) lds.group_top[tid / GROUP] = order_key(gm);
  if (tid == 0) lds.hits = 0;
  if (tid == 0) lds.bound = -INFINITY;
  team_sync<THREADS>();
  // (where all vectors may be put aside, a bound from them one by one is the better one, and comes with the ranking)
  if (nv > kHits<THREADS> && (THREADS == 64 || tid < 64)) {  // the leading 16 bits of the top-th greatest: a bound all the same
    const uint32_t bound = top_bound(lds.group_top[lane], top);
    if (lane == 0) lds.bound = bound <= 0x007FFFFFu ? -INFINITY : key_value(bound);  // key of -inf and the unused ones below it
  }
  team_sync<THREADS>();
  const float bound = lds.bound;
  auto look = [&](const u32x4& vec, int v) {
    float most = E::get(vec, 0);
#pragma unroll
    for (int i = 1; i < VEC; ++i) most = __builtin_elementwise_maximum(most, E::get(vec, i));  // NaN if there is one
    if (!(most < bound)) {
      const uint32_t place = atomicAdd(&lds.hits, 1u);
      if (place < (uint32_t)kHits<THREADS>) {
        lds.hit[place] = vec;
        lds.hit_at[place] = v;
      }
    }
  };
  if (!(m < bound) || odd) {
    const int full_ = forget(full), tid_ = forget_lane(tid);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * THREADS < full_ && j * THREADS + tid_ < full_) look(r[j], j * THREADS + tid_);
      one_by_one();
    }
    beyond_registers<E, THREADS, NV>(row, full, tid, look);
    if (full < nv && tid == 0) look(tail, full);
  }
  team_sync<THREADS>();
  const int hits = __builtin_amdgcn_readfirstlane((int)lds.hits);
  if (hits <= kHits<THREADS>) {
    if (THREADS > 64 && tid >= 64) return;
    int count = 0;
    for (int i0 = 0; i0 < hits * VEC; i0 += 64) {
      const int i = i0 + lane;
      bool pass = false;
      uint64_t entry = 0;
      if (i < hits * VEC) {
        const float x = E::to_float(reinterpret_cast<const typename E::T*>(lds.hit)[i]);
        const Slot<E> at = slot_of<E>(lds.hit_at[i / VEC], n);
        pass = !(x < bound) && i % VEC >= at.lo;
        entry = entry_of(x, first + at.base + i % VEC);
      }
      const uint64_t mask = __ballot(pass);
      if (pass) lds.cand[count + __builtin_popcountll(mask & ((1ull << lane) - 1))] = entry;
      count += (int)__builtin_popcountll(mask);
    }
    wave_sync();
    rank_entries(lds.cand, count, top, lane, out);
    for (int i = count + lane; i < top; i += 64) out(i, (uint64_t)0);  // a part shorter than that
    return;
  }
  uint64_t last = ~(uint64_t)0;
  for (int k = 0; k < top; ++k) {
    uint64_t best = 0;
    for (int v = tid; v < nv; v += THREADS) {
      const u32x4 vec = row_vec<E>(row, v, n);
      const Slot<E> at = slot_of<E>(v, n);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const uint64_t e = entry_of(E::get(vec, i), first + at.base + i);
        if (i >= at.lo && e < last && e > best) best = e;
      }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const uint64_t o = __shfl_xor((unsigned long long)best, d, 64);
      best = o > best ? o : best;
    }
    if constexpr (THREADS > 64) {
      if (lane == 0) lds.best[tid >> 6] = best;
      __syncthreads();
      for (int w = 0; w < THREADS / 64; ++w) best = lds.best[w] > best ? lds.best[w] : best;
      __syncthreads();
    }
    last = best;
    if (tid == 0) out(k, best);
  }
}

enum Mode { kScore, kTrain, kPart };

// A row (kPart: a part of one) is read once, into registers, up to NV vectors a thread; what is beyond them is read again by
// whatever needs it again.  THREADS 64: a wave for each row, several in a workgroup.
// STREAM: what is read and written once goes around the last-level cache.
template <int DTYPE, int THREADS, int NV, Mode MODE, bool ENT, bool STREAM>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS, THREADS == 64 ? 1 : NV > 20 ? 3 : 4) void lp_row_kernel(LpArgs a) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  constexpr int VEC = E::VEC, WAVES = THREADS / 64;
  extern __shared__ u32x4 team_memory[];  // TeamLds for each team, but where a wave trains
  TeamLds<THREADS>& lds = reinterpret_cast<TeamLds<THREADS>*>(team_memory)[THREADS == 64 ? threadIdx.x >> 6 : 0];
  const int lane = threadIdx.x & 63;
  const int teams = THREADS == 64 ? (int)(gridDim.x * (blockDim.x >> 6)) : (int)gridDim.x;
  int item = THREADS == 64 ? (int)(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6)) : (int)blockIdx.x;
  if constexpr (THREADS == 64) item = __builtin_amdgcn_readfirstlane(item);
  const int64_t items = MODE == kPart ? (int64_t)a.rows * a.splits : a.rows;
  for (int64_t it = item; it < items; it += teams) {
    const int r_ = MODE == kPart ? (int)(it / a.splits) : (int)it;
    const int first = MODE == kPart ? (int)(it % a.splits) * a.seg : 0;
    // (nothing that follows from these is worth a register from one row to the next)
    const int n = forget(MODE == kPart ? min(a.seg, a.vocab - first) : a.vocab);
    const int tid = forget_lane(THREADS == 64 ? threadIdx.x & 63 : threadIdx.x);
    const T* const row = static_cast<const T*>(a.logits) + (int64_t)r_ * a.stride + first;
    const int nv = (n + VEC - 1) / VEC, full = n / VEC;
    int token = -1;
    float at_token = 0.f;
    if (MODE != kPart && a.token) {
      token = a.token[r_];
      if ((uint32_t)token >= (uint32_t)a.vocab) token = -1;
      if (token >= 0) at_token = E::to_float(row[token]);
    }

    u32x4 r[NV], tail = lowest_vec<E>();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      r[j] = lowest_vec<E>();
      if (j * THREADS < full && j * THREADS + tid < full) r[j] = get_vec<E, STREAM>(row + (j * THREADS + tid) * VEC);
    }
    if (full < nv && tid == 0) tail = row_vec<E>(row, full, n);

    float m = -INFINITY, M = 0.f, s = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * THREADS < full) {
        add_vec<E, ENT>(r[j], a.c, m, M, s, s2);
        one_by_one();
      }
    beyond_registers<E, THREADS, NV>(row, full, tid, [&](const u32x4& vec, int) { add_vec<E, ENT>(vec, a.c, m, M, s, s2); });
    if (full < nv) add_vec<E, ENT>(tail, a.c, m, M, s, s2);

    forget(r);
    Sums sum = wave_merge(m, s, s2, a.c);
    if constexpr (WAVES > 1) {
      // through shared memory, so that it has arrived before another wave writes over it (d_logits may be logits)
      if (tid == 0) lds.at_token = at_token;
      if (lane == 0) lds.sums[tid >> 6] = make_float4(sum.m, sum.s, sum.s2, 0.f);
      __syncthreads();
      const float4 p = lane < WAVES ? lds.sums[lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
      sum = wave_merge(p.x, p.y, p.z, a.c);
      at_token = lds.at_token;
    }
    if (beyond(sum.m, a.c)) {  // rare: the sums again, with that row's t
      const float P = power_for(sum.m, a.c), M = sum.m * P;
      float count = 0.f;
      for (int v = tid; v < nv; v += THREADS) {
        const u32x4 vec = row_vec<E>(row, v, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) count += exp2_fast(fmaf(E::get(vec, i), P, -M));
      }
      count = wave_sum(count);
      if constexpr (WAVES > 1) {
        __syncthreads();
        if (lane == 0) lds.sums[tid >> 6].x = count;
        __syncthreads();
        count = wave_sum(lane < WAVES ? lds.sums[lane].x : 0.f);
      }
      sum.s = count;
      sum.s2 = 0.f;
    }

    if constexpr (MODE == kPart) {
      if (tid == 0) a.parts[it] = make_float4(sum.m, sum.s, sum.s2, 0.f);
      if (a.top) {
        uint64_t* const to = a.cand + it * a.top;
        team_top<E, THREADS, NV>(lds, r, tail, row, first, n, a.top, m, s != s, tid, [&](int rank, uint64_t e) { to[rank] = e; });
      }
    } else {
      const RowStat st = finish(sum, a.c, a.scale);
      if (tid == 0) {
        if (a.logp) a.logp[r_] = token >= 0 ? log_prob(st, at_token, a.scale) : 0.f;
        if (ENT && a.entropy) a.entropy[r_] = st.H;
        if (MODE == kScore && a.stats) put_stats<ENT>(a.stats + 4 * (int64_t)r_, st);
      }
      if constexpr (MODE == kScore) {
        if (a.top) {
          float* const logp = a.top_logp + (int64_t)r_ * a.top;
          int32_t* const tok = a.top_token + (int64_t)r_ * a.top;
          team_top<E, THREADS, NV>(lds, r, tail, row, 0, n, a.top, m, s != s, tid, [&](int rank, uint64_t e) {
            logp[rank] = log_prob(st, key_value((uint32_t)(e >> 32)), a.scale);
            tok[rank] = (int32_t)(0xFFFFFFFFu - (uint32_t)e);
          });
        }
      } else {
        const float w = token >= 0 ? a.d_logp[r_] : 0.f, u = ENT && a.d_entropy ? a.d_entropy[r_] : 0.f;
        const GradScale g = grad_scale(st, w, u, a.scale);
        T* const to = static_cast<T*>(a.d_logits) + (int64_t)r_ * a.d_stride;
        const int full_ = forget(full), tid_ = forget_lane(tid);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          if (j * THREADS < full_ && j * THREADS + tid_ < full_) {
            float x[VEC];
            grad_vec<E, ENT>(r[j], st, g, x);
            put_vec<E, STREAM>(to + (j * THREADS + tid_) * VEC, E::pack(x));
          }
          one_by_one();
        }
        beyond_registers<E, THREADS, NV>(row, full, tid, [&](const u32x4& vec, int v) {
          float x[VEC];
          grad_vec<E, ENT>(vec, st, g, x);
          put_vec<E, STREAM>(to + (int64_t)v * VEC, E::pack(x));
        });
        if (full < nv && tid == 0) {
          float x[VEC];
          grad_vec<E, ENT>(tail, st, g, x);
          store_row_vec<E, STREAM>(to, full, n, x);
        }
        // the token's own, by the thread that has just written it without
        if (token >= 0 && tid == (token < full * VEC ? token / VEC % THREADS : 0))
          to[token] = E::from_float(grad_of<ENT>(at_token, st, g) + g.at_token);
      }
    }
    team_sync<THREADS>();  // the next row's team memory
  }
}

// The sums of a row's parts, in every lane of a wave.
__device__ __forceinline__ Sums merge_parts(const float4* parts, int splits, int lane, float c) {
  const float4 p = lane < splits ? parts[lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  return wave_merge(p.x, p.y, p.z, c);
}

constexpr int kMaxSplits = 64;

// A row's parts in one: a workgroup for each row.  Each part's alternatives are in order; the leading ones of all parts, 64 together, give a
// bound as the groups' maxima do in team_top, and what passes it is ranked by one wave.
template <int DTYPE, bool ENT>
__global__ __launch_bounds__(256) void lp_join_kernel(LpArgs a) {
  typedef Elem<DTYPE> E;
  extern __shared__ uint64_t entries[];  // those that pass, at most [splits][top]
  __shared__ uint32_t passed;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int total = a.splits * a.top;
  float at_token = 0.f;
  int token = -1;
  if (a.logp) {
    token = a.token[row];
    if ((uint32_t)token >= (uint32_t)a.vocab) token = -1;
    if (token >= 0) at_token = E::to_float(static_cast<const typename E::T*>(a.logits)[(int64_t)row * a.stride + token]);
  }
  const uint64_t* const cand = a.cand + (int64_t)row * total;
  const int part = lane % a.splits, place = lane / a.splits;
  uint32_t sample = 0;
  if (place < a.top && (place + 1) * a.splits <= 64) sample = (uint32_t)(cand[part * a.top + place] >> 32);
  if (threadIdx.x == 0) passed = 0;
  const RowStat st = finish(merge_parts(a.parts + (int64_t)row * a.splits, a.splits, lane, a.c), a.c, a.scale);
  if (threadIdx.x == 0) {
    if (a.logp) a.logp[row] = token >= 0 ? log_prob(st, at_token, a.scale) : 0.f;
    if (ENT && a.entropy) a.entropy[row] = st.H;
    if (a.stats) put_stats<ENT>(a.stats + 4 * (int64_t)row, st);
  }
  if (total == 0) return;
  const uint32_t bound = top_bound(sample, a.top);
  __syncthreads();
  for (int i0 = 0; i0 < total; i0 += 256) {
    const int i = i0 + threadIdx.x;
    const uint64_t mine = i < total ? cand[i] : 0;
    const bool pass = mine != 0 && (uint32_t)(mine >> 32) >= bound;
    const uint64_t mask = __ballot(pass);
    uint32_t at = 0;
    if (lane == 0 && mask) at = atomicAdd(&passed, (uint32_t)__builtin_popcountll(mask));
    at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    if (pass) entries[at + __builtin_popcountll(mask & ((1ull << lane) - 1))] = mine;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  rank_entries(entries, (int)passed, a.top, lane, [&](int rank, uint64_t e) {
    a.top_logp[(int64_t)row * a.top + rank] = log_prob(st, key_value((uint32_t)(e >> 32)), a.scale);
    a.top_token[(int64_t)row * a.top + rank] = (int32_t)(0xFFFFFFFFu - (uint32_t)e);
  });
}

// The gradient where the row's statistics are known (PARTS: as parts), kGradVecs vectors a thread.
constexpr int kGradVecs = 4;

template <int DTYPE, bool ENT, bool PARTS, bool STREAM>
__global__ __launch_bounds__(256) void lp_grad_kernel(LpArgs a, int chunks) {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  constexpr int VEC = E::VEC, CHUNK = 256 * VEC * kGradVecs;
  const int64_t items = (int64_t)a.rows * chunks;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int r_ = (int)(it / chunks), first = (int)(it % chunks) * CHUNK;
    const int n = min(CHUNK, a.vocab - first), nv = (n + VEC - 1) / VEC;
    const T* const row = static_cast<const T*>(a.logits) + (int64_t)r_ * a.stride;
    u32x4 r[kGradVecs];
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      const int v = j * 256 + (int)threadIdx.x;
      r[j] = v < nv ? row_vec<E, STREAM>(row + first, v, n) : lowest_vec<E>();
    }
    int token = a.token[r_];
    if ((uint32_t)token >= (uint32_t)a.vocab) token = -1;
    // where d_logits is logits, this one is about to be overwritten, by this workgroup
    const bool mine = token >= first && token < first + n;
    const float at_token = mine ? E::to_float(row[token]) : 0.f;
    RowStat st;
    if constexpr (PARTS) {
      st = finish(merge_parts(a.parts + (int64_t)r_ * a.splits, a.splits, threadIdx.x & 63, a.c), a.c, a.scale);
    } else {
      const float* const q = a.stats + 4 * (int64_t)r_;
      st = RowStat{q[0], q[3], q[1], ENT && a.d_entropy ? q[2] : 0.f, 0.f};
    }
    const float w = token >= 0 ? a.d_logp[r_] : 0.f, u = ENT && a.d_entropy ? a.d_entropy[r_] : 0.f;
    const GradScale g = grad_scale(st, w, u, a.scale);
    T* const to = static_cast<T*>(a.d_logits) + (int64_t)r_ * a.d_stride + first;
    const int owner = (token - first) / VEC % 256;
    float own = 0.f, logp = 0.f;
    if (mine) {
      own = grad_of<ENT>(at_token, st, g) + g.at_token;
      logp = log_prob(st, at_token, a.scale);
    }
    asm volatile("" ::"v"(own), "v"(logp));  // the logit has arrived
    __syncthreads();
    if (PARTS && threadIdx.x == 0) {
      if (a.logp && mine) a.logp[r_] = logp;
      if (a.logp && token < 0 && first == 0) a.logp[r_] = 0.f;
      if (ENT && a.entropy && first == 0) a.entropy[r_] = st.H;
    }
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      const int v = j * 256 + (int)threadIdx.x;
      if (v < nv) {
        float x[VEC];
        grad_vec<E, ENT>(r[j], st, g, x);
        store_row_vec<E, STREAM>(to, v, n, x);
      }
    }
    if (mine && (int)threadIdx.x == owner) to[token - first] = E::from_float(own);
  }
}

// The team of a whole row: the smallest whose registers hold it, as several share a compute unit and one loads while another computes,
// and as a wave needs no barriers.  us, this team and the next larger one (rows x vocab):
//   wave4    8000 x 2000 bf16, 20 alternatives 17.4, 256 threads 33.3; training 17.8, 27.1
//   wave8    8000 x 3900 bf16, 20 alternatives 25.4, block8 40.1; training on 8000 x 3000 28.2, 37.6
//   block8   3000 x 12000 bf16, 20 alternatives 27.4, block16 32.0; 512 threads 47
//   block16  1000 x 30000 bf16, 20 alternatives 23.5, 512 threads 25.1; training on 3000 x 30000 73.2, 77.7
//   block26  8000 x 50257 f16 163, 512 threads 185; training on 2000 x 50257 90.0, 93.9
//   long     training on 4096 x 128256 bf16, through the cache: 512 threads 453, 1024 with 20 vectors 485, with 7 (most of a row read again) 470
// Where there is at most one row for a compute unit, 1024 threads: 1 x 32000 8.7 us, in parts 11.0; 200 x 30000 trained 9.8, in parts 15.
// What the long team cannot hold (81920 logits of 16 bits) is read again from the caches.  (Its kernels that score 16-bit rows keep 8 bytes a
// thread in scratch memory.)
enum Form { kWave4, kWave8, kSolo, kBlock8, kBlock16, kBlock26, kLong };
const char* const kFormNames[] = {"wave4", "wave8", "solo", "block8", "block16", "block26", "long"};

constexpr int kSoloVecs = 4, kLongVecs = 20;

// Whether three block26 teams on a compute unit finish before two long ones: they take 5/6 of the time for a row where all places are taken,
// but a last round that is not full costs more.  us, block26 and long, rows of 50257 fp16 with 20 alternatives, of 36000 bf16 trained, of 24000 fp32
// trained, the same logits from call to call:
//    300 rows  21.2 20.6,  18.3 17.8,  16.1 15.7      777 rows  32.6 34.1,  28.7 29.6,  33.2 32.3      2400 rows  71.7 86.7,  70.3 70.7,  84.8 82.1
//    700 rows  27.3 29.1,  25.1 25.6,  22.8 28.3     1300 rows  42.6 48.5,  48.6 50.1,  56.4 54.5      8000 rows   190  245,   216  214,   273  262
// Of 132 calls of 257 to 8000 rows the slower one is taken in 19, by 7 % at most.
bool dense(int64_t rows) { return (rows + 767) / 768 * 20 <= (rows + 511) / 512 * 16; }
constexpr int kUnits = 256;  // compute units
constexpr int kMostTeams = 1 << 20;

template <int DTYPE, int THREADS, int NV, Mode MODE, bool ENT, bool STREAM>
void launch_team(const LpArgs& a, int blocks, int threads, hipStream_t stream) {
  const size_t lds = MODE == kTrain && THREADS == 64 ? 0 : sizeof(TeamLds<THREADS>) * (threads / THREADS);
  hipLaunchKernelGGL((lp_row_kernel<DTYPE, THREADS, NV, MODE, ENT, STREAM>), dim3(std::min(blocks, kMostTeams)), dim3(threads), lds, stream, a);
}

template <int DTYPE, Mode MODE, bool ENT, bool STREAM>
int launch_row(const lp_desc* d, const LpArgs& a, hipStream_t stream) {
  if constexpr (MODE == kPart) {
    launch_team<DTYPE, 1024, kSoloVecs, kPart, ENT, false>(a, a.rows * a.splits, 1024, stream);
  } else {
    const int waves = a.rows >= 2048 ? 4 : 1;
    if (d->form == kWave4)
      launch_team<DTYPE, 64, 4, MODE, ENT, STREAM>(a, (int)(((int64_t)a.rows + waves - 1) / waves), 64 * waves, stream);
    else if (d->form == kWave8)
      launch_team<DTYPE, 64, 8, MODE, ENT, STREAM>(a, (int)(((int64_t)a.rows + waves - 1) / waves), 64 * waves, stream);
    else if (d->form == kBlock8)
      launch_team<DTYPE, 256, 8, MODE, ENT, STREAM>(a, a.rows, 256, stream);
    else if (d->form == kBlock16)
      launch_team<DTYPE, 256, 16, MODE, ENT, STREAM>(a, a.rows, 256, stream);
    else if (d->form == kBlock26)
      launch_team<DTYPE, 256, 26, MODE, ENT, STREAM>(a, a.rows, 256, stream);
    else if (d->form == kSolo)
      launch_team<DTYPE, 1024, kSoloVecs, MODE, ENT, false>(a, a.rows, 1024, stream);  // (at most 32 MB)
    else
      launch_team<DTYPE, 512, kLongVecs, MODE, ENT, STREAM>(a, a.rows, 512, stream);
  }
  return (int)hipGetLastError();
}

template <int DTYPE, bool ENT>
int launch_join(const LpArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((lp_join_kernel<DTYPE, ENT>), dim3(a.rows), dim3(256), (size_t)a.splits * a.top * 8, stream, a);
  return (int)hipGetLastError();
}

template <int DTYPE, bool ENT, bool PARTS, bool STREAM>
int launch_grad(const LpArgs& a, hipStream_t stream) {
  constexpr int CHUNK = 256 * Elem<DTYPE>::VEC * kGradVecs;
  const int chunks = (a.vocab + CHUNK - 1) / CHUNK;
  hipLaunchKernelGGL((lp_grad_kernel<DTYPE, ENT, PARTS, STREAM>), dim3((uint32_t)std::min<int64_t>((int64_t)a.rows * chunks, 1 << 22)), dim3(256), 0, stream, a, chunks);
  return (int)hipGetLastError();
}

// Whether the logits, or they and the gradient, are more than the last-level cache (256 MB) holds: they then go around it, and leave it to
// what is read a second time.  Training on 4096 x 128256: 455 us through it, 442 with the gradient around it, 417 with both.
bool streams(const lp_desc* d, int blobs) { return (double)d->p.rows * d->p.vocab * dtype_bytes(d->p.dtype) * blobs > (double)(256 << 20); }

// One of the descriptor's six kinds.
template <template <int, bool> class Op>
int by_kind(const lp_desc* d, const LpArgs& a, hipStream_t stream) {
  const bool ent = d->p.entropy != 0;
  switch (d->p.dtype) {
    case MI355_F32: return ent ? Op<MI355_F32, true>::run(d, a, stream) : Op<MI355_F32, false>::run(d, a, stream);
    case MI355_F16: return ent ? Op<MI355_F16, true>::run(d, a, stream) : Op<MI355_F16, false>::run(d, a, stream);
    default: return ent ? Op<MI355_BF16, true>::run(d, a, stream) : Op<MI355_BF16, false>::run(d, a, stream);
  }
}

template <int DTYPE, bool ENT>
struct Forward {
  static int run(const lp_desc* d, const LpArgs& a, hipStream_t stream) {
    if (d->splits == 1) return streams(d, 1) ? launch_row<DTYPE, kScore, ENT, true>(d, a, stream) : launch_row<DTYPE, kScore, ENT, false>(d, a, stream);
    const int e = launch_row<DTYPE, kPart, ENT, false>(d, a, stream);
    return e ? e : launch_join<DTYPE, ENT>(a, stream);
  }
};

template <int DTYPE, bool ENT>
struct Backward {
  static int run(const lp_desc* d, const LpArgs& a, hipStream_t stream) {
    return streams(d, 2) ? launch_grad<DTYPE, ENT, false, true>(a, stream) : launch_grad<DTYPE, ENT, false, false>(a, stream);
  }
};

template <int DTYPE, bool ENT>
struct ForwardBackward {
  static int run(const lp_desc* d, const LpArgs& a, hipStream_t stream) {
    if (d->splits == 1) return streams(d, 2) ? launch_row<DTYPE, kTrain, ENT, true>(d, a, stream) : launch_row<DTYPE, kTrain, ENT, false>(d, a, stream);
    const int e = launch_row<DTYPE, kPart, ENT, false>(d, a, stream);
    return e ? e : launch_grad<DTYPE, ENT, true, false>(a, stream);
  }
};

LpArgs base_args(const lp_desc* d, const void* logits, int64_t stride, const int32_t* token) {
  LpArgs a = {};
  a.logits = logits;
  a.stride = stride;
  a.token = token;
  a.rows = d->p.rows;
  a.vocab = d->p.vocab;
  a.splits = d->splits;
  a.seg = d->seg;
  a.scale = d->p.scale;
  a.c = d->c;
  return a;
}

void place_workspace(const lp_desc* d, LpArgs& a, void* ws) {
  a.parts = static_cast<float4*>(ws);
  a.cand = reinterpret_cast<uint64_t*>(a.parts + (size_t)d->p.rows * d->splits);
}

bool bad_rows(const lp_desc* d, const void* at, int64_t stride) { return !at || (d->p.rows > 1 && stride < d->p.vocab); }

}  // namespace

}  // namespace mi355conv

using namespace mi355conv;

extern "C" {

int lp_desc_create(lp_desc_t** out, const lp_params_t* pp) {
  if (!out || !pp) return CONV_EINVAL;
  const lp_params_t p = *pp;
  if (p.rows < 0 || p.vocab < 1 || (p.dtype != MI355_F32 && p.dtype != MI355_F16 && p.dtype != MI355_BF16)) return CONV_EINVAL;
  if (p.top < 0 || p.top > kMaxTop || p.top > p.vocab || (p.entropy != 0 && p.entropy != 1)) return CONV_EINVAL;
  if (!(p.scale >= 0x1p-60f && p.scale <= 0x1p60f)) return CONV_EINVAL;
  if (p.vocab >= 1 << 30) return CONV_ESHAPE;
  lp_desc* d = new (std::nothrow) lp_desc;
  if (!d) return CONV_EINVAL;
  memset(d, 0, sizeof(*d));
  d->p = p;
  d->c = (float)(p.scale * 1.44269504088896340736);
  const int vec = 16 / dtype_bytes(p.dtype);
  const int solo = 1024 * vec * kSoloVecs;
  d->form = p.vocab <= 64 * vec * 4                   ? kWave4
            : p.rows <= kUnits && p.vocab <= solo     ? kSolo
            : p.vocab <= 64 * vec * 8                 ? kWave8
            : p.vocab <= 256 * vec * 8                ? kBlock8
            : p.vocab <= 256 * vec * 16               ? kBlock16
            : p.vocab <= 256 * vec * 26 && dense(p.rows) ? kBlock26
                                                      : kLong;
  d->splits = 1;
  d->seg = p.vocab;
  // Where a workgroup of 1024 cannot hold a row and there are two compute units or more for each, rows are taken in parts: 64 x 128256
  // with 20 alternatives 14.4 us, whole rows 24.2; 8 x 128256 12.0, 23.2; 200 x 50257, one part, 15.0, and 14.7 in two.
  if (p.rows > 0 && p.rows <= kUnits / 2 && p.vocab > solo) {
    const int splits = std::min(std::min(kUnits / p.rows, (p.vocab + solo / 4 - 1) / (solo / 4)), kMaxSplits);
    d->seg = ((p.vocab + splits - 1) / splits + vec - 1) / vec * vec;
    d->splits = (p.vocab + d->seg - 1) / d->seg;
  }
  if (d->splits > 1) d->ws_bytes = (size_t)p.rows * d->splits * (16 + 8 * (size_t)p.top);
  const char* const form = kFormNames[d->form];
  auto around = [&](int blobs) { return d->form != kSolo && streams(d, blobs) ? ",stream" : ""; };
  if (d->splits > 1)
    snprintf(d->names, sizeof(d->names), "forward=lp_parts(S=%d)+join;backward=lp_grad%s;forward_backward=lp_parts(S=%d)+grad", d->splits,
             streams(d, 2) ? "[stream]" : "", d->splits);
  else
    snprintf(d->names, sizeof(d->names), "forward=lp_row[%s%s];backward=lp_grad%s;forward_backward=lp_row[%s%s]", form, around(1), streams(d, 2) ? "[stream]" : "",
             form, around(2));
  *out = d;
  return CONV_OK;
}

int lp_desc_destroy(lp_desc_t* d) {
  if (!d) return CONV_EINVAL;
  delete d;
  return CONV_OK;
}

int lp_desc_workspace_bytes(const lp_desc_t* d, size_t* bytes) {
  if (!d || !bytes) return CONV_EINVAL;
  *bytes = d->ws_bytes;
  return CONV_OK;
}

const char* lp_desc_kernel_names(const lp_desc_t* d) { return d ? d->names : ""; }

int lp_forward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, float* logp, float* entropy,
               float* stats, float* top_logp, int32_t* top_token, void* ws, size_t ws_bytes, void* hip_stream) {
  if (!d || (token != nullptr) != (logp != nullptr) || (entropy && !d->p.entropy)) return CONV_EINVAL;
  if (d->p.rows == 0) return CONV_OK;
  if ((top_logp != nullptr) != (d->p.top > 0) || (top_token != nullptr) != (d->p.top > 0)) return CONV_EINVAL;
  if (bad_rows(d, logits, stride)) return CONV_EINVAL;
  if (d->ws_bytes && (!ws || ws_bytes < d->ws_bytes)) return CONV_EWORKSPACE;
  if (d->ws_bytes && ((uintptr_t)ws & 15u)) return CONV_EINVAL;
  LpArgs a = base_args(d, logits, stride, token);
  a.logp = logp;
  a.entropy = entropy;
  a.stats = stats;
  a.top = d->p.top;
  a.top_logp = top_logp;
  a.top_token = top_token;
  place_workspace(d, a, ws);
  const int e = by_kind<Forward>(d, a, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int lp_backward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, const float* stats,
                const float* d_logp, const float* d_entropy, void* d_logits, int64_t d_stride, void* hip_stream) {
  if (!d || (d_entropy && !d->p.entropy)) return CONV_EINVAL;
  if (d->p.rows == 0) return CONV_OK;
  if (bad_rows(d, logits, stride) || bad_rows(d, d_logits, d_stride) || !token || !stats || !d_logp) return CONV_EINVAL;
  LpArgs a = base_args(d, logits, stride, token);
  a.stats = const_cast<float*>(stats);
  a.d_logp = d_logp;
  a.d_entropy = d_entropy;
  a.d_logits = d_logits;
  a.d_stride = d_stride;
  const int e = by_kind<Backward>(d, a, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

int lp_forward_backward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, const float* d_logp,
                        const float* d_entropy, float* logp, float* entropy, void* d_logits, int64_t d_stride, void* ws,
                        size_t ws_bytes, void* hip_stream) {
  if (!d || ((d_entropy || entropy) && !d->p.entropy)) return CONV_EINVAL;
  if (d->p.rows == 0) return CONV_OK;
  if (bad_rows(d, logits, stride) || bad_rows(d, d_logits, d_stride) || !token || !d_logp) return CONV_EINVAL;
  if (d->ws_bytes && (!ws || ws_bytes < d->ws_bytes)) return CONV_EWORKSPACE;
  if (d->ws_bytes && ((uintptr_t)ws & 15u)) return CONV_EINVAL;
  LpArgs a = base_args(d, logits, stride, token);
  a.logp = logp;
  a.entropy = entropy;
  a.d_logp = d_logp;
  a.d_entropy = d_entropy;
  a.d_logits = d_logits;
  a.d_stride = d_stride;
  place_workspace(d, a, ws);
  const int e = by_kind<ForwardBackward>(d, a, (hipStream_t)hip_stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
