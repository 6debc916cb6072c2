// Drawing tokens under a temperature, top-k, top-p and min-p from given uniform numbers (include/mi355sm.h).
//
// What is kept of a row is what its cut keeps, x > value or x = value and index <= last, and what min-p keeps: top-k and top-p only move the
// cut.  Its place is found by a histogram of the distances below the maximum, finer ones of a bin that holds many logits, and an exact order of the
// few of the last bin.  The token is then found from the weights' sums in the order of the indices: over groups of vectors, vectors, lanes, elements.
//
// Weights are 64 bits wide: with 128256 tokens borders lie 2^-17 of the whole apart, and a uniform number falls within fp32's error of one in
// every hundredth row.  exp(scale (x - m)) = 2^(n / 32) 2^(r / 32) with n a whole number and |r| <= 1/2: the 32 roots of 2 and a polynomial.
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
  int32_t large;  // a team of 1024 threads for a row, not 256
  char names[64];
};

namespace mi355conv {

namespace {

struct SmArgs {
  const void* logits;
  int64_t stride;
  const float *u, *scale, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logp;
  int32_t rows, vocab;
  int32_t shift;  // weights as whole numbers: 2^shift, so that a row's sum stays below 2^62
};

constexpr int kBins = 1024;       // of a histogram
constexpr int kList = 1024;       // logits that are put in order
constexpr int kGroups = 16;       // of a row's vectors, whose sums stand side by side
constexpr float kNear = 8.f;      // nats below the maximum that the first histogram looks at: weights from 3e-4 on

// 2^(i / 32), computed to 60 digits and rounded.
__device__ const double kRoots[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002,
};

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

template <int THREADS, int HELD>
struct TeamLds {
  static constexpr int WAVES = THREADS / 64;
  u32x4 held[HELD * THREADS];  // the row's first vectors, each read by the thread that wrote it
  double part[kGroups][WAVES];
  double root[32];
  double sum[WAVES];
  uint64_t whole[WAVES];
  uint64_t list[kList];
  uint64_t weight[kBins];
  int count[kBins];
  float most[WAVES], least[WAVES];
  int number[WAVES];
  uint32_t listed;
  int found, before, inside;
  double result;
};

struct Cut {
  float value;
  int last;
};

template <int DTYPE, int THREADS, int HELD>
struct Team {
  typedef Elem<DTYPE> E;
  typedef typename E::T T;
  typedef TeamLds<THREADS, HELD> Lds;
  static constexpr int VEC = E::VEC, WAVES = THREADS / 64;

  Lds& lds;
  const T* row;
  int n, nv, rounds, tid, lane, wave, shift;
  float m, scale;  // the maximum
  double top, c32, q;
  Cut cut;

  __device__ u32x4 vec(int j) const {
    const int v = j * THREADS + tid;
    if (j < HELD) return lds.held[v];
    return v < nv ? row_vec<E>(row, v, n) : lowest_vec<E>();
  }

  // f(vector, its number) for this thread's vectors of the rounds [j0, j1), four loads at a time.
  template <class F>
  __device__ __forceinline__ void each(int j0, int j1, F&& f) const {
    for (int j = j0; j < j1; j += 4) {
      u32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < j1) x[i] = vec(j + i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < j1) {
          f(x[i], (j + i) * THREADS + tid);
          __builtin_amdgcn_sched_barrier(0);  // (vectors side by side would take more registers than there are)
        }
    }
  }

  __device__ __forceinline__ double weight(float x) const {
    const double t = fmax(((double)x - top) * c32, -36000.);  // (2^-1125 is 0)
    const double whole = rint(t), r = t - whole;
    const int i = (int)whole;
    constexpr double L = 0.69314718055994530942 / 32;
    double p = L * L * L * L * L / 120;
    p = fma(p, r, L * L * L * L / 24);
    p = fma(p, r, L * L * L / 6);
    p = fma(p, r, L * L / 2);
    p = fma(p, r, L);
    p = fma(p, r, 1.);
    return ldexp(lds.root[i & 31] * p, i >> 5);
  }

  __device__ __forceinline__ bool keeps(float x, int index) const { return x > cut.value || (x == cut.value && index <= cut.last); }

  __device__ __forceinline__ float distance(float x) const { return fminf((m - x) * scale, FLT_MAX); }

  // The sum over the team, in the same order every time.
  __device__ double team_sum(double v) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) lds.sum[wave] = v;
    __syncthreads();
    return wave_sum(lane < WAVES ? lds.sum[lane] : 0.);
  }

  __device__ void team_range(float& most, float& least) {
    most = wave_most(most);
    least = -wave_most(-least);
    __syncthreads();
    if (lane == 0) {
      lds.most[wave] = most;
      lds.least[wave] = least;
    }
    __syncthreads();
    most = wave_most(lane < WAVES ? lds.most[lane] : -INFINITY);
    least = -wave_most(lane < WAVES ? -lds.least[lane] : -INFINITY);
  }

  // The groups' sums stand in the lanes: the first group with which they pass `target`, or the last one of any weight; target becomes what is left of
  // it before that group.
  __device__ static int pick(double s, int groups, double& target) {
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

  // The index of the first logit with which the sum of of(logit, index) passes the target: u times the whole (FRACTION), or as given.
  template <bool FRACTION, class W>
  __device__ int locate(double target, W&& of, double& whole) {
    int j0 = 0, j1 = rounds, place = 0;
    auto of_vec = [&](const u32x4& x, int v) {
      const Slot<E> at = slot_of<E>(v, n);
      double s = 0.;
#pragma unroll
      for (int i = 0; i < VEC; ++i) s += of(E::get(x, i), at.base + i);
      return s;
    };
    bool first = FRACTION;
    for (;;) {
      const int length = j1 - j0, per = length <= 4 ? 1 : max(4, (length + kGroups - 1) / kGroups), groups = (length + per - 1) / per;
      __syncthreads();
      for (int g = 0; g < groups; ++g) {
        double s = 0.;
        each(j0 + g * per, min(j0 + (g + 1) * per, j1), [&](const u32x4& x, int v) { s += of_vec(x, v); });
        s = wave_sum(s);
        if (lane == 0) lds.part[g][wave] = s;
      }
      __syncthreads();
      double s = 0.;
      if (lane < groups)
        for (int w = 0; w < WAVES; ++w) s += lds.part[lane][w];
      if (first) {
        whole = wave_sum(s);
        target *= whole;
        first = false;
      }
      const int g = pick(s, groups, target);
      j0 += g * per;
      j1 = min(j0 + per, j1);
      if (per == 1) {
        place = pick(lane < WAVES ? lds.part[g][lane] : 0., WAVES, target);
        break;
      }
    }
    if (wave == place) {
      const u32x4 x = vec(j0);
      const int v = j0 * THREADS + tid;
      const double mine = of_vec(x, v), up_to = wave_scan(mine);
      const uint64_t some = __ballot(mine > 0.), passed = __ballot(mine > 0. && up_to > target);
      const int at_lane = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some | 1);
      if (lane == at_lane) {
        const Slot<E> at = slot_of<E>(v, n);
        double sum = up_to - mine;
        int index = at.base + VEC - 1;
        bool done = false;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const double w = of(E::get(x, i), at.base + i);
          sum += w;
          if (w > 0. && !done) {
            index = at.base + i;
            done = sum > target;
          }
        }
        lds.found = index;
      }
    }
    __syncthreads();
    return lds.found;
  }

  // The first `entries` of the list in descending order.
  __device__ void sort_list(int entries) {
    int size = 2;
    while (size < entries) size *= 2;
    for (int i = entries + tid; i < size; i += THREADS) lds.list[i] = 0;
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        __syncthreads();
        for (int i = tid; i < size / 2; i += THREADS) {
          const int a = 2 * i - (i & (j - 1)), b = a + j;
          const uint64_t x = lds.list[a], y = lds.list[b];
          if ((x < y) == ((a & k) == 0)) {
            lds.list[a] = y;
            lds.list[b] = x;
          }
        }
      }
    __syncthreads();
  }

  // The bin in which the counts (WEIGHT: the weights) pass the target, counted from `carry` on: its number, or -1; lds.before and lds.inside are
  // the count before it and its own.  carry goes on to the end of the bins.
  template <bool WEIGHT>
  __device__ int find_bin(uint64_t target, uint64_t& carry, int& count_carry, bool surely) {
    constexpr int PER = kBins / THREADS;
    __syncthreads();
    int counts[PER], count = 0;
    uint64_t values[PER], value = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      counts[i] = lds.count[tid * PER + i];
      values[i] = WEIGHT ? lds.weight[tid * PER + i] : (uint64_t)counts[i];
      count += counts[i];
      value += values[i];
    }
    const int count_to = wave_scan(count);
    const uint64_t value_to = wave_scan(value);
    if (lane == 63) {
      lds.number[wave] = count_to;
      lds.whole[wave] = value_to;
    }
    if (tid == 0) lds.found = INT_MAX;
    __syncthreads();
    int count_before = count_carry, count_all = count_carry;
    uint64_t before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) {
        count_before += lds.number[w];
        before += lds.whole[w];
      }
      count_all += lds.number[w];
      all += lds.whole[w];
    }
    count_before += count_to - count;
    before += value_to - value;
    int mine = INT_MAX, last = -1, mine_before = 0, mine_count = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      before += values[i];
      if (counts[i] > 0) {
        last = tid * PER + i;
        if (mine == INT_MAX && before >= target) {
          mine = last;
          mine_before = count_before;
          mine_count = counts[i];
        }
      }
      count_before += counts[i];
    }
    if (mine != INT_MAX) atomicMin(&lds.found, mine);
    __syncthreads();
    int found = lds.found;
    if (found == INT_MAX && surely) {  // (a rounding: the last bin that holds any)
      __syncthreads();
      if (tid == 0) lds.found = -1;
      __syncthreads();
      if (last >= 0) atomicMax(&lds.found, last);
      __syncthreads();
      found = lds.found;
      if (found == last && found >= 0) {
        mine = found;
        mine_count = lds.count[found];
        mine_before = count_before - mine_count;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (tid * PER + i > found) mine_before -= counts[i];
      }
    }
    if (mine == found && mine != INT_MAX) {
      lds.before = mine_before;
      lds.inside = mine_count;
    }
    __syncthreads();
    carry = all;
    count_carry = count_all;
    return found == INT_MAX ? -1 : found;
  }

  __device__ void clear_bins() {
    __syncthreads();
    for (int i = tid; i < kBins; i += THREADS) {
      lds.count[i] = 0;
      lds.weight[i] = 0;
    }
    if (tid == 0) lds.listed = 0;
    __syncthreads();
  }

  __device__ __forceinline__ uint64_t fixed(double w) const { return (uint64_t)ldexp(w, shift); }

  // Moves the cut to where the counts (WEIGHT: the weights) of what it keeps reach the target, in descending order.  least: the least finite logit.
  template <bool WEIGHT>
  __device__ void find_cut(double target, float least) {
    // the first histograms: by distance, near the maximum, then beyond
    const float end = distance(least);
    float from = 0.f, per = 0.f;
    uint64_t carry = 0;
    int count_carry = 0, bin = -1;
    for (int phase = 0; phase < 2 && bin < 0; ++phase) {
      const float to = phase == 0 ? fminf(kNear, end) : end;
      if (phase == 1 && end <= kNear) break;
      from = phase == 0 ? 0.f : kNear;
      per = to > from ? fminf(kBins / (to - from), FLT_MAX) : 0.f;
      clear_bins();
      each(0, rounds, [&](const u32x4& x, int v) {
        const Slot<E> at = slot_of<E>(v, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float logit = E::get(x, i), d = distance(logit);
          if (logit > -INFINITY && (phase == 0 ? d <= to : d > from) && keeps(logit, at.base + i)) {
            const int b = min((int)((d - from) * per), kBins - 1);
            atomicAdd(&lds.count[b], 1);
            if (WEIGHT) atomicAdd((unsigned long long*)&lds.weight[b], (unsigned long long)fixed(weight(logit)));
          }
        }
      });
      bin = find_bin<WEIGHT>(WEIGHT ? fixed(target) : (uint64_t)target, carry, count_carry, false);
    }
    if (bin < 0) return;  // all that there is
    bool by_key = false;
    uint32_t high = 0;  // by key: bins of (high - key) >> bits
    int bits = 0, above = lds.before, inside = lds.inside;
    const bool far = from > 0.f;
    uint32_t low = 0;
    while (bin >= 0) {
      // what the bin holds: in the list if it is few; their range; the weight above them
      __syncthreads();
      if (tid == 0) lds.listed = 0;
      __syncthreads();
      float most = -INFINITY, least_in = INFINITY;
      double sum = 0.;
      each(0, rounds, [&](const u32x4& x, int v) {
        const Slot<E> at = slot_of<E>(v, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float logit = E::get(x, i);
          if (!(logit > -INFINITY) || !keeps(logit, at.base + i)) continue;
          int side;  // below 0: above the bin
          if (by_key) {
            const uint32_t key = order_key(logit);
            side = key > high ? -1 : key < low ? 1 : (int)((high - key) >> bits) - bin;
          } else {
            const float d = distance(logit);
            const bool other = far ? d <= from : d > kNear;
            side = other ? (far ? -1 : 1) : min((int)((d - from) * per), kBins - 1) - bin;
          }
          if (WEIGHT && side < 0) sum += weight(logit);
          if (side == 0) {
            most = fmaxf(most, logit);
            least_in = fminf(least_in, logit);
            if (inside <= kList) {
              const uint32_t place = atomicAdd(&lds.listed, 1u);
              if (place < (uint32_t)kList) lds.list[place] = entry_of(logit, at.base + i);
            }
          }
        }
      });
      if (WEIGHT) sum = team_sum(sum);
      if (inside <= kList) {
        __syncthreads();
        sort_list(inside);
        int place = (int)target - above - 1;
        if (WEIGHT) place = list_place(inside, sum, target);
        place = max(0, min(place, inside - 1));
        const uint64_t entry = lds.list[place];
        cut.value = key_value((uint32_t)(entry >> 32));
        cut.last = (int)(0xFFFFFFFFu - (uint32_t)entry);
        return;
      }
      team_range(most, least_in);
      if (most == least_in) {  // equal ones: by their indices
        double order = target - above;
        if (WEIGHT) order = fmin(fmax(ceil((target - sum) / weight(most)), 1.), (double)inside);
        const Cut kept = cut;
        double whole;
        const int index = locate<false>(order - 0.5, [&](float x, int at) { return x == most && keeps(x, at) ? 1. : 0.; }, whole);
        cut.value = most;
        cut.last = most == kept.value ? min(index, kept.last) : index;
        return;
      }
      const uint32_t next_high = order_key(most), next_low = order_key(least_in);
      by_key = true;
      high = next_high;
      low = next_low;
      bits = max(0, 32 - __builtin_clz(high - low) - 10);
      clear_bins();
      each(0, rounds, [&](const u32x4& x, int v) {
        const Slot<E> at = slot_of<E>(v, n);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float logit = E::get(x, i);
          const uint32_t key = order_key(logit);
          if (key <= high && key >= low && keeps(logit, at.base + i)) {
            const int b = (int)((high - key) >> bits);
            atomicAdd(&lds.count[b], 1);
            if (WEIGHT) atomicAdd((unsigned long long*)&lds.weight[b], (unsigned long long)fixed(weight(logit)));
          }
        }
      });
      uint64_t none = 0;
      int count_above = above;
      if (!WEIGHT) none = (uint64_t)above;
      bin = find_bin<WEIGHT>(WEIGHT ? fixed(fmax(target - sum, 0.)) : (uint64_t)target, none, count_above, true);
      above = lds.before;
      inside = lds.inside;
    }
  }

  // The list's first place with which the weights reach the target, counted from `sum` on.
  __device__ int list_place(int entries, double sum, double target) {
    constexpr int PER = kList / THREADS;
    double w[PER], mine = 0.;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      w[i] = at < entries ? weight(key_value((uint32_t)(lds.list[at] >> 32))) : 0.;
      mine += w[i];
    }
    const double to = wave_scan(mine);
    if (tid == 0) lds.found = entries - 1;
    if (lane == 63) lds.sum[wave] = to;
    __syncthreads();
#pragma unroll
    for (int o = 0; o < WAVES; ++o)
      if (o < wave) sum += lds.sum[o];
    sum += to - mine;
    bool done = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      sum += w[i];
      if (!done && tid * PER + i < entries && sum >= target) {
        atomicMin(&lds.found, tid * PER + i);
        done = true;
      }
    }
    __syncthreads();
    return lds.found;
  }
};

// A row for a team of threads, which reads it once from memory and keeps its first HELD vectors a thread in shared memory.
template <int DTYPE, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void sm_row_kernel(SmArgs a) {
  typedef Elem<DTYPE> E;
  typedef Team<DTYPE, THREADS, HELD> Rows;
  __shared__ TeamLds<THREADS, HELD> lds;
  const int tid = threadIdx.x;
  if (tid < 32) lds.root[tid] = kRoots[tid];
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    Rows t = {lds};
    t.tid = tid;
    t.lane = tid & 63;
    t.wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    t.row = static_cast<const typename E::T*>(a.logits) + (int64_t)r * a.stride;
    t.n = a.vocab;
    t.nv = (a.vocab + E::VEC - 1) / E::VEC;
    t.rounds = (t.nv + THREADS - 1) / THREADS;
    t.shift = a.shift;
    const float scale = a.scale ? a.scale[r] : 1.f, u = a.u[r], p = a.top_p ? a.top_p[r] : 1.f, q = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;

    __syncthreads();  // the row before this one
    float most = -INFINITY, least = INFINITY;
    bool bad = !(scale >= 0x1p-60f && scale <= 0x1p60f) || !(u >= 0.f && u <= 1.f) || p != p || q != q;
    for (int j0 = 0; j0 < t.rounds; j0 += 4) {
      u32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int v = (j0 + i) * THREADS + tid;
        x[i] = v < t.nv ? row_vec<E>(t.row, v, t.n) : lowest_vec<E>();
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (j0 + i < HELD) lds.held[(j0 + i) * THREADS + tid] = x[i];
#pragma unroll
        for (int e = 0; e < E::VEC; ++e) {
          const float logit = E::get(x[i], e);
          bad |= !(logit < INFINITY);
          most = fmaxf(most, logit);
          least = logit > -INFINITY ? fminf(least, logit) : least;
        }
      }
    }
    if (bad) most = INFINITY;
    t.team_range(most, least);
    if (!(fabsf(most) < INFINITY)) {
      if (tid == 0) {
        a.token[r] = -1;
        if (a.logp) a.logp[r] = most < 0.f ? -INFINITY : NAN;
      }
      continue;
    }
    t.m = most;
    t.top = most;
    t.scale = scale;
    t.c32 = (double)scale * (32 * 1.44269504088896340736);
    t.q = fmin((double)q, 1.);
    t.cut = Cut{-INFINITY, INT_MAX};
    if (k > 0 && k < t.n) t.template find_cut<false>((double)k, least);
    if (p < 1.f) {
      double sum = 0.;
      t.each(0, t.rounds, [&](const u32x4& x, int v) {
        const Slot<E> at = slot_of<E>(v, t.n);
#pragma unroll
        for (int i = 0; i < E::VEC; ++i) {
          const float logit = E::get(x, i);
          if (t.keeps(logit, at.base + i)) sum += t.weight(logit);
        }
      });
      t.template find_cut<true>(fmax(t.team_sum(sum) * (double)p, 0.), least);
    }
    double whole;
    const int token = t.template locate<true>(
        (double)u,
        [&](float x, int at) {
          double w = 0.;
          if (t.keeps(x, at)) {
            w = t.weight(x);
            w = w >= t.q ? w : 0.;
          }
          return w;
        },
        whole);
    if (tid == 0) {
      a.token[r] = token;
      if (a.logp) a.logp[r] = (float)log(t.weight(E::to_float(t.row[token])) / whole);
    }
  }
}

template <int DTYPE>
int launch(const sm_desc* d, const SmArgs& a, hipStream_t stream) {
  const dim3 grid(std::min(a.rows, 1 << 20));
  if (d->large)
    hipLaunchKernelGGL((sm_row_kernel<DTYPE, 1024, 8>), grid, dim3(1024), 0, stream, a);
  else
    hipLaunchKernelGGL((sm_row_kernel<DTYPE, 256, 4>), grid, dim3(256), 0, stream, a);
  return (int)hipGetLastError();
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
  d->large = p.vocab > 256 * 4 * 16 / dtype_bytes(p.dtype);
  snprintf(d->names, sizeof(d->names), "sample=sm_row[%d]", d->large ? 1024 : 256);
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
  *bytes = 0;
  return CONV_OK;
}

const char* sm_desc_kernel_names(const sm_desc_t* d) { return d ? d->names : ""; }

int sm_sample(const sm_desc_t* d, const void* logits, int64_t stride, const float* u, const float* scale, const int32_t* top_k,
              const float* top_p, const float* min_p, int32_t* token, float* logp, void* ws, size_t ws_bytes, void* hip_stream) {
  (void)ws, (void)ws_bytes;
  if (!d) return CONV_EINVAL;
  if (d->p.rows == 0) return CONV_OK;
  if (!logits || !u || !token || (d->p.rows > 1 && stride < d->p.vocab)) return CONV_EINVAL;
  int bits = 0;
  while (((int64_t)1 << bits) < d->p.vocab) ++bits;
  const SmArgs a = {logits, stride, u, scale, top_p, min_p, top_k, token, logp, d->p.rows, d->p.vocab, 61 - bits};
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int e = d->p.dtype == MI355_F32   ? launch<MI355_F32>(d, a, stream)
                : d->p.dtype == MI355_F16 ? launch<MI355_F16>(d, a, stream)
                                          : launch<MI355_BF16>(d, a, stream);
  return e ? record_hip_error(e) : CONV_OK;
}

}  // extern "C"
