// Sampling for gfx950: a token drawn from a row of logits under temperature, top-k, top-p and min-p, from a given random
// number.
//
// The row's tokens are ranked by falling logit, equal ones by rising index (NaN: not there).  With M the largest logit and
// w_i = exp((l_i - M) / T), each filter keeps a prefix of the ranking: the K best; of those the ones in front of which less
// than top_p of their weight lies; of those the ones of at least min_p (the largest weight is 1).  A prefix is described by
// its last element (thr, last): a token is kept if l > thr, or l == thr and its index <= last.  The token is the first, by
// index, whose running kept weight exceeds u times the kept weight.
//
// Weights are doubles: in a vocabulary of 150000 tokens a float sum is off by more than many tokens weigh, and the token
// next to a border would hang on the order of the sum.  Where weights are summed by atomics they are integers (w * 2^62,
// in two halves), so that the order does not matter there either: a row's result has the same bits on every run.
#include "sf_internal.h"
#include <float.h>
#include <limits.h>

namespace sf {
namespace {

constexpr int BUCKETS = 1024;    // of one refinement of the ranking
constexpr int LIST = 2048;       // elements that are ranked by sorting
constexpr int STEP = 256;        // elements per partial sum of the draw: four to a lane of a wave
constexpr int MAX_STEPS = SAMPLE_MAX_VOCAB / STEP;
constexpr float INF = __builtin_huge_valf();

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows of an odd vocabulary start off 16 bytes

// settings of one row, cleaned: top-k off is INT_MAX, top-p off is 1 (or more), min-p off is 0
struct Settings {
  float t, p, m;
  int k;
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int row) {
  const int e = row / a.group;
  Settings s;
  s.t = a.temperature ? a.temperature[e] : 1.f;
  s.k = a.top_k ? a.top_k[e] : 0;
  s.p = a.top_p ? a.top_p[e] : 1.f;
  s.m = a.min_p ? a.min_p[e] : 0.f;
  if (s.k <= 0) s.k = INT_MAX;
  if (!(s.t > 0.f)) { s.t = 1.f; s.k = 1; }  // greedy
  s.t = fminf(s.t, FLT_MAX);                 // keeps 1 / t above zero: -inf times it stays -inf
  if (!(s.p < 1.f)) s.p = 1.f;
  if (!(s.m > 0.f)) s.m = 0.f;
  return s;
}

__device__ __forceinline__ double weight(float l, float top, double inv_t) {
  return l == top ? 1.0 : exp(((double)l - (double)top) * inv_t);
}

// what the running weight has to exceed, within [0, z) whatever u is (NaN: the upper border)
__device__ __forceinline__ double target_of(float u, double z) {
  const double t = (double)u * z;
  return t < 0.0 ? 0.0 : fmin(t, z * (1.0 - 0x1p-53));
}

// ---- over a workgroup ----------------------------------------------------------------------------
template <int BS, class T, class F> __device__ __forceinline__ T block_reduce(T v, T *red, F f) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = red[0];
#pragma unroll
  for (int w = 1; w < BS / 64; ++w) r = f(r, red[w]);
  __syncthreads();
  return r;
}

// sum of v over the threads before this one; total: over all
template <int BS, class T> __device__ __forceinline__ T block_before(T v, T *red, T &total) {
  T x = v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) red[wave] = x;
  T incl = __shfl_up(x, 1);
  if (lane == 0) incl = 0;
  __syncthreads();
  T base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < BS / 64; ++w) {
    if (w == wave) base = all;
    all += red[w];
  }
  __syncthreads();
  total = all;
  return base + incl;
}

// key of the ranking: rises with the logit, among equal ones with falling index
__device__ __forceinline__ uint64_t rank_key(float l, int i) {
  uint32_t b = __float_as_uint(l + 0.f);  // -0 ranks as 0
  b = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)b << 32 | (uint32_t)(INT_MAX - i);
}
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t b = (uint32_t)(k >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int key_index(uint64_t k) { return INT_MAX - (int)(uint32_t)k; }

// the elements that a selection looks at, by rising index
struct Source {
  const float *l;
  const int32_t *idx;  // null: an element's place
  int n;
};

struct Shared {
  union {
    struct {
      uint32_t cnt[BUCKETS];
      uint64_t lo[BUCKETS], hi[BUCKETS];  // weight * 2^62, its lower 32 bits and the rest
    } h;
    double step[MAX_STEPS];
  };
  uint64_t list[LIST];
  double redd[16];
  int redi[16];
  uint32_t redu[16];
  int n_list;
  int at, found;
  double before, sum;
  int count;
};

template <int BS, class F> __device__ __forceinline__ void for_each(const Source &s, F f) {
  for (int i0 = threadIdx.x * 4; i0 < s.n; i0 += BS * 4) {
    if (i0 + 4 <= s.n) {
      const f32x4u v = *reinterpret_cast<const f32x4u *>(s.l + i0);
#pragma unroll
      for (int e = 0; e < 4; ++e) f(v[e], i0 + e);
    } else {
      for (int i = i0; i < s.n; ++i) f(s.l[i], i);
    }
  }
}

__device__ __forceinline__ double from_fixed(uint64_t lo, uint64_t hi) { return (double)hi * 0x1p-30 + (double)lo * 0x1p-62; }

// sorts sh.list[0, LIST) by falling key
template <int BS> __device__ void sort_list(Shared &sh, int n) {
  int m = 2;
  while (m < n) m <<= 1;
  for (int i = n + threadIdx.x; i < m; i += BS) sh.list[i] = 0;
  __syncthreads();
  for (int size = 2; size <= m; size <<= 1)
    for (int d = size >> 1; d; d >>= 1) {
      for (int x = threadIdx.x; x < m / 2; x += BS) {
        const int i = (x & (d - 1)) + 2 * (x & ~(d - 1)), j = i + d;
        const uint64_t a = sh.list[i], b = sh.list[j];
        if ((a < b) == ((i & size) == 0)) { sh.list[i] = b; sh.list[j] = a; }
      }
      __syncthreads();
    }
}

// The j-th (from 0) element by index among those equal to v.
template <int BS> __device__ int nth_equal(Shared &sh, const Source &s, float v, int j) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) sh.found = -1;
  __syncthreads();
  // waves own consecutive stretches; the one that holds the j-th walks it again
  const int per = (s.n + BS / 64 - 1) / (BS / 64), lo = min(s.n, wave * per), hi = min(s.n, lo + per);
  int c = 0;
  for (int i = lo + lane; i < hi; i += 64) c += s.l[i] == v;
#pragma unroll
  for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
  if (lane == 0) sh.redi[wave] = c;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += sh.redi[w];
  if (before <= j && j < before + c)
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const bool eq = i0 + lane < hi && s.l[min(i0 + lane, hi - 1)] == v;
      const uint64_t m = __ballot(eq);
      const int here = __popcll(m & ((1ull << lane) - 1));
      if (eq && before + here == j) sh.found = s.idx ? s.idx[i0 + lane] : i0 + lane;
      before += __popcll(m);
    }
  __syncthreads();
  const int r = sh.found;
  __syncthreads();
  return r;
}

// Cuts the ranking of the elements that are kept so far (l > thr or l == thr and index <= last): by_mass, behind the last
// element in front of which less than `target` of weight lies; else behind the k best.  thr and last receive the last kept
// element; returns the kept weight.  lo_hint: nothing of interest is expected below.
//
// A refinement sorts the elements of an interval of logits into buckets by a linear map (it never puts a smaller logit in
// front of a larger one), finds the bucket of the cut from the running counts and weights, and goes on with that bucket's
// interval, until it has few elements, which are sorted, or equal ones, which are counted.
template <int BS>
__device__ double cut(Shared &sh, const Source &s, bool by_mass, int k, double share, float top, double inv_t, float lo_hint,
                      float &thr, int &last) {
  constexpr int PER = BUCKETS / BS > 0 ? BUCKETS / BS : 1;
  const int tid = threadIdx.x;
  const float thr0 = thr;
  const int last0 = last;
  auto kept = [&](float l, int i) { return l > thr0 || (l == thr0 && (s.idx ? s.idx[i] : i) <= last0); };
  float lo = fmaxf(lo_hint, thr0), hi = top;  // the interval; what lies above is kept whole
  bool below = true;                          // elements below lo belong to the last bucket
  double mass0 = 0.0, target = share;         // weight above the interval
  int count0 = 0;
  bool first = true;
  for (;;) {
    const double scale = hi > lo ? (BUCKETS - 2) / ((double)hi - (double)lo) : 0.0;
    auto bucket = [&](float l) {
      if (l == hi) return 0;
      if (l < lo || hi == INF) return BUCKETS - 1;
      return min(BUCKETS - 2, (int)(((double)hi - (double)l) * scale));
    };
    auto inside = [&](float l, int i) { return l <= hi && (below || l >= lo) && kept(l, i); };
    for (int x = tid; x < BUCKETS; x += BS) { sh.h.cnt[x] = 0; sh.h.lo[x] = 0; sh.h.hi[x] = 0; }
    __syncthreads();
    for_each<BS>(s, [&](float l, int i) {
      if (!inside(l, i)) return;
      const int b = bucket(l);
      atomicAdd(&sh.h.cnt[b], 1u);
      const uint64_t fx = (uint64_t)(weight(l, top, inv_t) * 0x1p62);
      atomicAdd((unsigned long long *)&sh.h.lo[b], (unsigned long long)(fx & 0xffffffffu));
      atomicAdd((unsigned long long *)&sh.h.hi[b], (unsigned long long)(fx >> 32));
    });
    __syncthreads();
    // running counts and weights; each thread has PER consecutive buckets
    int c[PER], cs = 0;
    double w[PER], ws = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int b = tid * PER + e;
      c[e] = b < BUCKETS ? (int)sh.h.cnt[b] : 0;
      w[e] = b < BUCKETS ? from_fixed(sh.h.lo[b], sh.h.hi[b]) : 0.0;
      cs += c[e]; ws += w[e];
    }
    int ctot;
    double wtot;
    int cb = count0 + block_before<BS>(cs, sh.redi, ctot);
    double wb = mass0 + block_before<BS>(ws, sh.redd, wtot);
    if (first && by_mass) target = share * wtot;  // share of the kept weight
    first = false;
    if (tid == 0) sh.at = -1;
    __syncthreads();
    // the last bucket that the cut reaches into: its first element is kept
    int mine = -1;
    double mine_w = 0.0;
    int mine_c = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const bool in = by_mass ? wb < target || cb == 0 : cb < k;
      if (c[e] > 0 && in) { mine = tid * PER + e; mine_w = wb; mine_c = cb; }
      cb += c[e]; wb += w[e];
    }
    const int at = block_reduce<BS>(mine, sh.redi, [](int a, int b) { return max(a, b); });
    if (at < 0) { thr = thr0; last = last0; return 0.0; }  // nothing there
    if (mine == at) { sh.before = mine_w; sh.count = mine_c; }
    if (tid == 0) sh.n_list = 0;
    const int n_at = (int)sh.h.cnt[at];
    __syncthreads();
    mass0 = sh.before; count0 = sh.count;
    if (n_at <= LIST) {
      for_each<BS>(s, [&](float l, int i) {
        if (inside(l, i) && bucket(l) == at) sh.list[atomicAdd(&sh.n_list, 1)] = rank_key(l, s.idx ? s.idx[i] : i);
      });
      __syncthreads();
      sort_list<BS>(sh, n_at);
      // running weight of the sorted elements
      constexpr int EACH = LIST / BS;
      double x[EACH], xs = 0.0, xt;
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int i = tid * EACH + e;
        x[e] = i < n_at ? weight(key_logit(sh.list[i]), top, inv_t) : 0.0;
        xs += x[e];
      }
      double run = mass0 + block_before<BS>(xs, sh.redd, xt);
      int keep = -1;
      double sum = 0.0;
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int i = tid * EACH + e;
        const bool in = by_mass ? run < target || count0 + i == 0 : count0 + i < k;
        run += x[e];
        if (i < n_at && in) { keep = i; sum = run; }
      }
      const int end = block_reduce<BS>(keep, sh.redi, [](int a, int b) { return max(a, b); });
      if (keep == end && end >= 0) sh.sum = sum;
      __syncthreads();
      thr = key_logit(sh.list[end]);
      last = key_index(sh.list[end]);
      const double r = sh.sum;
      __syncthreads();
      return r;
    }
    // too many: the bucket's own interval
    float mn = INF, mx = -INF;
    for_each<BS>(s, [&](float l, int i) {
      if (inside(l, i) && bucket(l) == at) { mn = fminf(mn, l); mx = fmaxf(mx, l); }
    });
    mn = block_reduce<BS>(mn, (float *)sh.redu, [](float a, float b) { return fminf(a, b); });
    mx = block_reduce<BS>(mx, (float *)sh.redu, [](float a, float b) { return fmaxf(a, b); });
    if (mn == mx) {
      const double w1 = weight(mn, top, inv_t);
      int j = n_at;
      if (!by_mass) j = min(n_at, k - count0);
      else if (w1 > 0.0) j = (int)fmin((double)n_at, fmax(1.0, ceil((target - mass0) / w1)));
      thr = mn;
      last = j == n_at && mn > thr0 ? INT_MAX : nth_equal<BS>(sh, s, mn, j - 1);
      return mass0 + w1 * j;
    }
    // -inf apart from the rest: elements below lo
    below = mn == -INF;
    if (below) {
      mn = INF;
      for_each<BS>(s, [&](float l, int i) {
        if (inside(l, i) && bucket(l) == at && l > -INF) mn = fminf(mn, l);
      });
      mn = block_reduce<BS>(mn, (float *)sh.redu, [](float a, float b) { return fminf(a, b); });
    }
    lo = mn; hi = mx;
  }
}

template <int BS>
__global__ __launch_bounds__(BS) void sample_row_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  const float *x = a.logits + (size_t)row * a.V;
  const Settings st = settings_of(a, row);
  const Source src{x, nullptr, a.V};
  // largest, lowest index
  float best = -INF, low = INF;
  int at = INT_MAX;
  for_each<BS>(src, [&](float l, int i) {
    if (l > best || (l == best && i < at)) { best = l; at = i; }
    if (l > -INF) low = fminf(low, l);
  });
  const float top = block_reduce<BS>(best, (float *)sh.redu, [](float p, float q) { return fmaxf(p, q); });
  const int arg = block_reduce<BS>(best == top ? at : INT_MAX, sh.redi, [](int p, int q) { return min(p, q); });
  low = block_reduce<BS>(low, (float *)sh.redu, [](float p, float q) { return fminf(p, q); });
  const double inv_t = 1.0 / (double)st.t;
  SampleDist d{top, top, arg == INT_MAX ? -1 : arg, st.t, 1.0, arg == INT_MAX ? 0 : arg, arg == INT_MAX ? 0.f : 1.f};
  if (d.last < 0) d.z = 0.0;
  const bool one = arg == INT_MAX || st.k == 1 || top == -INF || st.m > 1.f;
  if (!one) {
    float thr = -INF;
    int last = INT_MAX;
    const float hint = fmaxf(low, top - fminf(40.f * st.t, FLT_MAX));
    if (st.k < a.V) (void)cut<BS>(sh, src, false, st.k, 0.0, top, inv_t, hint, thr, last);
    if (st.p < 1.f) (void)cut<BS>(sh, src, true, 0, (double)st.p, top, inv_t, hint, thr, last);
    if (st.m > 0.f) {
      float mn = top;
      for_each<BS>(src, [&](float l, int i) {
        if (l > thr && l < mn && weight(l, top, inv_t) >= (double)st.m) mn = l;
      });
      mn = block_reduce<BS>(mn, (float *)sh.redu, [](float p, float q) { return fminf(p, q); });
      if (weight(thr, top, inv_t) < (double)st.m) { thr = mn; last = INT_MAX; }
    }
    // the draw: kept weight of every step, the step that the target falls into, the token in it
    const int lane = tid & 63, wave = tid >> 6, n_steps = (a.V + STEP - 1) / STEP;
    auto step_weights = [&](int s, double (&w)[4]) {
      const int i0 = s * STEP + lane * 4;
      double sum = 0.0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + e;
        const float l = i < a.V ? x[i] : -INF;
        w[e] = i < a.V && (l > thr || (l == thr && i <= last)) ? weight(l, top, inv_t) : 0.0;
        sum += w[e];
      }
      return sum;
    };
    double w[4];
    for (int s = wave; s < n_steps; s += BS / 64) {
      double sum = step_weights(s, w);
#pragma unroll
      for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
      if (lane == 0) sh.step[s] = sum;
    }
    __syncthreads();
    const int per = (n_steps + BS - 1) / BS, s0 = min(n_steps, tid * per), s1 = min(n_steps, s0 + per);
    double own = 0.0, z;
    for (int s = s0; s < s1; ++s) own += sh.step[s];
    double run = block_before<BS>(own, sh.redd, z);
    const double target = a.u ? target_of(a.u[row], z) : 0.0;
    int mine = -1;
    double before = 0.0;
    for (int s = s0; s < s1; ++s) {
      if (sh.step[s] > 0.0 && run <= target) { mine = s; before = run; }
      run += sh.step[s];
    }
    const int hit = block_reduce<BS>(mine, sh.redi, [](int p, int q) { return max(p, q); });
    if (mine == hit && hit >= 0) sh.before = before;
    __syncthreads();
    d.thr = thr; d.last = last; d.z = z;
    if (a.ids && wave == 0 && hit >= 0) {
      double own_w = step_weights(hit, w), incl = own_w;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      double r = sh.before + (incl - own_w);
      int id = -1, any = -1;
      double wid = 0.0, wany = 0.0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        r += w[e];
        if (w[e] > 0.0) { any = hit * STEP + lane * 4 + e; wany = w[e]; }
        if (id < 0 && w[e] > 0.0 && r > target) { id = any; wid = w[e]; }
      }
      // the first lane that passes the target; where rounding lets none, the last token of weight
      const uint64_t over = __ballot(id >= 0), some = __ballot(any >= 0);
      const int lane_at = over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll(some);
      d.id = __shfl(over ? id : any, lane_at);
      d.prob = (float)(__shfl(over ? wid : wany, lane_at) / z);
    }
  }
  if (tid == 0) {
    if (a.ids) a.ids[row] = d.id;
    if (a.prob) a.prob[row] = d.prob;
    if (a.dist) a.dist[row] = d;
  }
}

// ---- acceptance --------------------------------------------------------------------------------
__device__ __forceinline__ bool kept_by(const SampleDist &d, float l, int i) {
  return l > d.thr || (l == d.thr && i <= d.last);
}
__device__ __forceinline__ double share_of(const SampleDist &d, double inv_t, double inv_z, float l, int i) {
  return kept_by(d, l, i) ? weight(l, d.top, inv_t) * inv_z : 0.0;
}

// What is left of the target's distribution at the block row behind the last accepted slot.
struct Rest {
  const float *p, *q;  // rows of logits; q null: no draft distribution there
  SampleDist pd, qd;
  double p_t, p_z, q_t, q_z;
  int dead;            // token that a draft without logits is certain of (-1: none)
  __device__ __forceinline__ double at(int i) const {
    const double pi = share_of(pd, p_t, p_z, p[i], i);
    if (q) return fmax(pi - share_of(qd, q_t, q_z, q[i], i), 0.0);
    return i == dead ? 0.0 : pi;
  }
};
__device__ __forceinline__ double inv_of(double z) { return z > 0.0 ? 1.0 / z : 0.0; }

// Accepted slots of sequence b: slot i stays if all before it do and u * q(d) < p(d).  Every thread returns the number.
__device__ int accepted(const SampleAcceptArgs &a, int b, int *red) {
  const int q = a.k + 1;
  int fail = a.k;
  if (threadIdx.x < a.k) {
    const int i = threadIdx.x, d = a.draft[(size_t)b * a.k + i];
    bool stays = false;
    if (d >= 0 && d < a.V) {
      const SampleDist pd = a.dist[(size_t)b * q + i];
      const double p = share_of(pd, 1.0 / (double)pd.temp, inv_of(pd.z), a.target[((size_t)b * q + i) * a.V + d], d);
      double qd = 1.0;
      if (a.draft_logits) {
        const SampleDist dd = a.draft_dist[(size_t)b * a.k + i];
        qd = share_of(dd, 1.0 / (double)dd.temp, inv_of(dd.z), a.draft_logits[((size_t)b * a.k + i) * a.V + d], d);
      }
      stays = (double)a.u_accept[(size_t)b * a.k + i] * qd < p;
    }
    if (!stays) fail = i;
  }
  return block_reduce<256>(fail, red, [](int x, int y) { return min(x, y); });
}

__device__ Rest rest_of(const SampleAcceptArgs &a, int b, int n) {
  const size_t row = (size_t)b * (a.k + 1) + n, slot = (size_t)b * a.k + n;
  Rest r;
  r.p = a.target + row * a.V;
  r.pd = a.dist[row];
  r.p_t = 1.0 / (double)r.pd.temp; r.p_z = inv_of(r.pd.z);
  r.q = nullptr; r.q_t = r.q_z = 0.0; r.dead = -1;
  if (n < a.k && a.draft_logits) {
    r.q = a.draft_logits + slot * a.V;
    r.qd = a.draft_dist[slot];
    r.q_t = 1.0 / (double)r.qd.temp; r.q_z = inv_of(r.qd.z);
  } else if (n < a.k) {
    r.dead = a.draft[slot];
  }
  return r;
}

// One workgroup per (sequence, segment of the vocabulary): the segment's rest.
__global__ __launch_bounds__(256) void rest_sum_kernel(const SampleAcceptArgs a, int segs) {
  __shared__ int redi[4];
  __shared__ double redd[4];
  const int b = blockIdx.x / segs, seg = blockIdx.x % segs;
  const Rest r = rest_of(a, b, accepted(a, b, redi));
  double sum = 0.0;
  for (int i = seg * SAMPLE_SEG + threadIdx.x; i < min(a.V, (seg + 1) * SAMPLE_SEG); i += 256) sum += r.at(i);
  sum = block_reduce<256>(sum, redd, [](double x, double y) { return x + y; });
  if (threadIdx.x == 0) a.part[(size_t)b * segs + seg] = sum;
}

// One workgroup per sequence: the token behind the accepted slots.
__global__ __launch_bounds__(256) void rest_draw_kernel(const SampleAcceptArgs a, int segs) {
  __shared__ int redi[4];
  __shared__ double redd[4], step[SAMPLE_SEG / 64], found;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = accepted(a, b, redi);
  Rest r = rest_of(a, b, n);
  double *part = a.part + (size_t)b * segs;
  double own = tid < segs ? part[tid] : 0.0, z, before = block_before<256>(own, redd, z);
  if (!(z > 0.0)) {
    // nothing is left (target and draft agree, and the drafted token has no share in either): the target's own
    r.q = nullptr; r.dead = -1;
    for (int s = 0; s < segs; ++s) {
      double sum = 0.0;
      for (int i = s * SAMPLE_SEG + tid; i < min(a.V, (s + 1) * SAMPLE_SEG); i += 256) sum += r.at(i);
      sum = block_reduce<256>(sum, redd, [](double x, double y) { return x + y; });
      if (tid == s) own = sum;
    }
    before = block_before<256>(own, redd, z);
  }
  const double target = target_of(a.u_sample[b], z);
  const int seg = block_reduce<256>(own > 0.0 && before <= target ? tid : -1, redi, [](int x, int y) { return max(x, y); });
  int id = max(r.pd.id, 0);
  if (seg >= 0) {
    if (tid == seg) found = before;
    const int i0 = seg * SAMPLE_SEG, i1 = min(a.V, i0 + SAMPLE_SEG), steps = (i1 - i0 + 63) / 64;
    for (int s = wave; s < steps; s += 4) {
      const int i = i0 + s * 64 + lane;
      double v = i < i1 ? r.at(i) : 0.0;
#pragma unroll
      for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
      if (lane == 0) step[s] = v;
    }
    __syncthreads();
    const double x = tid < steps ? step[tid] : 0.0;
    double tot;
    const double run = found + block_before<256>(x, redd, tot);
    const int hit = block_reduce<256>(x > 0.0 && run <= target ? tid : -1, redi, [](int p, int q) { return max(p, q); });
    // rounding may put the segment's first token behind the target
    const int s = hit >= 0 ? hit : block_reduce<256>(x > 0.0 ? tid : INT_MAX, redi, [](int p, int q) { return min(p, q); });
    if (tid == s) found = run;
    __syncthreads();
    if (wave == 0 && s < steps) {
      const int i = i0 + s * 64 + lane;
      const double v = i < i1 ? r.at(i) : 0.0;
      double incl = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      const uint64_t some = __ballot(v > 0.0), over = __ballot(v > 0.0 && found + incl > target);
      if (some) id = i0 + s * 64 + (over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll(some));
    }
  }
  if (tid <= n) a.tokens[(size_t)b * (a.k + 1) + tid] = tid < n ? a.draft[(size_t)b * a.k + tid] : -1;
  __syncthreads();
  if (tid == 0) {
    a.tokens[(size_t)b * (a.k + 1) + n] = id;
    a.accept[b] = n + 1;
  }
}

}  // namespace

hipError_t launch_sample_accept(const SampleAcceptArgs &a, hipStream_t s) {
  const int segs = (a.V + SAMPLE_SEG - 1) / SAMPLE_SEG;
  rest_sum_kernel<<<a.B * segs, 256, 0, s>>>(a, segs);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  rest_draw_kernel<<<a.B, 256, 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t launch_sample(const SampleArgs &a, hipStream_t s) {
  sample_row_kernel<1024><<<a.M, 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sf
