// Sampling for gfx950: a token drawn from a row of logits under temperature, top-k, top-p and min-p, from a given random
// number.
//
// The row's tokens are ranked by falling logit, equal ones by rising index (NaN: not there).  With M the largest logit and
// w_i = exp((l_i - M) / T), each filter keeps a prefix of the ranking: the K best; of those the ones in front of which less
// than top_p of their weight lies; of those the ones of at least min_p (the largest weight is 1).  A prefix is described by
// its last element (thr, last): a token is kept if l > thr, or l == thr and its index <= last.  The token is the first, by
// index, whose running kept weight exceeds u times the kept weight.
//
// Two launches, so that the logits leave memory once.  segment_kernel holds 8192 tokens of a row in the registers of a
// workgroup and leaves what the row needs of them: the largest, the sum of weights, a histogram of weights (nucleus), the
// tokens that may lie in the kept prefix.  row_kernel joins the segments, finds the prefix, finds the segment that u falls
// into by the segments' kept weights, and reads that one again for the token.  What a segment had no room for (a flat row's
// nucleus of tens of thousands) is read from the logits again, for that row alone.
//
// Weights are doubles: in a vocabulary of 150000 tokens a float sum is off by more than many tokens weigh, and the token
// next to a border would hang on the order of the sum.  Where weights are summed by atomics they are integers (multiples of
// 2^-62 in two halves, or of 2^-36 of a bucket's edge), so that the order does not matter there either: a row's result has the
// same bits on every run.
#include "sf_internal.h"
#include <float.h>
#include <limits.h>

namespace sf {
namespace {

constexpr int BUCKETS = 1024;    // of one refinement of the ranking
constexpr int LIST = 2048;       // elements that are ranked by sorting
constexpr int STEP = 256;        // elements per partial sum of the draw: four to a lane of a wave
constexpr int SEG = SAMPLE_SEG, MAX_SEGS = SAMPLE_MAX_VOCAB / SEG;
constexpr int BINS = SAMPLE_BINS, ROOM = SAMPLE_ROOM;
constexpr float INF = __builtin_huge_valf();

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows of an odd vocabulary start off 16 bytes

// Settings of one row, cleaned: top-k off is INT_MAX, top-p off is 1, min-p off is 0; and what they ask of a row.
enum { ONE, ALL, NUCLEUS, FEW };  // the first alone; all; top-p of all; a count or a least weight limits the prefix
struct Settings {
  float t, p, m;
  int k, kind;
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int row) {
  const int e = row / a.group;
  Settings s;
  s.t = a.temperature ? a.temperature[e] : 1.f;
  s.k = a.top_k ? a.top_k[e] : 0;
  s.p = a.top_p ? a.top_p[e] : 1.f;
  s.m = a.min_p ? a.min_p[e] : 0.f;
  if (s.k <= 0 || s.k >= a.V) s.k = INT_MAX;
  if (a.V == 1 || !(s.t > 0.f)) { s.t = 1.f; s.k = 1; }  // greedy
  s.t = fminf(s.t, FLT_MAX);                 // keeps 1 / t above zero: -inf times it stays -inf
  if (!(s.p < 1.f)) s.p = 1.f;
  if (!(s.m > 0.f)) s.m = 0.f;
  s.kind = s.k == 1 || s.m > 1.f ? ONE : s.k != INT_MAX ? FEW : s.p < 1.f ? NUCLEUS : s.m > 0.f ? FEW : ALL;
  return s;
}

// 2^y for y <= 0 (or a little above), to about 2^-50: the power series of 2^f, |f| <= 1/2, to the twelfth term.  The device
// library's exp takes twice as many instructions, and double precision is a third of what these kernels do.
__device__ __forceinline__ double power_of_two(double y) {
  y = fmax(y, -1200.0);  // 0 from there on, for -inf too
  const double n = rint(y), f = y - n;
  double p = 2.5678435993488196e-11;
  p = fma(p, f, 4.4455382718708101e-10);
  p = fma(p, f, 7.0549116208011209e-09);
  p = fma(p, f, 1.0178086009239696e-07);
  p = fma(p, f, 1.3215486790144305e-06);
  p = fma(p, f, 1.5252733804059838e-05);
  p = fma(p, f, 1.5403530393381606e-04);
  p = fma(p, f, 1.3333558146428441e-03);
  p = fma(p, f, 9.6181291076284769e-03);
  p = fma(p, f, 5.5504108664821576e-02);
  p = fma(p, f, 2.4022650695910069e-01);
  p = fma(p, f, 6.9314718055994529e-01);
  p = fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n);
}

constexpr double LOG2E = 1.4426950408889634;

// scale: log2(e) / T
__device__ __forceinline__ double weight(float l, float top, double scale) {
  return l == top ? 1.0 : power_of_two(((double)l - (double)top) * scale);
}

// The grid of a row's buckets: bucket b holds the logits of [b, b + 1) / g.  Nucleus: eight to a factor of e in weight.
// Counts: as wide at T >= 1/2, not narrower below, so that the tokens of a count are within reach at any temperature.
__device__ __forceinline__ double grid_of(const Settings &s) { return 8.0 / (double)(s.kind == NUCLEUS ? s.t : fmaxf(s.t, 0.5f)); }
constexpr double GRID_END = 1 << 20;  // beyond, a place on the grid is too coarse for the weights: the row goes without it
__device__ __forceinline__ int bucket_of(float l, double g) {
  return (int)floor(fmin(fmax((double)l * g, -2.0 * GRID_END), 2.0 * GRID_END));
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
  struct {
    uint32_t cnt[BUCKETS];
    uint64_t lo[BUCKETS], hi[BUCKETS];  // weight * 2^62, its lower 32 bits and the rest
  } h;
  uint64_t list[LIST];
  double seg[MAX_SEGS], step[SEG / STEP];  // kept weight of the segments, of a segment's steps
  uint64_t seg_lo[MAX_SEGS], seg_hi[MAX_SEGS];
  int32_t seg_n[MAX_SEGS], seg_at[MAX_SEGS];
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
// element in front of which less than `target` of weight lies (share >= 0: that share of the weight of these and `rest`, what
// else there is); else behind the k best.  mass0: weight of elements that rank in front of all of these and are not among them.  thr and last receive the last
// kept element; returns the kept weight.  lo_hint: nothing of interest is expected below; hi: nothing lies above.
//
// A refinement sorts the elements of an interval of logits into buckets by a linear map (it never puts a smaller logit in
// front of a larger one), finds the bucket of the cut from the running counts and weights, and goes on with that bucket's
// interval, until it has few elements, which are sorted, or equal ones, which are counted.
template <int BS>
__device__ double cut(Shared &sh, const Source &s, bool by_mass, int k, double share, double target, double mass0, double rest,
                      float top, double scale, float lo_hint, float hi, float &thr, int &last) {
  constexpr int PER = BUCKETS / BS > 0 ? BUCKETS / BS : 1;
  const int tid = threadIdx.x;
  const float thr0 = thr;
  const int last0 = last;
  auto kept = [&](float l, int i) { return l > thr0 || (l == thr0 && (s.idx ? s.idx[i] : i) <= last0); };
  float lo = fmaxf(lo_hint, thr0);            // the interval [lo, hi]; what lies above is kept whole
  bool below = true;                          // elements below lo belong to the last bucket
  int count0 = mass0 > 0.0 ? 1 : 0;           // by weight only whether there is one in front matters
  bool whole = s.n <= LIST;                   // few elements: sorted as they are
  for (;;) {
    const double places = hi > lo ? (BUCKETS - 2) / ((double)hi - (double)lo) : 0.0;
    auto bucket = [&](float l) {
      if (whole || l == hi) return 0;
      if (l < lo || hi == INF) return BUCKETS - 1;
      return min(BUCKETS - 2, (int)(((double)hi - (double)l) * places));
    };
    auto inside = [&](float l, int i) { return l <= hi && (below || l >= lo) && kept(l, i); };
    int at = 0, n_at = s.n;
    if (!whole) {
      for (int x = tid; x < BUCKETS; x += BS) { sh.h.cnt[x] = 0; sh.h.lo[x] = 0; sh.h.hi[x] = 0; }
      __syncthreads();
      for_each<BS>(s, [&](float l, int i) {
        if (!inside(l, i)) return;
        const int b = bucket(l);
        atomicAdd(&sh.h.cnt[b], 1u);
        const uint64_t fx = (uint64_t)(weight(l, top, scale) * 0x1p62);
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
      if (share >= 0.0) target = share * (rest + wtot);
      share = -1.0;
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
      at = block_reduce<BS>(mine, sh.redi, [](int a, int b) { return max(a, b); });
      if (at < 0) { thr = thr0; last = last0; return mass0; }  // nothing there
      if (mine == at) { sh.before = mine_w; sh.count = mine_c; }
      n_at = (int)sh.h.cnt[at];
      __syncthreads();
      mass0 = sh.before; count0 = sh.count;
    }
    if (n_at <= LIST) {
      if (tid == 0) sh.n_list = 0;
      __syncthreads();
      for_each<BS>(s, [&](float l, int i) {
        if (inside(l, i) && bucket(l) == at) sh.list[atomicAdd(&sh.n_list, 1)] = rank_key(l, s.idx ? s.idx[i] : i);
      });
      __syncthreads();
      n_at = sh.n_list;
      if (n_at == 0) { thr = thr0; last = last0; return mass0; }
      sort_list<BS>(sh, n_at);
      // running weight of the sorted elements
      constexpr int EACH = LIST / BS;
      double x[EACH], xs = 0.0, xt;
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const int i = tid * EACH + e;
        x[e] = i < n_at ? weight(key_logit(sh.list[i]), top, scale) : 0.0;
        xs += x[e];
      }
      double run = mass0 + block_before<BS>(xs, sh.redd, xt);
      if (share >= 0.0) target = share * (rest + xt);
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
      double r = mass0;
      if (end >= 0) {
        thr = key_logit(sh.list[end]);
        last = key_index(sh.list[end]);
        r = sh.sum;
      }
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
      const double w1 = weight(mn, top, scale);
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

// The smallest float whose weight reaches m in (0, 1].
__device__ float least_of(float m, float top, double scale) {
  auto order = [](float l) { const uint32_t b = __float_as_uint(l); return b & 0x80000000u ? ~b : b | 0x80000000u; };
  auto value = [](uint32_t b) { return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b); };
  uint32_t lo = order(-INF), hi = order(top);  // the weight of lo is below m, that of hi is not
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (weight(value(mid), top, scale) >= (double)m) hi = mid; else lo = mid;
  }
  return value(hi);
}

// Appends the elements (l, i) of a tile that are wanted to the row's list, by rising index: every thread passes its N
// consecutive ones.  count: entries so far (the same in all threads); beyond `room` nothing is written.
template <int BS, int N>
__device__ __forceinline__ void append(Shared &sh, const float (&l)[N], const int (&i)[N], const bool (&want)[N], float *to_l,
                                       int32_t *to_i, int room, int &count) {
  int own = 0, all;
#pragma unroll
  for (int e = 0; e < N; ++e) own += want[e];
  int at = count + block_before<BS>(own, sh.redi, all);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (want[e]) {
      if (at < room) { to_l[at] = l[e]; to_i[at] = i[e]; }
      ++at;
    }
  count += all;
}

struct SegStat {
  float top;
  int32_t arg;    // lowest index of the largest; INT_MAX: no comparable value
  int32_t bucket; // of the largest on the row's grid: the histogram's first
  int32_t cut;    // the list holds all of the segment's elements from this bucket on; INT_MAX: not even the first
  int32_t n;      // entries of the list
  int32_t off;    // the grid does not reach the values
  double z;       // ALL: sum of weights against the segment's largest
};
static_assert(sizeof(SegStat) == SAMPLE_STAT_BYTES, "workspace");

__device__ __forceinline__ SegStat *stats(const SampleArgs &a) { return reinterpret_cast<SegStat *>(a.ws); }
__device__ __forceinline__ size_t cells(const SampleArgs &a) { return (size_t)a.M * a.segs; }
__device__ __forceinline__ uint64_t *bins(const SampleArgs &a) { return reinterpret_cast<uint64_t *>(a.ws + cells(a) * SAMPLE_STAT_BYTES); }
__device__ __forceinline__ float *list_l(const SampleArgs &a) { return reinterpret_cast<float *>(bins(a) + cells(a) * BINS); }
__device__ __forceinline__ int32_t *list_i(const SampleArgs &a) { return reinterpret_cast<int32_t *>(list_l(a) + cells(a) * ROOM); }

// A bin: count in the upper 14 bits, below it the sum of 2^36 exp((l - edge) / T), edge the bucket's upper end.
constexpr int BIN_COUNT = 50;
constexpr uint64_t BIN_MASS = (1ull << BIN_COUNT) - 1;
static_assert(SEG < 1 << 14, "a bin counts a segment");

// One workgroup per (row, segment): 32 tokens of each thread stay in registers.
__global__ __launch_bounds__(256) void segment_kernel(const SampleArgs a) {
  __shared__ uint64_t hist[4][BINS];  // one a wave
  __shared__ float redf[4];
  __shared__ int32_t redi[4], counts[SEG / 1024][4];
  __shared__ double redd[4];
  constexpr int N = SEG / 1024;
  const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float *x = a.logits + (size_t)row * a.V + seg * SEG;
  const int n = min(SEG, a.V - seg * SEG);
  float l[N][4];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = (j * 256 + tid) * 4;
    if (i + 4 <= n) {
      const f32x4u v = __builtin_nontemporal_load(reinterpret_cast<const f32x4u *>(x + i));
#pragma unroll
      for (int e = 0; e < 4; ++e) l[j][e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) l[j][e] = i + e < n ? x[i + e] : __builtin_nanf("");
    }
  }
  const Settings st = settings_of(a, row);
  float best = -INF;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) best = fmaxf(best, l[j][e]);  // NaN never wins
  const float top = block_reduce<256>(best, redf, [](float p, float q) { return fmaxf(p, q); });
  int arg = INT_MAX;
  if (best == top) {
#pragma unroll
    for (int j = N - 1; j >= 0; --j)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (l[j][e] == top) arg = seg * SEG + (j * 256 + tid) * 4 + e;
  }
  arg = block_reduce<256>(arg, redi, [](int p, int q) { return min(p, q); });
  SegStat out{top, arg, 0, INT_MAX, 0, 0, 0.0};
  const size_t cell = (size_t)row * a.segs + seg;
  const double scale = LOG2E / (double)st.t;
  if (arg == INT_MAX || st.kind == ONE) {
    // nothing more
  } else if (st.kind == ALL) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += l[j][e] == l[j][e] ? weight(l[j][e], top, scale) : 0.0;
    out.z = block_reduce<256>(sum, redd, [](double p, double q) { return p + q; });
  } else {
    const double g = grid_of(st);
    out.off = !(fabs((double)top * g) < GRID_END);
    if (!out.off) {
      out.bucket = bucket_of(top, g);
      for (int b = lane; b < BINS; b += 64) hist[wave][b] = 0;  // a wave's own: no barrier
      const bool mass = st.kind == NUCLEUS;
      const double last_edge = (double)(out.bucket - BINS + 2);
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = l[j][e];
          if (!(v > -INF)) continue;
          const double t = (double)v * g, fl = floor(fmax(t, -2.0 * GRID_END));
          const int rel = min(out.bucket - (int)fl, BINS - 1);
          uint64_t add = 1ull << BIN_COUNT;
          if (mass) {
            double w;
            if (rel < BINS - 1) {
              // exp(f / 8), f in [-1, 0): the power series to the ninth term
              const double f = t - (fl + 1.0);
              w = 2.0531802791346530e-14;
              w = fma(w, f, 1.4782898009769500e-12);
              w = fma(w, f, 9.4610547262524802e-11);
              w = fma(w, f, 5.2981906467013891e-09);
              w = fma(w, f, 2.5431315104166666e-07);
              w = fma(w, f, 1.0172526041666666e-05);
              w = fma(w, f, 3.2552083333333332e-04);
              w = fma(w, f, 7.8125e-03);
              w = fma(w, f, 0.125);
              w = fma(w, f, 1.0);
            } else {
              w = power_of_two((t - last_edge) * (LOG2E / 8.0));
            }
            add += __builtin_bit_cast(uint64_t, fma(w, 0x1p36, 0x1p52)) & ((1ull << 52) - 1);
          }
          atomicAdd((unsigned long long *)&hist[wave][rel], (unsigned long long)add);
        }
      __syncthreads();
      static_assert(BINS == 256, "a bin for each thread");
      const uint64_t bin = hist[0][tid] + hist[1][tid] + hist[2][tid] + hist[3][tid];
      if (mass) bins(a)[cell * BINS + tid] = bin;
      // How deep the list goes: as far as it has room; with a count, until the segment alone has so many; with a least
      // weight (where no share of a count's weight hangs on what lies below), until below it even against this segment's largest;
      // with a share, until what lies below is a quarter of what the share leaves out.
      int total;
      const int cnt = (int)(bin >> BIN_COUNT), upto = cnt + block_before<256>(cnt, redi, total);
      bool take = upto <= ROOM;
      if (st.k != INT_MAX) take = take && upto - cnt < st.k;
      if (st.m > 0.f && !(st.k != INT_MAX && st.p < 1.f))
        take = take && (double)(out.bucket - tid + 1) >= ((double)top + (double)st.t * log((double)st.m)) * g - 1.0;
      if (mass) {
        const double here = (double)(bin & BIN_MASS) * power_of_two((double)-tid * (LOG2E / 8.0));
        double z;
        const double before = block_before<256>(here, redd, z);
        take = take && z - before > 0.25 * (1.0 - (double)st.p) * z;
      }
      const int deep = block_reduce<256>(take ? BINS : tid, redi, [](int p, int q) { return min(p, q); });
      // the last bin also holds what lies below it: a list that takes it holds everything
      const int cut = deep == 0 ? INT_MAX : deep >= BINS ? INT_MIN : out.bucket - deep + 1;
      out.cut = cut;
      if (cut != INT_MAX) {
        auto want = [&](float v) { return v > -INF && bucket_of(v, g) >= cut; };
        uint32_t flags = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int c = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool w = want(l[j][e]);
            flags |= (uint32_t)w << (j * 4 + e);
            c += __popcll(__ballot(w));
          }
          if (lane == 0) counts[j][wave] = c;
        }
        __syncthreads();
        int base = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          int at = base;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (w < wave) at += counts[j][w];
            base += counts[j][w];
          }
          const uint32_t mine = flags >> (j * 4) & 15;
          if (!__any(mine != 0)) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) at += __popcll(__ballot(mine >> e & 1) & ((1ull << lane) - 1));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (mine >> e & 1) {
              list_l(a)[cell * ROOM + at] = l[j][e];
              list_i(a)[cell * ROOM + at] = seg * SEG + (j * 256 + tid) * 4 + e;
              ++at;
            }
        }
        out.n = base;
      }
    }
  }
  if (tid == 0) stats(a)[cell] = out;
}

// One workgroup per row.
template <int BS>
__global__ __launch_bounds__(BS) void row_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, segs = a.segs;
  const float *x = a.logits + (size_t)row * a.V;
  const SegStat *stat = stats(a) + (size_t)row * segs;
  const Settings st = settings_of(a, row);
  SegStat mine{-INF, INT_MAX, 0, INT_MIN, 0, 0, 0.0};
  if (tid < segs) mine = stat[tid];
  const float top = block_reduce<BS>(mine.top, (float *)sh.redu, [](float p, float q) { return fmaxf(p, q); });
  const int arg = block_reduce<BS>(mine.top == top ? mine.arg : INT_MAX, sh.redi, [](int p, int q) { return min(p, q); });
  const double scale = LOG2E / (double)st.t;
  SampleDist d{top, top, arg == INT_MAX ? -1 : arg, st.t, arg == INT_MAX ? 0.0 : 1.0, arg == INT_MAX ? 0 : arg, arg == INT_MAX ? 0.f : 1.f};
  if (arg != INT_MAX && st.kind != ONE && top > -INF) {
    float thr = -INF;
    int last = INT_MAX;
    const Source all{x, nullptr, a.V};
    const float hint = top - fminf(40.f * st.t, FLT_MAX);
    const float least = st.m > 0.f ? least_of(st.m, top, scale) : -INF;
    const double g = grid_of(st);
    float *mem_l = list_l(a) + (size_t)row * segs * ROOM;
    int32_t *mem_i = list_i(a) + (size_t)row * segs * ROOM;
    const int room = segs * ROOM;
    // a segment that weighs nothing beside the row's largest, to the last bit, is left out
    const bool absent = tid >= segs || mine.arg == INT_MAX || weight(mine.top, top, scale) == 0.0;
    const float lowest = block_reduce<BS>(tid < segs && absent ? mine.top : -INF, (float *)sh.redu, [](float p, float q) { return fmaxf(p, q); });
    // the deepest bucket from which on every segment's list is whole
    const int whole = block_reduce<BS>(!absent ? mine.cut : INT_MIN, sh.redi, [](int p, int q) { return max(p, q); });
    const bool off = block_reduce<BS>(!absent && mine.off ? 1 : 0, sh.redi, [](int p, int q) { return p | q; });
    // joins the segments' lists from bucket `from` up to bucket `upto`, by rising index, in the place of the first
    auto join = [&](int from, int upto) {
      int n = 0;
      if (tid < segs) sh.seg_n[tid] = absent ? 0 : mine.n;
      __syncthreads();
      for (int s = 0; s < segs; ++s) {
        const int ns = sh.seg_n[s];
        for (int i0 = 0; i0 < ns; i0 += BS) {
          const int i = i0 + tid;
          float l[1] = {0.f};
          int idx[1] = {0};
          bool want[1] = {false};
          if (i < ns) {
            l[0] = mem_l[s * ROOM + i];
            idx[0] = mem_i[s * ROOM + i];
            const int b = bucket_of(l[0], g);
            want[0] = b >= from && b <= upto;
          }
          append<BS>(sh, l, idx, want, mem_l, mem_i, room, n);  // its barrier stands between these reads and its writes
        }
      }
      __syncthreads();
      return n;
    };
    // kept weight of the segments from the elements of a source, exact whatever the order
    auto add_kept = [&](const Source &s) {
      for_each<BS>(s, [&](float l, int i) {
        const int idx = s.idx ? s.idx[i] : i;
        if (!(l > thr || (l == thr && idx <= last))) return;
        const uint64_t fx = (uint64_t)(weight(l, top, scale) * 0x1p62);
        atomicAdd((unsigned long long *)&sh.seg_lo[idx / SEG], (unsigned long long)(fx & 0xffffffffu));
        atomicAdd((unsigned long long *)&sh.seg_hi[idx / SEG], (unsigned long long)(fx >> 32));
      });
      __syncthreads();
    };
    for (int s = tid; s < segs; s += BS) { sh.seg_lo[s] = 0; sh.seg_hi[s] = 0; sh.seg[s] = 0.0; }
    __syncthreads();
    bool done = false;
    if (st.kind == ALL) {
      if (tid < segs) sh.seg[tid] = mine.arg == INT_MAX ? 0.0 : mine.z * weight(mine.top, top, scale);
      __syncthreads();
      done = true;
    } else if (st.kind == NUCLEUS && !off) {
      // the row's histogram, from the bucket of its largest downward; a segment's starts at its own largest
      const int first = bucket_of(top, g);
      if (tid < segs) sh.seg_at[tid] = absent ? INT_MIN : mine.bucket;
      __syncthreads();
      const uint64_t *h = bins(a) + (size_t)row * segs * BINS;
      // thread b < BINS - 1 has the row's bucket first - b; all that lies deeper is summed by segment
      double here = 0.0;
      int cnt = 0;
      if (tid < BINS - 1) {
        uint64_t m = 0;
        for (int s = 0; s < segs; ++s) {
          const int fs = sh.seg_at[s], rel = tid - (first - fs);
          if (fs == INT_MIN || rel < 0) continue;  // deeper than BINS - 1 it cannot be: fs <= first
          const uint64_t bin = h[(size_t)s * BINS + rel];
          m += bin & BIN_MASS;
          cnt += (int)(bin >> BIN_COUNT);
        }
        here = (double)m * 0x1p-36 * power_of_two(((double)(first - tid + 1) - (double)top * g) * (LOG2E / 8.0));
      }
      double deep = 0.0;
      for (int c = tid; c < segs * BINS; c += BS) {
        const int s = c / BINS, rel = c % BINS, fs = sh.seg_at[s];
        if (fs == INT_MIN || rel + (first - fs) < BINS - 1) continue;
        deep += (double)(h[c] & BIN_MASS) * 0x1p-36 * power_of_two(((double)(fs - rel + 1) - (double)top * g) * (LOG2E / 8.0));
      }
      deep = block_reduce<BS>(deep, sh.redd, [](double p, double q) { return p + q; });
      double z;
      const double before = block_before<BS>(here, sh.redd, z);
      const double target = (double)st.p * (z + deep);
      int ctot;
      const int cbefore = block_before<BS>(cnt, sh.redi, ctot);
      const int at = block_reduce<BS>(cnt > 0 && (before < target || cbefore == 0) ? tid : -1, sh.redi, [](int p, int q) { return max(p, q); });
      // target lies in what is deeper: the histogram does not tell where
      const bool reach = z >= target && at >= 0;
      if (at == tid) { sh.before = before; sh.count = cnt; sh.sum = z - here; }
      __syncthreads();
      if (reach) {
        const int b = first - at, n_b = sh.count;
        const double mass0 = sh.before, rest = sh.sum + deep;
        Source mem{mem_l, mem_i, 0};
        bool have = true;
        if (b >= whole) {
          mem.n = join(b, b);
        } else if (n_b <= room) {
          // not in the lists: from the logits
          int n = 0;
          for (int i0 = 0; i0 < a.V; i0 += BS * 4) {
            float l[4];
            int idx[4];
            bool want[4];
            const int i = i0 + tid * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              l[e] = i + e < a.V ? x[i + e] : -INF;
              idx[e] = i + e;
              want[e] = l[e] > -INF && bucket_of(l[e], g) == b;
            }
            append<BS>(sh, l, idx, want, mem_l, mem_i, room, n);
          }
          __syncthreads();
          mem.n = n;
        } else {
          have = false;
        }
        if (have) {
          // the bucket's ends, a little wider
          const float lo_b = (float)((b - 0.01) / g), hi_b = fminf(top, (float)((b + 1.01) / g));
          // The bucket's weight anew from its elements: histogram and weights differ in the last bits, and among equal
          // logits the border may fall on an element exactly.
          (void)cut<BS>(sh, mem, true, 0, (double)st.p, 0.0, mass0, rest, top, scale, lo_b, hi_b, thr, last);
          if (least > thr) { thr = least; last = INT_MAX; }
          if (bucket_of(thr, g) == b) {
            // of every segment: the buckets above, and what is kept of this one
            for (int s = wave; s < segs; s += BS / 64) {
              const int fs = sh.seg_at[s];
              double sum = 0.0;
              if (fs != INT_MIN)
                for (int rel = lane; rel < min(BINS - 1, fs - b); rel += 64)
                  sum += (double)(h[(size_t)s * BINS + rel] & BIN_MASS) * 0x1p-36 *
                         power_of_two(((double)(fs - rel + 1) - (double)top * g) * (LOG2E / 8.0));
#pragma unroll
              for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
              if (lane == 0) sh.seg[s] = sum;
            }
            __syncthreads();
            add_kept(mem);
            done = true;
          }  // else the least weight cuts higher: below, over the row
        } else {
          thr = -INF;
        }
        if (!done && have) { add_kept(all); done = true; }
      }
    } else if (st.kind == FEW && !off) {
      if (whole != INT_MAX) {
        const int n = join(whole, INT_MAX);
        const Source mem{mem_l, mem_i, n};
        if (n >= st.k) {
          const double w = cut<BS>(sh, mem, false, st.k, -1.0, 0.0, 0.0, 0.0, top, scale, hint, top, thr, last);
          if (st.p < 1.f) (void)cut<BS>(sh, mem, true, 0, -1.0, (double)st.p * w, 0.0, 0.0, top, scale, hint, top, thr, last);
          done = thr > lowest;  // else a segment without a list may have one of them
          if (least > thr) { thr = least; last = INT_MAX; }
        } else if ((st.k == INT_MAX || st.p >= 1.f) && (whole == INT_MIN || bucket_of(least, g) >= whole) && st.m > 0.f) {
          thr = least;
          done = true;
        }
        if (done) add_kept(mem);
      }
    }
    if (!done) {
      // the whole row, refinement by refinement
      thr = -INF; last = INT_MAX;
      double w = -1.0;
      if (st.k != INT_MAX) w = cut<BS>(sh, all, false, st.k, -1.0, 0.0, 0.0, 0.0, top, scale, hint, top, thr, last);
      if (st.p < 1.f) (void)cut<BS>(sh, all, true, 0, w < 0.0 ? (double)st.p : -1.0, (double)st.p * w, 0.0, 0.0, top, scale, hint, top, thr, last);
      if (least > thr) { thr = least; last = INT_MAX; }
      add_kept(all);
    }
    // kept weight in front of every segment; the segment that the target falls into
    double own = 0.0, z;
    if (tid < segs) own = sh.seg[tid] + from_fixed(sh.seg_lo[tid], sh.seg_hi[tid]);
    const double before = block_before<BS>(own, sh.redd, z);
    d.thr = thr; d.last = last; d.z = z;
    if (a.u) {
      const double target = target_of(a.u[row], z);
      const int seg = block_reduce<BS>(own > 0.0 && before <= target ? tid : -1, sh.redi, [](int p, int q) { return max(p, q); });
      if (tid == seg) sh.before = before;
      const int i0 = seg * SEG, n_steps = (min(a.V - i0, SEG) + STEP - 1) / STEP;
      auto step_weights = [&](int s, double (&w)[4]) {
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + s * STEP + lane * 4 + e;
          const float l = i < a.V ? x[i] : -INF;
          w[e] = i < a.V && (l > thr || (l == thr && i <= last)) ? weight(l, top, scale) : 0.0;
          sum += w[e];
        }
        return sum;
      };
      double w[4];
      if (seg >= 0) {
        for (int s = wave; s < n_steps; s += BS / 64) {
          double sum = step_weights(s, w);
#pragma unroll
          for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
          if (lane == 0) sh.step[s] = sum;
        }
      }
      __syncthreads();
      if (seg >= 0 && wave == 0) {
        // the step: the last that starts at or before the target (rounding may put all behind it: the first of weight)
        const double v = lane < n_steps ? sh.step[lane] : 0.0;
        double incl = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const double y = __shfl_up(incl, o);
          if (lane >= o) incl += y;
        }
        const double start = sh.before + (incl - v);
        const uint64_t some = __ballot(v > 0.0), fit = __ballot(v > 0.0 && start <= target);
        if (some) {
          const int s = fit ? 63 - __clzll(fit) : __ffsll((unsigned long long)some) - 1;
          double run = __shfl(start, s);
          const double own_w = step_weights(s, w);
          double in = own_w;
#pragma unroll
          for (int o = 1; o < 64; o <<= 1) {
            const double y = __shfl_up(in, o);
            if (lane >= o) in += y;
          }
          run += in - own_w;
          int id = -1, any = -1;
          double wid = 0.0, wany = 0.0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            run += w[e];
            if (w[e] > 0.0) { any = i0 + s * STEP + lane * 4 + e; wany = w[e]; }
            if (id < 0 && w[e] > 0.0 && run > target) { id = any; wid = w[e]; }
          }
          // the first lane that passes the target; where rounding lets none, the last token of weight
          const uint64_t over = __ballot(id >= 0), has = __ballot(any >= 0);
          const int lane_at = over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll(has);
          d.id = __shfl(over ? id : any, lane_at);
          d.prob = (float)(__shfl(over ? wid : wany, lane_at) / z);
        }
      }
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
__device__ __forceinline__ double share_of(const SampleDist &d, double scale, double inv_z, float l, int i) {
  return kept_by(d, l, i) ? weight(l, d.top, scale) * inv_z : 0.0;
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
      const double p = share_of(pd, LOG2E / (double)pd.temp, inv_of(pd.z), a.target[((size_t)b * q + i) * a.V + d], d);
      double qd = 1.0;
      if (a.draft_logits) {
        const SampleDist dd = a.draft_dist[(size_t)b * a.k + i];
        qd = share_of(dd, LOG2E / (double)dd.temp, inv_of(dd.z), a.draft_logits[((size_t)b * a.k + i) * a.V + d], d);
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
  r.p_t = LOG2E / (double)r.pd.temp; r.p_z = inv_of(r.pd.z);
  r.q = nullptr; r.q_t = r.q_z = 0.0; r.dead = -1;
  if (n < a.k && a.draft_logits) {
    r.q = a.draft_logits + slot * a.V;
    r.qd = a.draft_dist[slot];
    r.q_t = LOG2E / (double)r.qd.temp; r.q_z = inv_of(r.qd.z);
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
  segment_kernel<<<a.M * a.segs, 256, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.M <= 256) row_kernel<1024><<<a.M, 1024, 0, s>>>(a);
  else row_kernel<256><<<a.M, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sf
