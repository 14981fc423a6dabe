// Sampling for gfx950: a token drawn from a row of logits under temperature, top-k, top-p and min-p, from a given random
// number.
//
// The row's tokens are ranked by falling logit, equal ones by rising index (NaN: not there).  With M the largest logit and
// w_i = exp((l_i - M) / T), each filter keeps a prefix of the ranking: the K best; of those the ones in front of which less
// than top_p of their weight lies; of those the ones of at least min_p (the largest weight is 1).  A prefix is described by
// its last element (thr, last): a token is kept if l > thr, or l == thr and its index <= last.  The token is the first, by
// index, whose running kept weight exceeds u times the kept weight.
//
// Two launches, so that most of the logits leave memory once.  segment_kernel holds 8192 tokens of a row in the registers of a
// workgroup and leaves what the row needs of them: the largest, the sum of weights, a histogram of weights (nucleus), the
// tokens that may lie in the kept prefix.  row_kernel joins the segments, finds the prefix, finds the segment that u falls
// into by the segments' kept weights, and reads that one again for the token.  What a segment had no room for (a flat row's
// nucleus of tens of thousands, a count behind a lead of more than 32) is read from the logits again, for that row alone.
//
// What bounds them: the first launch the vector instructions, at half the rate that the logits could be read with when all
// rows ask for a nucleus (640 rows of 152064: 127 us, 3.1 TB/s) and 3.3 TB/s for settings of all kinds (256 of 128256: 40 us);
// the second one the latency of a row's dozen dependent steps, 17 to 25 us, a compute unit to a row (640 rows 116 us, 256 rows
// 49, one row 14).  A single workgroup per row, which reads the row in each of its steps, takes 691 us for the 640 rows.
//
// Weights are doubles: in a vocabulary of 150000 tokens a float sum is off by more than many tokens weigh, and the token
// next to a border would hang on the order of the sum.  Where weights are summed by atomics they are integers (multiples of
// 2^-62 in two halves, or of 2^-36 of a bucket's edge), so that the order does not matter there either: a row's result has the
// same bits on every run.  A nucleus takes the bins' rounding: a token weighs e^-1/8 of its edge at least, so its sums are off by
// 2^-36.8 of themselves, and the segments' shares, cut to 2^-49 in each of up to 128 x 255 bins, by 2^-34 together: less than 2^-33
// of the kept weight, which is 1 at least.
#include "sf_internal.h"
#include <float.h>
#include <limits.h>

namespace sf {
namespace {

constexpr int BUCKETS = 1024;    // of one refinement of the ranking
constexpr int LIST = 1536;       // elements that are ranked one by one: a count of a thousand, with what shares its last bucket
constexpr int MEM = 8192;        // elements of a row that LDS has room for
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
  s.p = s.p < 1.f ? fmaxf(s.p, 0.f) : 1.f;
  if (!(s.m > 0.f)) s.m = 0.f;
  s.kind = s.k == 1 || s.m > 1.f ? ONE : s.k != INT_MAX ? FEW : s.p < 1.f ? NUCLEUS : s.m > 0.f ? FEW : ALL;
  return s;
}

// Polynomials of doubles.  pinned: the coefficients once in scalar registers, where the compiler cannot see their values; one that
// it sees it moves into two vector registers in front of every product that adds it, three instructions for one.
template <int N> struct Poly {
  double c[N];  // from the highest power
  __device__ __forceinline__ double operator()(double x) const {
    double p = c[0];
#pragma unroll
    for (int i = 1; i < N; ++i) p = fma(p, x, c[i]);
    return p;
  }
};
template <int N> __device__ __forceinline__ Poly<N> pinned(Poly<N> p) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+s"(p.c[i]));
  return p;
}

// 2^y for y <= 0 (or a little above), to 2^-50: (2^f - 1) / f on |f| <= 1/2 as a polynomial of degree nine through its values at
// the Chebyshev points.  The device library's exp takes twice as many instructions, and double precision is a third of what
// these kernels do.
#define POW2_POLY                                                                                                              \
  Poly<11> {                                                                                                                   \
    {7.07097786650813908e-09, 1.02059054137655955e-07, 1.32154516332214336e-06, 1.52526729248507372e-05,                     \
     1.54035304247765285e-04, 1.33335582007945925e-03, 9.61812910761866528e-03, 5.55041086646516704e-02,                     \
     2.40226506959100750e-01, 6.93147180559946174e-01, 1.0}                                                                    \
  }
__device__ __forceinline__ double power_of_two(double y, const Poly<11> &poly) {
  y = fmax(y, -1200.0);  // 0 from there on, for -inf too
  const double n = rint(y);
  return __builtin_ldexp(poly(y - n), (int)n);
}
__device__ __forceinline__ double power_of_two(double y) { return power_of_two(y, POW2_POLY); }
__device__ __noinline__ double power_of_two_apart(double y) { return power_of_two(y); }  // where it is rare and the code long

constexpr double LOG2E = 1.4426950408889634;

// scale: log2(e) / T
__device__ __forceinline__ double weight(float l, float top, double scale) {
  return l == top ? 1.0 : power_of_two(((double)l - (double)top) * scale);
}

// The grid of a row's buckets: bucket b holds the logits of about [b, b + 1) / g (a product in float, which never puts a
// smaller logit into a higher bucket).  Nucleus: eight to a factor of e in weight.  Counts: likewise between T = 1 and 2, not
// narrower below nor wider above, so that the tokens of a count are within reach at any temperature: 256 buckets reach 32 below a
// segment's largest (at 19, a row with a lead of 26 lost sight of its crowd: 465 us for a count of 1000, 44 so).
__device__ __forceinline__ double grid_of(const Settings &s) {
  return 8.0 / (double)(s.kind == NUCLEUS ? s.t : fminf(fmaxf(s.t, 1.f), 2.f));
}
constexpr float GRID_END = 1 << 16;  // beyond, a float's place on the grid is too coarse: the row goes without it
__device__ __forceinline__ float grid_place(float l, float g) { return floorf(fmaxf(l * g, -2.f * GRID_END)); }
__device__ __forceinline__ int bucket_of(float l, float g) { return (int)fminf(grid_place(l, g), 2.f * GRID_END); }

__device__ __forceinline__ uint32_t float_order(float l) {
  const uint32_t b = __float_as_uint(l);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_float(uint32_t b) { return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b); }

// The smallest float of a rising condition, from a guess that is mostly a few floats off.  It holds for hi, not for -inf.
template <class F> __device__ __forceinline__ float first_float(float guess, float hi, F holds) {
  uint32_t a = float_order(-INF), b = float_order(hi);
  const uint32_t g = min(max(float_order(guess), a + 1), b);
  if (holds(order_float(g))) {
    b = g;
    for (int i = 0; i < 4 && b - a > 1; ++i)
      if (holds(order_float(b - 1))) --b; else a = b - 1;
  } else {
    a = g;
    for (int i = 0; i < 4 && b - a > 1; ++i)
      if (holds(order_float(a + 1))) b = a + 1; else ++a;
  }
  while (b - a > 1) {
    const uint32_t mid = a + (b - a) / 2;
    if (holds(order_float(mid))) b = mid; else a = mid;
  }
  return order_float(b);
}
// the first float of bucket b, b at most that of hi
__device__ __forceinline__ float bucket_start(int b, double g, float hi) {
  return first_float((float)((double)b / g), hi, [&](float l) { return bucket_of(l, (float)g) >= b; });
}
// the smallest float whose weight reaches m in (0, 1]
__device__ __forceinline__ float least_of(float m, float t, float top, double scale) {
  return first_float((float)((double)top + (double)t * log((double)m)), top, [&](float l) { return weight(l, top, scale) >= (double)m; });
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
  const uint32_t b = float_order(l + 0.f);  // -0 ranks as 0
  return (uint64_t)b << 32 | (uint32_t)(INT_MAX - i);
}
__device__ __forceinline__ float key_logit(uint64_t k) {
  return order_float((uint32_t)(k >> 32));
}
__device__ __forceinline__ int key_index(uint64_t k) { return INT_MAX - (int)(uint32_t)k; }

// the elements that a selection looks at: a row of logits, or a list of ranking keys in LDS
struct Row {
  const float *l;
  int n;
};
struct List {
  const uint64_t *key;
  int n;
};

struct Shared {
  struct {
    uint32_t cnt[BUCKETS];
    uint64_t lo[2 * BUCKETS];  // weight * 2^62: its lower 32 bits, and BUCKETS on the rest
  } h;
  uint64_t mem[MEM], list[LIST], sorted[LIST];
  double seg[MAX_SEGS], step[SEG / STEP];  // kept weight of the segments, of a segment's steps
  uint64_t seg_lo[MAX_SEGS], seg_hi[MAX_SEGS];
  int32_t seg_n[MAX_SEGS], seg_at[MAX_SEGS], seg_task[MAX_SEGS];
  double redd[16];
  int redi[16];
  uint32_t redu[16];
  double factor[BINS];  // of the row's bins
  int n_list, n_mem;
  int at, found;
  double before, sum;
  int count;
};

// x[i, i + 4) of n
__device__ __forceinline__ f32x4u four(const float *x, int i, int n) {
  if (i + 4 <= n) return *reinterpret_cast<const f32x4u *>(x + i);
  f32x4u v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = i + e < n ? x[i + e] : __builtin_nanf("");
  return v;
}

// f(logit, index) for all but NaN.  Four requests of a thread are on their way at a time.
template <int BS, class F> __device__ __forceinline__ void for_each(const Row &s, F f) {
  constexpr int AHEAD = 4;
  for (int i0 = threadIdx.x * 4; i0 < s.n; i0 += BS * 4 * AHEAD) {
    f32x4u v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) v[j] = four(s.l, i0 + j * BS * 4, s.n);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v[j][e] == v[j][e]) f(v[j][e], i0 + j * BS * 4 + e);
  }
}
template <int BS, class F> __device__ __forceinline__ void for_each(const List &s, F f) {
  for (int i = threadIdx.x; i < s.n; i += BS) f(key_logit(s.key[i]), key_index(s.key[i]));
}

__device__ __forceinline__ double from_fixed(uint64_t lo, uint64_t hi) { return (double)hi * 0x1p-30 + (double)lo * 0x1p-62; }

// sh.sorted = list[0, n) by falling key.  An element's place is the number of larger ones; a wave's comparison of 64 elements
// with one is four cycles of LDS, so that few are compared with all, and of more (COUNT) each with those of its own bucket of
// a linear map (of equal logits there is one).  A network of exchanges with a barrier in each of its steps is slower from 512 on.
template <int BS> __device__ void sort_list(Shared &sh, const uint64_t *list, int n) {
  constexpr int COUNT = 320, EACH = (LIST + BS - 1) / BS, PER = BUCKETS / BS;
  const int tid = threadIdx.x;
  if (n <= COUNT) {
    for (int e = tid; e < n; e += BS) {
      const uint64_t key = list[e];
      int place = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) place += list[j] > key;
      sh.sorted[place] = key;
    }
    __syncthreads();
    return;
  }
  uint64_t key[EACH];
  float mn = INF, mx = -INF;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = e * BS + tid;
    key[e] = i < n ? list[i] : 0;
    if (i < n) { mn = fminf(mn, key_logit(key[e])); mx = fmaxf(mx, key_logit(key[e])); }
  }
  for (int b = tid; b < BUCKETS; b += BS) sh.h.cnt[b] = 0;
  mn = block_reduce<BS>(mn, (float *)sh.redu, [](float p, float q) { return fminf(p, q); });
  mx = block_reduce<BS>(mx, (float *)sh.redu, [](float p, float q) { return fmaxf(p, q); });
  const bool map = mn > -INF && mx < INF && mn < mx;
  const double places = map ? (BUCKETS - 1) / ((double)mx - (double)mn) : 0.0;
  int bucket[EACH], at[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    bucket[e] = map ? min(BUCKETS - 1, (int)(((double)mx - (double)key_logit(key[e])) * places)) : 0;
    if (e * BS + tid < n) at[e] = (int)atomicAdd(&sh.h.cnt[bucket[e]], 1u);
  }
  __syncthreads();
  // counts to starts
  int c[PER], own = 0, all;
#pragma unroll
  for (int e = 0; e < PER; ++e) own += c[e] = (int)sh.h.cnt[tid * PER + e];
  int run = block_before<BS>(own, sh.redi, all);
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    sh.h.cnt[tid * PER + e] = (uint32_t)run;
    run += c[e];
  }
  __syncthreads();
  uint64_t *const grouped = sh.h.lo;
  static_assert(LIST <= 2 * BUCKETS, "the list by buckets");
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (e * BS + tid < n) grouped[(int)sh.h.cnt[bucket[e]] + at[e]] = key[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if (e * BS + tid >= n) continue;
    const int lo = (int)sh.h.cnt[bucket[e]], hi = bucket[e] + 1 < BUCKETS ? (int)sh.h.cnt[bucket[e] + 1] : n;
    int place = lo;
#pragma unroll 8  // of equal logits the bucket is long
    for (int j = lo; j < hi; ++j) place += grouped[j] > key[e];
    sh.sorted[place] = key[e];
  }
  __syncthreads();
}

// The j-th (from 0) element by index among those equal to v.
template <int BS> __device__ int nth_equal(Shared &sh, const Row &s, float v, int j) {
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
      if (eq && before + here == j) sh.found = i0 + lane;
      before += __popcll(m);
    }
  __syncthreads();
  const int r = sh.found;
  __syncthreads();
  return r;
}

// Of list[0, n), n <= LIST: ranks them and cuts behind the k best, and of those (share < 1) behind the last in front of
// which less than share of the weight lies: of the k best's, or, without a count, of all these and `rest`'s.  target >= 0: the
// weight itself.  mass0: weight of elements that rank in front and are not among them.  Returns how many stay (sh.sorted) and
// their weight, mass0 with it.
template <int BS>
__device__ int ranked(Shared &sh, const uint64_t *list, int n, int k, double share, double target, double mass0, double rest,
                      float top, double scale, double &kept) {
  constexpr int EACH = LIST / BS > 0 ? LIST / BS : 1;
  const int tid = threadIdx.x;
  sort_list<BS>(sh, list, n);
  double x[EACH], xs = 0.0, all;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = tid * EACH + e;
    x[e] = i < n && i < k ? weight(key_logit(sh.sorted[i]), top, scale) : 0.0;
    xs += x[e];
  }
  double run = mass0 + block_before<BS>(xs, sh.redd, all);
  if (target < 0.0) target = share < 1.0 ? share * (k == INT_MAX ? rest + all : mass0 + all) : INF;
  int keep = -1;
  double sum = 0.0;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = tid * EACH + e;
    const bool in = i < n && i < k && (run < target || (i == 0 && !(mass0 > 0.0)));
    run += x[e];
    if (in) { keep = i; sum = run; }
  }
  const int end = block_reduce<BS>(keep, sh.redi, [](int a, int b) { return max(a, b); });
  if (keep == end && end >= 0) sh.sum = sum;
  __syncthreads();
  kept = end >= 0 ? sh.sum : mass0;
  return end + 1;
}

// Cuts the ranking of the elements that are kept so far (l > thr or l == thr and index <= last): by_mass, behind the last
// element in front of which less than `target` of weight lies (share >= 0: that share of the weight of these and `rest`, what
// else there is); else behind the k best.  mass0: weight of elements that rank in front of all of these and are not among
// them.  thr and last receive the last kept element; returns the kept weight.  ties: where the j-th of equal elements is looked up
// (s may be in any order).  lo_hint: nothing of interest is expected below; hi: nothing lies above.
//
// A refinement sorts the elements of an interval of logits into buckets by a linear map (it never puts a smaller logit in
// front of a larger one), finds the bucket of the cut from the running counts and weights, and goes on with that bucket's
// interval, until it has few elements, which are sorted, or equal ones, which are counted.
template <int BS, class Source>
__device__ double cut(Shared &sh, const Source &s, const Row &ties, bool by_mass, int k, double share, double target, double mass0, double rest,
                      float top, double scale, float lo_hint, float hi, float &thr, int &last) {
  constexpr int PER = BUCKETS / BS > 0 ? BUCKETS / BS : 1;
  const int tid = threadIdx.x;
  const float thr0 = thr;
  const int last0 = last;
  auto kept = [&](float l, int i) { return l > thr0 || (l == thr0 && i <= last0); };
  float lo = fmaxf(lo_hint, thr0);            // the interval [lo, hi]; what lies above is kept whole
  bool below = true;                          // elements below lo belong to the last bucket
  int count0 = mass0 > 0.0 ? 1 : 0;           // by weight only whether there is one in front matters
  const bool whole = s.n <= LIST;             // few elements: ranked as they are
  for (;;) {
    const double places = hi > lo ? (BUCKETS - 2) / ((double)hi - (double)lo) : 0.0;
    auto bucket = [&](float l) {
      if (whole || l == hi) return 0;
      if (l < lo || l == -INF || hi == INF) return BUCKETS - 1;
      return min(BUCKETS - 2, (int)(((double)hi - (double)l) * places));
    };
    auto inside = [&](float l, int i) { return l <= hi && (below || l >= lo) && kept(l, i); };
    int at = 0, n_at = s.n;
    if (!whole) {
      for (int x = tid; x < BUCKETS; x += BS) { sh.h.cnt[x] = 0; sh.h.lo[x] = 0; sh.h.lo[BUCKETS + x] = 0; }
      __syncthreads();
      int minus = 0;  // -inf weighs nothing: counted apart, a mask's thousands would queue for one address
      for_each<BS>(s, [&](float l, int i) {
        if (!inside(l, i)) return;
        if (l == -INF && l < hi) { ++minus; return; }
        const int b = bucket(l);
        atomicAdd(&sh.h.cnt[b], 1u);
        const uint64_t fx = (uint64_t)(weight(l, top, scale) * 0x1p62);
        atomicAdd((unsigned long long *)&sh.h.lo[b], (unsigned long long)(fx & 0xffffffffu));
        atomicAdd((unsigned long long *)&sh.h.lo[BUCKETS + b], (unsigned long long)(fx >> 32));
      });
      if (minus) atomicAdd(&sh.h.cnt[BUCKETS - 1], (uint32_t)minus);
      __syncthreads();
      // running counts and weights; each thread has PER consecutive buckets
      int c[PER], cs = 0;
      double w[PER], ws = 0.0;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int b = tid * PER + e;
        c[e] = b < BUCKETS ? (int)sh.h.cnt[b] : 0;
        w[e] = b < BUCKETS ? from_fixed(sh.h.lo[b], sh.h.lo[BUCKETS + b]) : 0.0;
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
        if (inside(l, i) && bucket(l) == at) sh.list[atomicAdd(&sh.n_list, 1)] = rank_key(l, i);
      });
      __syncthreads();
      n_at = sh.n_list;
      if (n_at == 0) { thr = thr0; last = last0; return mass0; }
      if (share >= 0.0) target = -1.0;
      double r;
      const int n_kept = ranked<BS>(sh, sh.list, n_at, by_mass ? INT_MAX : k - count0, by_mass && share >= 0.0 ? share : 1.0,
                                    by_mass ? target : -1.0, mass0, rest, top, scale, r);
      if (n_kept > 0) {
        thr = key_logit(sh.sorted[n_kept - 1]);
        last = key_index(sh.sorted[n_kept - 1]);
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
      last = j == n_at && mn > thr0 ? INT_MAX : nth_equal<BS>(sh, ties, mn, j - 1);
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

// Appends N elements of each lane of a wave, where wanted, to sh.mem, in any order; sh.n_mem counts those that find no room too.
template <int N>
__device__ __forceinline__ void collect(Shared &sh, const bool (&want)[N], const float (&l)[N], const int (&i)[N]) {
  uint64_t m[N];
  int c = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    m[e] = __ballot(want[e]);
    c += __popcll(m[e]);
  }
  if (c == 0) return;
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (lane == 0) at = atomicAdd(&sh.n_mem, c);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (want[e]) {
      const int p = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[e], 0));
      if (p < MEM) sh.mem[p] = rank_key(l[e], i[e]);
    }
    at += __popcll(m[e]);
  }
}

struct SegStat {
  float top;
  int32_t arg;    // lowest index of the largest; INT_MAX: no comparable value
  int32_t bucket; // of the largest on the row's grid: the histogram's first
  int32_t cut;    // the list holds all of the segment's elements from this bucket on; INT_MAX: not even the first
  int32_t n;      // entries of the list, in any order
  int32_t off;    // the grid does not reach the values
  double z;       // ALL: sum of weights against the segment's largest.  Behind a row kernel that draws no token: the kept weight
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
  __shared__ int32_t redi[4], n_list;
  __shared__ double redd[4];
  constexpr int N = SEG / 1024;
  const int row = blockIdx.x / a.segs, seg = blockIdx.x % a.segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float *x = a.logits + (size_t)row * a.V + seg * SEG;
  const int n = min(SEG, a.V - seg * SEG);
  float l[N][4];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = (j * 256 + tid) * 4;
    const f32x4u v = n == SEG ? *reinterpret_cast<const f32x4u *>(x + i) : four(x, i, n);
#pragma unroll
    for (int e = 0; e < 4; ++e) l[j][e] = v[e];
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
    if (fabsf(top) < INF) {
      const Poly<11> poly = pinned(POW2_POLY);
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += power_of_two(((double)l[j][e] - (double)top) * scale, poly);  // NaN weighs nothing
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += l[j][e] == top ? 1.0 : 0.0;
    }
    out.z = block_reduce<256>(sum, redd, [](double p, double q) { return p + q; });
  } else {
    const double g = grid_of(st);
    const float gf = (float)g;
    out.off = !(fabsf(top * gf) < GRID_END);
    if (!out.off) {
      out.bucket = bucket_of(top, gf);
      if (tid == 0) n_list = 0;
      for (int b = lane; b < BINS; b += 64) hist[wave][b] = 0;  // a wave's own: no barrier
      const bool mass = st.kind == NUCLEUS;
      const float first = (float)out.bucket;
      int limit = BINS;  // bins from there on have not counted all
      if (mass) {
        // 2^36 exp(f / 8) + 2^52, f in [-1, 0] (the float product's roundings beside): the lower 52 bits are the bin's part.  A
        // polynomial of degree six in f + 1/2 through the values at the Chebyshev points: to 2^-45, the bin takes 2^-37.
        const Poly<7> poly = pinned(Poly<7>{{4.97784668590196699e-09 * 0x1p36, 2.38947156470155655e-07 * 0x1p36,
                                             9.55620375649920453e-06 * 0x1p36, 3.05798517364579050e-04 * 0x1p36,
                                             7.33916455323328255e-03 * 0x1p36, 1.17426632851876683e-01 * 0x1p36,
                                             9.39413062813475808e-01 * 0x1p36 + 0x1p52}});
        const float from = bucket_start(out.bucket - (BINS - 2), g, top);  // below it the last bin
        float low = top;
        char *const mine = reinterpret_cast<char *>(&hist[wave][0]);
        auto add = [&](uint32_t place, double fixed) __attribute__((always_inline)) {
          uint64_t v = __builtin_bit_cast(uint64_t, fixed);  // off with the exponent of 2^52, on with a count of one
          v += (uint64_t)((1u << (BIN_COUNT - 32)) - 0x43300000u) << 32;
          atomicAdd(reinterpret_cast<unsigned long long *>(mine + place), (unsigned long long)v);
        };
        const float first8 = first * 8.f;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = l[j][e], fl = floorf(v * gf);
            low = fminf(low, v);
            if (!(v >= from)) continue;
            const double f = fma((double)v, g, -(double)(fl + 0.5f));
            add((uint32_t)(int)fmaf(fl, -8.f, first8), poly(f));
          }
        if (__any(low < from)) {
          const double last_edge = (double)(out.bucket - BINS + 2);
#pragma unroll
          for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = l[j][e];
              if (v > -INF && v < from) add((BINS - 1) * 8, fma(power_of_two_apart(((double)v * g - last_edge) * (LOG2E / 8.0)), 0x1p36, 0x1p52));
            }
        }
      } else {
        // only what may get into the list is counted: nothing below the least of the threads' largest, of which there are 256
        float bound = block_reduce<256>(best, redf, [](float p, float q) { return fminf(p, q); });
        if (st.k != INT_MAX && st.k > 256) bound = -INF;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = l[j][e];
            if (!(v > -INF) || v < bound) continue;
            const int rel = (int)fminf(first - grid_place(v, gf), (float)(BINS - 1));
            atomicAdd((unsigned long long *)&hist[wave][rel], 1ull << BIN_COUNT);
          }
        limit = sample_whole_bins(bound > -INF, out.bucket, bucket_of(bound, gf));
      }
      __syncthreads();
      static_assert(BINS == 256, "a bin for each thread");
      const uint64_t bin = hist[0][tid] + hist[1][tid] + hist[2][tid] + hist[3][tid];
      if (mass) bins(a)[cell * BINS + tid] = bin;
      // How deep the list goes (sample_takes): as far as it has room; with a count, until the segment alone has so many; with a least
      // weight (where no share of a count's weight hangs on what lies below), until below it even against this segment's largest;
      // with a share, until it has 64 and what lies below is a quarter of what the share leaves out.
      int total;
      const int cnt = (int)(bin >> BIN_COUNT), upto = cnt + block_before<256>(cnt, redi, total);
      bool take = sample_takes(tid, cnt, upto, limit, st.k);
      if (st.m > 0.f && !(st.k != INT_MAX && st.p < 1.f))
        take = take && (double)(out.bucket - tid + 1) >= ((double)top + (double)st.t * log((double)st.m)) * g - 1.0;
      if (mass) {
        const double here = (double)(bin & BIN_MASS) * power_of_two((double)-tid * (LOG2E / 8.0));
        double z;
        const double before = block_before<256>(here, redd, z);
        take = take && (upto - cnt < 64 || z - before > 0.25 * (1.0 - (double)st.p) * z);
      }
      const int deep = block_reduce<256>(take ? BINS : tid, redi, [](int p, int q) { return min(p, q); });
      // the last bin also holds what lies below it: a list that takes it holds everything
      out.cut = deep == 0 ? INT_MAX : deep >= BINS ? INT_MIN : out.bucket - deep + 1;
      if (deep > 0) {
        const float from = deep >= BINS ? -FLT_MAX : bucket_start(out.cut, g, top);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          uint64_t m[4];
          int c = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m[e] = __ballot(l[j][e] >= from);
            c += __popcll(m[e]);
          }
          if (c == 0) continue;
          int at = 0;
          if (lane == 0) at = atomicAdd(&n_list, c);
          at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (m[e] >> lane & 1) {
              const int p = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[e], 0));
              if (p < ROOM) {
                list_l(a)[cell * ROOM + p] = l[j][e];
                list_i(a)[cell * ROOM + p] = seg * SEG + (j * 256 + tid) * 4 + e;
              }
            }
            at += __popcll(m[e]);
          }
        }
        __syncthreads();
        out.n = n_list;
        if (n_list > ROOM) { out.n = 0; out.cut = INT_MAX; }  // not by the counts; what lies behind the list does not hang on them
      }
    }
  }
  if (tid == 0) stats(a)[cell] = out;
}

// over the lanes of a wave
template <class T, class F> __device__ __forceinline__ T wave_reduce(T v, F f) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = f(v, __shfl_xor(v, o));
  return v;
}
template <class T> __device__ __forceinline__ T wave_before(T v) {  // sum over the lanes below
  T x = v;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  x = __shfl_up(x, 1);
  return lane == 0 ? T(0) : x;
}

// One workgroup per row.
template <int BS>
__global__ __launch_bounds__(BS, BS / 256) void row_kernel(const SampleArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Shared &sh = *reinterpret_cast<Shared *>(smem);
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, segs = a.segs;
  const float *x = a.logits + (size_t)row * a.V;
  const SegStat *stat = stats(a) + (size_t)row * segs;
  const Settings st = settings_of(a, row);
  // every wave has all the segments, two to a lane
  static_assert(MAX_SEGS == 128, "two segments to a lane");
  SegStat own[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    own[e] = SegStat{-INF, INT_MAX, 0, INT_MIN, 0, 0, 0.0};
    if (lane + e * 64 < segs) own[e] = stat[lane + e * 64];
  }
  const float top = wave_reduce(fmaxf(own[0].top, own[1].top), [](float p, float q) { return fmaxf(p, q); });
  const int arg = wave_reduce(min(own[0].top == top ? own[0].arg : INT_MAX, own[1].top == top ? own[1].arg : INT_MAX),
                              [](int p, int q) { return min(p, q); });
  const double scale = LOG2E / (double)st.t;
  SampleDist d{top, top, arg == INT_MAX ? -1 : arg, st.t, arg == INT_MAX ? 0.0 : 1.0, arg == INT_MAX ? 0 : arg, arg == INT_MAX ? 0.f : 1.f};
  int writer = 0;  // wave that knows the token
  if (arg != INT_MAX && st.kind != ONE && top > -INF) {
    const float u = a.u ? a.u[row] : 0.f;
    float thr = -INF;
    int last = INT_MAX;
    const Row all{x, a.V};
    const float hint = top - fminf(40.f * st.t, FLT_MAX);
    const float least = st.m > 0.f ? least_of(st.m, st.t, top, scale) : -INF;
    const double g = grid_of(st);
    const float gf = (float)g;
    const size_t cell0 = (size_t)row * segs * ROOM;
    int whole = INT_MIN, off = 0;  // the deepest bucket from which on every segment's list is whole; off the grid
    float lowest = -INF;           // the largest of the segments that are left out
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      // a segment that weighs nothing beside the row's largest, to the last bit, is left out
      if (own[e].arg == INT_MAX || weight(own[e].top, top, scale) == 0.0) {
        lowest = fmaxf(lowest, own[e].top);
        own[e].arg = INT_MAX;
      } else {
        whole = max(whole, own[e].cut);
        off |= own[e].off;
      }
    }
    whole = wave_reduce(whole, [](int p, int q) { return max(p, q); });
    off = wave_reduce(off, [](int p, int q) { return p | q; });
    lowest = wave_reduce(lowest, [](float p, float q) { return fmaxf(p, q); });
    // the lists in pieces of 64 entries: the pieces of the segments up to each lane's
    int n0 = own[0].arg != INT_MAX ? (own[0].n + 63) / 64 : 0, n1 = own[1].arg != INT_MAX ? (own[1].n + 63) / 64 : 0;
    const int all0 = wave_reduce(n0, [](int p, int q) { return p + q; });
    const int end0 = wave_before(n0) + n0, end1 = all0 + wave_before(n1) + n1;
    const int pieces = all0 + wave_reduce(n1, [](int p, int q) { return p + q; });
    if (wave == 0) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int s = lane + e * 64;
        const bool there = own[e].arg != INT_MAX;
        sh.seg_n[s] = there ? own[e].n : 0;
        sh.seg_at[s] = there ? own[e].bucket : INT_MIN;
        sh.seg_task[s] = e ? end1 - n1 : end0 - n0;
        sh.seg_lo[s] = 0; sh.seg_hi[s] = 0;
        sh.seg[s] = there && st.kind == ALL ? own[e].z * weight(own[e].top, top, scale) : 0.0;
      }
      if (lane == 0) sh.n_mem = 0;
    }
    __syncthreads();
    // f(l[], i[]) for the entries of the segments' lists, four pieces of a wave at a time; NaN: not there
    constexpr int PIECES = 4;
    auto visit = [&](auto f) {
      for (int t0 = wave; t0 < pieces; t0 += BS / 64 * PIECES) {
        float l[PIECES];
        int i[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          const int t = t0 + j * (BS / 64);
          l[j] = __builtin_nanf(""); i[j] = 0;
          if (t < pieces) {
            // the segment: the first whose pieces end behind t
            const int s = __popcll(__ballot(end0 <= t)) + __popcll(__ballot(end1 <= t));
            const int at = (t - sh.seg_task[s]) * 64 + lane;
            if (at < sh.seg_n[s]) {
              l[j] = list_l(a)[cell0 + s * ROOM + at];
              i[j] = list_i(a)[cell0 + s * ROOM + at];
            }
          }
        }
        f(l, i);
      }
      __syncthreads();
    };
    // selects what lies in [from, to) of the segments' lists
    auto join = [&](float from, float to) {
      visit([&](const float (&l)[PIECES], const int (&i)[PIECES]) {
        bool want[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) want[j] = l[j] >= from && l[j] < to;
        collect(sh, want, l, i);
      });
      return sh.n_mem;
    };
    // The bucket of 1024, by rising number, that the k-th lies in: sh.at, and how many lie up to its end: sh.count (at: BUCKETS if
    // there are fewer than k).
    auto bucket_of_kth = [&]() {
      constexpr int PER = BUCKETS / BS;
      int c[PER], own_c = 0, ctot;
#pragma unroll
      for (int e = 0; e < PER; ++e) own_c += c[e] = (int)sh.h.cnt[tid * PER + e];
      int run = block_before<BS>(own_c, sh.redi, ctot);
      if (tid == 0 && ctot < st.k) sh.at = BUCKETS;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        if (run < st.k && run + c[e] >= st.k) { sh.at = tid * PER + e; sh.count = run + c[e]; }
        run += c[e];
      }
      __syncthreads();
    };
    // kept weight of the segments from the selection, exact whatever the order
    auto add_one = [&](float l, int idx) {
      const uint64_t fx = (uint64_t)(weight(l, top, scale) * 0x1p62);
      atomicAdd((unsigned long long *)&sh.seg_lo[idx / SEG], (unsigned long long)(fx & 0xffffffffu));
      atomicAdd((unsigned long long *)&sh.seg_hi[idx / SEG], (unsigned long long)(fx >> 32));
    };
    auto add_kept = [&](const List &s) {
      for_each<BS>(s, [&](float l, int i) {
        if (l > thr || (l == thr && i <= last)) add_one(l, i);
      });
    };
    // of a list of up to LIST elements: see ranked; its kept ones added
    auto cut_list = [&](const uint64_t *list, int n, int k, double mass0, double rest) {
      double kept;
      const int n_kept = ranked<BS>(sh, list, n, k, (double)st.p, -1.0, mass0, rest, top, scale, kept);
      if (n_kept > 0) {
        thr = key_logit(sh.sorted[n_kept - 1]);
        last = key_index(sh.sorted[n_kept - 1]);
      }
      if (least > thr) { thr = least; last = INT_MAX; }
      for (int i = tid; i < n_kept; i += BS) {
        const float l = key_logit(sh.sorted[i]);
        if (l >= thr) add_one(l, key_index(sh.sorted[i]));
      }
    };
    // the same from the logits
    auto add_row = [&]() {
      for (int s = wave; s < segs; s += BS / 64) {
        const int n = min(a.V - s * SEG, SEG);
        double sum = 0.0;
        for (int i0 = lane * 4; i0 < n; i0 += STEP * 4) {
          f32x4u v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = four(x + s * SEG, i0 + j * STEP, n);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v[j][e] > thr || (v[j][e] == thr && s * SEG + i0 + j * STEP + e <= last)) sum += weight(v[j][e], top, scale);
        }
        sum = wave_reduce(sum, [](double p, double q) { return p + q; });
        if (lane == 0) sh.seg[s] = sum;
      }
    };
    bool done = st.kind == ALL;
    if (st.kind == NUCLEUS && !off) {
      // The row's histogram, from the bucket of its largest downward (a segment's starts at its own largest), and what lies
      // deeper.  Whole numbers until they are weighed.
      const int first = bucket_of(top, gf);
      const uint64_t *h = bins(a) + (size_t)row * segs * BINS;
      const double edge = (double)top * g;
      for (int b = tid; b < BINS; b += BS) {
        sh.h.lo[b] = 0;
        sh.h.cnt[b] = 0;
        sh.factor[b] = power_of_two(((double)(first - b + 1) - edge) * (LOG2E / 8.0)) * 0x1p-36;
      }
      __syncthreads();
      double deep = 0.0;
      constexpr int AHEAD = 8;
      for (int c0 = tid; c0 < segs * BINS; c0 += BS * AHEAD) {
        uint64_t v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          const int c = c0 + j * BS;
          v[j] = c < segs * BINS && sh.seg_at[c / BINS] != INT_MIN ? h[c] : 0;
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          if (v[j] == 0) continue;
          const int c = c0 + j * BS, rel = c % BINS + (first - sh.seg_at[c / BINS]);
          if (c % BINS < BINS - 1 && rel < BINS - 1) {
            atomicAdd((unsigned long long *)&sh.h.lo[rel], (unsigned long long)(v[j] & BIN_MASS));
            atomicAdd(&sh.h.cnt[rel], (uint32_t)(v[j] >> BIN_COUNT));
          } else {
            deep += (double)(v[j] & BIN_MASS) * power_of_two(((double)(first - rel + 1) - edge) * (LOG2E / 8.0));
          }
        }
      }
      deep = block_reduce<BS>(deep, sh.redd, [](double p, double q) { return p + q; }) * 0x1p-36;
      const int cnt = tid < BINS - 1 ? (int)sh.h.cnt[tid] : 0;
      const double here = tid < BINS - 1 ? (double)sh.h.lo[tid] * sh.factor[tid] : 0.0;
      double z;
      const double before = block_before<BS>(here, sh.redd, z);
      const double target = (double)st.p * (z + deep);
      const int at = block_reduce<BS>(cnt > 0 && (before < target || tid == 0) ? tid : -1, sh.redi, [](int p, int q) { return max(p, q); });
      if (at == tid) { sh.before = before; sh.count = cnt; sh.sum = z - here; }
      __syncthreads();
      int b = first - at, n_b = sh.count;
      // the least weight may cut higher: then its bucket alone is looked at, from there on all stay
      const bool by_least = st.m > 0.f && bucket_of(least, gf) > b;
      if (by_least) {
        b = bucket_of(least, gf);
        n_b = (int)sh.h.cnt[first - b];
      }
      const double mass0 = sh.before, rest = sh.sum + deep;
      // Where the target lies in what is deeper, the histogram does not tell; a bucket of too many is left to the row.
      if (z >= target && at >= 0 && n_b <= MEM) {
        const float lo_b = by_least ? least : bucket_start(b, g, top), hi_b = b == first ? INF : bucket_start(b + 1, g, top);
        if (b >= whole) {
          (void)join(lo_b, hi_b);
        } else {
          // Not in the lists: from the logits.  A thread marks which of its 32 it wants and a wave makes room for all of
          // them at once; their indexes first, the logits follow from the cache.  (Element by element with its key, 256 to a
          // request for room, a row of 128000 took 34 us.)
          constexpr int N = 8;  // 64 KiB of a workgroup on their way
          f32x4u v[N], ahead[N];
          auto request = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < N; ++j) ahead[j] = four(x, i0 + (j * BS + tid) * 4, a.V);
          };
          request(0);
          for (int i0 = 0; i0 < a.V; i0 += BS * 4 * N) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = ahead[j];
            if (i0 + BS * 4 * N < a.V) request(i0 + BS * 4 * N);
            uint32_t want = 0;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) want |= v[j][e] >= lo_b && v[j][e] < hi_b ? 1u << (j * 4 + e) : 0u;
            if (!__any(want != 0)) continue;
            const int c = __popc(want), before = wave_before(c);
            int at = 0;
            if (lane == 63) at = atomicAdd(&sh.n_mem, before + c);
            at = __shfl(at, 63) + before;
            while (want) {
              const int e = __ffs(want) - 1;
              want &= want - 1;
              if (at < MEM) sh.mem[at] = (uint64_t)(i0 + (e / 4 * BS + tid) * 4 + e % 4);
              ++at;
            }
          }
          __syncthreads();
          for (int i = tid; i < min(sh.n_mem, MEM); i += BS) {
            const int idx = (int)sh.mem[i];
            sh.mem[i] = rank_key(x[idx], idx);
          }
          __syncthreads();
        }
        const List mem{sh.mem, sh.n_mem};
        if (by_least) {
          thr = least;
          add_kept(mem);
        } else if (mem.n <= LIST) {
          // The bucket's weight anew from its elements: histogram and weights differ in the last bits, and among equal
          // logits the border may fall on an element exactly.
          cut_list(sh.mem, mem.n, INT_MAX, mass0, rest);
        } else {
          (void)cut<BS>(sh, mem, all, true, 0, (double)st.p, 0.0, mass0, rest, top, scale, lo_b, fminf(top, hi_b), thr, last);
          if (least > thr) { thr = least; last = INT_MAX; }
          add_kept(mem);
        }
        {
          // of every segment: the buckets above, and what is kept of this one
          for (int c0 = wave * 64; c0 < segs * BINS; c0 += BS * AHEAD) {
            uint64_t v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
              const int c = c0 + j * BS + lane, fs = sh.seg_at[min(c / BINS, segs - 1)];
              v[j] = c < segs * BINS && fs != INT_MIN && fs - c % BINS > b ? h[c] & BIN_MASS : 0;
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
              if (!__any(v[j] != 0)) continue;
              const int c = c0 + j * BS + lane, s = c / BINS;
              // in multiples of 2^-49: a segment's tokens weigh less than 2^14 together
              const uint64_t fx = v[j] ? (uint64_t)((double)v[j] * sh.factor[first - sh.seg_at[s] + c % BINS] * 0x1p49) : 0;
              const uint64_t sum = wave_reduce(fx, [](uint64_t p, uint64_t q) { return p + q; });
              if (lane == 0) {
                atomicAdd((unsigned long long *)&sh.seg_lo[s], (unsigned long long)((sum << 13) & 0xffffffffu));
                atomicAdd((unsigned long long *)&sh.seg_hi[s], (unsigned long long)(sum >> 19));
              }
            }
          }
        }
        done = true;
      }
    } else if (st.kind == FEW && !off && whole != INT_MAX) {
      const float from = whole == INT_MIN ? -FLT_MAX : bucket_start(whole, g, top);
      int n = join(from, INF);
      if (n > MEM && st.k <= MEM / 2) {
        // more than there is room for: the bucket of the grid that the k-th lies in, and what lies from there on
        const int first = bucket_of(top, gf);
        for (int b = tid; b < BUCKETS; b += BS) sh.h.cnt[b] = 0;
        __syncthreads();
        visit([&](const float (&l)[PIECES], const int (&)[PIECES]) {
#pragma unroll
          for (int j = 0; j < PIECES; ++j)
            if (l[j] >= from) atomicAdd(&sh.h.cnt[min(BUCKETS - 1, first - bucket_of(l[j], gf))], 1u);
        });
        if (tid == 0) sh.n_mem = 0;
        bucket_of_kth();
        if (sh.at < BUCKETS - 1) n = join(fmaxf(from, bucket_start(first - sh.at, g, top)), INF);
      }
      const List mem{sh.mem, min(n, MEM)};
      // lists of all there is and a share of its weight: the count drops none that weighs anything
      const bool enough = n <= MEM && (n >= st.k || (whole == INT_MIN && st.p < 1.f));
      const uint64_t *list = sh.mem;
      int few = n;  // elements of it
      if (enough && n > LIST && st.k <= LIST) {
        // too many to rank: those in front of and in the bucket, of a linear map, that the k-th lies in
        const double places = top > from ? (BUCKETS - 1) / ((double)top - (double)from) : 0.0;
        auto bucket = [&](float l) { return min(BUCKETS - 1, (int)(((double)top - (double)l) * places)); };
        for (int b = tid; b < BUCKETS; b += BS) sh.h.cnt[b] = 0;
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
        for_each<BS>(mem, [&](float l, int) { atomicAdd(&sh.h.cnt[bucket(l)], 1u); });
        __syncthreads();
        bucket_of_kth();
        few = sh.count;
        list = sh.list;
        if (few <= LIST)
          for_each<BS>(mem, [&](float l, int i) {
            if (bucket(l) <= sh.at) sh.list[atomicAdd(&sh.n_list, 1)] = rank_key(l, i);
          });
        __syncthreads();
      }
      const bool in_list = enough && few <= LIST;
      if (in_list) {
        cut_list(list, few, st.k, 0.0, 0.0);
        done = thr > lowest;  // else a segment without a list may have one of them
      } else if (enough) {
        const double w = cut<BS>(sh, mem, all, false, st.k, -1.0, 0.0, 0.0, 0.0, top, scale, hint, top, thr, last);
        if (st.p < 1.f) (void)cut<BS>(sh, mem, all, true, 0, -1.0, (double)st.p * w, 0.0, 0.0, top, scale, hint, top, thr, last);
        done = thr > lowest;
        if (least > thr) { thr = least; last = INT_MAX; }
      } else if (n <= MEM && n < st.k && (st.k == INT_MAX || st.p >= 1.f) && st.m > 0.f && (whole == INT_MIN || bucket_of(least, gf) >= whole)) {
        thr = least;
        done = true;
      }
      if (done && !in_list) add_kept(mem);
    }
    if (!done) {
      // the whole row, refinement by refinement
      __syncthreads();
      for (int s = tid; s < segs; s += BS) { sh.seg_lo[s] = 0; sh.seg_hi[s] = 0; }
      thr = -INF; last = INT_MAX;
      double w = -1.0;
      if (st.k != INT_MAX) w = cut<BS>(sh, all, all, false, st.k, -1.0, 0.0, 0.0, 0.0, top, scale, hint, top, thr, last);
      if (st.p < 1.f)
        (void)cut<BS>(sh, all, all, true, 0, w < 0.0 ? (double)st.p : -1.0, (double)st.p * w, 0.0, 0.0, top, scale, hint, top, thr, last);
      if (least > thr) { thr = least; last = INT_MAX; }
      add_row();
    }
    __syncthreads();
    // kept weight in front of every segment; the segment that the target falls into (every wave by itself)
    const double w0 = sh.seg[lane] + from_fixed(sh.seg_lo[lane], sh.seg_hi[lane]);
    const double w1 = sh.seg[lane + 64] + from_fixed(sh.seg_lo[lane + 64], sh.seg_hi[lane + 64]);
    const double z0 = wave_reduce(w0, [](double p, double q) { return p + q; });
    const double z = z0 + wave_reduce(w1, [](double p, double q) { return p + q; });
    d.thr = thr; d.last = last; d.z = z;
    if (!a.u && wave == 0) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (lane + e * 64 < segs) stats(a)[(size_t)row * segs + lane + e * 64].z = e ? w1 : w0;
    }
    if (a.u) {
      const double target = target_of(u, z), b0 = wave_before(w0), b1 = z0 + wave_before(w1);
      const uint64_t in0 = __ballot(w0 > 0.0 && b0 <= target), in1 = __ballot(w1 > 0.0 && b1 <= target);
      if (in0 | in1) {
        const int seg = in1 ? 127 - __clzll(in1) : 63 - __clzll(in0);
        const double seg_before = __shfl(seg < 64 ? b0 : b1, seg & 63);
        const int n = min(a.V - seg * SEG, SEG), n_steps = (n + STEP - 1) / STEP;
        const float *xs = x + seg * SEG;
        auto weights = [&](const f32x4u &l, int i, double (&w)[4]) {
          double sum = 0.0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = 0.0;
            if (l[e] > thr || (l[e] == thr && seg * SEG + i + e <= last)) w[e] = weight(l[e], top, scale);
            sum += w[e];
          }
          return sum;
        };
        constexpr int PER = SEG / STEP / (BS / 64);  // steps of a wave
        f32x4u v[PER];
        double w[4];
#pragma unroll
        for (int j = 0; j < PER; ++j) v[j] = four(xs, (j * (BS / 64) + wave) * STEP + lane * 4, n);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const int s = j * (BS / 64) + wave;
          const double sum = wave_reduce(weights(v[j], s * STEP + lane * 4, w), [](double p, double q) { return p + q; });
          if (lane == 0) sh.step[s] = sum;
        }
        __syncthreads();
        // the step: the last that starts at or before the target (rounding may put all behind it: the first of weight)
        const double sum = lane < n_steps ? sh.step[lane] : 0.0, start = seg_before + wave_before(sum);
        const uint64_t some = __ballot(sum > 0.0), fit = __ballot(sum > 0.0 && start <= target);
        if (some) {
          const int s = fit ? 63 - __clzll(fit) : __ffsll((unsigned long long)some) - 1, i = s * STEP + lane * 4;
          writer = s % (BS / 64);
          if (wave == writer) {  // it has the step's logits
            f32x4u l = v[0];
#pragma unroll
            for (int j = 1; j < PER; ++j)
              if (s == j * (BS / 64) + wave) l = v[j];
            const double mine = weights(l, i, w);
            double run = __shfl(start, s) + wave_before(mine);
            int id = -1, any = -1;
            double wid = 0.0, wany = 0.0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              run += w[e];
              if (w[e] > 0.0) { any = seg * SEG + i + e; wany = w[e]; }
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
  }
  if (!a.u && !(arg != INT_MAX && st.kind != ONE && top > -INF)) {  // the first alone
    __syncthreads();
    for (int s = tid; s < segs; s += BS) stats(a)[(size_t)row * segs + s].z = arg != INT_MAX && s == arg / SEG ? 1.0 : 0.0;
  }
  if (wave == writer && lane == 0) {
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
  // of the four tokens from i on, whose logits are lp and lq
  __device__ __forceinline__ double at(const f32x4u &lp, const f32x4u &lq, int i, double (&r)[4]) const {
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r[e] = 0.0;
      if (kept_by(pd, lp[e], i + e) && i + e != dead) {
        r[e] = weight(lp[e], pd.top, p_t) * p_z;
        if (q) r[e] = fmax(r[e] - share_of(qd, q_t, q_z, lq[e], i + e), 0.0);
      }
      sum += r[e];
    }
    return sum;
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

// Four consecutive tokens of a lane in each of the segment's steps of 256; of NW waves this one's.
template <int NW, class F> __device__ __forceinline__ void rest_steps(const Rest &r, int i0, int V, F f) {
  constexpr int PER = SEG / STEP / NW, AHEAD = PER < 4 ? PER : 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int j0 = 0; j0 < PER; j0 += AHEAD) {
    f32x4u p[AHEAD], q[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = i0 + ((j0 + j) * NW + wave) * STEP + lane * 4;
      p[j] = four(r.p, i, V);
      q[j] = r.q ? four(r.q, i, V) : p[j];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int s = (j0 + j) * NW + wave;
      double w[4];
      f(s, r.at(p[j], q[j], i0 + s * STEP + lane * 4, w));
    }
  }
}

// One workgroup per (sequence, segment of the vocabulary): the segment's rest, and by the first one the accepted slots.  Without
// a draft distribution at that place the rest is the target's own but for one token, and a segment without it weighs what the row kernel
// found (read again, 128 rows of 152064 took 38 us).
__global__ __launch_bounds__(256) void rest_sum_kernel(const SampleAcceptArgs a, int segs) {
  __shared__ int redi[4];
  __shared__ double redd[4];
  const int b = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int n = accepted(a, b, redi);
  const Rest r = rest_of(a, b, n);
  double sum = 0.0;
  if (!r.q && (r.dead < 0 || r.dead / SEG != seg)) {
    sum = static_cast<const SegStat *>(a.stat)[((size_t)b * (a.k + 1) + n) * segs + seg].z * r.p_z;
  } else {
    rest_steps<4>(r, seg * SEG, a.V, [&](int, double s) { sum += s; });
    sum = block_reduce<256>(sum, redd, [](double x, double y) { return x + y; });
  }
  if (threadIdx.x == 0) {
    a.part[(size_t)b * segs + seg] = sum;
    if (seg == 0) a.n[b] = n;
  }
}

// One workgroup per sequence: the token behind the accepted slots.
__global__ __launch_bounds__(1024) void rest_draw_kernel(const SampleAcceptArgs a, int segs) {
  __shared__ double part[MAX_SEGS], step[SEG / STEP];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.n[b];
  Rest r = rest_of(a, b, n);
  if (tid < MAX_SEGS) part[tid] = tid < segs ? a.part[(size_t)b * segs + tid] : 0.0;
  __syncthreads();
  double w0 = part[lane], w1 = part[lane + 64];
  auto add = [](double p, double q) { return p + q; };
  double z0 = wave_reduce(w0, add), z = z0 + wave_reduce(w1, add);
  if (!(z > 0.0)) {
    // nothing is left (target and draft agree, and the drafted token has no share in either): the target's own
    r.q = nullptr; r.dead = -1;
    __syncthreads();
    for (int s = wave; s < segs; s += 16) {
      double sum = 0.0, w[4];
      for (int i = s * SEG + lane * 4; i < min(a.V, (s + 1) * SEG); i += STEP) {
        const f32x4u p = four(r.p, i, a.V);
        sum += r.at(p, p, i, w);
      }
      sum = wave_reduce(sum, add);
      if (lane == 0) part[s] = sum;
    }
    __syncthreads();
    w0 = part[lane]; w1 = part[lane + 64];
    z0 = wave_reduce(w0, add); z = z0 + wave_reduce(w1, add);
  }
  const double target = target_of(a.u_sample[b], z), b0 = wave_before(w0), b1 = z0 + wave_before(w1);
  const uint64_t in0 = __ballot(w0 > 0.0 && b0 <= target), in1 = __ballot(w1 > 0.0 && b1 <= target);
  int id = max(r.pd.id, 0);
  if (in0 | in1) {
    const int seg = in1 ? 127 - __clzll(in1) : 63 - __clzll(in0), i0 = seg * SEG;
    const double seg_before = __shfl(seg < 64 ? b0 : b1, seg & 63);
    rest_steps<16>(r, i0, a.V, [&](int s, double mine) {
      const double sum = wave_reduce(mine, add);
      if (lane == 0) step[s] = sum;
    });
    __syncthreads();
    if (wave == 0) {
      // the step: the last that starts at or before the target (rounding may put all behind it: the first of weight)
      const double sum = lane < SEG / STEP ? step[lane] : 0.0, start = seg_before + wave_before(sum);
      const uint64_t some = __ballot(sum > 0.0), fit = __ballot(sum > 0.0 && start <= target);
      if (some) {
        const int s = fit ? 63 - __clzll(fit) : __ffsll((unsigned long long)some) - 1, i = i0 + s * STEP + lane * 4;
        const f32x4u p = four(r.p, i, a.V);
        double w[4];
        const double mine = r.at(p, r.q ? four(r.q, i, a.V) : p, i, w);
        double run = __shfl(start, s) + wave_before(mine);
        int hit = -1, any = -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          run += w[e];
          if (w[e] > 0.0) any = i + e;
          if (hit < 0 && w[e] > 0.0 && run > target) hit = any;
        }
        const uint64_t over = __ballot(hit >= 0), has = __ballot(any >= 0);
        id = __shfl(over ? hit : any, over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll(has));
      }
    }
  }
  int32_t *tokens = a.tokens + (size_t)b * (a.k + 1);
  if (tid < n) tokens[tid] = a.draft[(size_t)b * a.k + tid];
  if (tid == 0) {
    tokens[n] = id;
    a.accept[b] = n + 1;
  }
}

// the row kernel's LDS is more than a launch may ask for by default
hipError_t ensure_row_lds() {
  static bool raised[64] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (raised[dev]) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&row_kernel<512>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
  if (e == hipSuccess) raised[dev] = true;
  return e;
}

}  // namespace

hipError_t launch_sample_accept(const SampleAcceptArgs &a, hipStream_t s) {
  const int segs = (a.V + SAMPLE_SEG - 1) / SAMPLE_SEG;
  rest_sum_kernel<<<a.B * segs, 256, 0, s>>>(a, segs);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  rest_draw_kernel<<<a.B, 1024, 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t sample_prepare_device() { return ensure_row_lds(); }

hipError_t launch_sample(const SampleArgs &a, hipStream_t s) {
  segment_kernel<<<a.M * a.segs, 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = ensure_row_lds();
  if (e != hipSuccess) return e;
  row_kernel<512><<<a.M, 512, sizeof(Shared), s>>>(a);
  return hipGetLastError();
}

}  // namespace sf
