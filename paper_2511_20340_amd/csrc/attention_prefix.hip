// Attention of a batch whose sequences all continue one shared prefix, for gfx950.
//
// A query row attends to the P keys of the prefix, then to its sequence's own keys and block.  softmax over the union is
// the join of softmaxes over the parts: with (m, l, O) the running maximum, sum and weighted values of each part,
//   m = max m_i,  l = sum l_i 2^(m_i - m),  O = sum O_i 2^(m_i - m) / l.
// The own part is what the attention of the steps computes (attention.hip), sequence by sequence, at the rate of memory.  For
// the prefix the rows of ALL sequences that share a kv head are one matrix: its keys and values are read once per 32 * waves
// rows instead of once per sequence, which makes that part a matrix product, bound by the matrix cores and the softmax between
// the two products.
#include "attention_rows.h"
#include <algorithm>
#include <type_traits>

namespace sf {
namespace {

constexpr int STEP_TILES = 2;  // 32-key tiles between two meetings of a workgroup's waves

#ifdef __HIP_DEVICE_COMPILE__
typedef __amdgpu_buffer_rsrc_t buffer_t;
#endif

// Both parts for 128 x 5 rows of 40 / 8 heads of 128 over 8192 keys and 32 to 512 own ones take 144 us, 0.77 PFLOP/s (138
// in a step, with the rotation and the append): the matrix instructions of a stage and the exponentials between them do not overlap
// within a wave, and two waves to a SIMD fill a part of each other's gaps.  64 rows to a wave, which halves the LDS reads, take 200 (registers); the small batches are latency: 32 x 5
// rows over 2048 keys of heads of 64 13 us.
//
// One workgroup: 128 rows of one kv head, chunk_tiles tiles of the prefix.  The cache's tiles are MFMA operands as they are: they
// go to LDS by direct loads, two stages of STEP_TILES tiles, and every wave reads the fragments it needs from there.
template <int HD> constexpr int PREFIX_LDS_BYTES = 2 * 2 * STEP_TILES * HD * 64;
template <int HD, int FUSE>
__device__ __forceinline__ void prefix_rows(const int id, char *smem, const bf16_t *__restrict__ Q, const void *Pk, const void *Pv,
                                            float *__restrict__ part_o, float *__restrict__ part_ml, int R, int rows, int Hq,
                                            int Hkv, int len, int cap, int chunk_tiles, int n_chunks, float scale_log2e,
                                            const float2 *__restrict__ table) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int KS = HD / 16, NT = HD / 32, NW = 4;
  constexpr int TILE = HD * 64;                    // bytes of a 32-key tile
  constexpr int STAGE = 2 * STEP_TILES * TILE;     // K tiles, then V tiles
  constexpr int LOADS = STAGE / 1024 / NW;         // of one wave for a stage
  // kv heads fastest: eight of them are eight XCDs, each with its head's keys in an L2 of its own; then the rows of a chunk
  const int tiles_r = rows / (32 * NW), g = id % Hkv, rt = id / Hkv % tiles_r, chunk = id / Hkv / tiles_r;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int n_tiles = (len + TK - 1) / TK, t0 = chunk * chunk_tiles, t1 = min(n_tiles, t0 + chunk_tiles);
  const int steps = (t1 - t0 + STEP_TILES - 1) / STEP_TILES;
  const size_t slab = (size_t)g * (cap / TK) * TILE;
  const buffer_t buf_k = __builtin_amdgcn_make_buffer_rsrc((char *)const_cast<void *>(Pk) + slab, 0, (uint32_t)n_tiles * TILE, 0x00020000);
  const buffer_t buf_v = __builtin_amdgcn_make_buffer_rsrc((char *)const_cast<void *>(Pv) + slab, 0, (uint32_t)n_tiles * TILE, 0x00020000);
  auto load = [&](int step) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = wave * LOADS + i, tile = (u % (STAGE / 2048)) / (TILE / 1024), unit = u % (TILE / 1024);
      char *to = smem + (step & 1) * STAGE + u * 1024;
      const uint32_t at = (uint32_t)min(t0 + step * STEP_TILES + tile, n_tiles - 1) * TILE + unit * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(u < STAGE / 2048 ? buf_k : buf_v, (__attribute__((address_space(3))) void *)to, 16,
                                               lane * 16, at, 0, 0);
    }
  };
  load(0);

  // Q^T operand: lane (n, h), k-step s holds features [(2s+h)*8, +8) of its row
  const int r = (rt * NW + wave) * 32 + n;
  const bool row_ok = r < R;
  const bool idle = (rt * NW + wave) * 32 >= R;  // few rows: the other waves only load
  const int bi = row_ok ? r / G : 0, qh = g * G + (row_ok ? r % G : 0);  // bi = b * n_q + block row
  bf16x8 qf[KS];
  if (FUSE) {
    const uint4 *qp = reinterpret_cast<const uint4 *>(Q + ((size_t)bi * (Hq + 2 * Hkv) + qh) * HD);
    const float2 *tab = table + (size_t)bi * (HD / 2);
#pragma unroll
    for (int s = 0; s < KS / 2; ++s) {
      const uint4 lo4 = row_ok ? qp[2 * s + h] : make_uint4(0, 0, 0, 0);
      const uint4 hi4 = row_ok ? qp[2 * (s + KS / 2) + h] : make_uint4(0, 0, 0, 0);
      const bf16x8 lo = __builtin_bit_cast(bf16x8, lo4), hi = __builtin_bit_cast(bf16x8, hi4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float q0, q1;
        rope_pair((float)lo[i], (float)hi[i], tab[(2 * s + h) * 8 + i], q0, q1);
        qf[s][i] = (__bf16)q0;
        qf[s + KS / 2][i] = (__bf16)q1;
      }
    }
  } else {
    const uint4 *qp = reinterpret_cast<const uint4 *>(Q + ((size_t)bi * Hq + qh) * HD);
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, row_ok ? qp[2 * s + h] : make_uint4(0, 0, 0, 0));
  }

  f32x16 acc[NT];
  float m_run = NEG_INF, l_run = 0.f;
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[c][v] = 0.f;
  const int end = min(len, t1 * TK);  // keys of this chunk

  auto tiles = [&](int step, auto tail_c) __attribute__((always_inline)) {
    constexpr bool TAIL = decltype(tail_c)::value;  // the stage holds keys behind the end: they may be anything (even NaN)
    const bf16x8 *kb = reinterpret_cast<const bf16x8 *>(smem + (step & 1) * STAGE) + lane;
    const bf16x8 *vb = kb + STEP_TILES * TILE / 16;
    const int p0 = (t0 + step * STEP_TILES) * TK;
    // All of the keys' fragments on their way, then products that do not wait for one another next to each other (fragment by
    // fragment, as the compiler orders them by itself: 163 us where this takes 134).
    bf16x8 kf[STEP_TILES][KS], vf[STEP_TILES][KS];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int t = 0; t < STEP_TILES; ++t) kf[t][s] = kb[(t * KS + s) * 64];
    __builtin_amdgcn_sched_barrier(0);
    f32x16 sc[STEP_TILES];
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[t][v] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int t = 0; t < STEP_TILES; ++t)
        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t][s], qf[s], sc[t], 0, 0, 0);
    // the values' fragments arrive while the softmax runs
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s) vf[t][s] = vb[(t * KS + s) * 64];
    __builtin_amdgcn_sched_barrier(0);
    if (TAIL) {
#pragma unroll
      for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (p0 + t * TK + c_row(v, h) >= end) sc[t][v] = NEG_INF;
    }
    float mx = NEG_INF;
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sc[t][v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale_log2e;
    // The maximum follows the scores in strides: as long as they stay below 2^8 times its weight, sums and products in float
    // lose nothing by an old one, and the accumulators need not be scaled.  A row goes by its own scores, which decide how its p are
    // rounded; the wave's other rows (of other sequences) only by whether the branch is taken.
    const bool rises = mx > m_run + 8.f;
    if (__any(rises)) {
      const float m_new = rises ? mx : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == NEG_INF ? 0.f : m_new));
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[c][v] *= alpha;
    }
    const float m_use = m_run == NEG_INF ? 0.f : m_run;
    bf16x8 pf[STEP_TILES][2];
    float psum[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][v], scale_log2e, -m_use));
        psum[v & 1] += p;
        pf[t][v >> 3][v & 7] = (__bf16)p;
      }
    l_run += psum[0] + psum[1];
    if (TAIL) {
#pragma unroll
      for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const uint4 w4 = __builtin_bit_cast(uint4, vf[t][s]);
          uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (p0 + t * TK + 16 * (s / NT) + 8 * (e >> 2) + 4 * h + (e & 3) >= end) w[e >> 1] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
          vf[t][s] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < NT; ++c)
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][u * NT + c], pf[t][u], acc[c], 0, 0, 0);
  };
  // this wave's loads of the stage have landed, everyone's have behind the barrier; the other stage has been read by all
  auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  const int whole = (end - t0 * TK) / (STEP_TILES * TK) == steps ? steps : steps - 1;  // steps without such keys
  for (int step = 0; step < whole; ++step) {
    meet();
    if (step + 1 < steps) load(step + 1);
    if (!idle) tiles(step, std::integral_constant<bool, false>{});
  }
  if (whole < steps) {
    meet();
    if (!idle) tiles(whole, std::integral_constant<bool, true>{});
  }
  const float l = l_run + __shfl_xor(l_run, 32);
  if (!row_ok) return;
  const size_t at = ((size_t)g * n_chunks + chunk) * rows + r;
  if (h == 0) *reinterpret_cast<float2 *>(part_ml + at * 2) = make_float2(m_run, l);
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<float4 *>(part_o + at * HD + 32 * c + 8 * j + 4 * h) =
          make_float4(acc[c][4 * j], acc[c][4 * j + 1], acc[c][4 * j + 2], acc[c][4 * j + 3]);
#endif
}

// Both parts in one launch: the prefix's workgroups, bound by the matrix cores, first, those of the own keys, bound by memory and
// short, where they leave room and at the end (dealt out in turn, or the own ones first: 171 and 157 us where this takes 147).
struct PrefixKernelArgs {
  const bf16_t *q;
  const void *pk, *pv;
  const uint4 *kc, *vc;
  const int32_t *kv_len, *order, *slots;
  const float2 *table;
  float *pre_o, *pre_ml, *own_o, *own_ml;
  int B, n_q, Hq, Hkv, cap, mode, own_tiles, own_chunks, n_rt;  // own keys
  int len, pcap, pre_tiles, pre_chunks, rows;                   // prefix
  int pre_blocks, own_blocks;
  float scale_log2e;
};
template <int HD> constexpr int BOTH_LDS_BYTES = ATTN_LDS_BYTES<HD> > PREFIX_LDS_BYTES<HD> ? ATTN_LDS_BYTES<HD> : PREFIX_LDS_BYTES<HD>;
template <int HD, int FUSE, int ONCE>
__global__ __launch_bounds__(256, 2) void prefix_attn_kernel(const PrefixKernelArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  if ((int)blockIdx.x < a.pre_blocks) {
    prefix_rows<HD, FUSE>(blockIdx.x, smem, a.q, a.pk, a.pv, a.pre_o, a.pre_ml, a.B * a.n_q * (a.Hq / a.Hkv), a.rows, a.Hq, a.Hkv,
                          a.len, a.pcap, a.pre_tiles, a.pre_chunks, a.scale_log2e, a.table);
    return;
  }
  const int id = blockIdx.x - a.pre_blocks;
  const int y = a.Hkv * a.n_rt;
  attn_rows<HD, FUSE, ONCE, 1>(make_uint3(id % a.own_chunks, id / a.own_chunks % y, id / a.own_chunks / y), reinterpret_cast<float *>(smem),
                               a.q, a.kc, a.vc, a.kv_len, nullptr, a.own_o, a.own_ml, a.n_q, a.Hq, a.Hkv, a.cap, a.mode,
                               a.own_tiles, a.own_chunks, a.n_rt, a.scale_log2e, a.table, a.order, a.slots);
}

// Joins the partials of the prefix and of the own keys: 32 lanes per query row, 8 rows per workgroup, every lane HD / 32
// features.
template <int HD>
__global__ __launch_bounds__(256) void prefix_combine_kernel(const float *__restrict__ pre_o, const float *__restrict__ pre_ml,
                                                             int pre_chunks, int pre_rows, const float *__restrict__ own_o,
                                                             const float *__restrict__ own_ml, int own_chunks, int own_rows,
                                                             int chunk_tiles, const int32_t *__restrict__ kv_len,
                                                             bf16_t *__restrict__ O, int total_rows, int n_q, int Hq, int Hkv,
                                                             int cap) {
  constexpr int E = HD / 32;
  typedef float vec __attribute__((ext_vector_type(E)));
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;  // row = (b, block row, query head)
  if (row >= total_rows) return;
  const int hq = row % Hq, bi = row / Hq, i = bi % n_q, b = bi / n_q;
  const int G = Hq / Hkv, g = hq / G;
  const size_t pre = (size_t)g * pre_chunks * pre_rows + (size_t)bi * G + hq % G;
  const size_t own = ((size_t)b * Hkv + g) * own_chunks * own_rows + i * G + hq % G;
  const int n_tiles = (max(0, min(kv_len[b], cap - n_q)) + n_q + TK - 1) / TK;
  const int sc = min((n_tiles + chunk_tiles - 1) / chunk_tiles, own_chunks), n = pre_chunks + sc;
  float m = NEG_INF, l = 0.f;
  vec o = 0.f;
  for (int c = 0; c < n; ++c) {
    const bool p = c < pre_chunks;
    const size_t at = p ? pre + (size_t)c * pre_rows : own + (size_t)(c - pre_chunks) * own_rows;
    const float2 ml = *reinterpret_cast<const float2 *>((p ? pre_ml : own_ml) + at * 2);
    const vec x = *reinterpret_cast<const vec *>((p ? pre_o : own_o) + at * HD + lane * E);
    const float m_new = fmaxf(m, ml.x), m_use = m_new == NEG_INF ? 0.f : m_new;
    const float f0 = __builtin_amdgcn_exp2f(m - m_use), f1 = __builtin_amdgcn_exp2f(ml.x - m_use);
    l = l * f0 + ml.y * f1;
    o = o * f0 + x * f1;
    m = m_new;
  }
  o *= 1.f / l;
  uint32_t *out = reinterpret_cast<uint32_t *>(O + (size_t)row * HD + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) out[e / 2] = pack2bf(o[e], o[e + 1]);
}

// fp32 (small models): one workgroup per (query head, block row, sequence) walks the prefix, then the own keys, in pieces
// of CK with a workgroup-wide running maximum, as the fp32 attention of the steps does.
constexpr int CK = 512;
__global__ __launch_bounds__(256) void prefix_f32_kernel(const float *__restrict__ Q, const float *__restrict__ Pk,
                                                         const float *__restrict__ Pv, int plen, int pcap,
                                                         const float *__restrict__ Kc, const float *__restrict__ Vc,
                                                         const int32_t *__restrict__ kv_len, float *__restrict__ O, int n_q,
                                                         int Hq, int Hkv, int hd, int cap, int mode, float scale,
                                                         const int32_t *__restrict__ slots) {
  __shared__ __attribute__((aligned(16))) float sq[256];
  __shared__ float sc[CK], red[8];
  __shared__ f32x4 so[256];
  const int hq = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = hq / (Hq / Hkv);
  const int len = max(0, min(kv_len[b], cap - n_q)), own = len + (mode == SF_MASK_BIDIR ? n_q : i + 1);
  const size_t slab = ((size_t)(slots ? slots[b] : b) * Hkv + g) * (size_t)cap * hd, pslab = (size_t)g * pcap * hd;
  const size_t row = (((size_t)b * n_q + i) * Hq + hq) * hd;
  if (tid < hd) sq[tid] = Q[row + tid];
  __syncthreads();
  const int cols = hd / 4, groups = 256 / cols, col = tid % cols, grp = tid / cols;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m_run = NEG_INF, l_run = 0.f;
  for (int part = 0; part < 2; ++part) {
    const float *K = part ? Kc + slab : Pk + pslab, *V = part ? Vc + slab : Pv + pslab;
    const int total = part ? own : plen;
    for (int p0 = 0; p0 < total; p0 += CK) {
      const int nk = min(CK, total - p0);
      float mx = NEG_INF;
      for (int x = tid >> 1; x < nk; x += 128) {
        const float *kr = K + (size_t)(p0 + x) * hd + (tid & 1) * 4, *qr = sq + (tid & 1) * 4;
        float s = 0.f;
        for (int e = 0; e < hd; e += 8) {
          const f32x4 k4 = *reinterpret_cast<const f32x4 *>(kr + e), q4 = *reinterpret_cast<const f32x4 *>(qr + e);
          s += k4[0] * q4[0] + k4[1] * q4[1] + k4[2] * q4[2] + k4[3] * q4[3];
        }
        s = (s + __shfl_xor(s, 1)) * scale;
        if ((tid & 1) == 0) sc[x] = s;
        mx = fmaxf(mx, s);
      }
      for (int w = 32; w; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w));
      if (lane == 0) red[wave] = mx;
      __syncthreads();
      const float m_new = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m_run);
      const float m_use = m_new == NEG_INF ? 0.f : m_new;
      float sum = 0.f;
      for (int x = tid; x < nk; x += 256) {
        const float p = expf(sc[x] - m_use);
        sc[x] = p;
        sum += p;
      }
      for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w);
      if (lane == 0) red[4 + wave] = sum;
      __syncthreads();
      const float alpha = expf(m_run - m_use);
      l_run = l_run * alpha + ((red[4] + red[5]) + (red[6] + red[7]));
      m_run = m_new;
      o *= alpha;
      if (grp < groups)
        for (int x = grp; x < nk; x += groups)
          o += sc[x] * *reinterpret_cast<const f32x4 *>(V + (size_t)(p0 + x) * hd + col * 4);
      __syncthreads();
    }
  }
  so[tid] = o;
  __syncthreads();
  if (tid < cols) {
    for (int x = 1; x < groups; ++x) o += so[x * cols + tid];
    *reinterpret_cast<f32x4 *>(O + row + tid * 4) = o / l_run;
  }
}

template <int HD, int FUSE, int ONCE> hipError_t run_prefix(const PrefixKernelArgs &a, hipStream_t s) {
  static bool raised[64] = {};  // LDS beyond what a launch may ask for by default
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!raised[dev]) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&prefix_attn_kernel<HD, FUSE, ONCE>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, BOTH_LDS_BYTES<HD>);
    if (e != hipSuccess) return e;
    raised[dev] = true;
  }
  prefix_attn_kernel<HD, FUSE, ONCE><<<a.pre_blocks + a.own_blocks, 256, BOTH_LDS_BYTES<HD>, s>>>(a);
  return hipGetLastError();
}

template <int HD> hipError_t pick_prefix(const PrefixKernelArgs &a, bool fuse, hipStream_t s) {
  if (fuse) return a.n_rt == 1 ? run_prefix<HD, 1, 1>(a, s) : run_prefix<HD, 1, 0>(a, s);
  return a.n_rt == 1 ? run_prefix<HD, 0, 1>(a, s) : run_prefix<HD, 0, 0>(a, s);
}

}  // namespace

PrefixPlan prefix_plan(int B, int n_q, int Hq, int Hkv, int len, int plan_rows) {
  const int G = Hq / Hkv, n_tiles = (len + TK - 1) / TK;
  PrefixPlan p;
  p.rows = (B * n_q * G + 127) / 128 * 128;
  const int row_tiles = (plan_rows * G + 127) / 128;
  // As many workgroups as the chip holds at once (two to a compute unit), not more: a chunk more costs its partials.  128 x 5
  // rows, 8192 keys, in 1, 2, 3, 4 chunks: 173, 157, 163, 161 us with the join; 37 x 4 rows, 1500 keys: 38, 27, 25, 25, in 5
  // and 6 26 and 26.  Below 12 tiles to a chunk nothing is gained unless the rows are one tile and all is latency.
  const int want = std::max(1, 512 / (Hkv * row_tiles));
  p.chunk_tiles = std::max((n_tiles + want - 1) / want, row_tiles == 1 ? 8 : 12);
  p.chunk_tiles = (p.chunk_tiles + STEP_TILES - 1) / STEP_TILES * STEP_TILES;
  p.n_chunks = (n_tiles + p.chunk_tiles - 1) / p.chunk_tiles;
  return p;
}

size_t prefix_rows_bound(int B, int n_q, int Hq, int Hkv) {
  const size_t R = (size_t)B * n_q * (Hq / Hkv);
  // rows x chunks, with at most 512 / (Hkv x row tiles) chunks rounded up: one more of all rows, or 512 row tiles in all
  return (size_t)Hkv * ((R + 127) / 128 * 128 + 128 * (512 / Hkv + 1));
}

hipError_t launch_prefix_bf16(const PrefixArgs &a, hipStream_t s) {
  const AttnArgs &o = a.own;
  PrefixKernelArgs k{};
  k.q = (const bf16_t *)(o.qkv ? o.qkv : o.q);
  k.pk = a.pk; k.pv = a.pv; k.kc = (const uint4 *)o.kc; k.vc = (const uint4 *)o.vc;
  k.kv_len = o.kv_len; k.order = o.order; k.slots = o.slots; k.table = o.table;
  k.pre_o = a.part_o; k.pre_ml = a.part_ml; k.own_o = o.part_o; k.own_ml = o.part_ml;
  k.B = o.B; k.n_q = o.n_q; k.Hq = o.Hq; k.Hkv = o.Hkv; k.cap = o.cap; k.mode = o.mode;
  k.own_tiles = o.chunk_tiles; k.own_chunks = o.n_chunks; k.n_rt = (o.Hq / o.Hkv * o.n_q + 31) / 32;
  k.len = a.len; k.pcap = a.cap; k.pre_tiles = a.chunk_tiles; k.pre_chunks = a.n_chunks; k.rows = a.rows;
  k.pre_blocks = o.Hkv * (a.rows / 128) * a.n_chunks;
  k.own_blocks = o.n_chunks * o.Hkv * k.n_rt * o.B;
  k.scale_log2e = 1.4426950408889634f / sqrtf((float)o.hd);
  return o.hd == 128 ? pick_prefix<128>(k, o.qkv != nullptr, s) : pick_prefix<64>(k, o.qkv != nullptr, s);
}

hipError_t launch_prefix_combine(const PrefixArgs &a, hipStream_t s) {
  const AttnArgs &o = a.own;
  const int total = o.B * o.n_q * o.Hq, own_rows = (o.Hq / o.Hkv * o.n_q + 31) / 32 * 32;
  auto launch = [&](auto kernel) {
    kernel<<<(total + 7) / 8, 256, 0, s>>>(a.part_o, a.part_ml, a.n_chunks, a.rows, o.part_o, o.part_ml, o.n_chunks, own_rows,
                                           o.chunk_tiles, o.kv_len, (bf16_t *)o.out, total, o.n_q, o.Hq, o.Hkv, o.cap);
  };
  if (o.hd == 128) launch(&prefix_combine_kernel<128>); else launch(&prefix_combine_kernel<64>);
  return hipGetLastError();
}

hipError_t launch_prefix_f32(const PrefixArgs &a, hipStream_t s) {
  const AttnArgs &o = a.own;
  prefix_f32_kernel<<<dim3(o.Hq, o.n_q, o.B), 256, 0, s>>>((const float *)o.q, (const float *)a.pk, (const float *)a.pv, a.len,
                                                           a.cap, (const float *)o.kc, (const float *)o.vc, o.kv_len,
                                                           (float *)o.out, o.n_q, o.Hq, o.Hkv, o.hd, o.cap, o.mode,
                                                           1.f / sqrtf((float)o.hd), o.slots);
  return hipGetLastError();
}

}  // namespace sf
