// Attention of a batch whose sequences all continue one shared prefix, for gfx950.
//
// A query row attends to the P keys of the prefix, then to its sequence's own keys and block.  softmax over the union is
// the join of softmaxes over the parts: with (m, l, O) the running maximum, sum and weighted values of each part,
//   m = max m_i,  l = sum l_i 2^(m_i - m),  O = sum O_i 2^(m_i - m) / l.
// The own part is what the attention of the steps computes (attention.hip), sequence by sequence, at the rate of memory.  For
// the prefix the rows of ALL sequences that share a kv head are one matrix: its keys and values are read once per 32 * waves
// rows instead of once per sequence, which makes that part a matrix product, bound by the matrix cores and the softmax between
// the two products.
#include "sf_internal.h"

namespace sf {
namespace {

constexpr float NEG_INF = -__builtin_huge_valf();
constexpr int STEP_TILES = 2;  // 32-key tiles between two meetings of a workgroup's waves

#ifdef __HIP_DEVICE_COMPILE__
typedef __amdgpu_buffer_rsrc_t buffer_t;
#endif

// One workgroup: 32 * NW rows of one kv head, chunk_tiles tiles of the prefix.  The cache's tiles are MFMA operands as they
// are: they go to LDS by direct loads, two stages of STEP_TILES tiles, and every wave reads the fragments it needs from there.
template <int HD, int NW, int FUSE>
__global__ __launch_bounds__(64 * NW, 2) void prefix_bf16_kernel(const bf16_t *__restrict__ Q, const void *Pk, const void *Pv,
                                                                 float *__restrict__ part_o, float *__restrict__ part_ml, int R,
                                                                 int rows, int n_q, int Hq, int Hkv, int len, int cap,
                                                                 int chunk_tiles, int n_chunks, float scale_log2e,
                                                                 const float2 *__restrict__ table) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int KS = HD / 16, NT = HD / 32;
  constexpr int TILE = HD * 64;                    // bytes of a 32-key tile
  constexpr int STAGE = 2 * STEP_TILES * TILE;     // K tiles, then V tiles
  constexpr int LOADS = STAGE / 1024 / NW;         // of one wave for a stage
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  // kv heads fastest: eight of them are eight XCDs, each with its head's keys in an L2 of its own; then the rows of a chunk
  const int g = blockIdx.x % Hkv, rt = blockIdx.x / Hkv % (rows / (32 * NW)), chunk = blockIdx.x / (Hkv * (rows / (32 * NW)));
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
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[c][v] = 0.f;
  float m_run = NEG_INF, l_run = 0.f;

  for (int step = 0; step < steps; ++step) {
    // this wave's loads of the stage have landed, everyone's have behind the barrier; the other stage has been read by all
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (step + 1 < steps) load(step + 1);
    const bf16x8 *kb = reinterpret_cast<const bf16x8 *>(smem + (step & 1) * STAGE) + lane;
    const bf16x8 *vb = kb + STEP_TILES * TILE / 16;
    f32x16 sc[STEP_TILES];
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[t][v] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[(t * KS + s) * 64], qf[s], sc[t], 0, 0, 0);
    }
    const int p0 = (t0 + step * STEP_TILES) * TK;
    const int end = min(len, t1 * TK);       // keys of this chunk
    const bool tail = p0 + STEP_TILES * TK > end;
    float mx = NEG_INF;
    if (tail) {
#pragma unroll
      for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (p0 + t * TK + c_row(v, h) >= end) sc[t][v] = NEG_INF;
    }
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sc[t][v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale_log2e;
    // The maximum follows the scores in strides: as long as they stay below 2^8 times its weight, sums and products in float
    // lose nothing by an old one, and the accumulators need not be scaled.
    if (__any(mx > m_run + 8.f)) {
      const float m_new = fmaxf(m_run, mx);
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
    float psum = 0.f;
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][v], scale_log2e, -m_use));
        psum += p;
        pf[t][v >> 3][v & 7] = (__bf16)p;
      }
    l_run += psum;
#pragma unroll
    for (int t = 0; t < STEP_TILES; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          bf16x8 vf = vb[(t * KS + u * NT + c) * 64];
          if (tail) {  // dead slots may hold anything (even NaN)
            uint4 w4 = __builtin_bit_cast(uint4, vf);
            uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (p0 + t * TK + 16 * u + 8 * (e >> 2) + 4 * h + (e & 3) >= end) w[e >> 1] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
            vf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
          }
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t][u], acc[c], 0, 0, 0);
        }
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

template <int HD, int NW, int FUSE> hipError_t run_prefix(const PrefixArgs &a, hipStream_t s) {
  constexpr int LDS = 2 * 2 * STEP_TILES * HD * 64;
  const AttnArgs &o = a.own;
  prefix_bf16_kernel<HD, NW, FUSE><<<o.Hkv * (a.rows / (32 * NW)) * a.n_chunks, 64 * NW, LDS, s>>>(
      (const bf16_t *)(FUSE ? o.qkv : o.q), a.pk, a.pv, a.part_o, a.part_ml, o.B * o.n_q * (o.Hq / o.Hkv), a.rows, o.n_q, o.Hq,
      o.Hkv, a.len, a.cap, a.chunk_tiles, a.n_chunks, 1.4426950408889634f / sqrtf((float)HD), o.table);
  return hipGetLastError();
}

template <int HD> hipError_t pick_prefix(const PrefixArgs &a, hipStream_t s) {
  if (a.own.qkv) return a.waves == 4 ? run_prefix<HD, 4, 1>(a, s) : a.waves == 2 ? run_prefix<HD, 2, 1>(a, s) : run_prefix<HD, 1, 1>(a, s);
  return a.waves == 4 ? run_prefix<HD, 4, 0>(a, s) : a.waves == 2 ? run_prefix<HD, 2, 0>(a, s) : run_prefix<HD, 1, 0>(a, s);
}

}  // namespace

PrefixPlan prefix_plan(int B, int n_q, int Hq, int Hkv, int len) {
  const int R = B * n_q * (Hq / Hkv), n_tiles = (len + TK - 1) / TK;
  PrefixPlan p;
  p.waves = R <= 32 ? 1 : R <= 64 ? 2 : 4;
  const int row_tiles = (R + 32 * p.waves - 1) / (32 * p.waves);
  p.rows = row_tiles * 32 * p.waves;
  const int want = (512 + Hkv * row_tiles - 1) / (Hkv * row_tiles);
  p.chunk_tiles = (n_tiles + want - 1) / want;
  if (p.chunk_tiles < 8) p.chunk_tiles = 8;
  p.n_chunks = (n_tiles + p.chunk_tiles - 1) / p.chunk_tiles;
  return p;
}

size_t prefix_rows_bound(int B, int n_q, int Hq, int Hkv) {
  const size_t R = (size_t)B * n_q * (Hq / Hkv);
  // rows x chunks, with at most 512 / (Hkv x row tiles) chunks rounded up: one more of all rows, or 512 row tiles in all
  return (size_t)Hkv * ((R + 127) / 128 * 128 + 128 * (512 / Hkv + 1));
}

hipError_t launch_prefix_bf16(const PrefixArgs &a, hipStream_t s) {
  return a.own.hd == 128 ? pick_prefix<128>(a, s) : pick_prefix<64>(a, s);
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
