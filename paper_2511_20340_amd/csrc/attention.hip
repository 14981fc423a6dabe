// Hybrid-mask ragged-prefix attention for gfx950 (SpecFormer: causal along the cached context,
// bidirectional -- or causal -- inside the block of n_q new rows).
//
// bf16 path.  One workgroup (4 wavefronts) owns one chunk of `chunk_tiles` 32-key tiles of one
// (sequence, kv head, 32-row group).  All G*n_q query rows that share the kv head form the N side
// of a 32x32x16 MFMA, so every K/V byte is read from HBM once for the whole GQA group and block.
// Per tile a wave computes   S^T = K . Q^T   (keys on the MFMA M side, loaded straight from the
// tiled cache into operand registers: `blob[i*64+lane]`, 1 KiB contiguous per instruction),
// an online softmax in fp32 registers with the mask built from (key position, row's block
// index), and   O^T += V^T . P^T   whose P operand is exactly the S^T accumulator layout.
// The 4 waves interleave tiles; they merge (m, l, O) through LDS at the end.  A sequence that
// spans several chunks leaves fp32 partials that a small combine kernel merges.
#include "attention_rows.h"

namespace sf {

namespace {

template <int HD, int FUSE, int ONCE>
__global__ __launch_bounds__(256, HD == 64 ? 4 : 2) void attn_bf16_kernel(
    const bf16_t *__restrict__ Q, const uint4 *Kc, const uint4 *Vc, const int32_t *__restrict__ kv_len, bf16_t *__restrict__ O,
    float *__restrict__ part_o, float *__restrict__ part_ml, int n_q, int Hq, int Hkv, int cap, int mode, int chunk_tiles,
    int n_chunks, int n_rt, float scale_log2e, const float2 *__restrict__ table, const int32_t *__restrict__ order,
    const int32_t *__restrict__ slots) {
  extern __shared__ float lds[];
  attn_rows<HD, FUSE, ONCE, 0>(make_uint3(blockIdx.x, blockIdx.y, blockIdx.z), lds, Q, Kc, Vc, kv_len, O, part_o, part_ml, n_q,
                               Hq, Hkv, cap, mode, chunk_tiles, n_chunks, n_rt, scale_log2e, table, order, slots);
}

// Merge the split-KV partials of sequences that span more than one chunk.  32 lanes per query row, 8 rows per
// workgroup: lane c holds the (max, sum) of chunk c, each lane HD / 32 features of the output, and the chunks' outputs
// are requested eight at a time (one row per workgroup walking them one by one takes 8.1 us at 11 chunks and 160 rows a sequence, this 4.7).
template <int HD>
__global__ __launch_bounds__(256) void attn_combine_kernel(
    const float *__restrict__ part_o, const float *__restrict__ part_ml, const int32_t *__restrict__ kv_len,
    bf16_t *__restrict__ O, int rows, int n_q, int Hq, int Hkv, int cap, int chunk_tiles, int n_chunks, int n_rt) {
  constexpr int E = HD / 32, AHEAD = 8;
  typedef float vec __attribute__((ext_vector_type(E)));
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;  // row = (b, block row, query head)
  if (row >= rows) return;
  const int hq = row % Hq, i = row / Hq % n_q, b = row / (Hq * n_q);
  const int G = Hq / Hkv, g = hq / G, rr = i * G + hq % G;
  const size_t slot0 = ((size_t)b * Hkv + g) * n_chunks * (n_rt * 32) + rr;
  const size_t step = n_rt * 32;
  const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + slot0;
  // the first chunks are requested before the sequence's length is known (slots past it hold anything and are not used)
  float2 first = lane < n_chunks ? ml[lane * step] : make_float2(NEG_INF, 0.f);
  vec x[AHEAD];
  auto request = [&](int c, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      x[u] = *reinterpret_cast<const vec *>(part_o + (slot0 + min(c + u, last) * step) * HD + lane * E);
  };
  request(0, n_chunks - 1);
  const int n_tiles = (min(kv_len[b], cap - n_q) + n_q + TK - 1) / TK;
  const int sc = min((n_tiles + chunk_tiles - 1) / chunk_tiles, n_chunks);
  if (sc <= 1) return;
  if (lane >= sc) first = make_float2(NEG_INF, 0.f);
  float m = first.x;
  for (int c = lane + 32; c < sc; c += 32) m = fmaxf(m, ml[c * step].x);
#pragma unroll
  for (int w = 16; w; w >>= 1) m = fmaxf(m, __shfl_xor(m, w, 32));
  const float m_use = m == NEG_INF ? 0.f : m;
  float l = 0.f;
  vec o = 0.f;
  for (int c0 = 0; c0 < sc; c0 += 32) {
    const int n = min(32, sc - c0);
    const float2 mine = c0 == 0 ? first : lane < n ? ml[(c0 + lane) * step] : make_float2(NEG_INF, 0.f);
    const float f_c = __builtin_amdgcn_exp2f(mine.x - m_use);  // of chunk c0 + lane
    for (int c = 0; c < n; c += AHEAD) {
      if (c0 + c > 0) request(c0 + c, sc - 1);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (c + u < n) {
          // one rounding per chunk for the row's sum as for its outputs: the products are not rounded by themselves
          const float f = __shfl(f_c, c + u, 32);
          l = fmaf(__shfl(mine.y, c + u, 32), f, l);
          o += x[u] * f;
        }
    }
  }
  o *= 1.f / l;
  uint32_t *out = reinterpret_cast<uint32_t *>(O + (size_t)row * HD + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) out[e / 2] = pack2bf(o[e], o[e + 1]);
}

// fp32 path (small models): plain cache layout, one workgroup per (query head, block row, sequence).
// Keys are processed in chunks of CK with a workgroup-wide online softmax.  A pair of lanes scores one key (its
// features in alternating groups of four), so 128 keys are scored at once; for the weighted sum of the values
// the threads form hd/4 columns of four features times 256/(hd/4) key groups, which meet in LDS at the end.  At 64 keys everything is latency: one workgroup per row keeps
// every chain short (4 sequences x 4 heads x 5 rows: 36 us with one workgroup per head walking all rows).
constexpr int CK = 512;
__global__ __launch_bounds__(256) void attn_f32_kernel(const float *__restrict__ Q, const float *__restrict__ Kc,
                                                       const float *__restrict__ Vc,
                                                       const int32_t *__restrict__ kv_len, float *__restrict__ O,
                                                       int n_q, int Hq, int Hkv, int hd, int cap, int mode,
                                                       float scale, const int32_t *__restrict__ slots) {
  __shared__ __attribute__((aligned(16))) float sq[256];
  __shared__ float sc[CK], red[8];
  __shared__ f32x4 so[256];
  const int hq = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = hq / (Hq / Hkv);
  const int len = min(kv_len[b], cap - n_q), total = len + (mode == SF_MASK_BIDIR ? n_q : i + 1);
  const size_t cache = ((size_t)(slots ? slots[b] : b) * Hkv + g) * (size_t)cap * hd;
  const float *K = Kc + cache, *V = Vc + cache;
  const size_t row = (((size_t)b * n_q + i) * Hq + hq) * hd;
  if (tid < hd) sq[tid] = Q[row + tid];
  __syncthreads();
  const int cols = hd / 4, groups = 256 / cols, col = tid % cols, grp = tid / cols;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m_run = NEG_INF, l_run = 0.f;
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
    const float m_use = m_new == NEG_INF ? 0.f : m_new;  // no finite score yet: keep exp finite
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
    __syncthreads();  // sc and red are written again
  }
  so[tid] = o;
  __syncthreads();
  if (tid < cols) {
    for (int x = 1; x < groups; ++x) o += so[x * cols + tid];
    *reinterpret_cast<f32x4 *>(O + row + tid * 4) = o / l_run;
  }
}

}  // namespace

// Chunk size (in 32-key tiles) of the split-KV decomposition.  The grid is sized from the host's
// upper bound of the lengths: split only when there are fewer (sequence, head, row tile) groups
// than CUs, and never below 16 tiles (4 per wave) per chunk; with >= 256 groups every group is one
// workgroup and no combine pass is needed (measured fastest at every batch >= 32).
int attn_chunk_tiles(int groups, int keys_upper) {
  const int n_tiles = (keys_upper + TK - 1) / TK;
  const int want_chunks = (256 + groups - 1) / (groups > 0 ? groups : 1);
  int ct = (n_tiles + want_chunks - 1) / want_chunks;
  return ct < 16 ? 16 : ct;
}

size_t attn_workspace_bytes(int B, int Hkv, int hd, int G, int n_q, int len_upper) {
  const int n_rt = (G * n_q + 31) / 32;
  // sized for the smallest chunk any launch may pick (16 tiles)
  const int ct = 16;
  const int n_tiles = (len_upper + n_q + TK - 1) / TK;
  const int n_chunks = (n_tiles + ct - 1) / ct;
  if (n_chunks <= 1) return 0;
  return (size_t)B * Hkv * n_chunks * (n_rt * 32) * (hd + 2) * sizeof(float);
}

hipError_t launch_attention_bf16(const AttnArgs &a, hipStream_t s) {
  const int G = a.Hq / a.Hkv;
  const int n_rt = (G * a.n_q + 31) / 32;
  const float scale_log2e = 1.4426950408889634f / sqrtf((float)a.hd);
  dim3 grid(a.n_chunks, a.Hkv * n_rt, a.B), block(256);
  const size_t lds = (size_t)WAVES * 32 * (a.hd + 4 + 2) * sizeof(float);
  static bool attr_done = false;
  if (!attr_done) {
#define SF_ATTN_LDS(HD_, FUSE_, ONCE_)                                                                    \
  (void)hipFuncSetAttribute(reinterpret_cast<const void *>(attn_bf16_kernel<HD_, FUSE_, ONCE_>),         \
                            hipFuncAttributeMaxDynamicSharedMemorySize, ATTN_LDS_BYTES<HD_>)
    SF_ATTN_LDS(128, 0, 0); SF_ATTN_LDS(128, 1, 0); SF_ATTN_LDS(64, 0, 0); SF_ATTN_LDS(64, 1, 0);
    SF_ATTN_LDS(128, 0, 1); SF_ATTN_LDS(128, 1, 1); SF_ATTN_LDS(64, 0, 1); SF_ATTN_LDS(64, 1, 1);
#undef SF_ATTN_LDS
    attr_done = true;
  }
  // One row tile per (sequence, kv head): every K/V byte is read by exactly one workgroup and the loads are
  // non-temporal -- on this chip a read-once stream runs at 6.7 TB/s with them and 5.9 TB/s without (256
  // workgroups, 16-byte loads).  128 sequences of 1024-4096 keys, 8 kv heads of 128: 230 us against 245 us per
  // launch.  Several row tiles read the same keys from different workgroups: those keep the caching loads.
  // a.qkv: the raw QKV projection; the kernel rotates and appends the block's rows itself
  const bf16_t *q = (const bf16_t *)(a.qkv ? a.qkv : a.q);
#define SF_ATTN_LAUNCH(HD_, FUSE_, ONCE_)                                                                   \
  attn_bf16_kernel<HD_, FUSE_, ONCE_><<<grid, block, lds, s>>>(                                             \
      q, (const uint4 *)a.kc, (const uint4 *)a.vc, a.kv_len, (bf16_t *)a.out, a.part_o, a.part_ml, a.n_q,   \
      a.Hq, a.Hkv, a.cap, a.mode, a.chunk_tiles, a.n_chunks, n_rt, scale_log2e, a.table, a.order, a.slots)
#define SF_ATTN_PICK(HD_)                                                                                   \
  do {                                                                                                      \
    if (n_rt == 1) { if (a.qkv) SF_ATTN_LAUNCH(HD_, 1, 1); else SF_ATTN_LAUNCH(HD_, 0, 1); }                \
    else           { if (a.qkv) SF_ATTN_LAUNCH(HD_, 1, 0); else SF_ATTN_LAUNCH(HD_, 0, 0); }                \
  } while (0)
  if (a.hd == 128) SF_ATTN_PICK(128); else SF_ATTN_PICK(64);
#undef SF_ATTN_PICK
#undef SF_ATTN_LAUNCH
  return hipGetLastError();
}

hipError_t launch_attention_combine(const AttnArgs &a, hipStream_t s) {
  const int G = a.Hq / a.Hkv, n_rt = (G * a.n_q + 31) / 32, rows = a.B * a.n_q * a.Hq;
  auto launch = [&](auto kernel) {
    kernel<<<(rows + 7) / 8, 256, 0, s>>>(a.part_o, a.part_ml, a.kv_len, (bf16_t *)a.out, rows, a.n_q, a.Hq, a.Hkv, a.cap,
                                          a.chunk_tiles, a.n_chunks, n_rt);
  };
  if (a.hd == 128) launch(&attn_combine_kernel<128>); else launch(&attn_combine_kernel<64>);
  return hipGetLastError();
}

hipError_t launch_attention_f32(const AttnArgs &a, hipStream_t s) {
  attn_f32_kernel<<<dim3(a.Hq, a.n_q, a.B), 256, 0, s>>>((const float *)a.q, (const float *)a.kc, (const float *)a.vc,
                                                         a.kv_len, (float *)a.out, a.n_q, a.Hq, a.Hkv, a.hd, a.cap,
                                                         a.mode, 1.f / sqrtf((float)a.hd), a.slots);
  return hipGetLastError();
}

}  // namespace sf
