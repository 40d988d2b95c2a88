// Rotary decode attention over 8-bit pages with the key factor in registers.
//
// The rebuild K^T = B_k^T C_k^T takes the codes as they are: the fp8 matrix instructions multiply e4m3 operands with a power of two
// per lane, which is the scale of the lane's position, and run at twice the bf16 rate.  An entry of B_k, eight significant bits, is
// the sum of two e4m3 codes (packed once per layer), so that two such products replace one bf16 product in the same matrix time; the
// codes need no conversion, half the LDS and half the LDS reads.  The unit's sums of 1024 products are off by 1.6e-5 of the result in the
// 2-norm (512 latents with the power-law spectrum), an order below the fp16 rounding of the rotated keys that follows.
//
// One workgroup of eight waves (two per SIMD) owns a pair of KV heads of one (sequence, context split).  Wave w holds the 32 columns
// of its head, 16 coordinates and their partners, for the whole kernel (16 registers per 64 latent indices) and walks the pages:
// tiles go global -> LDS by direct copies, a whole tile ahead (K, V and scales in two buffers each).  The stream of tile t:
//   units (k-steps of 64, position block 0 then 1) of its rebuild, and between them
//   the previous tile's second position block: rotation, scores;  barrier;  its softmax, this tile's queries;  barrier;
//   its P' codes_V;  this tile's first block: rotation, scores.
// Keys are rotated by their offset in the tile (fp16 constants), queries by the distance to its first position.  Weights carry the
// values' scales: see lorc_decode_q8.hip.
//
// Bound by the matrix cores beside the vector instructions of rotation, softmax and conversion: 32/8 heads, rank 512, 16 x 4096 positions
// 70 us (68.7 GFLOP of rebuild, taken twice), matrix cores busy 61 %; a longer context adds 1147 TFLOP/s, a bf16 product of 8192^3 on the
// same card 1200.  bf16 pages: 76 us.  64/8 heads, 64 x 8192: 527 us (579).  Two waves per SIMD, not one: the waits of one are the
// products of the other (the wide form takes 122 us for the first shape).
#include "lorc_device.h"
#include "lorc_kernels.h"
#include "lorc_q8.h"
#include "lorc_stationary.h"

namespace lorc {

namespace {
constexpr int kQ8Tiles = 128;      // pages a workgroup walks at most (their ids live in LDS)
constexpr int kQ8ScaleBytes = 256; // scale bytes of a tile's K (or V) codes: up to four groups

__host__ __device__ inline size_t q8_stat_lds_bytes(int ns, int r_v, int heads) {
  size_t b = (size_t)2 * ns * 4096;                 // K codes, two buffers, padded to whole k-steps of 64
  b += (size_t)2 * 64 * r_v;                        // V codes
  b += 4 * kQ8ScaleBytes;                           // scale bytes of K, then of V
  b += (size_t)4 * kStatMaxHeads * 64 * 4;          // partial scores of the four quarters of a head
  b += 4 * 2048;                                    // P' operands per group
  b += (size_t)heads * kStatQPitch * 4;             // rotated queries, fp16 pairs
  b += (size_t)3 * kStatMaxHeads * 4;               // alpha; running max and sum at the end
  b += 64 * 8;                                      // frequencies in turns per position
  b += kQ8Tiles * 4;
  return b;
}

__device__ __forceinline__ f32x4s mfma16_f16(f16x8 a, f16x8 b, f32x4s c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
}  // namespace

// NS: k-steps of 64 latent indices.  PPH: query heads whose softmax a wave takes (1: up to eight heads per workgroup, 2: up to sixteen).
template <int NS, int PPH>
__global__ __launch_bounds__(kStatThreads, 2) void decode_q8_stationary_kernel(DecodeParams p) {
  constexpr int HD = 128, HALF = 64, T = 64, NW = kStatWaves, NT = kStatThreads, U = 2 * NS, HW = 8 * PPH;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroup -> (sequence, split, head pair): the pairs of one (sequence, split) sit on one XCD, next to each other
  const int NQ = (p.h_kv + 1) >> 1;
  const int grp = blockIdx.x / (8 * NQ), rem = blockIdx.x % (8 * NQ);
  const int hp = rem >> 3, unit_id = grp * 8 + (rem & 7);
  if (unit_id >= p.b * p.n_splits) return;
  const int seq = unit_id / p.n_splits, split = unit_id % p.n_splits;
  const int G = p.G, r_k = p.r_k, r_v = p.r_v, gk = q8_groups(r_k), gv = q8_groups(r_v);
  const int h0 = hp * 2 * G, n_heads = p.h_q - h0 < 2 * G ? p.h_q - h0 : 2 * G;

  unsigned char* kbuf = smem;
  unsigned char* vbuf = kbuf + (size_t)2 * NS * 4096;
  unsigned char* sbytes = vbuf + (size_t)2 * 64 * r_v;
  float* sp = reinterpret_cast<float*>(sbytes + 4 * kQ8ScaleBytes);
  uint16_t* pbuf = reinterpret_cast<uint16_t*>(sp + 4 * kStatMaxHeads * T);
  uint32_t* qrot = reinterpret_cast<uint32_t*>(pbuf + 4 * 1024);
  float* alpha = reinterpret_cast<float*>(qrot + HW * kStatQPitch);
  float* m_fin = alpha + kStatMaxHeads;
  float* l_fin = m_fin + kStatMaxHeads;
  double* turns_tab = reinterpret_cast<double*>(l_fin + kStatMaxHeads);
  int* ids = reinterpret_cast<int*>(turns_tab + HALF);
  const uint32_t k_lds = (uint32_t)(uintptr_t)kbuf, v_lds = (uint32_t)(uintptr_t)vbuf, s_lds = (uint32_t)(uintptr_t)sbytes;

  // ---- set-up: everything that is asked of memory goes out at once, the page ids first
  const int tile_begin = split * p.tiles_per_split;
  const int* table = p.block_table + (size_t)seq * p.max_pages;
  const int id0 = table[tile_begin < p.max_pages ? tile_begin : p.max_pages - 1];
  int ctx = p.ctx_len[seq];
  const int q_pos = p.q_pos[seq];
  int my_id = -1;  // (the split has at most kQ8Tiles pages)
  if (tid < p.tiles_per_split && tile_begin + tid < p.max_pages) my_id = table[tile_begin + tid];
  const uint32_t page_bytes = (uint32_t)p.page_elems * 2u;
  const int kvh = w >> 2, wq = w & 3;
  // softmax of head w (and w + 8); waves past the last head repeat it (same values to the same words)
  int sm_h[PPH];
  uint32_t q_raw[PPH];  // the head's coordinates lane and lane + 64, bf16
  float m_run[PPH], l_run[PPH];
#pragma unroll
  for (int u = 0; u < PPH; ++u) {
    sm_h[u] = w + 8 * u < n_heads ? w + 8 * u : n_heads - 1;
    const uint16_t* src = p.q + ((size_t)seq * p.h_q + h0 + sm_h[u]) * HD + lane;
    q_raw[u] = (uint32_t)src[0] | (uint32_t)src[HALF] << 16;
    m_run[u] = kNegInfS;
    l_run[u] = 0.f;
  }
  const double theta_lane = p.rope_tab[lane] * kInvTwoPi;
  i32x8 fac[NS][2];  // the factor: see the head of this file
  int fac_scale[2];
  {
    const int n = p.h_kv * HD, steps = coded_steps(r_k), block = (2 * hp + kvh) * 4 + wq;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p.coded, (uint32_t)(steps * 128 + kCodedMaxSteps) * (uint32_t)n);
    const bool real = 2 * hp + kvh < p.h_kv;  // (the last pair of an odd number of heads)
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // (past the end: zeros)
        const uint32_t at = real && s < steps ? (uint32_t)((block * steps + s) * 2 + u) * 2048u + lane * 16u : 0x7fff0000u;
        const u32x4 a = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
        const u32x4 b = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + 1024u, 0, 0));
        fac[s][u] = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
      }
    const u32x2 sc = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(
        r, real ? (uint32_t)steps * n * 128u + (uint32_t)(block * 32 + l32) * (uint32_t)kCodedMaxSteps : 0x7fff0000u, 0, 0));
    fac_scale[0] = (int)sc[0];
    fac_scale[1] = (int)sc[1];
  }
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  int tile_end = tile_begin + p.tiles_per_split;
  const int n_tiles = (ctx + T - 1) / T;
  if (tile_end > n_tiles) tile_end = n_tiles;
  const int nt = tile_end > tile_begin ? tile_end - tile_begin : 0;

  // ---- copies of a tile: blocks of 1 KiB, wave w moves w, w + 8, ...
  auto fresh_lane = [&]() {  // (rebuilt where it is used: no register is kept for what is derived from it)
    int l = lane_id();
    asm volatile("" : "+v"(l));
    return l;
  };
  const int k_rows = r_k >> 5, k_blocks = 2 * k_rows, v_blocks = r_v >> 4;
  auto tile_id = [&](int t) {
    const bool in = t < nt;
    const int id = __builtin_amdgcn_readfirstlane(ids[in ? t : 0]);
    return in ? id : -1;
  };
  auto rsrc_of = [&](int id) {
    const bool ok = id >= 0;
    return dma_rsrc(reinterpret_cast<const unsigned char*>(p.cache) + (ok ? (size_t)id * page_bytes : 0), ok ? page_bytes : 0u);
  };
  auto copy_k = [&](int id, int buf) {
    const u32x4 r = rsrc_of(id);
    const uint32_t lane4 = 4u * (uint32_t)fresh_lane(), lane16 = 4u * lane4;
#pragma unroll
    for (int i = 0; i < (4 * NS + NW - 1) / NW; ++i) {
      const int b = w + NW * i, pb = b >= k_rows ? 1 : 0, c = b - pb * k_rows;
      if (b < k_blocks) dma_1k(r, uniform_u32(k_lds + (uint32_t)(buf * NS * 4096 + pb * NS * 2048 + c * 1024)), lane16, uniform_u32((uint32_t)b * 1024u));
    }
    // (the scales of K: the copy begins in the page, lanes behind its end read zeros)
    if (w == 0) dma_256(r, uniform_u32(s_lds + (uint32_t)(buf * kQ8ScaleBytes)), lane4, uniform_u32((uint32_t)(64 * (r_k + r_v))));
  };
  auto copy_v = [&](int id, int buf) {
    const u32x4 r = rsrc_of(id);
    const uint32_t lane4 = 4u * (uint32_t)fresh_lane(), lane16 = 4u * lane4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = w + NW * i;
      if (b < v_blocks) dma_1k(r, uniform_u32(v_lds + (uint32_t)(buf * 64 * r_v + b * 1024)), lane16, uniform_u32((uint32_t)(64 * r_k + b * 1024)));
    }
    if (w == NW - 1) dma_256(r, uniform_u32(s_lds + (uint32_t)((2 + buf) * kQ8ScaleBytes)), lane4, uniform_u32((uint32_t)(64 * (r_k + r_v + gk))));
  };
  {  // what is read before it is written: K's padding, the V tile and the weights "before" the first tile
    const u32x4 z = {0u, 0u, 0u, 0u};
    if (r_k < 64 * NS) {
      for (int i = tid; i < 2 * NS * 4096 / 16; i += NT) reinterpret_cast<u32x4*>(kbuf)[i] = z;
      lds_barrier();  // (the first copies land beside it)
    }
    const int first = __builtin_amdgcn_readfirstlane(id0);
    copy_k(nt > 0 && first >= 0 && first < p.n_pages ? first : -1, 0);
    for (int i = tid; i < 64 * r_v / 16; i += NT) reinterpret_cast<u32x4*>(vbuf + 64 * r_v)[i] = z;
    for (int i = tid; i < 4 * 128; i += NT) reinterpret_cast<u32x4*>(pbuf)[i] = z;
    for (int i = tid; i < HW * kStatQPitch; i += NT) qrot[i] = 0u;
    if (tid < kStatMaxHeads) {
      alpha[tid] = 1.f;
      l_fin[tid] = 0.f;
    }
    if (tid < HALF) turns_tab[tid] = theta_lane;
    if (tid < kQ8Tiles) ids[tid] = my_id >= 0 && my_id < p.n_pages ? my_id : -1;
  }
  lds_barrier();
  f16x2 rot[2][8];  // (cos, sin) of the offset in the tile, position block b, the lane's eight frequencies
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const double theta = turns_tab[16 * wq + acc_row(j, hf)];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const double turns = (32 * b + l32) * theta;
      const float fr = (float)(turns - rint(turns));
      rot[b][j][0] = static_cast<_Float16>(__builtin_amdgcn_cosf(fr));
      rot[b][j][1] = static_cast<_Float16>(__builtin_amdgcn_sinf(fr));
    }
  }
  f32x4s o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x4s{0.f, 0.f, 0.f, 0.f};
  f32x16 acc[2], zero16;
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[0][j] = acc[1][j] = zero16[j] = 0.f;

  __builtin_amdgcn_s_waitcnt(0);  // the factor's loads too: none of them may be waited for inside the loop

  // ---- pieces of the stream
  const unsigned char* k_src = kbuf + lane * 8;
  auto k_operand = [&](int buf, auto u_c) {  // unit u: position block u / NS, k-step u % NS
    constexpr int u = decltype(u_c)::value, b = u / NS, s = u % NS;
    const unsigned char* at = k_src + buf * NS * 4096 + b * NS * 2048 + s * 2048;
    const u32x2 x0 = *reinterpret_cast<const u32x2*>(at), x1 = *reinterpret_cast<const u32x2*>(at + 512);
    const u32x2 x2 = *reinterpret_cast<const u32x2*>(at + 1024), x3 = *reinterpret_cast<const u32x2*>(at + 1536);
    return i32x8{(int)x0[0], (int)x0[1], (int)x1[0], (int)x1[1], (int)x2[0], (int)x2[1], (int)x3[0], (int)x3[1]};
  };
  auto k_scales = [&](int buf, int b) {  // scale bytes of position 32 b + l32, a byte per group
    const unsigned char* at = sbytes + buf * kQ8ScaleBytes + 32 * b + l32;
    uint32_t v = at[0];
    if constexpr (NS > 2) v |= (uint32_t)at[64] << 8;
    if constexpr (NS > 4) v |= (uint32_t)at[128] << 16;
    if constexpr (NS > 6) v |= (uint32_t)at[192] << 24;
    return (int)v;
  };
  auto rotate = [&](f16x8 (&kf)[2], auto b_c, auto part_c) {  // rows 2 part, 2 part + 1 (of eight) and their partners
    constexpr int b = decltype(b_c)::value, part = decltype(part_c)::value;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * part + i;
      uint32_t cs = __builtin_bit_cast(uint32_t, rot[b][j]);
      asm volatile("" : "+v"(cs));  // (else all of them are widened ahead of the loop, and spilled)
      const f16x2 h = __builtin_bit_cast(f16x2, cs);
      const float x = acc[b][j], y = acc[b][j + 8], c = (float)h[0], s = (float)h[1];
      kf[j >> 2][2 * (j & 3)] = static_cast<_Float16>(x * c - y * s);
      kf[j >> 2][2 * (j & 3) + 1] = static_cast<_Float16>(y * c + x * s);
    }
  };
  const uint32_t* q_src = qrot + (size_t)(kvh * G + (l32 < G && kvh * G + l32 < n_heads ? l32 : 0)) * kStatQPitch + 16 * wq + 4 * hf;
  float* s_dst = sp + (size_t)((wq * 2 + kvh) * 8 + 4 * hf) * T + l32;  // (rows past the group: filed, not read)
  auto score = [&](f32x16& sa, const f16x8 (&kf)[2], auto part_c) {
    constexpr int part = decltype(part_c)::value;
    sa = mfma32_f16(__builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(q_src + 8 * part)), kf[part], part ? sa : zero16);
  };
  auto score_store = [&](const f32x16& sa, auto b_c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s_dst[j * T + 32 * decltype(b_c)::value] = sa[j];
  };
  struct Softmax {
    float a[4], s, mx, e;
    uint32_t ub[4];
  };
  auto softmax_load = [&](Softmax& sm, int u, int buf) {
    const int h = sm_h[u], l = PPH == 2 ? fresh_lane() : lane;
    const float* src = sp + (size_t)(h < G ? h : 8 + h - G) * T + l;
#pragma unroll
    for (int q = 0; q < 4; ++q) sm.a[q] = src[q * kStatMaxHeads * T];
    const unsigned char* at = sbytes + (2 + buf) * kQ8ScaleBytes + l;
#pragma unroll
    for (int g = 0; g < 4; ++g) sm.ub[g] = at[g < gv ? 64 * g : 0];
  };
  auto softmax_max = [&](Softmax& sm, int valid) {
    sm.s = lane < valid ? (sm.a[0] + sm.a[1]) + (sm.a[2] + sm.a[3]) : kNegInfS;
    uint32_t top = sm.ub[0] > sm.ub[1] ? sm.ub[0] : sm.ub[1];
    const uint32_t t2 = sm.ub[2] > sm.ub[3] ? sm.ub[2] : sm.ub[3];
    top = top > t2 ? top : t2;
    top = top > 127 + kLeastExp ? top : 127 + kLeastExp;
    sm.mx = sm.s + ((float)top - (127.f + kTopExp));
  };
  auto softmax_rows = [&](Softmax& sm) {
    sm.mx = row_max_step<0>(sm.mx);
    sm.mx = row_max_step<1>(sm.mx);
    sm.mx = row_max_step<2>(sm.mx);
    sm.mx = row_max_step<3>(sm.mx);
  };
  auto softmax_weight = [&](Softmax& sm, int u) {
    const float2 rows = row_pair(sm.mx);
    const float2 halves = half_pair(fmaxf(rows.x, rows.y));
    const float m_new = fmaxf(fmaxf(m_run[u], fmaxf(halves.x, halves.y)), kNoWeight);
    const float al = __builtin_amdgcn_exp2f(m_run[u] - m_new);
    m_run[u] = m_new;
    sm.e = __builtin_amdgcn_exp2f(sm.s - m_new);
    l_run[u] = l_run[u] * al + sm.e;
    alpha[sm_h[u]] = al;
  };
  auto softmax_store = [&](const Softmax& sm, int u) {
    const int l = PPH == 2 ? fresh_lane() : lane;
    uint16_t* dst = pbuf + ((size_t)((l >> 5) * 64 + sm_h[u] + 16 * ((l & 31) >> 3)) * 8 + (l & 7));
#pragma unroll
    for (int g = 0; g < 4; ++g)  // (groups past the rank: filed, not read)
      dst[g * 1024] = f16_bits(below_f16_max(__builtin_amdgcn_ldexpf(sm.e, (int)sm.ub[g] - 127)));
  };
  struct Query {
    double turns;
    float cs, sn;
  };
  auto query_angle = [&](Query& qr) {
    const float fr = (float)(qr.turns - rint(qr.turns));
    qr.cs = __builtin_amdgcn_cosf(fr) * p.q_scale;
    qr.sn = __builtin_amdgcn_sinf(fr) * p.q_scale;
  };
  auto query_store = [&](const Query& qr) {
#pragma unroll
    for (int u = 0; u < PPH; ++u) {
      const float x = __uint_as_float(q_raw[u] << 16), y = __uint_as_float(q_raw[u] & 0xffff0000u);
      f16x2 v;
      v[0] = static_cast<_Float16>(x * qr.cs - y * qr.sn);
      v[1] = static_cast<_Float16>(y * qr.cs + x * qr.sn);
      qrot[(size_t)sm_h[u] * kStatQPitch + lane] = __builtin_bit_cast(uint32_t, v);
    }
  };
  // O += P' codes: wave w owns latents 64 w .. 64 w + 63; block (jb, b): latents 64 w + 32 jb + 2 n16 + b
  const int n16 = lane & 15, kg = lane >> 4;
  // (There is no branch in the stream: the compiler would move the products behind it, and their operands into scratch memory.  Waves
  // and blocks past the rank work on the first ones and keep the result to themselves.)
  const bool has_v = 64 * w < r_v, has_v2 = 64 * w + 32 < r_v;
  const int wv = has_v ? w : 0, jb_off = has_v2 ? 4 * 512 : 0;
  const unsigned char* v_src = vbuf + (size_t)(wv * 8 + (kg >> 1)) * 512 + ((kg & 1) * 32 + 2 * n16) * 8;
  const uint16_t* p_src = pbuf + (size_t)(wv >> 1) * 1024 + lane * 8;
  struct PV {
    f32x4s al;
    f16x8 pf[2];
    u32x4 v[2];
  };
  auto pv_prep = [&](PV& x) {
    x.al = *reinterpret_cast<const f32x4s*>(alpha + 4 * kg);
    x.pf[0] = load_frag_f16(p_src);
    x.pf[1] = load_frag_f16(p_src + 512);
  };
  auto pv_load = [&](PV& x, int buf, int jb, int valid, bool ragged) {
#pragma unroll
    for (int ph = 0; ph < 2; ++ph) {
      x.v[ph] = *reinterpret_cast<const u32x4*>(v_src + buf * 64 * r_v + jb * jb_off + ph * 1024);
      if (ragged) {  // slots past the context hold anything, NaN codes too
        const u32x2 lo = keep_bytes(u32x2{x.v[ph][0], x.v[ph][1]}, valid - 32 * ph - 8 * kg);
        const u32x2 hi = keep_bytes(u32x2{x.v[ph][2], x.v[ph][3]}, valid - 32 * ph - 8 * kg);
        x.v[ph] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  };
  auto pv_mul = [&](const PV& x, auto i_c) {  // block i = 2 jb + b
    constexpr int i = decltype(i_c)::value, b = i & 1;
    o[i] *= x.al;
    o[i] = mfma16_f16(x.pf[0], codes_f16(u32x2{x.v[0][2 * b], x.v[0][2 * b + 1]}), o[i]);
    o[i] = mfma16_f16(x.pf[1], codes_f16(u32x2{x.v[1][2 * b], x.v[1][2 * b + 1]}), o[i]);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  // Where the pieces sit in the stream: behind the x-th of 32 products (two per unit).  A product occupies the matrix core for 64
  // cycles and the next of the same wave waits for it, so a piece between them costs nothing while it is short.
  auto at = [](int x) constexpr { return x * (2 * U) / 32; };

  int valid_prev = 0;  // the tile before the first one has no positions
  for (int t = 0; t < nt; ++t) {
    const int pos0 = (tile_begin + t) * T, buf = t & 1, prev = buf ^ 1;
    dma_barrier<0>();  // this tile's K codes and scales, the previous tile's V codes; every wave is through the previous tile
    {
      const int id = tile_id(t), next = tile_id(t + 1);
      copy_v(id, buf);
      copy_k(next, prev);
    }
    f16x8 kf[2];
    f32x16 sa;
    Softmax sm[PPH];
    Query qr;
    PV pv;
    i32x8 c[2];
    c[0] = k_operand(buf, I0{});
    const int k_scale[2] = {k_scales(buf, 0), k_scales(buf, 1)};
    static_for<2 * U>([&](auto x_c) {
      constexpr int x = decltype(x_c)::value, u = x / 2, part = x % 2, b = u / NS, s = u % NS;
      if constexpr (part == 0 && u + 1 < U) c[(u + 1) % 2] = k_operand(buf, std::integral_constant<int, u + 1 < U ? u + 1 : 0>{});
      __builtin_amdgcn_sched_barrier(0);
      acc[b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fac[s][part], c[u % 2], s == 0 && part == 0 ? zero16 : acc[b], 0, 0, s & 3,
                                                               fac_scale[s >> 2], s >> 1, k_scale[b]);
      // -- the previous tile's second position block
      if constexpr (x == at(0)) rotate(kf, I1{}, I0{});
      if constexpr (x == at(1)) rotate(kf, I1{}, I1{});
      if constexpr (x == at(2)) rotate(kf, I1{}, I2{});
      if constexpr (x == at(3)) rotate(kf, I1{}, I3{});
      if constexpr (x == at(4)) score(sa, kf, I0{});
      if constexpr (x == at(5)) score(sa, kf, I1{});
      if constexpr (x == at(7)) score_store(sa, I1{});
      if constexpr (x == at(8)) lds_barrier();  // its scores are complete
      // -- its softmax, a head after the other
      static_for<PPH>([&](auto h_c) {
        constexpr int h = decltype(h_c)::value, x0 = 8 + 4 * h;
        if constexpr (x == at(x0)) softmax_load(sm[h], h, prev);
        if constexpr (x == at(x0 + 1)) softmax_max(sm[h], valid_prev);
        if constexpr (x == at(x0 + 2)) softmax_rows(sm[h]);
        if constexpr (x == at(x0 + 3)) softmax_weight(sm[h], h);
        if constexpr (x == at(x0 + 4)) softmax_store(sm[h], h);
      });
      // -- this tile's queries
      if constexpr (x == at(14)) qr.turns = (double)(q_pos - pos0) * turns_tab[lane];
      if constexpr (x == at(15)) query_angle(qr);
      if constexpr (x == at(17)) query_store(qr);
      if constexpr (x == at(18)) lds_barrier();  // weights and queries are complete
      // -- the previous tile's P' codes
      if constexpr (x == at(18)) pv_prep(pv);
      if constexpr (x == at(18)) pv_load(pv, prev, 0, T, false);
      if constexpr (x == at(19)) pv_mul(pv, I0{});
      if constexpr (x == at(20)) pv_mul(pv, I1{});
      if constexpr (x == at(21)) pv_load(pv, prev, 1, T, false);
      if constexpr (x == at(22)) pv_mul(pv, I2{});
      if constexpr (x == at(23)) pv_mul(pv, I3{});
      // -- this tile's first position block
      if constexpr (x == at(24)) rotate(kf, I0{}, I0{});
      if constexpr (x == at(25)) rotate(kf, I0{}, I1{});
      if constexpr (x == at(26)) rotate(kf, I0{}, I2{});
      if constexpr (x == at(27)) rotate(kf, I0{}, I3{});
      if constexpr (x == at(28)) score(sa, kf, I0{});
      if constexpr (x == at(29)) score(sa, kf, I1{});
      if constexpr (x == at(31)) score_store(sa, I0{});
      __builtin_amdgcn_sched_barrier(0);
    });
    valid_prev = ctx - pos0 < T ? ctx - pos0 : T;
  }

  if (nt > 0) {  // the last tile's second half
    const int prev = (nt - 1) & 1;
    f16x8 kf[2];
    f32x16 sa;
    Softmax sm[PPH];
    PV pv;
    rotate(kf, I1{}, I0{});
    rotate(kf, I1{}, I1{});
    rotate(kf, I1{}, I2{});
    rotate(kf, I1{}, I3{});
    score(sa, kf, I0{});
    score(sa, kf, I1{});
    score_store(sa, I1{});
    dma_barrier<0>();  // scores complete; its V codes and scales have landed
#pragma unroll
    for (int h = 0; h < PPH; ++h) {
      softmax_load(sm[h], h, prev);
      softmax_max(sm[h], valid_prev);
      softmax_rows(sm[h]);
      softmax_weight(sm[h], h);
      softmax_store(sm[h], h);
    }
    lds_barrier();  // weights visible
    pv_prep(pv);
    pv_load(pv, prev, 0, valid_prev, valid_prev < T);
    pv_mul(pv, I0{});
    pv_mul(pv, I1{});
    pv_load(pv, prev, 1, valid_prev, valid_prev < T);
    pv_mul(pv, I2{});
    pv_mul(pv, I3{});
  }

  // ---- partials: every copy has to land before its memory is used again
  __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
  for (int u = 0; u < PPH; ++u) {
    float l = l_run[u];
    l += half_wave_peer<0>(l);
    l += half_wave_peer<1>(l);
    l += half_wave_peer<2>(l);
    l += half_wave_peer<3>(l);
    const float2 rows = row_pair(l);
    const float2 halves = half_pair(rows.x + rows.y);
    m_fin[sm_h[u]] = m_run[u];
    l_fin[sm_h[u]] = halves.x + halves.y;
  }
  __syncthreads();
  const size_t row0 = ((size_t)seq * p.n_splits + split) * p.h_q + h0;
  if (tid < n_heads) {
    p.part_ml[(row0 + tid) * 2] = nt > 0 ? m_fin[tid] : kNegInfS;
    p.part_ml[(row0 + tid) * 2 + 1] = l_fin[tid];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int h = 4 * kg + j;
    const float l = l_fin[h], inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    if (h < n_heads) {
#pragma unroll
      for (int jb = 0; jb < 2; ++jb)
        if (jb ? has_v2 : has_v)
          *reinterpret_cast<uint32_t*>(p.part_o + (row0 + h) * r_v + 64 * w + 32 * jb + 2 * n16) =
              (uint32_t)f16_bits(o[2 * jb][j] * inv) | ((uint32_t)f16_bits(o[2 * jb + 1][j] * inv) << 16);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
namespace {
using Q8StatKernel = void (*)(DecodeParams);
template <int PPH>
Q8StatKernel q8_stat_kernel(int ns) {
  switch (ns) {
    case 2: return decode_q8_stationary_kernel<2, PPH>;
    case 3: return decode_q8_stationary_kernel<3, PPH>;
    case 4: return decode_q8_stationary_kernel<4, PPH>;
    case 5: return decode_q8_stationary_kernel<5, PPH>;
    case 6: return decode_q8_stationary_kernel<6, PPH>;
    case 7: return decode_q8_stationary_kernel<7, PPH>;
    default: return decode_q8_stationary_kernel<8, PPH>;
  }
}
int q8_stat_ns(int r_k) { return r_k <= 128 ? 2 : coded_steps(r_k); }
}  // namespace

bool q8_stationary_shape_ok(const lorc_layer_desc& d) {
  return d.head_dim == 128 && d.n_q_heads / d.n_kv_heads <= kStatMaxHeads / 2 && d.rank_k <= 512 && d.rank_v <= 512;
}

int q8_stationary_max_tiles() { return kQ8Tiles; }

int set_kernel_attributes_decode_q8_stationary() {
  for (int ns = 2; ns <= 8; ++ns)
    for (Q8StatKernel k : {q8_stat_kernel<1>(ns), q8_stat_kernel<2>(ns)})
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess)
        return LORC_EHIP;
  return LORC_OK;
}

int launch_decode_q8_stationary(const DecodeParams& p, hipStream_t s) {
  const int ns = q8_stat_ns(p.r_k), nq = (p.h_kv + 1) / 2, units = p.b * p.n_splits;
  const bool one = 2 * p.G <= 8;
  const size_t lds = q8_stat_lds_bytes(ns, p.r_v, one ? 8 : 16);
  if (lds > 160 * 1024 || p.tiles_per_split > kQ8Tiles) return LORC_EUNSUPPORTED;
  return launch_kernel(one ? q8_stat_kernel<1>(ns) : q8_stat_kernel<2>(ns), dim3(((units + 7) / 8) * 8 * nq), dim3(kStatThreads), lds, s, p);
}

}  // namespace lorc
