// Rotary decode attention over 8-bit pages for what lorc_decode_q8_stat.hip has no room for: ranks from 544 to 1024, groups of 9 to 32
// query heads, head_dim 64.
//
// The same products (the pages' codes against B_k as pairs of e4m3 codes, held in registers), with one wave per SIMD: four waves of up
// to 512 registers own one KV head of head_dim 128 (or two of 64) of one (sequence, context split) and up to sixteen query heads; a wave
// holds 32 columns, 16 registers per 64 latent indices (256 at rank 1024).  Half pages of 32 positions keep K and V in two buffers each
// within the LDS.  A product takes 64 cycles of the matrix core and the next one of the wave waits for it, so everything else is laid
// between the products of the next half page's rebuild: rotation and scores;  barrier;  softmax, queries;  barrier;  P' codes_V.
//
// Bound by what a single wave cannot hide (rank 768: matrix cores busy 36 %, vector instructions 29 %, waits 22 %).  32/8 heads, 16 x 4096
// positions, with the merge (bf16 pages in brackets): rank 576 120 us (90), 768 126 to 139 (110 to 127), 1024 157 (192); 32/2 heads rank 256
// 39 (88); 24/8 heads of 64, rank 256 51 (44), rank 512 62 (68).
#include "lorc_device.h"
#include "lorc_kernels.h"
#include "lorc_q8.h"
#include "lorc_stationary.h"

namespace lorc {

namespace {
constexpr int kWideWaves = 4, kWideThreads = 64 * kWideWaves, kWideTiles = 256;  // half pages a workgroup walks at most
constexpr int kWideScales = 512;  // scale bytes of a page's K (or V): up to eight groups

__host__ __device__ constexpr size_t q8_wide_lds_bytes(int ns, int vb, int heads) {
  return (size_t)2 * ns * 2048            // K codes, two buffers, padded to whole k-steps of 64
         + (size_t)2 * vb * 4096          // V codes
         + 4 * kWideScales                // scale bytes of K, then of V
         + (size_t)4 * 16 * 32 * 4        // partial scores of the four quarters of the head
         + 8 * 1024                       // P' operands per group
         + (size_t)heads * kStatQPitch * 4
         + 3 * 16 * 4 + 64 * 8 + kWideTiles / 2 * 4;
}
}  // namespace

// NS: k-steps of 64 latent indices of K; VB: blocks of 32 value latents per wave; PPH: pairs of heads whose softmax a wave takes.
template <int HD, int NS, int VB, int PPH>
__global__ __launch_bounds__(kWideThreads, 1) void decode_q8_wide_kernel(DecodeParams p) {
  constexpr int HALF = HD / 2, T = 32, NW = kWideWaves, NT = kWideThreads, HW = 8 * PPH, X = 2 * NS;
  constexpr int QW = HD / 32, KVW = NW / QW, HP = 16 / KVW;  // waves of a KV head, KV heads of a workgroup, query heads of each at most
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31, n16 = lane & 15, kg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroup -> (sequence, split, KV heads, HP query heads of each); those of one (sequence, split) sit on one XCD
  const int parts = (p.G + HP - 1) / HP, NQ = (p.h_kv + KVW - 1) / KVW * parts;
  const int grp = blockIdx.x / (8 * NQ), rem = blockIdx.x % (8 * NQ);
  const int hp = rem >> 3, unit_id = grp * 8 + (rem & 7);
  if (unit_id >= p.b * p.n_splits) return;
  const int seq = unit_id / p.n_splits, split = unit_id % p.n_splits, g_kv = hp / parts * KVW;
  const int r_k = p.r_k, r_v = p.r_v, gk = q8_groups(r_k), gv = q8_groups(r_v);
  const int part0 = HP * (hp % parts), left = p.G - part0, gp = left < HP ? left : HP;  // query heads of a KV head here
  const int n_heads = (p.h_kv - g_kv < KVW ? p.h_kv - g_kv : KVW) * gp;
  auto head_of = [&](int h) { return KVW == 1 ? g_kv * p.G + part0 + h : (g_kv + h / gp) * p.G + part0 + h % gp; };
  const int kvh = w / QW, wq = w % QW;

  unsigned char* kbuf = smem;
  unsigned char* vbuf = kbuf + (size_t)2 * NS * 2048;
  unsigned char* sbytes = vbuf + (size_t)2 * VB * 4096;
  float* sp = reinterpret_cast<float*>(sbytes + 4 * kWideScales);
  uint16_t* pbuf = reinterpret_cast<uint16_t*>(sp + 4 * 16 * T);
  uint32_t* qrot = reinterpret_cast<uint32_t*>(pbuf + 8 * 512);
  float* alpha = reinterpret_cast<float*>(qrot + HW * kStatQPitch);
  float* m_fin = alpha + 16;
  float* l_fin = m_fin + 16;
  double* turns_tab = reinterpret_cast<double*>(l_fin + 16);
  int* ids = reinterpret_cast<int*>(turns_tab + 64);
  const uint32_t k_lds = (uint32_t)(uintptr_t)kbuf, v_lds = (uint32_t)(uintptr_t)vbuf, s_lds = (uint32_t)(uintptr_t)sbytes;

  // ---- set-up
  const int page_begin = split * p.tiles_per_split;
  const int* table = p.block_table + (size_t)seq * p.max_pages;
  int ctx = p.ctx_len[seq];
  const int q_pos = p.q_pos[seq];
  int my_id = -1;  // (the split has at most kWideTiles / 2 pages)
  if (tid < p.tiles_per_split && page_begin + tid < p.max_pages) my_id = table[page_begin + tid];
  const uint32_t page_bytes = (uint32_t)p.page_elems * 2u;
  // softmax: lanes 32 hf .. 32 hf + 31 take head 2 w + hf (and 8 more); lanes past the last head repeat it (same values to the same words)
  int sm_h[PPH];
  uint32_t q_raw[2 * PPH];  // queries: head w, w + 4, ... (repeated past the last), coordinates lane and lane + 64, bf16
  float m_run[PPH], l_run[PPH];
#pragma unroll
  for (int u = 0; u < PPH; ++u) {
    sm_h[u] = 2 * w + hf + 8 * u < n_heads ? 2 * w + hf + 8 * u : n_heads - 1;
    m_run[u] = kNegInfS;
    l_run[u] = 0.f;
  }
  int q_head[2 * PPH];
#pragma unroll
  for (int u = 0; u < 2 * PPH; ++u) {
    q_head[u] = w + 4 * u < n_heads ? w + 4 * u : n_heads - 1;
    const uint16_t* src = p.q + ((size_t)seq * p.h_q + head_of(q_head[u])) * HD + lane % HALF;
    q_raw[u] = (uint32_t)src[0] | (uint32_t)src[HALF] << 16;
  }
  const double theta_lane = p.rope_tab[lane % HALF] * kInvTwoPi;
  half2_t rot[8];  // (cos, sin) of the position's offset in the half page, the lane's eight frequencies
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 cs = p.lane_cs[l32 * HALF + 16 * wq + acc_row(j, hf)];
    rot[j][0] = static_cast<_Float16>(cs.x);
    rot[j][1] = static_cast<_Float16>(cs.y);
  }
  i32x8 fac[NS][2];
  int fac_scale[4];
  {
    const int n = p.h_kv * HD, steps = coded_steps(r_k), block = (g_kv + kvh) * QW + wq;
    const bool real = g_kv + kvh < p.h_kv;  // (the last pair of an odd number of heads)
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p.coded, (uint32_t)(steps * 128 + kCodedMaxSteps) * (uint32_t)n);
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
    const u32x4 sc = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
        r, real ? (uint32_t)steps * n * 128u + (uint32_t)(block * 32 + l32) * (uint32_t)kCodedMaxSteps : 0x7fff0000u, 0, 0));
#pragma unroll
    for (int c = 0; c < 4; ++c) fac_scale[c] = (int)sc[c];
  }
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  const int begin = page_begin * kPage;
  int end = begin + p.tiles_per_split * kPage;
  if (end > ctx) end = ctx;
  const int nt = end > begin ? (end - begin + T - 1) / T : 0;  // half pages

  {  // what is read before it is written
    const u32x4 z = {0u, 0u, 0u, 0u};
    for (int i = tid; i < 2 * NS * 2048 / 16; i += NT) reinterpret_cast<u32x4*>(kbuf)[i] = z;
    for (int i = tid; i < 2 * VB * 4096 / 16; i += NT) reinterpret_cast<u32x4*>(vbuf)[i] = z;
    for (int i = tid; i < 8 * 64; i += NT) reinterpret_cast<u32x4*>(pbuf)[i] = z;
    for (int i = tid; i < HW * kStatQPitch; i += NT) qrot[i] = 0u;
    if (tid < 16) {
      alpha[tid] = 1.f;
      l_fin[tid] = 0.f;
    }
    if (tid < 64) turns_tab[tid] = theta_lane;
    if (tid < kWideTiles / 2) ids[tid] = my_id >= 0 && my_id < p.n_pages ? my_id : -1;
  }
  lds_barrier();

  // ---- copies of a half page: blocks of 1 KiB, wave w moves w, w + 4, ...; blocks past the rank repeat the last one (no branch in the
  // stream: see lorc_decode_q8_stat.hip)
  const int k_rows = r_k >> 5, v_rows = r_v >> 5;
  auto id_read = [&](int t) { return ids[(t >> 1) < kWideTiles / 2 ? t >> 1 : kWideTiles / 2 - 1]; };
  auto id_use = [&](int raw, int t) { return __builtin_amdgcn_readfirstlane(raw) | ((nt - 1 - t) >> 31); };
  auto rsrc_of = [&](int id) {
    const uint32_t ok = ~(uint32_t)(id >> 31);
    return dma_rsrc(reinterpret_cast<const unsigned char*>(p.cache) + (size_t)((uint32_t)id & ok) * page_bytes, page_bytes & ok);
  };
  const uint32_t lane4 = 4u * (uint32_t)lane, lane16 = 16u * (uint32_t)lane;
  constexpr int NKC = (2 * NS + NW - 1) / NW, NVC = VB;  // copies per wave, and two of scale bytes each
  auto copy_scales = [&](const u32x4& r, int part, int buf, int i) {  // part: 0 K, 1 V
    // (of few groups the second block begins behind the page: its lanes read zeros, the bound counts lane and scalar offset)
    const uint32_t from = 64u * (uint32_t)(r_k + r_v + (part ? gk : 0)) + 256u * (uint32_t)i;
    dma_256(r, uniform_u32(s_lds + (uint32_t)((2 * part + buf) * kWideScales + 256 * i)), lane4 + from, 0u);
  };
  auto copy_k = [&](const u32x4& r, int t, int i) {
    const int buf = t & 1, sb = t & 1;
    if (i >= NKC) return copy_scales(r, 0, buf, i - NKC);
    const int c = w + NW * i < k_rows ? w + NW * i : k_rows - 1;
    dma_1k(r, uniform_u32(k_lds + (uint32_t)(buf * NS * 2048 + c * 1024)), lane16, uniform_u32((uint32_t)(sb * k_rows + c) * 1024u));
  };
  auto copy_v = [&](const u32x4& r, int t, int i) {
    const int buf = t & 1, sb = t & 1;
    if (i >= NVC) return copy_scales(r, 1, buf, i - NVC);
    const int c = w + NW * i < v_rows ? w + NW * i : v_rows - 1;
    dma_1k(r, uniform_u32(v_lds + (uint32_t)(buf * VB * 4096 + c * 1024)), lane16, uniform_u32((uint32_t)(64 * r_k + (c * 4 + 2 * sb) * 512)));
  };
  int id_cur = id_use(id_read(0), 0), id_next = id_use(id_read(1), 1);
  {
    const u32x4 r = rsrc_of(id_cur);
#pragma unroll
    for (int i = 0; i < NKC + 2; ++i) copy_k(r, 0, i);
  }

  f32x4s o[2 * VB];
#pragma unroll
  for (int i = 0; i < 2 * VB; ++i) o[i] = f32x4s{0.f, 0.f, 0.f, 0.f};
  f32x16 acc, prev_acc, zero16;
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[j] = prev_acc[j] = zero16[j] = 0.f;
  __builtin_amdgcn_s_waitcnt(0);  // the factor's loads too: none of them may be waited for inside the loop
  // The factor lives in the accumulation half of the register file, which the products read as well; o does not, because it is rescaled by
  // vector instructions on every half page (96 moves between the halves otherwise).
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int u = 0; u < 2; ++u) asm volatile("" : "+a"(fac[s][u]));

  // ---- pieces of the stream
  const unsigned char* k_src = kbuf + lane * 8;
  auto k_operand = [&](int buf, auto s_c) {
    const unsigned char* at = k_src + buf * NS * 2048 + decltype(s_c)::value * 2048;
    const u32x2 x0 = *reinterpret_cast<const u32x2*>(at), x1 = *reinterpret_cast<const u32x2*>(at + 512);
    const u32x2 x2 = *reinterpret_cast<const u32x2*>(at + 1024), x3 = *reinterpret_cast<const u32x2*>(at + 1536);
    return i32x8{(int)x0[0], (int)x0[1], (int)x1[0], (int)x1[1], (int)x2[0], (int)x2[1], (int)x3[0], (int)x3[1]};
  };
  auto k_scales = [&](int t, int first) {  // bytes of groups first .. first + 3 of the lane's position
    const unsigned char* at = sbytes + (t & 1) * kWideScales + 64 * first + 32 * (t & 1) + l32;
    return (int)((uint32_t)at[0] | (uint32_t)at[64] << 8 | (uint32_t)at[128] << 16 | (uint32_t)at[192] << 24);
  };
  auto rotate = [&](f16x8 (&kf)[2], auto part_c) {  // rows 2 part, 2 part + 1 (of eight) and their partners
    constexpr int part = decltype(part_c)::value;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * part + i;
      uint32_t cs = __builtin_bit_cast(uint32_t, rot[j]);
      asm volatile("" : "+v"(cs));
      const half2_t h = __builtin_bit_cast(half2_t, cs);
      const float x = prev_acc[j], y = prev_acc[j + 8], c = (float)h[0], s = (float)h[1];
      kf[j >> 2][2 * (j & 3)] = static_cast<_Float16>(x * c - y * s);
      kf[j >> 2][2 * (j & 3) + 1] = static_cast<_Float16>(y * c + x * s);
    }
  };
  const uint32_t* q_src = qrot + (size_t)(kvh * gp + (l32 < gp && kvh * gp + l32 < n_heads ? l32 : 0)) * kStatQPitch + 16 * wq + 4 * hf;
  float* s_dst = sp + (size_t)(w * 16 + 4 * hf) * T + l32;
  auto query_operand = [&](auto part_c) { return *reinterpret_cast<const u32x4*>(q_src + 8 * decltype(part_c)::value); };
  auto score = [&](f32x16& sa, const f16x8 (&kf)[2], const u32x4& q, auto part_c) {
    constexpr int part = decltype(part_c)::value;
    sa = mfma32_f16(__builtin_bit_cast(f16x8, q), kf[part], part ? sa : zero16);
  };
  auto score_store = [&](const f32x16& sa) {  // rows 8 (j / 4) + 4 hf + j % 4 (rows past the last head: filed, not read)
#pragma unroll
    for (int j = 0; j < 4 * PPH; ++j) s_dst[(8 * (j >> 2) + (j & 3)) * T] = sa[j];
  };
  int sm_src[PPH];  // first partial score of the head at the lane's position
#pragma unroll
  for (int u = 0; u < PPH; ++u)
    sm_src[u] = ((KVW == 1 ? 0 : sm_h[u] / gp) * QW * 16 + (KVW == 1 ? sm_h[u] : sm_h[u] % gp)) * T + l32;
  struct Softmax {
    float a[QW], s, mx, e;
    uint32_t ub[8];
  };
  auto softmax_load = [&](Softmax& sm, int u, int t) {
    const float* src = sp + sm_src[u];
#pragma unroll
    for (int q = 0; q < QW; ++q) sm.a[q] = src[q * 16 * T];
    const unsigned char* at = sbytes + (2 + (t & 1)) * kWideScales + 32 * (t & 1) + l32;
#pragma unroll
    for (int g = 0; g < 8; ++g) sm.ub[g] = at[g < gv ? 64 * g : 0];
  };
  auto softmax_max = [&](Softmax& sm, int valid) {
    sm.s = l32 < valid ? (QW == 4 ? (sm.a[0] + sm.a[1]) + (sm.a[2] + sm.a[3]) : sm.a[0] + sm.a[1]) : kNegInfS;
    uint32_t top = 127 + kLeastExp;
#pragma unroll
    for (int g = 0; g < 8; ++g) top = top > sm.ub[g] ? top : sm.ub[g];
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
    const float m_new = fmaxf(fmaxf(m_run[u], fmaxf(rows.x, rows.y)), kNoWeight);
    const float al = __builtin_amdgcn_exp2f(m_run[u] - m_new);
    m_run[u] = m_new;
    sm.e = __builtin_amdgcn_exp2f(sm.s - m_new);
    l_run[u] = l_run[u] * al + sm.e;
    alpha[sm_h[u]] = al;
  };
  auto softmax_store = [&](const Softmax& sm, int u) {
    uint16_t* dst = pbuf + (size_t)(sm_h[u] + 16 * (l32 >> 3)) * 8 + (l32 & 7);
#pragma unroll
    for (int g = 0; g < 8; ++g) dst[g * 512] = f16_bits(below_f16_max(__builtin_amdgcn_ldexpf(sm.e, (int)sm.ub[g] - 127)));  // (groups past the rank: filed, not read)
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
    for (int u = 0; u < 2 * PPH; ++u) {
      const float x = __uint_as_float(q_raw[u] << 16), y = __uint_as_float(q_raw[u] & 0xffff0000u);
      half2_t v;
      v[0] = static_cast<_Float16>(x * qr.cs - y * qr.sn);
      v[1] = static_cast<_Float16>(y * qr.cs + x * qr.sn);
      qrot[(size_t)q_head[u] * kStatQPitch + lane % HALF] = __builtin_bit_cast(uint32_t, v);
    }
  };
  // O += P' codes: wave w owns blocks w, w + 4, ... of 32 value latents; accumulator 2 i + b: latents 32 (w + 4 i) + 2 n16 + b
  const uint32_t v_lane = (uint32_t)((kg >> 1) * 512 + ((kg & 1) * 32 + 2 * n16) * 8);
  struct PV {
    f16x8 pf;
    u32x4 v;
  };
  auto pv_load = [&](PV& x, int buf, int i, int valid, bool ragged) {
    const int jb = w + NW * i < v_rows ? w + NW * i : 0;  // (past the rank: the first block, and the result is not kept)
    x.pf = load_frag_f16(pbuf + (size_t)(jb >> 2) * 512 + lane * 8);
    x.v = *reinterpret_cast<const u32x4*>(vbuf + buf * VB * 4096 + jb * 1024 + v_lane);
    if (ragged) {  // slots past the context hold anything, NaN codes too
      const u32x2 lo = keep_bytes(u32x2{x.v[0], x.v[1]}, valid - 8 * kg), hi = keep_bytes(u32x2{x.v[2], x.v[3]}, valid - 8 * kg);
      x.v = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  auto pv_mul = [&](const PV& x, const f32x4s& al, auto i_c) {
    constexpr int i = decltype(i_c)::value;
    o[2 * i] *= al;
    o[2 * i + 1] *= al;
    o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.pf, codes_f16(u32x2{x.v[0], x.v[1]}), o[2 * i], 0, 0, 0);
    o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.pf, codes_f16(u32x2{x.v[2], x.v[3]}), o[2 * i + 1], 0, 0, 0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  auto at = [](int x) constexpr { return x * X / 32; };  // pieces sit behind the x-th of 32 products

  int valid_prev = 0;  // the half page before the first one has no positions
  for (int t = 0; t < nt; ++t) {
    const int pos0 = begin + t * T, buf = t & 1, prev = buf ^ 1;
    dma_barrier<0>();  // this half page's K, the previous one's V; every wave is through the previous stream
    const int id_raw = id_read(t + 2);
    const u32x4 r_next = rsrc_of(id_next), r_cur = rsrc_of(id_cur);
    f16x8 kf[2];
    f32x16 sa;
    Softmax sm;
    Query qr;
    PV pv[2];
    f32x4s al;
    i32x8 c[2];
    u32x4 qf[2];
    c[0] = k_operand(buf, I0{});
    const int k_scale[2] = {k_scales(t, 0), k_scales(t, 4)};
    prev_acc = acc;
    static_for<X>([&](auto x_c) {
      constexpr int x = decltype(x_c)::value, s = x / 2, part = x % 2;
      if constexpr (part == 0 && s + 1 < NS) c[(s + 1) % 2] = k_operand(buf, std::integral_constant<int, s + 1 < NS ? s + 1 : 0>{});
      __builtin_amdgcn_sched_barrier(0);
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fac[s][part], c[s % 2], x == 0 ? zero16 : acc, 0, 0, s & 3, fac_scale[s >> 2], (s >> 1) & 3,
                                                            k_scale[s >> 3]);
      // -- the copies, spread over the first half of the stream: the next half page's K, this one's V
      static_for<NKC + NVC + 4>([&](auto i_c) {
        constexpr int i = decltype(i_c)::value;
        if constexpr (x == at(i * 16 / (NKC + NVC + 4))) {
          if constexpr (i < NKC + 2) copy_k(r_next, t + 1, i);
          else copy_v(r_cur, t, i - NKC - 2);
        }
      });
      // -- the previous half page: rotation and scores
      static_for<4>([&](auto i_c) {
        if constexpr (x == at(2 * decltype(i_c)::value)) rotate(kf, i_c);
      });
      if constexpr (x == at(0)) qf[0] = query_operand(I0{});
      if constexpr (x == at(2)) qf[1] = query_operand(I1{});
      if constexpr (x == at(4)) score(sa, kf, qf[0], I0{});
      if constexpr (x == at(7)) score(sa, kf, qf[1], I1{});
      if constexpr (x == at(9)) score_store(sa);
      if constexpr (x == at(10)) lds_barrier();  // its scores are complete
      // -- its softmax, a pair of heads after the other
      static_for<PPH>([&](auto h_c) {
        constexpr int h = decltype(h_c)::value, x0 = 10 + 4 * h;
        if constexpr (x == at(x0)) softmax_load(sm, h, t + 1);  // (its buffers are those of the parity of t + 1)
        if constexpr (x == at(x0 + 1)) softmax_max(sm, valid_prev);
        if constexpr (x == at(x0 + 2)) softmax_rows(sm);
        if constexpr (x == at(x0 + 3)) softmax_weight(sm, h);
        if constexpr (x == at(x0 + 3)) softmax_store(sm, h);
      });
      // -- this half page's queries
      if constexpr (x == at(11)) qr.turns = (double)(q_pos - pos0) * turns_tab[lane];
      if constexpr (x == at(12)) query_angle(qr);
      if constexpr (x == at(14)) query_store(qr);
      if constexpr (x == at(18)) lds_barrier();  // weights and queries are complete
      // -- P' codes of the previous half page, a block's operands ahead
      if constexpr (x == at(18)) al = *reinterpret_cast<const f32x4s*>(alpha + 4 * kg);
      if constexpr (x == at(18)) pv_load(pv[0], prev, 0, T, false);
      static_for<VB>([&](auto i_c) {
        constexpr int i = decltype(i_c)::value;
        if constexpr (x == at(19 + i * 13 / VB)) {
          if constexpr (i + 1 < VB) pv_load(pv[(i + 1) % 2], prev, i + 1, T, false);
          pv_mul(pv[i % 2], al, i_c);
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    valid_prev = end - pos0 < T ? end - pos0 : T;
    id_cur = id_next;
    id_next = id_use(id_raw, t + 2);
  }

  if (nt > 0) {  // the last half page
    f16x8 kf[2];
    f32x16 sa;
    prev_acc = acc;
    static_for<4>([&](auto i_c) { rotate(kf, i_c); });
    score(sa, kf, query_operand(I0{}), I0{});
    score(sa, kf, query_operand(I1{}), I1{});
    score_store(sa);
    dma_barrier<0>();  // scores complete; its V and scales have landed
#pragma unroll
    for (int h = 0; h < PPH; ++h) {
      Softmax sm;
      softmax_load(sm, h, nt - 1);
      softmax_max(sm, valid_prev);
      softmax_rows(sm);
      softmax_weight(sm, h);
      softmax_store(sm, h);
    }
    lds_barrier();
    const f32x4s al = *reinterpret_cast<const f32x4s*>(alpha + 4 * kg);
    static_for<VB>([&](auto i_c) {
      PV pv;
      pv_load(pv, (nt - 1) & 1, decltype(i_c)::value, valid_prev, valid_prev < T);
      pv_mul(pv, al, i_c);
    });
  }

  // ---- partials: every copy has to land before the workgroup ends
  __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
  for (int u = 0; u < PPH; ++u) {
    float l = l_run[u];
    l += half_wave_peer<0>(l);
    l += half_wave_peer<1>(l);
    l += half_wave_peer<2>(l);
    l += half_wave_peer<3>(l);
    const float2 rows = row_pair(l);
    m_fin[sm_h[u]] = m_run[u];
    l_fin[sm_h[u]] = rows.x + rows.y;
  }
  __syncthreads();
  const size_t row0 = ((size_t)seq * p.n_splits + split) * p.h_q;
  if (tid < n_heads) {
    p.part_ml[(row0 + head_of(tid)) * 2] = nt > 0 ? m_fin[tid] : kNegInfS;
    p.part_ml[(row0 + head_of(tid)) * 2 + 1] = l_fin[tid];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int h = 4 * kg + j;
    const float l = l_fin[h], inv = l > 0.f ? __builtin_amdgcn_rcpf(l) : l == 0.f ? 0.f : l;
    if (h < n_heads) {
#pragma unroll
      for (int i = 0; i < VB; ++i)
        if (w + NW * i < v_rows)
          *reinterpret_cast<uint32_t*>(p.part_o + (row0 + head_of(h)) * r_v + 32 * (w + NW * i) + 2 * n16) =
              (uint32_t)f16_bits(o[2 * i][j] * inv) | ((uint32_t)f16_bits(o[2 * i + 1][j] * inv) << 16);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
namespace {
using Q8WideKernel = void (*)(DecodeParams);
// latents that a kernel is padded to (the larger of K's and V's)
int q8_wide_class(int r_k, int r_v) {
  const int r = r_k > r_v ? r_k : r_v;
  return r <= 128 ? 128 : r <= 256 ? 256 : r <= 512 ? 512 : r <= 640 ? 640 : r <= 768 ? 768 : 1024;
}
template <int HD, int PPH>
Q8WideKernel q8_wide_kernel(int cls) {
  switch (cls) {
    case 128: return decode_q8_wide_kernel<HD, 2, 1, PPH>;
    case 256: return decode_q8_wide_kernel<HD, 4, 2, PPH>;
    case 512: return decode_q8_wide_kernel<HD, 8, 4, PPH>;
    case 640: return decode_q8_wide_kernel<HD, 10, 5, PPH>;
    case 768: return decode_q8_wide_kernel<HD, 12, 6, PPH>;
    default: return decode_q8_wide_kernel<HD, 16, 8, PPH>;
  }
}
Q8WideKernel q8_wide_kernel(int head_dim, int cls, bool one) {
  if (head_dim == 128) return one ? q8_wide_kernel<128, 1>(cls) : q8_wide_kernel<128, 2>(cls);
  return one ? q8_wide_kernel<64, 1>(cls) : q8_wide_kernel<64, 2>(cls);
}
}  // namespace

// Workgroups of a (sequence, split): one KV head of 128 coordinates and sixteen of its query heads, or two of 64 and eight of each.
int q8_wide_units(const lorc_layer_desc& d) {
  const int G = d.n_q_heads / d.n_kv_heads;
  return d.head_dim == 128 ? d.n_kv_heads * ((G + 15) / 16) : (d.n_kv_heads + 1) / 2 * ((G + 7) / 8);
}

int q8_wide_max_tiles() { return kWideTiles / 2; }

int set_kernel_attributes_decode_q8_wide() {
  for (int head_dim : {64, 128})
    for (int cls : {128, 256, 512, 640, 768, 1024})
      for (bool one : {false, true})
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(q8_wide_kernel(head_dim, cls, one)), hipFuncAttributeMaxDynamicSharedMemorySize,
                                160 * 1024) != hipSuccess)
          return LORC_EHIP;
  return LORC_OK;
}

int launch_decode_q8_wide(const lorc_layer_desc& d, const DecodeParams& p, hipStream_t s) {
  const int cls = q8_wide_class(p.r_k, p.r_v), nq = q8_wide_units(d), units = p.b * p.n_splits;
  const bool one = p.head_dim == 128 ? p.G <= 8 : p.G <= 4;  // up to eight query heads in a workgroup
  const size_t lds = q8_wide_lds_bytes(cls / 64, cls / 128, one ? 8 : 16);
  if (lds > 160 * 1024 || 2 * p.tiles_per_split > kWideTiles) return LORC_EUNSUPPORTED;
  return launch_kernel(q8_wide_kernel(p.head_dim, cls, one), dim3(((units + 7) / 8) * 8 * nq), dim3(kWideThreads), lds, s, p);
}

}  // namespace lorc
