// Decode attention over the 8-bit latent cache: e4m3 codes with a power of two per position and 128 latents.
//
// What the scales cost: a key's scale belongs to one position, and a lane of a key operand holds one position, so it goes into the
// conversion of the codes (which takes a power of two for free).  A value's scale belongs to a position too, which is the
// contraction index of P V: it goes into the weights, P'_t = p_t 2^(k_t), and the codes are multiplied as they are.
// Weights and codes are fp16 there (a code has four significant bits, the weights keep eleven).  To keep P' in range whatever the
// scales are, the running reference of the softmax is M = max_t (s_t + k_t) - kTopExp instead of max_t s_t: the largest P' is then 2^15, the
// top of fp16, and the sum of the weights is taken relative to the same M, l = sum 2^(s_t - M), in fp32.  (k_t counts as at least kLeastExp in
// M, which bounds l; values below 448 x 2^kLeastExp are far below what the fp16 partials hold.)
// k_t is the largest over the groups of the position, as one reference serves all of them.  In a group that is 2^-j of the largest, a weight
// that is 2^-i of the largest has P' = 2^(15 - i - j): all eleven bits to i + j = 29, none beyond 40.  (With the largest P' at one, it would be 14
// and 25: groups that lie 2^16 apart and count alike in the output cost 2 to 3 % of it.)  An uncompressed layer's groups are its KV heads, which
// have a reference each; there the largest P' is one.
#include <climits>

#include "lorc_device.h"
#include "lorc_kernels.h"
#include "lorc_q8.h"

namespace lorc {

namespace {
constexpr float kNegInfQ = -__builtin_huge_valf();
constexpr double kTurns = 0.15915494309189533576888;  // 1 / 2 pi
}  // namespace

// ------------------------------------------------------------------------------------------------ absorbed query, ranks above 512
// One workgroup of four waves per (sequence, context split, block of 32 query heads), 32 positions at a time.  The step's K codes are
// widened once into LDS (bf16, operand order), wave w takes every fourth k-step of the scores, partial scores meet in LDS, eight lanes
// per head take the softmax, and wave w owns every fourth block of 32 value latents, whose codes it loads itself, ahead of the scores.
// Bound by the chain of four phases and the three barriers between them, one workgroup per compute unit: rank 1024, 16 x 4096 positions 118 us with the merge
// (bf16 pages, twice the bytes: 90).  The kernel for ranks up to 512 keeps two buffers of whole pages in LDS, which do not fit here (two of half
// pages would: that form is not built); where both can serve (16 x 8192, rank 512) it takes 42 us and a form like this one 172.
__global__ __launch_bounds__(256, 1) void decode_q8_kernel(DecodeParams p) {
  constexpr int T = 32, NBW = 8;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r_k = p.r_k, r_v = p.r_v, nks = r_k >> 4, gk = q8_groups(r_k), gv = q8_groups(r_v), nb = r_v >> 5;
  const int n_units = (p.h_q + 31) / 32;
  const int unit = blockIdx.x % n_units, ss = blockIdx.x / n_units, split = ss % p.n_splits, seq = ss / p.n_splits;
  const int h0 = 32 * unit, nh = p.h_q - h0 < 32 ? p.h_q - h0 : 32;
  uint16_t* kt = reinterpret_cast<uint16_t*>(smem);                       // [nks][64 lanes][8]
  float* sp = reinterpret_cast<float*>(smem + (size_t)r_k * 64);          // [4 waves][32 heads][32 positions]
  uint16_t* pb = reinterpret_cast<uint16_t*>(sp + 4 * 32 * T);            // [gv][2][64 lanes][8]
  float* al = reinterpret_cast<float*>(pb + (size_t)gv * 1024);           // [32]
  float* l_fin = al + 32;

  int ctx = p.ctx_len[seq];
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  const int t_begin = split * p.tiles_per_split * kPage;
  int t_end = t_begin + p.tiles_per_split * kPage;
  if (t_end > ctx) t_end = ctx;
  const unsigned char* pool = reinterpret_cast<const unsigned char*>(p.cache);
  const uint32_t page_bytes = (uint32_t)p.page_elems * 2u, codes = (uint32_t)kPage * (r_k + r_v);

  f32x16 o[NBW], zero16;
#pragma unroll
  for (int j = 0; j < 16; ++j) zero16[j] = 0.f;
#pragma unroll
  for (int i = 0; i < NBW; ++i) o[i] = zero16;
  const int sh = tid >> 3, s8 = tid & 7;  // softmax: head, and which four of the positions
  float m_run = kNoWeight, l_run = 0.f;

  for (int pos0 = t_begin; pos0 < t_end; pos0 += T) {
    const int id = __builtin_amdgcn_readfirstlane(p.block_table[(size_t)seq * p.max_pages + pos0 / kPage]), sb = (pos0 / T) & 1;
    const bool ok = id >= 0 && id < p.n_pages;
    const __amdgpu_buffer_rsrc_t page = make_rsrc(uniform_ptr(pool + (ok ? (size_t)id * page_bytes : 0)), ok ? page_bytes : 0u);
    // ---- K codes of the step, widened into LDS: a thread takes sixteen, eight of each of two positions
    for (int c = tid; c < 2 * r_k; c += 256) {
      const int slot = 32 * sb + ((2 * c) & 31), g = c >> 8;
      const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(page, c * 16, sb * r_k * 32, 0));
      const uint32_t sc = __builtin_amdgcn_raw_buffer_load_b16(page, g * kPage + slot, codes, 0);
      u32x4* dst = reinterpret_cast<u32x4*>(kt + (size_t)c * 16);
      dst[0] = codes_bf16(u32x2{v[0], v[1]}, pow2_of(sc & 255u));
      dst[1] = codes_bf16(u32x2{v[2], v[3]}, pow2_of((sc >> 8) & 255u));
    }
    // ---- what the later phases need of the page travels meanwhile
    uint32_t ub[8];  // value scale bytes of the thread's four positions, per group
#pragma unroll
    for (int g = 0; g < 8; ++g)
      ub[g] = g < gv ? (ok ? __builtin_amdgcn_raw_buffer_load_b32(page, (gk + g) * kPage + 32 * sb + 4 * s8, codes, 0) : 0x7f7f7f7fu) : 0u;
    u32x2 vraw[NBW][2];
#pragma unroll
    for (int i = 0; i < NBW; ++i)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int jb = w + 4 * i < nb ? w + 4 * i : 0;
        vraw[i][ks] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(page, lane * 8, kPage * r_k + (jb * 4 + 2 * sb + ks) * 512, 0));
      }
    __syncthreads();
    // ---- scores
    {
      const uint16_t* kl = kt + (size_t)lane * 8;
      const uint16_t* qsrc = p.q + ((size_t)seq * p.h_q + h0 + (l32 < nh ? l32 : 0)) * r_k + 8 * hf;
      f32x16 sa = zero16;
#pragma unroll 4
      for (int ks = w; ks < nks; ks += 4) sa = mfma32(load_frag(qsrc + 16 * ks), load_frag(kl + (size_t)ks * 512), sa);
#pragma unroll
      for (int j = 0; j < 16; ++j) sp[(w * 32 + acc_row(j, hf)) * T + l32] = sa[j] * p.q_scale;
    }
    __syncthreads();
    // ---- softmax: eight lanes per head, four positions each
    {
      float s[4], mx = kNegInfQ;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = 4 * s8 + e;
        s[e] = (sp[sh * T + pos] + sp[(32 + sh) * T + pos]) + (sp[(64 + sh) * T + pos] + sp[(96 + sh) * T + pos]);
        if (pos0 + pos >= t_end) s[e] = kNegInfQ;
        uint32_t top = 127 + kLeastExp;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const uint32_t b = (ub[g] >> (8 * e)) & 255u;
          top = g < gv && b > top ? b : top;
        }
        mx = fmaxf(mx, s[e] + ((float)top - (127.f + kTopExp)));
      }
#pragma unroll
      for (int step = 1; step < 8; step <<= 1) mx = fmaxf(mx, __shfl_xor(mx, step, 64));
      const float m_new = fmaxf(m_run, mx), alpha = exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
      if (s8 == 0) al[sh] = alpha;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = 4 * s8 + e;
        const float pe = pos0 + pos < t_end ? exp2f(s[e] - m_new) : 0.f;
        l_run += pe;
#pragma unroll
        for (int g = 0; g < 8; ++g)
          if (g < gv)
            pb[((size_t)(g * 2 + (pos >> 4)) * 64 + sh + 32 * ((pos & 15) >> 3)) * 8 + (pos & 7)] =
                f16_bits(below_f16_max(__builtin_amdgcn_ldexpf(pe, (int)((ub[g] >> (8 * e)) & 255u) - 127)));
      }
    }
    __syncthreads();
    // ---- o = alpha o + P' codes
    {
      const int left = t_end - pos0;
#pragma unroll
      for (int i = 0; i < NBW; ++i) {
        const int jb = w + 4 * i;
        if (jb < nb) {
#pragma unroll
          for (int j = 0; j < 16; ++j) o[i][j] *= al[acc_row(j, hf)];
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            u32x2 v = vraw[i][ks];
            if (left < T) v = keep_bytes(v, left - 16 * ks - 8 * hf);  // slots past the context hold anything, NaN codes too
            const f16x8 pf = load_frag_f16(pb + ((size_t)((jb >> 2) * 2 + ks) * 64 + lane) * 8);
            o[i] = mfma32_f16(pf, codes_f16(v), o[i]);
          }
        }
      }
    }
  }

  // ---- partials, normalised by the split's own sum
#pragma unroll
  for (int step = 1; step < 8; step <<= 1) l_run += __shfl_xor(l_run, step, 64);
  const size_t row0 = ((size_t)seq * p.n_splits + split) * p.h_q + h0;
  if (s8 == 0) {
    l_fin[sh] = l_run;
    if (sh < nh) {
      p.part_ml[(row0 + sh) * 2] = t_end > t_begin ? m_run : kNegInfQ;
      p.part_ml[(row0 + sh) * 2 + 1] = l_run;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NBW; ++i) {
    const int jb = w + 4 * i;
    if (jb < nb) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int h = acc_row(j, hf);
        const float l = l_fin[h];
        if (h < nh) p.part_o[(row0 + h) * r_v + jb * 32 + l32] = f16_bits(l > 0.f ? o[i][j] / l : l == 0.f ? 0.f : l);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ uncompressed layer
// One wave per (sequence, context split, KV head, 16 query heads of its group): it walks the split 32 positions at a time and
// exchanges nothing with others.  16x16x32 products: S^T = K Q^T and O^T = V^T P^T.  A 16 byte load gives a lane of a K operand eight
// coordinates of two neighbouring positions, 2 m and 2 m + 1 for row m, and a lane of a V operand eight positions of two neighbouring
// coordinates, so that row r of block b is position (coordinate) 2 r + b of the step and a lane's eight scores are those of eight
// consecutive positions, which is what it holds of V.  Keys take the angles of their offset in the step, constants in fp16 like the
// keys themselves; the base goes to the queries (one frequency per lane, handed round through LDS).
// Bound by the page stream: 16 x 4096 positions of 2 KiB in 28.9 us, 4.7 TB/s (bf16 pages: 46 us), the merge 4.8 more.
template <bool BOTH>
__global__ __launch_bounds__(256, 2) void decode_plain_q8_kernel(DecodeParams p) {
  constexpr int HD = 128, HALF = 64, T = 32;
  __shared__ __align__(16) float2 base_cs[4][HALF];
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, q = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nq = BOTH ? (p.G + 15) / 16 : 1, n_units = p.h_kv * nq, n_blocks = (n_units + 3) / 4;
  const int unit = (blockIdx.x % n_blocks) * 4 + w, ss = blockIdx.x / n_blocks;
  if (unit >= n_units) return;  // (a wave on its own: there is no barrier in this kernel)
  const int split = ss % p.n_splits, seq = ss / p.n_splits, g = unit / nq, h0 = g * p.G + 16 * (unit % nq);
  const int nh = p.G - 16 * (unit % nq) < 16 ? p.G - 16 * (unit % nq) : 16;
  int ctx = p.ctx_len[seq];
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  const int n = p.h_kv * HD;
  const int t_begin = split * p.tiles_per_split * kPage;
  int t_end = t_begin + p.tiles_per_split * kPage;
  if (t_end > ctx) t_end = ctx;
  const int n_steps = t_end > t_begin ? (t_end - t_begin + T - 1) / T : 0;
  const unsigned char* pool = reinterpret_cast<const unsigned char*>(p.cache);
  const uint32_t page_bytes = (uint32_t)p.page_elems * 2u, codes = 2u * kPage * n;
  const uint32_t lane_off = (uint32_t)(q >> 1) * 512u + (uint32_t)((q & 1) * 32 + 2 * m) * 8u;

  u32x4 kraw[4], vraw[4];
  u32x2 vs;
  uint32_t ks;
  bool v_ok = false;
  auto page_of = [&](int i, bool& ok) {
    const int tile = i < n_steps ? (t_begin + i * T) / kPage : 0;
    const int id = __builtin_amdgcn_readfirstlane(i < n_steps ? p.block_table[(size_t)seq * p.max_pages + tile] : -1);
    ok = id >= 0 && id < p.n_pages;
    return make_rsrc(uniform_ptr(pool + (ok ? (size_t)id * page_bytes : 0)), ok ? page_bytes : 0u);
  };
  auto k_request = [&](int i) {
    bool ok;
    const __amdgpu_buffer_rsrc_t r = page_of(i, ok);
    const int row = (i & 1) * (n >> 4) + g * 8;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) kraw[kk] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_off, (row + 2 * kk) * 512, 0));
    ks = __builtin_amdgcn_raw_buffer_load_b16(r, 2 * m, codes + g * kPage + (i & 1) * T, 0);
  };
  auto v_request = [&](int i) {
    const __amdgpu_buffer_rsrc_t r = page_of(i, v_ok);
#pragma unroll
    for (int jb = 0; jb < 4; ++jb)
      vraw[jb] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_off, kPage * n + ((g * 4 + jb) * 4 + 2 * (i & 1)) * 512, 0));
    vs = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, 8 * q, codes + (p.h_kv + g) * kPage + (i & 1) * T, 0));
  };
  k_request(0);
  v_request(0);

  float qx[2][8], qy[2][8];  // scaled query pairs of head m: frequencies 32 kk + 8 q + e; rows past the group are zeros
  {
    const uint16_t* row = p.q + ((size_t)seq * p.h_q + h0 + (m < nh ? m : 0)) * HD + 8 * q;
    const float scale = m < nh ? p.q_scale : 0.f;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const bf16x8 lo = load_frag(row + 32 * kk), hi = load_frag(row + 32 * kk + HALF);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qx[kk][e] = m < nh ? (float)lo[e] * scale : 0.f;
        qy[kk][e] = m < nh ? (float)hi[e] * scale : 0.f;
      }
    }
  }
  f16x8 lc[2][2], ls[2][2];  // rotation of the lane's two positions inside a step
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = p.lane_cs[(2 * m + b) * HALF + 32 * kk + 8 * q + e];
        lc[b][kk][e] = static_cast<_Float16>(cs.x);
        ls[b][kk][e] = static_cast<_Float16>(cs.y);
      }
  const double theta = p.rope_tab[lane] * kTurns;
  const int q_pos = p.q_pos[seq];

  float m_run = kNoWeight, l_run = 0.f;
  f32x4 o[8];
#pragma unroll
  for (int jb = 0; jb < 8; ++jb) o[jb] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int i = 0; i < n_steps; ++i) {
    const int pos0 = t_begin + i * T;
    {
      const double turns = (double)(q_pos - pos0) * theta;
      const float fr = (float)(turns - rint(turns));
      base_cs[w][lane] = make_float2(__builtin_amdgcn_cosf(fr), __builtin_amdgcn_sinf(fr));
      __builtin_amdgcn_wave_barrier();  // a wave's LDS operations run in order
    }
    // ---- scores
    f32x4 S[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    const float k_scale[2] = {pow2_of(ks & 255u), pow2_of((ks >> 8) & 255u)};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      f16x8 q_lo, q_hi;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = base_cs[w][32 * kk + 8 * q + e];
        q_lo[e] = static_cast<_Float16>(qx[kk][e] * cs.x - qy[kk][e] * cs.y);
        q_hi[e] = static_cast<_Float16>(qy[kk][e] * cs.x + qx[kk][e] * cs.y);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f16x8 x = codes_f16(u32x2{kraw[kk][2 * b], kraw[kk][2 * b + 1]}, k_scale[b]);
        const f16x8 y = codes_f16(u32x2{kraw[kk + 2][2 * b], kraw[kk + 2][2 * b + 1]}, k_scale[b]);
        const f16x8 lo = x * lc[b][kk] - y * ls[b][kk], hi = y * lc[b][kk] + x * ls[b][kk];
        S[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, q_lo, S[b], 0, 0, 0);
        S[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, q_hi, S[b], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
    k_request(i + 1);
    // ---- online softmax: a lane holds eight positions of query head m; the four lane groups meet in the maximum
    f16x8 pf;
    float alpha;
    {
      float s[8], t[8], mx = kNegInfQ;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[e] = pos0 + 8 * q + e < t_end ? S[e & 1][e >> 1] : kNegInfQ;
        const uint32_t byte = v_ok ? (vs[e >> 2] >> (8 * (e & 3))) & 255u : 127u;
        const float k = (float)byte - 127.f;
        t[e] = s[e] + k;
        mx = fmaxf(mx, s[e] + fmaxf(k, (float)kLeastExp));
      }
      const float2 a = row_pair(mx);
      mx = fmaxf(a.x, a.y);
      const float2 c = half_pair(mx);
      mx = fmaxf(c.x, c.y);
      const float m_new = fmaxf(m_run, mx);
      alpha = exp2f(m_run - m_new);
      m_run = m_new;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = pos0 + 8 * q + e < t_end;
        pf[e] = static_cast<_Float16>(in ? exp2f(t[e] - m_new) : 0.f);
        sum += in ? exp2f(s[e] - m_new) : 0.f;
      }
      l_run = l_run * alpha + sum;
    }
    // ---- o += V^T P'^T
#pragma unroll
    for (int jb = 0; jb < 4; ++jb)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        u32x2 v = {vraw[jb][2 * b], vraw[jb][2 * b + 1]};
        if (pos0 + T > t_end) v = keep_bytes(v, t_end - pos0 - 8 * q);  // slots past the context hold anything, NaN codes too
#pragma unroll
        for (int j = 0; j < 4; ++j) o[2 * jb + b][j] *= alpha;
        o[2 * jb + b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(v), pf, o[2 * jb + b], 0, 0, 0);
      }
    v_request(i + 1);
  }

  // ---- partials: O^T has coordinates along the accumulator rows (32 jb + 2 (4 q + j) + b) and query head m
  const float2 a = row_pair(l_run);
  const float2 c = half_pair(a.x + a.y);
  const float l = c.x + c.y, inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  if (m < nh) {
    const size_t row = ((size_t)seq * p.n_splits + split) * p.h_q + h0 + m;
    if (q == 0) {
      p.part_ml[row * 2] = n_steps > 0 ? m_run : kNegInfQ;
      p.part_ml[row * 2 + 1] = l;
    }
#pragma unroll
    for (int jb = 0; jb < 4; ++jb) {
      u32x4 pk;
#pragma unroll
      for (int j = 0; j < 4; ++j) pk[j] = (uint32_t)f16_bits(o[2 * jb][j] * inv) | ((uint32_t)f16_bits(o[2 * jb + 1][j] * inv) << 16);
      *reinterpret_cast<u32x4*>(p.part_o + row * HD + 32 * jb + 8 * q) = pk;
    }
  }
}

// ------------------------------------------------------------------------------------------------ host
namespace {
size_t align256q(size_t x) { return (x + 255) & ~(size_t)255; }
size_t q8_lds_bytes(const lorc_layer_desc& d) {
  return (size_t)d.rank_k * 64 + 4 * 32 * 32 * 4 + (size_t)q8_groups(d.rank_v) * 2048 + 2 * 32 * 4;
}
}  // namespace

namespace {
// Which kernel, and how it divides a sequence.  Rotary: stationary where its registers hold the factor, wide for the rest (16 x 4096 positions
// on either: 32/8 heads rank 512 77 / 122 us, rank 128 43 / 76, 16/16 heads rank 192 78 / 209).  Absorbed: the two page buffers decide.
// Walk: workgroups per (sequence, split), those that share a compute unit, the pages that a split
// walks at most (their ids live in LDS).
struct Q8Walk {
  long units, per_cu, most;
  int kernel;  // rotary: 1 stationary, 2 wide; absorbed: 1 ranks to 512, 0 above
};
Q8Walk q8_walk(const lorc_layer_desc& d, Q8Form form) {
  constexpr long kAny = (1 << 30) / kPage;
  if (form == Q8Form::kPlain) return {(d.n_kv_heads * ((d.n_q_heads / d.n_kv_heads + 15) / 16) + 3) / 4, 2, kAny, 0};
  if (form == Q8Form::kAbsorbed) {
    const bool fast = q8_absorbed_shape_ok(d);
    return {(d.n_q_heads + 31) / 32, 1, fast ? q8_absorbed_max_tiles() : kAny, fast};
  }
  if (q8_stationary_shape_ok(d)) return {(d.n_kv_heads + 1) / 2, 1, q8_stationary_max_tiles(), 1};
  return {q8_wide_units(d), 1, q8_wide_max_tiles(), 2};
}
}  // namespace

bool q8_shape_ok(const lorc_layer_desc& d, Q8Form form, int max_ctx) {
  if (form == Q8Form::kPlain ? !plain_shape_ok(d) : d.rank_k > kStreamMaxRank || d.rank_v > kStreamMaxRank) return false;
  // the merge joins 512 splits; and a split's end has to stay below 2^31
  return max_ctx <= (1 << 30) && (max_ctx + kPage - 1) / kPage <= 512 * q8_walk(d, form).most;
}

// Splits: the workgroups run in rounds of what the device holds, a round lasts as long as its pages and the set-up of a workgroup,
// which costs about two pages.  One workgroup too many is a whole round: against the fewest splits that give every compute unit one, rank
// 512, 12 x 4096 positions 95 -> 64 us, 24 x 4096 161 -> 121, 40 KV heads 8 x 2000 125 -> 98, absorbed 24 x 4096 54 -> 41.  (Lengths are on the
// device: sequences count as max_ctx here.)
constexpr long kQ8Rounds = 6, kQ8Setup = 2;
DecodePlan make_q8_plan(const lorc_layer_desc& d, Q8Form form, int b, int max_ctx, int n_cus, int max_splits) {
  DecodePlan pl{};
  if (!q8_shape_ok(d, form, max_ctx)) return pl;
  pl.tile = kPage;
  int n_tiles = (max_ctx + kPage - 1) / kPage;
  if (n_tiles < 1) n_tiles = 1;
  const auto [units, per_cu, most, kernel] = q8_walk(d, form);
  pl.stationary = kernel;
  const long least = (n_tiles + most - 1) / most;
  const long slots = per_cu * (n_cus > 0 ? n_cus : 256), first = (b * units + slots - 1) / slots;
  long ns = 1, best = LONG_MAX;
  for (long rounds = first; rounds < first + kQ8Rounds; ++rounds) {
    const long most_here = rounds * slots / (b * units);
    const long here = most_here > 64 ? 64 : most_here > n_tiles ? n_tiles : most_here;
    const long cost = rounds * ((n_tiles + here - 1) / here + kQ8Setup);
    if (cost < best) {
      best = cost;
      ns = here;
    }
  }
  if (ns > max_splits) ns = max_splits;
  if (ns < least) ns = least;
  if (ns > n_tiles) ns = n_tiles;
  pl.tiles_per_split = (int)((n_tiles + ns - 1) / ns);
  pl.n_splits = (n_tiles + pl.tiles_per_split - 1) / pl.tiles_per_split;
  const int out_w = form == Q8Form::kPlain ? d.head_dim : d.rank_v;
  size_t off = 0;
  pl.off_ml = off;
  off = align256q(off + (size_t)b * pl.n_splits * d.n_q_heads * 2 * 4);
  pl.off_o = off;
  off = align256q(off + (size_t)b * pl.n_splits * d.n_q_heads * out_w * 2);
  pl.total_bytes = off;
  return pl;
}

// A plan of as many splits as a workspace of `bytes` holds.  The fewest that a kernel can do with grow with the context and with b: a
// larger call's size always holds them.
DecodePlan make_q8_plan_within(const lorc_layer_desc& d, Q8Form form, int b, int max_ctx, int n_cus, size_t bytes) {
  DecodePlan pl = make_q8_plan(d, form, b, max_ctx, n_cus, kAnySplits);
  while (pl.total_bytes > bytes && pl.n_splits > 1) {
    const DecodePlan fewer = make_q8_plan(d, form, b, max_ctx, n_cus, pl.n_splits - 1);
    if (fewer.n_splits >= pl.n_splits) break;  // the fewest that the kernel can walk
    pl = fewer;
  }
  return pl;
}

int set_kernel_attributes_decode_q8() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(decode_q8_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess
             ? LORC_OK : LORC_EHIP;
}

int launch_decode_q8(const lorc_layer_desc& d, Q8Form form, const DecodeParams& p, const DecodePlan& plan, hipStream_t s) {
  if (plan.total_bytes == 0) return LORC_EUNSUPPORTED;
  const int units = p.b * p.n_splits;
  if (form == Q8Form::kPlain) {
    const int n_units = p.h_kv * ((p.G + 15) / 16);
    const dim3 grid(units * ((n_units + 3) / 4));
    if (int rc = launch_kernel(p.G > 16 ? decode_plain_q8_kernel<true> : decode_plain_q8_kernel<false>, grid, dim3(256), 0, s, p)) return rc;
    return launch_decode_merge(p, true, s);
  }
  if (plan.stationary) {
    if (int rc = form == Q8Form::kAbsorbed ? launch_decode_q8_absorbed(p, s)
                 : plan.stationary == 2    ? launch_decode_q8_wide(d, p, s)
                                           : launch_decode_q8_stationary(p, s))
      return rc;
    return launch_decode_merge(p, false, s);
  }
  const size_t lds = q8_lds_bytes(d);
  if (lds > 160 * 1024) return LORC_EUNSUPPORTED;
  if (int rc = launch_kernel(decode_q8_kernel, dim3(units * ((p.h_q + 31) / 32)), dim3(256), lds, s, p)) return rc;
  return launch_decode_merge(p, false, s);
}

}  // namespace lorc
