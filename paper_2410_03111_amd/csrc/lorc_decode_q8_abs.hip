// Absorbed-query decode over 8-bit pages (no positional rotation: scores are taken on the K codes themselves), ranks up to 512.
//
// Bound by the page stream.  One workgroup of eight waves per (sequence, context split, 32 query heads); pages go global -> LDS by
// direct copies, nearly two pages ahead (K and V in two buffers each, every buffer requested again as soon as its last reader is through).
// Scores: wave w takes 16 heads and 16 of the page's 64 positions over the whole rank, on the fp8 matrix instructions: the codes as
// they are, with the scale of the lane's position, against the query as a sum of two e4m3 codes (a bf16 entry has eight significant
// bits), made once.  So a score is complete in one wave and only row maxima are exchanged.  Weights carry the values' scales (see
// lorc_decode_q8.hip); wave w owns 64 value latents for all heads.
//
// Rank 512, 32 heads, 16 x 8192 positions: 33 us, 4.0 TB/s of pages (bf16 pages, twice the bytes: 52), the merge 8 more; 64 heads 57 us with
// the merge (144).  Short lists are a chain of launch, page id, page, softmax, store: 3 x 2000 positions, rank 384: 11.4 us + 5.7.
#include "lorc_device.h"
#include "lorc_kernels.h"
#include "lorc_q8.h"
#include "lorc_stationary.h"

namespace lorc {

namespace {
constexpr int kAbsHeads = 32, kAbsTiles = 1024;  // heads of a workgroup; pages it walks at most (their ids live in LDS)

__host__ __device__ constexpr size_t q8_abs_lds_bytes(int n) {
  return (size_t)n * 32768            // K and V codes, two buffers each, padded to whole groups of 128
         + 4 * 256                    // scale bytes of K, V
         + (size_t)n * 4096           // P' operands per group
         + kAbsHeads * 4 * 4          // row maxima of the four position blocks
         + 3 * kAbsHeads * 4          // alpha; running max and sum at the end
         + 4 * kAbsHeads * 4          // sums of the four position blocks
         + kAbsTiles * 4;
}
}  // namespace

// N: groups of 128 latents that K and V are padded to.
template <int N>
__global__ __launch_bounds__(kStatThreads, 2) void decode_q8_absorbed_kernel(DecodeParams p) {
  constexpr int T = 64, NW = kStatWaves, NT = kStatThreads, KB = N * 8192, VB = N * 8192;  // bytes of a K (V) buffer
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31, n16 = lane & 15, kg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_hb = (p.h_q + kAbsHeads - 1) / kAbsHeads, hblk = blockIdx.x % n_hb, ss = blockIdx.x / n_hb;
  const int split = ss % p.n_splits, seq = ss / p.n_splits;
  const int r_k = p.r_k, r_v = p.r_v, gk = q8_groups(r_k), gv = q8_groups(r_v);
  const int h0 = hblk * kAbsHeads, nh = p.h_q - h0 < kAbsHeads ? p.h_q - h0 : kAbsHeads;
  unsigned char* kbuf = smem;
  unsigned char* vbuf = kbuf + 2 * KB;
  unsigned char* sbytes = vbuf + 2 * VB;
  uint16_t* pbuf = reinterpret_cast<uint16_t*>(sbytes + 4 * 256);
  float* xm = reinterpret_cast<float*>(pbuf + N * 2048);
  float* alpha = xm + kAbsHeads * 4;
  float* m_fin = alpha + kAbsHeads;
  float* l_fin = m_fin + kAbsHeads;
  float* xs = l_fin + kAbsHeads;
  int* ids = reinterpret_cast<int*>(xs + 4 * kAbsHeads);
  const uint32_t k_lds = (uint32_t)(uintptr_t)kbuf, v_lds = (uint32_t)(uintptr_t)vbuf, s_lds = (uint32_t)(uintptr_t)sbytes;

  int ctx = p.ctx_len[seq];
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  const int tile_begin = split * p.tiles_per_split;
  int tile_end = tile_begin + p.tiles_per_split;
  const int n_tiles = (ctx + T - 1) / T;
  if (tile_end > n_tiles) tile_end = n_tiles;
  const int nt = tile_end > tile_begin ? tile_end - tile_begin : 0;
  const uint32_t page_bytes = (uint32_t)p.page_elems * 2u;
  const int* table = p.block_table + (size_t)seq * p.max_pages;
  auto fetch_id = [&](int t) {  // (in bounds whatever the context is, so that it does not wait for it)
    const int tile = tile_begin + t < p.max_pages ? tile_begin + t : p.max_pages - 1;
    return table[tile];
  };
  const int id0 = fetch_id(0), id1 = fetch_id(1);
  // this wave's share of the query, see below
  const int pb16 = w & 3, hb = w >> 2;
  u32x4 qv[4];
  {
    const int h = 16 * hb + n16, j0 = 128 * pb16 + 32 * kg;
    const bool real = h < nh && j0 < r_k;  // (ranks are multiples of 32)
    const uint16_t* row = p.q + ((size_t)seq * p.h_q + h0 + (h < nh ? h : 0)) * r_k + (real ? j0 : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      qv[i] = *reinterpret_cast<const u32x4*>(row + 8 * i);
#pragma unroll
      for (int c = 0; c < 4; ++c) qv[i][c] = real ? qv[i][c] : 0u;
    }
  }
  for (int i = tid; i < nt; i += NT) {
    const int id = table[tile_begin + i];
    ids[i] = id >= 0 && id < p.n_pages ? id : -1;
  }
  if (r_k < 128 * N) {  // the padding of the K tiles
    const u32x4 z = {0u, 0u, 0u, 0u};
    for (int i = tid; i < 2 * KB / 16; i += NT) reinterpret_cast<u32x4*>(kbuf)[i] = z;
  }
  __syncthreads();

  // ---- copies of a page: N blocks of 1 KiB per wave and part (blocks past the rank repeat the last one: the waits count copies); the
  // scale bytes of both parts, by every wave, come with K: the softmax reference takes the values' scales
  const uint32_t lane16 = (uint32_t)lane * 16u;
  const int k_rows = r_k >> 5, k_blocks = 2 * k_rows, v_blocks = r_v >> 4;
  auto tile_id = [&](int t) {
    const int id = __builtin_amdgcn_readfirstlane(ids[t < nt ? t : 0]);
    return t < nt ? id : -1;
  };
  auto rsrc_of = [&](int id) {
    const bool ok = id >= 0;
    return dma_rsrc(reinterpret_cast<const unsigned char*>(p.cache) + (ok ? (size_t)id * page_bytes : 0), ok ? page_bytes : 0u);
  };
  auto copy_k = [&](int id, int buf) {
    const u32x4 r = rsrc_of(id);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int b = w + NW * i;
      b = b < k_blocks ? b : k_blocks - 1;
      const int pb = b >= k_rows ? 1 : 0, c = b - pb * k_rows;
      dma_1k(r, uniform_u32(k_lds + (uint32_t)(buf * KB + pb * (KB / 2) + c * 1024)), lane16, uniform_u32((uint32_t)b * 1024u));
    }
    // (both begin in the page, lanes behind its end read zeros)
    dma_256(r, uniform_u32(s_lds + (uint32_t)(buf * 512)), lane16 >> 2, uniform_u32((uint32_t)(64 * (r_k + r_v))));
    dma_256(r, uniform_u32(s_lds + (uint32_t)(buf * 512 + 256)), lane16 >> 2, uniform_u32((uint32_t)(64 * (r_k + r_v + gk))));
  };
  auto copy_v = [&](int id, int buf) {
    const u32x4 r = rsrc_of(id);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int b = w + NW * i;
      b = b < v_blocks ? b : v_blocks - 1;
      dma_1k(r, uniform_u32(v_lds + (uint32_t)(buf * VB + b * 1024)), lane16, uniform_u32((uint32_t)(64 * r_k + b * 1024)));
    }
  };
  constexpr int kKCopies = N + 2, kVCopies = N;
  {
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(qv[i]));  // here, not behind the copies: the counter of loads is one for both
    auto valid_id = [&](int id_raw, int t) {
      const int id = __builtin_amdgcn_readfirstlane(id_raw);
      return t < nt && id >= 0 && id < p.n_pages ? id : -1;
    };
    const int first = valid_id(id0, 0);
    copy_k(first, 0);
    copy_v(first, 0);
    copy_k(valid_id(id1, 1), 1);
  }

  // ---- the query: head 16 hb + n16, latents 128 g + 32 kg .. + 31, under one power of two per head and group.  The four waves of a head
  // block make a group each and hand it round through the V buffer that is not in use yet.
  i32x8 qa[N][2];
  int q_bytes = 0;
  {
    unsigned char* shared = vbuf + VB;
    int* byte_of = reinterpret_cast<int*>(xm);  // [2 head blocks][4 groups][16 heads]
    const int g = pb16;
    if (g < N) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t a = magnitude(qv[i][c] & 0xffffu), b = magnitude(qv[i][c] >> 16);
          most = most > a ? most : a;
          most = most > b ? most : b;
        }
#pragma unroll
      for (int step = 16; step < 64; step <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)most, step, 64);
        most = most > o ? most : o;
      }
      const int byte = scale_byte(most);
      const float inv = inverse_scale(byte);
      if (kg == 0) byte_of[(hb * 4 + g) * 16 + n16] = byte;
      int hi[8], lo[8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t x = qv[i][2 * c], y = qv[i][2 * c + 1];
          code_pair(__uint_as_float(x << 16) * inv, __uint_as_float(x & 0xffff0000u) * inv, __uint_as_float(y << 16) * inv,
                    __uint_as_float(y & 0xffff0000u) * inv, hi[2 * i + c], lo[2 * i + c]);
        }
      u32x4* dst = reinterpret_cast<u32x4*>(shared + (size_t)(hb * N + g) * 4096) + lane;
      dst[0] = u32x4{(uint32_t)hi[0], (uint32_t)hi[1], (uint32_t)hi[2], (uint32_t)hi[3]};
      dst[64] = u32x4{(uint32_t)hi[4], (uint32_t)hi[5], (uint32_t)hi[6], (uint32_t)hi[7]};
      dst[128] = u32x4{(uint32_t)lo[0], (uint32_t)lo[1], (uint32_t)lo[2], (uint32_t)lo[3]};
      dst[192] = u32x4{(uint32_t)lo[4], (uint32_t)lo[5], (uint32_t)lo[6], (uint32_t)lo[7]};
    }
    lds_barrier();
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const u32x4* src = reinterpret_cast<const u32x4*>(shared + (size_t)(hb * N + u) * 4096) + lane;
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        const u32x4 a = src[128 * part], b = src[128 * part + 64];
        qa[u][part] = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
      }
      q_bytes |= byte_of[(hb * 4 + u) * 16 + n16] << (8 * u);
    }
  }
  float m_run[4], l_run[4];  // of heads 16 hb + 4 kg + j: reference, and this lane's share of the sum
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m_run[j] = kNoWeight;
    l_run[j] = 0.f;
  }
  f32x16 o[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  __builtin_amdgcn_s_waitcnt(0);  // no load but the copies is waited for from here on

  const int pos = 16 * pb16 + n16;  // this lane's position of the page (scores)
  const unsigned char* k_src = kbuf + (pb16 >> 1) * (KB / 2) + kg * 1024 + (16 * (pb16 & 1) + n16) * 8;
  // value latents 64 w + 32 i + l32; waves past the rank work on the first block and keep the result to themselves
  const bool has_v[2] = {64 * w < r_v, 64 * w + 32 < r_v};
  const unsigned char* v_src[2] = {vbuf + (has_v[0] ? 2 * w : 0) * 2048 + lane * 8, vbuf + (has_v[1] ? 2 * w + 1 : 0) * 2048 + lane * 8};
  const uint16_t* p_src = pbuf + (has_v[0] ? w >> 1 : 0) * 2048 + lane * 8;

  for (int t = 0; t < nt; ++t) {
    const int buf = t & 1, valid = ctx - (tile_begin + t) * T;
    dma_barrier<kVCopies + kKCopies>();  // this page's K has landed (younger: its V, the next K); every wave is through the previous V
    copy_v(tile_id(t + 1), buf ^ 1);
    // ---- scores
    int k_bytes = 0;
    uint32_t ub[N], top = 127 + kLeastExp;
#pragma unroll
    for (int g = 0; g < N; ++g) {
      k_bytes |= (int)sbytes[buf * 512 + 64 * g + pos] << (8 * g);
      ub[g] = sbytes[buf * 512 + 256 + (g < gv ? 64 * g : 0) + pos];
      top = ub[g] > top ? ub[g] : top;
    }
    f32x4 s4 = {0.f, 0.f, 0.f, 0.f};
    static_for<N>([&](auto g_c) {
      constexpr int g = decltype(g_c)::value;
      const unsigned char* at = k_src + buf * KB + g * 4096;
      const u32x2 x0 = *reinterpret_cast<const u32x2*>(at), x1 = *reinterpret_cast<const u32x2*>(at + 256);
      const u32x2 x2 = *reinterpret_cast<const u32x2*>(at + 512), x3 = *reinterpret_cast<const u32x2*>(at + 768);
      const i32x8 kb = {(int)x0[0], (int)x0[1], (int)x1[0], (int)x1[1], (int)x2[0], (int)x2[1], (int)x3[0], (int)x3[1]};
      s4 = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(qa[g][0], kb, s4, 0, 0, g, q_bytes, g, k_bytes);
      s4 = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(qa[g][1], kb, s4, 0, 0, g, q_bytes, g, k_bytes);
    });
    // ---- softmax: row maxima of the wave's 16 positions, exchanged between the four position blocks
    const float k_top = (float)top - (127.f + kTopExp);
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = pos < valid ? s4[j] * p.q_scale : kNegInfS;
      float mx = s[j] + k_top;
      mx = row_max_step<0>(mx);
      mx = row_max_step<1>(mx);
      mx = row_max_step<2>(mx);
      mx = row_max_step<3>(mx);
      xm[(16 * hb + 4 * kg + j) * 4 + pb16] = mx;  // (sixteen lanes, the same value)
    }
    lds_barrier();  // every wave is through this page's K and scales
    copy_k(tile_id(t + 2), buf);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int h = 16 * hb + 4 * kg + j;
      const f32x4 m4 = *reinterpret_cast<const f32x4*>(xm + h * 4);
      const float m_new = fmaxf(m_run[j], fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])));
      const float al = __builtin_amdgcn_exp2f(m_run[j] - m_new), e = __builtin_amdgcn_exp2f(s[j] - m_new);
      m_run[j] = m_new;
      l_run[j] = l_run[j] * al + e;
      alpha[h] = al;  // (four waves and sixteen lanes, the same value)
      uint16_t* dst = pbuf + ((size_t)pb16 * 64 + h + 32 * (n16 >> 3)) * 8 + (n16 & 7);
#pragma unroll
      for (int g = 0; g < N; ++g) dst[g * 2048] = f16_bits(below_f16_max(__builtin_amdgcn_ldexpf(e, (int)ub[g] - 127)));
    }
    dma_barrier<2 * kKCopies + kVCopies>();  // weights in place; this page's V has landed (younger: two K, one V)
    // ---- o = alpha o + P' codes
    f32x4 al[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) al[q] = *reinterpret_cast<const f32x4*>(alpha + 8 * q + 4 * hf);
    const bool ragged = valid < T;  // slots past the context hold anything, NaN codes too
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] *= al[j >> 2][j & 3];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        u32x2 v = *reinterpret_cast<const u32x2*>(v_src[i] + buf * VB + ks * 512);
        if (ragged) v = keep_bytes(v, valid - 16 * ks - 8 * hf);
        o[i] = mfma32_f16(load_frag_f16(p_src + ks * 512), codes_f16(v), o[i]);
      }
    }
  }

  // ---- partials
  __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float l = l_run[j];
    l += half_wave_peer<0>(l);
    l += half_wave_peer<1>(l);
    l += half_wave_peer<2>(l);
    l += half_wave_peer<3>(l);
    const int h = 16 * hb + 4 * kg + j;
    xs[h * 4 + pb16] = l;
    if (pb16 == 0) m_fin[h] = m_run[j];
  }
  __syncthreads();
  if (tid < kAbsHeads) l_fin[tid] = (xs[tid * 4] + xs[tid * 4 + 1]) + (xs[tid * 4 + 2] + xs[tid * 4 + 3]);
  __syncthreads();
  const size_t row0 = ((size_t)seq * p.n_splits + split) * p.h_q + h0;
  if (tid < nh) {
    p.part_ml[(row0 + tid) * 2] = nt > 0 ? m_fin[tid] : kNegInfS;
    p.part_ml[(row0 + tid) * 2 + 1] = l_fin[tid];
  }
  // rows through LDS, so that memory sees 16 bytes per lane: two bytes per lane took 4.4 us
  const int pitch = r_v * 2 + 16;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const int h = acc_row(j, hf);
    const float l = l_fin[h], inv = l > 0.f ? __builtin_amdgcn_rcpf(l) : l == 0.f ? 0.f : l;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (has_v[i]) *reinterpret_cast<uint16_t*>(smem + (size_t)h * pitch + (64 * w + 32 * i + l32) * 2) = f16_bits(o[i][j] * inv);
  }
  __syncthreads();
  const int per_row = r_v >> 3;
  for (int c = tid; c < nh * per_row; c += NT) {
    const int h = c / per_row, cc = c - h * per_row;
    *reinterpret_cast<u32x4*>(p.part_o + (row0 + h) * r_v + cc * 8) = *reinterpret_cast<const u32x4*>(smem + (size_t)h * pitch + cc * 16);
  }
}

// ------------------------------------------------------------------------------------------------ host
namespace {
using Q8AbsKernel = void (*)(DecodeParams);
Q8AbsKernel q8_abs_kernel(int n) {
  switch (n) {
    case 1: return decode_q8_absorbed_kernel<1>;
    case 2: return decode_q8_absorbed_kernel<2>;
    case 3: return decode_q8_absorbed_kernel<3>;
    default: return decode_q8_absorbed_kernel<4>;
  }
}
}  // namespace

bool q8_absorbed_shape_ok(const lorc_layer_desc& d) { return d.rank_k <= 512 && d.rank_v <= 512; }

int q8_absorbed_max_tiles() { return kAbsTiles; }

int set_kernel_attributes_decode_q8_absorbed() {
  for (int n = 1; n <= 4; ++n)
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(q8_abs_kernel(n)), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess)
      return LORC_EHIP;
  return LORC_OK;
}

int launch_decode_q8_absorbed(const DecodeParams& p, hipStream_t s) {
  const int gk = q8_groups(p.r_k), gv = q8_groups(p.r_v), n = gk > gv ? gk : gv;
  if (n > 4 || p.tiles_per_split > kAbsTiles) return LORC_EUNSUPPORTED;
  return launch_kernel(q8_abs_kernel(n), dim3(p.b * p.n_splits * ((p.h_q + kAbsHeads - 1) / kAbsHeads)), dim3(kStatThreads),
                       q8_abs_lds_bytes(n), s, p);
}

}  // namespace lorc
