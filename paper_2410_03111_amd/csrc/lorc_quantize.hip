// Latents from bf16 pages into 8-bit pages: e4m3 codes with a power of two per position and 128 latents.
//
// The scale of a group is 2^k, k the least exponent with amax <= 448 2^k (448: the largest e4m3 value).  A code keeps its four
// significant bits under any scale, so a power of two loses nothing against amax / 448, and it makes every product with a
// scale exact wherever it is applied.  One position per scale: a block of several positions would have to be rounded again
// whenever a later token of it is larger, and the cache would depend on how tokens were batched.
//
// Both pages hold their latents in the same element order, in which a wave's 64 lanes own 8 elements each of a 1 KiB (512 byte)
// tile.  K: a lane's elements belong to one position, a group is eight tiles and the two halves of the wave.  V: a lane's
// elements are eight positions of one latent, a group is four tiles and the 32 lanes of a half.  Either way the maximum of a
// group stays inside one wave, and a page is 2 (groups of K) + 4 (groups of V) units of work, one wave each.
// Bound by memory: 2 bytes read and 1 written per latent (+ 1 per 128).  4 prompts of 8192 positions, rank 512: 19 us, 5.2 TB/s; one token of
// each of 64 sequences: 6.0 us, the chain position -> page id -> latents -> maximum -> codes.
#include "lorc_device.h"
#include "lorc_kernels.h"
#include "lorc_q8.h"

namespace lorc {

namespace {
__device__ __forceinline__ uint32_t max_half(uint32_t v) {  // over the two halves of the wave
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const uint32_t a = r[0], b = r[1];
  return a > b ? a : b;
}
__device__ __forceinline__ int codes4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
__device__ __forceinline__ float elem(const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
}  // namespace

__global__ __launch_bounds__(256) void quantize_latents_kernel(QuantizeParams p) {
  const int gk = q8_groups(p.r_k), gv = q8_groups(p.r_v), units = 2 * gk + 4 * gv, blocks = (units + 3) / 4;
  const int lane = threadIdx.x & 63, hf = lane >> 5, l32 = lane & 31;
  int i = p.first + (int)blockIdx.x;
  const int unit = (i % blocks) * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  i /= blocks;
  const int seq = i / p.span, nth = i % p.span;
  if (unit >= units) return;
  int begin = p.pos_begin[seq], end = p.pos_end[seq];
  if (begin < 0) begin = 0;
  if (end <= begin) return;
  if (end - begin > p.max_tokens) end = begin + p.max_tokens;
  const int page = begin / kPage + nth;
  if (page >= p.src_max_pages || page >= p.dst_max_pages || end <= page * kPage) return;
  const int from = __builtin_amdgcn_readfirstlane(p.src_table[(size_t)seq * p.src_max_pages + page]);
  const int to = __builtin_amdgcn_readfirstlane(p.dst_table[(size_t)seq * p.dst_max_pages + page]);
  if (from < 0 || from >= p.src_pages || to < 0 || to >= p.dst_pages) return;
  const int lo = begin - page * kPage, hi = end - page * kPage;  // slots [lo, hi) of the page
  const uint16_t* src = p.src + (size_t)from * kPage * (p.r_k + p.r_v);
  unsigned char* dst = p.dst + (size_t)to * q8_page_bytes(p.r_k, p.r_v);
  unsigned char* scales = dst + (size_t)kPage * (p.r_k + p.r_v);

  if (unit < 2 * gk) {
    const int sb = unit & 1, g = unit >> 1, slot = 32 * sb + l32;
    if (32 * sb >= hi || 32 * sb + 32 <= lo) return;
    const int nks = p.r_k >> 4, n_t = nks - 8 * g < 8 ? nks - 8 * g : 8;
    const size_t at = ((size_t)(sb * nks + 8 * g) * 64 + lane) * 8;
    u32x4 v[8];
    uint32_t most = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (t < n_t) v[t] = *reinterpret_cast<const u32x4*>(src + at + (size_t)t * 512);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t < n_t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t a = magnitude(v[t][c] & 0xffffu), b = magnitude(v[t][c] >> 16);
          most = most > a ? most : a;
          most = most > b ? most : b;
        }
      }
    }
    most = max_half(most);
    const int byte = scale_byte(most);
    const float inv = inverse_scale(byte);
    if (slot < lo || slot >= hi) return;
    if (hf == 0) scales[g * kPage + slot] = (unsigned char)byte;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t < n_t) {
        u32x2 o;
#pragma unroll
        for (int c = 0; c < 2; ++c)
          o[c] = (uint32_t)codes4(elem(v[t], 4 * c) * inv, elem(v[t], 4 * c + 1) * inv, elem(v[t], 4 * c + 2) * inv, elem(v[t], 4 * c + 3) * inv);
        *reinterpret_cast<u32x2*>(dst + at + (size_t)t * 512) = o;
      }
    }
    return;
  }

  const int u = unit - 2 * gk, sq = u & 3, g = u >> 2;  // 16 slots of group g
  if (16 * sq >= hi || 16 * sq + 16 <= lo) return;
  const int nj = p.r_v >> 5, n_t = nj - 4 * g < 4 ? nj - 4 * g : 4;
  const size_t at = (size_t)kPage * p.r_k + ((size_t)(16 * g + sq) * 64 + lane) * 8;  // tile (4 g, sq); the next one is 4 tiles on
  u32x4 v[4];
  uint32_t most[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t < n_t) v[t] = *reinterpret_cast<const u32x4*>(src + at + (size_t)t * 2048);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (t < n_t) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t a = magnitude(e & 1 ? v[t][e >> 1] >> 16 : v[t][e >> 1] & 0xffffu);
        most[e] = most[e] > a ? most[e] : a;
      }
    }
  }
  int byte[8];
  float inv[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int step = 1; step < 32; step <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)most[e], step, 64);
      most[e] = most[e] > o ? most[e] : o;
    }
    byte[e] = scale_byte(most[e]);
    inv[e] = inverse_scale(byte[e]);
  }
  const int slot0 = 16 * sq + 8 * hf;  // the lane's eight slots
  if (l32 < 8) {
    int mine = byte[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mine = l32 == e ? byte[e] : mine;
    if (slot0 + l32 >= lo && slot0 + l32 < hi) scales[(gk + g) * kPage + slot0 + l32] = (unsigned char)mine;
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (t < n_t) {
      u32x2 o;
#pragma unroll
      for (int c = 0; c < 2; ++c)
        o[c] = (uint32_t)codes4(elem(v[t], 4 * c) * inv[4 * c], elem(v[t], 4 * c + 1) * inv[4 * c + 1], elem(v[t], 4 * c + 2) * inv[4 * c + 2],
                                elem(v[t], 4 * c + 3) * inv[4 * c + 3]);
      unsigned char* d = dst + at + (size_t)t * 2048;
      if (slot0 >= lo && slot0 + 8 <= hi) {
        *reinterpret_cast<u32x2*>(d) = o;
      } else {  // slots of other tokens share the word: single bytes
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (slot0 + e >= lo && slot0 + e < hi) d[e] = (unsigned char)(o[e >> 2] >> (8 * (e & 3)));
      }
    }
  }
}

int launch_quantize(const QuantizeParams& p, hipStream_t s) {
  const int units = 2 * q8_groups(p.r_k) + 4 * q8_groups(p.r_v);
  const size_t blocks = (size_t)p.b * p.span * ((units + 3) / 4);
  if (blocks > 0x7fffffffu) return LORC_EINVAL;
  return launch_parts((int)blocks, launch_blocks(256), [&](int first, int count) {
    QuantizeParams part = p;
    part.first = first;
    return launch_kernel(quantize_latents_kernel, dim3((uint32_t)count), dim3(256), 0, s, part);
  });
}

}  // namespace lorc
