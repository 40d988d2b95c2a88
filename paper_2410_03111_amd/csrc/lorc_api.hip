// C ABI of the device entry points: argument validation on the host, then kernel launches on the caller's
// stream.  Nothing here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>

#include "lorc.h"
#include "lorc_kernels.h"
#include "lorc_layout.h"

using namespace lorc;

namespace {
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The only state the library keeps: per device, whether the large-LDS function attributes have been set and how
// many compute units it has.  Filled by the first entry point called with that device current (normally
// lorc_pack_factors); the attribute call cannot be captured into a HIP graph, every later call can.
constexpr int kMaxDevices = 64;
std::atomic<int> g_device_cus[kMaxDevices];  // 0 = not initialised yet

// Split partials of lorc_decode_attention_static: device memory that belongs to the library's code object, one
// copy per GPU.  Host code never uses the array's name as an address; it asks the runtime for the device address
// once per device (below) and passes that pointer on.
constexpr size_t kStaticScratchBytes = LORC_STATIC_WORKSPACE_BYTES;
static __device__ __align__(256) __attribute__((used)) unsigned char scratch[kStaticScratchBytes];
void* g_scratch_ptr[kMaxDevices];  // device address of `scratch` on each device; valid once g_device_cus is set

int device_ready(int* n_cus) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return LORC_EHIP;
  int v = g_device_cus[dev].load(std::memory_order_acquire);
  if (v == 0) {
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) return LORC_EHIP;
    if (int rc = set_kernel_attributes_append()) return rc;
    if (int rc = set_kernel_attributes_decode()) return rc;
    if (int rc = set_kernel_attributes_prefill()) return rc;
    if (int rc = set_kernel_attributes_decode_q8()) return rc;
    if (int rc = set_kernel_attributes_decode_q8_stationary()) return rc;
    if (int rc = set_kernel_attributes_decode_q8_absorbed()) return rc;
    if (int rc = set_kernel_attributes_decode_q8_wide()) return rc;
    void* sp = nullptr;
    if (hipGetSymbolAddress(&sp, HIP_SYMBOL(scratch)) != hipSuccess || sp == nullptr) return LORC_EHIP;
    g_scratch_ptr[dev] = sp;
    g_device_cus[dev].store(v, std::memory_order_release);
  }
  if (n_cus) *n_cus = v;
  return LORC_OK;
}

// Compute-unit count for the workspace-size helpers, which must agree with the launch: the current device's if it
// can be asked, else the MI355X's.
int cu_count_or_default() {
  int dev = 0, v = 0;
  if (hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < kMaxDevices) {
    v = g_device_cus[dev].load(std::memory_order_acquire);
    if (v > 0) return v;
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0) return v;
  }
  (void)hipGetLastError();  // no device: not an error of this call
  return 256;
}

float softmax_scale_log2(const lorc_layer_desc& d) {
  const float scale = d.softmax_scale > 0.f ? d.softmax_scale : 1.0f / std::sqrt((float)d.head_dim);
  return scale * 1.4426950408889634f;
}

// Argument checks shared by the decode entry points (rotary, latent-space output, absorbed query): everything that
// can be refused without asking the device.
int decode_args(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos, bool needs_q_pos, const int32_t* ctx_len,
                int32_t b, int32_t max_ctx, const void* packed, const void* cache, const int32_t* block_table,
                int32_t max_pages, int32_t n_pages, const void* out, const void* workspace) {
  if (!desc || !q || (needs_q_pos && !q_pos) || !ctx_len || !packed || !cache || !block_table || !out || !workspace) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  if (b <= 0 || max_ctx < 0 || max_pages <= 0 || n_pages <= 0) return LORC_EINVAL;
  if ((long)max_pages * kPage < max_ctx) return LORC_EINVAL;
  if (!aligned16(q) || !aligned16(packed) || !aligned16(cache) || !aligned16(out)) return LORC_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return LORC_EINVAL;
  return LORC_OK;
}

// Workspace check and the parameter block of the decode kernels.
int decode_params(DecodeParams& p, const lorc_layer_desc* desc, const void* q, const int32_t* q_pos, bool needs_q_pos,
                  const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed, const void* cache,
                  const int32_t* block_table, int32_t max_pages, int32_t n_pages, void* out, void* workspace,
                  size_t workspace_bytes, const DecodePlan& plan, int latent_out, int n_cus) {
  if (plan.total_bytes == 0) return LORC_EUNSUPPORTED;  // no kernel path takes this shape
  if (workspace_bytes < plan.total_bytes) return LORC_EWORKSPACE;
  const int n = desc->n_kv_heads * desc->head_dim;
  const uint16_t* pk = static_cast<const uint16_t*>(packed);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.q = static_cast<const uint16_t*>(q);
  p.q_pos = q_pos;
  p.ctx_len = ctx_len;
  p.bk = pk + packed_off_bk(desc->d_model, desc->rank_k, desc->rank_v);
  p.bv = pk + packed_off_bv(desc->d_model, desc->rank_k, desc->rank_v, n);
  p.cache = static_cast<const uint16_t*>(cache);
  p.block_table = block_table;
  p.out = static_cast<uint16_t*>(out);
  p.latent_out = latent_out;
  p.rope_tab = reinterpret_cast<const double*>(pk + packed_off_rope(desc->d_model, desc->rank_k, desc->rank_v, n));
  p.lane_cs = reinterpret_cast<const float2*>(p.rope_tab + 64);
  p.part_ml = reinterpret_cast<float*>(ws + plan.off_ml);
  p.part_o = reinterpret_cast<uint16_t*>(ws + plan.off_o);
  p.scores = reinterpret_cast<float*>(ws + plan.off_scores);
  p.score_stride = plan.score_stride;
  p.v_chunks = plan.v_chunks;
  p.b = b;
  p.h_q = desc->n_q_heads;
  p.h_kv = desc->n_kv_heads;
  p.G = desc->n_q_heads / desc->n_kv_heads;
  p.head_dim = desc->head_dim;
  p.r_k = desc->rank_k;
  p.r_v = desc->rank_v;
  p.n_tasks = n / 64;
  p.max_ctx = max_ctx;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.n_splits = plan.n_splits;
  p.tiles_per_split = plan.tiles_per_split;
  p.page_elems = page_elems(desc->rank_k, desc->rank_v);
  p.rope_base = desc->rope_base;
  p.q_scale = softmax_scale_log2(*desc);
  p.n_cus = n_cus;
  return LORC_OK;
}

int decode_rotary(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos, const int32_t* ctx_len, int32_t b,
                  int32_t max_ctx, const void* packed, const void* cache, const int32_t* block_table, int32_t max_pages,
                  int32_t n_pages, void* out, void* workspace, size_t workspace_bytes, void* stream, void* ev_begin,
                  void* ev_end, int latent_out, bool plain = false) {
  if (int rc = decode_args(desc, q, q_pos, true, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out, workspace))
    return rc;
  if (plain && !plain_shape_ok(*desc)) return LORC_EUNSUPPORTED;
  int n_cus = 0;
  if (int rc = device_ready(&n_cus)) return rc;
  const DecodePlan plan = plain ? make_wide_plan(*desc, b, max_ctx, n_cus, true)
                                : make_decode_plan_within(*desc, b, max_ctx, n_cus, workspace_bytes);
  DecodeParams p;
  if (int rc = decode_params(p, desc, q, q_pos, true, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages,
                             out, workspace, workspace_bytes, plan, latent_out, n_cus))
    return rc;
  return launch_decode(p, plan, static_cast<hipStream_t>(stream), static_cast<hipEvent_t>(ev_begin),
                       static_cast<hipEvent_t>(ev_end));
}
}  // namespace

extern "C" {

size_t lorc_packed_bytes(const lorc_layer_desc* desc) {
  if (!desc || check_desc(*desc) != LORC_OK) return 0;
  return packed_total_elems(desc->d_model, desc->rank_k, desc->rank_v, desc->n_kv_heads * desc->head_dim) * 2;
}

int lorc_pack_factors(const lorc_layer_desc* desc, const void* A_k, const void* A_v, const void* B_k,
                      const void* B_v, void* packed, void* stream) {
  if (!desc || !A_k || !A_v || !packed) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  // an uncompressed layer (rank = n on both sides) has identity read-side factors, which are never stored
  const int n_cols = desc->n_kv_heads * desc->head_dim;
  const bool no_b = !B_k && !B_v;
  if ((!B_k || !B_v) && !(no_b && desc->rank_k == n_cols && desc->rank_v == n_cols)) return LORC_EINVAL;
  if (!aligned16(packed)) return LORC_EINVAL;
  if (int rc = device_ready(nullptr)) return rc;
  return launch_pack(*desc, A_k, A_v, B_k, B_v, packed, static_cast<hipStream_t>(stream));
}

int lorc_append_latent(const lorc_layer_desc* desc, const void* x, int32_t T, const void* packed,
                       const int32_t* slot_seq, const int32_t* slot_pos, const int32_t* block_table,
                       int32_t n_seqs, int32_t max_pages, int32_t n_pages, void* cache, void* stream) {
  if (!desc || !x || !packed || !slot_seq || !slot_pos || !block_table || !cache) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  if (T < 0 || n_seqs <= 0 || max_pages <= 0 || n_pages <= 0) return LORC_EINVAL;
  if (!aligned16(x) || !aligned16(packed) || !aligned16(cache)) return LORC_EINVAL;
  if (T == 0) return LORC_OK;
  int n_cus = 0;
  if (int rc = device_ready(&n_cus)) return rc;
  AppendParams p;
  p.x = static_cast<const uint16_t*>(x);
  p.at = static_cast<const uint16_t*>(packed);
  p.at_tiled = p.at + packed_off_at_tiled(desc->d_model, desc->rank_k, desc->rank_v, desc->n_kv_heads * desc->head_dim);
  p.slot_seq = slot_seq;
  p.slot_pos = slot_pos;
  p.block_table = block_table;
  p.cache = static_cast<uint16_t*>(cache);
  p.T = T;
  p.D = desc->d_model;
  p.r_k = desc->rank_k;
  p.r_v = desc->rank_v;
  p.n_seqs = n_seqs;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.page_elems = page_elems(desc->rank_k, desc->rank_v);
  return launch_append(p, n_cus, static_cast<hipStream_t>(stream));
}

const char* lorc_append_plan_info(const lorc_layer_desc* desc, int32_t T) {
  if (!desc || check_desc(*desc) != LORC_OK || T <= 0) return nullptr;
  return append_kernel_name(desc->d_model, desc->rank_k, desc->rank_v, T, cu_count_or_default());
}

const char* lorc_append_kernel_info(const lorc_layer_desc* desc, int32_t T) {
  if (!desc || check_desc(*desc) != LORC_OK || T <= 0) return nullptr;
  return append_kernel_symbol(desc->d_model, desc->rank_k, desc->rank_v, T, cu_count_or_default());
}

size_t lorc_decode_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_ctx < 0) return 0;
  return make_decode_plan(*desc, b, max_ctx, cu_count_or_default()).total_bytes;
}

const char* lorc_decode_plan_info(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx, int32_t* n_splits,
                                  int32_t* tiles_per_split) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_ctx < 0) return nullptr;
  const DecodePlan plan = make_decode_plan(*desc, b, max_ctx, cu_count_or_default());
  if (plan.total_bytes == 0) return nullptr;
  if (n_splits) *n_splits = plan.n_splits;
  if (tiles_per_split) *tiles_per_split = plan.tiles_per_split;
  return plan.wide ? "wide_scores_kernel" : (plan.stationary == 1 && desc->rank_k > kStatSmallRank ? "decode_stationary_kernel" : "decode_split_kernel");
}

const char* lorc_decode_kernel_info(const lorc_layer_desc* desc, int32_t absorbed, int32_t b, int32_t max_ctx,
                                    size_t workspace_bytes, int32_t* n_splits, int32_t* tiles_per_split) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_ctx < 0) return nullptr;
  const int cus = cu_count_or_default();
  const DecodePlan plan = absorbed ? make_absorbed_plan_within(*desc, b, max_ctx, cus, workspace_bytes)
                                   : make_decode_plan_within(*desc, b, max_ctx, cus, workspace_bytes);
  if (plan.total_bytes == 0 || plan.total_bytes > workspace_bytes) return nullptr;
  if (n_splits) *n_splits = plan.n_splits;
  if (tiles_per_split) *tiles_per_split = plan.tiles_per_split;
  return decode_kernel_symbol(*desc, plan, absorbed != 0);
}

size_t lorc_decode_plain_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  if (!desc || check_desc(*desc) != LORC_OK || !plain_shape_ok(*desc) || b <= 0 || max_ctx < 0) return 0;
  return make_wide_plan(*desc, b, max_ctx, cu_count_or_default(), true).total_bytes;
}

int lorc_decode_attention_plain(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos,
                                const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed,
                                const void* cache, const int32_t* block_table, int32_t max_pages, int32_t n_pages,
                                void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return decode_rotary(desc, q, q_pos, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out, workspace,
                       workspace_bytes, stream, nullptr, nullptr, 0, true);
}

int lorc_decode_attention(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos,
                          const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed,
                          const void* cache, const int32_t* block_table, int32_t max_pages, int32_t n_pages,
                          void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return decode_rotary(desc, q, q_pos, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out, workspace,
                       workspace_bytes, stream, nullptr, nullptr, 0);
}

int lorc_decode_attention_timed(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos,
                                const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed,
                                const void* cache, const int32_t* block_table, int32_t max_pages,
                                int32_t n_pages, void* out, void* workspace, size_t workspace_bytes,
                                void* stream, void* ev_split_begin, void* ev_split_end) {
  return decode_rotary(desc, q, q_pos, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out, workspace,
                       workspace_bytes, stream, ev_split_begin, ev_split_end, 0);
}

int lorc_decode_attention_latent(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos,
                                 const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed,
                                 const void* cache, const int32_t* block_table, int32_t max_pages,
                                 int32_t n_pages, void* out_latent, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  return decode_rotary(desc, q, q_pos, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out_latent,
                       workspace, workspace_bytes, stream, nullptr, nullptr, 1);
}

int lorc_decode_attention_static(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos,
                                 const int32_t* ctx_len, int32_t b, int32_t max_ctx, const void* packed,
                                 const void* cache, const int32_t* block_table, int32_t max_pages, int32_t n_pages,
                                 void* out, void* stream) {
  if (!desc) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  if (int rc = device_ready(nullptr)) return rc;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return LORC_EHIP;
  // a problem whose partials do not fit the array in any plan is refused by the workspace check (LORC_EWORKSPACE)
  return decode_rotary(desc, q, q_pos, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out,
                       g_scratch_ptr[dev], kStaticScratchBytes, stream, nullptr, nullptr, 0);
}

// ---- decode without positional rotation, absorbed query (Section 4.1, Eq. 7)
size_t lorc_decode_absorbed_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_ctx < 0) return 0;
  return make_absorbed_plan(*desc, b, max_ctx, cu_count_or_default()).total_bytes;
}

int lorc_decode_attention_absorbed_timed(const lorc_layer_desc* desc, const void* q_lat, const int32_t* ctx_len, int32_t b,
                                         int32_t max_ctx, const void* packed, const void* cache,
                                         const int32_t* block_table, int32_t max_pages, int32_t n_pages, void* out,
                                         void* workspace, size_t workspace_bytes, void* stream, void* ev_split_begin,
                                         void* ev_split_end) {
  if (int rc = decode_args(desc, q_lat, nullptr, false, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out,
                           workspace))
    return rc;
  int n_cus = 0;
  if (int rc = device_ready(&n_cus)) return rc;
  const DecodePlan plan = make_absorbed_plan_within(*desc, b, max_ctx, n_cus, workspace_bytes);
  DecodeParams p;
  if (int rc = decode_params(p, desc, q_lat, nullptr, false, ctx_len, b, max_ctx, packed, cache, block_table, max_pages,
                             n_pages, out, workspace, workspace_bytes, plan, 0, n_cus))
    return rc;
  return launch_decode_absorbed(p, plan, static_cast<hipStream_t>(stream), static_cast<hipEvent_t>(ev_split_begin),
                                static_cast<hipEvent_t>(ev_split_end));
}

int lorc_decode_attention_absorbed(const lorc_layer_desc* desc, const void* q_lat, const int32_t* ctx_len, int32_t b,
                                   int32_t max_ctx, const void* packed, const void* cache, const int32_t* block_table,
                                   int32_t max_pages, int32_t n_pages, void* out, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  return lorc_decode_attention_absorbed_timed(desc, q_lat, ctx_len, b, max_ctx, packed, cache, block_table, max_pages,
                                              n_pages, out, workspace, workspace_bytes, stream, nullptr, nullptr);
}

size_t lorc_prefill_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_seqlen) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_seqlen < 0) return 0;
  return make_prefill_plan(*desc, b, max_seqlen).total_bytes;
}

namespace {
int prefill_common(const lorc_layer_desc* desc, const void* q, const int32_t* cu_seqlens, int32_t b,
                   int32_t total_tokens, int32_t max_seqlen, const void* packed, const void* cache,
                   const int32_t* block_table, int32_t max_pages, int32_t n_pages, void* out,
                   void* workspace, size_t workspace_bytes, void* stream, bool plain) {
  if (!desc || !q || !cu_seqlens || !packed || !cache || !block_table || !out || !workspace) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  if (b <= 0 || total_tokens < 0 || max_seqlen < 0 || max_seqlen > total_tokens || max_pages <= 0 || n_pages <= 0)
    return LORC_EINVAL;
  if ((long)max_pages * kPage < max_seqlen) return LORC_EINVAL;
  if (!aligned16(q) || !aligned16(packed) || !aligned16(cache) || !aligned16(out)) return LORC_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return LORC_EINVAL;
  if (plain && !plain_shape_ok(*desc)) return LORC_EUNSUPPORTED;
  if (total_tokens == 0) return LORC_OK;
  const PrefillPlan plan = make_prefill_plan(*desc, b, max_seqlen);
  const int n = desc->n_kv_heads * desc->head_dim;
  // the attention kernel addresses one sequence's rebuilt keys with 32-bit byte offsets
  if ((size_t)plan.lp * n * 2 > 0x7fffffffu) return LORC_EUNSUPPORTED;
  if (workspace_bytes < plan.total_bytes) return LORC_EWORKSPACE;
  int n_cus = 0;
  if (int rc = device_ready(&n_cus)) return rc;
  const uint16_t* pk = static_cast<const uint16_t*>(packed);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  PrefillParams p;
  p.q = static_cast<const uint16_t*>(q);
  p.cu_seqlens = cu_seqlens;
  p.bk = pk + packed_off_bk(desc->d_model, desc->rank_k, desc->rank_v);
  p.bv = pk + packed_off_bv(desc->d_model, desc->rank_k, desc->rank_v, n);
  p.cache = static_cast<const uint16_t*>(cache);
  p.block_table = block_table;
  p.out = static_cast<uint16_t*>(out);
  p.rope_tab = reinterpret_cast<const double*>(pk + packed_off_rope(desc->d_model, desc->rank_k, desc->rank_v, n));
  p.lane_cs = reinterpret_cast<const float2*>(p.rope_tab + 64);
  p.krot = reinterpret_cast<uint16_t*>(ws + plan.off_krot);
  p.vt = reinterpret_cast<uint16_t*>(ws + plan.off_vt);
  p.b = b;
  p.h_q = desc->n_q_heads;
  p.h_kv = desc->n_kv_heads;
  p.G = desc->n_q_heads / desc->n_kv_heads;
  p.head_dim = desc->head_dim;
  p.r_k = desc->rank_k;
  p.r_v = desc->rank_v;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  p.tiles_per_seq = plan.tiles_per_seq;
  p.lp = plan.lp;
  p.page_elems = page_elems(desc->rank_k, desc->rank_v);
  p.rope_base = desc->rope_base;
  p.q_scale = softmax_scale_log2(*desc);
  return launch_prefill(p, n_cus, static_cast<hipStream_t>(stream), plain);
}
}  // namespace

int lorc_prefill_attention(const lorc_layer_desc* desc, const void* q, const int32_t* cu_seqlens, int32_t b,
                           int32_t total_tokens, int32_t max_seqlen, const void* packed, const void* cache,
                           const int32_t* block_table, int32_t max_pages, int32_t n_pages, void* out,
                           void* workspace, size_t workspace_bytes, void* stream) {
  return prefill_common(desc, q, cu_seqlens, b, total_tokens, max_seqlen, packed, cache, block_table, max_pages, n_pages, out,
                        workspace, workspace_bytes, stream, false);
}

int lorc_prefill_attention_plain(const lorc_layer_desc* desc, const void* q, const int32_t* cu_seqlens, int32_t b,
                                 int32_t total_tokens, int32_t max_seqlen, const void* packed, const void* cache,
                                 const int32_t* block_table, int32_t max_pages, int32_t n_pages, void* out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  return prefill_common(desc, q, cu_seqlens, b, total_tokens, max_seqlen, packed, cache, block_table, max_pages, n_pages, out,
                        workspace, workspace_bytes, stream, true);
}

// ---- pages
namespace {
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr int kMostEntries = 1 << 30;  // of tables, counts and lists: what a plan adds up and steps over stays below 2^31
// (asked before a list's pointers are: a list of no entries needs none, and an empty tensor has none)
bool list_ok(int32_t n) { return n >= 0 && n <= kMostEntries; }
int table_args(const void* block_table, int32_t n_seqs, int32_t max_pages, const void* page_refs, int32_t n_pages) {
  if (!block_table || !page_refs || n_seqs <= 0 || max_pages <= 0 || n_pages <= 0) return LORC_EINVAL;
  if (max_pages > INT32_MAX / kPage || (long)n_seqs * max_pages > kMostEntries || n_pages > kMostEntries) return LORC_EINVAL;
  return LORC_OK;
}
}  // namespace

size_t lorc_pages_workspace_bytes(int32_t n_seqs, int32_t n_pages) {
  if (n_seqs <= 0 || n_pages <= 0) return 0;
  return 2 * align256((size_t)n_seqs * 4) + align256((size_t)n_pages * 4);
}

int lorc_copy_pages(void* pool, size_t page_bytes, int32_t n_pages, const int32_t* src, const int32_t* dst, int32_t count, void* stream) {
  if (!pool || n_pages <= 0 || !list_ok(count) || page_bytes == 0 || (page_bytes & 15) || !aligned16(pool)) return LORC_EINVAL;
  if (count == 0) return LORC_OK;
  if (!src || !dst) return LORC_EINVAL;
  return launch_copy_pages(pool, page_bytes, n_pages, src, dst, count, static_cast<hipStream_t>(stream));
}

int lorc_fork_sequences(int32_t* block_table, int32_t n_seqs, int32_t max_pages, int32_t* page_refs, int32_t n_pages,
                        const int32_t* parents, const int32_t* children, const int32_t* lens, int32_t n, int32_t* copy_src,
                        int32_t* copy_dst, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = table_args(block_table, n_seqs, max_pages, page_refs, n_pages)) return rc;
  if (!workspace || !list_ok(n)) return LORC_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return LORC_EINVAL;
  if (workspace_bytes < lorc_pages_workspace_bytes(n_seqs, n_pages)) return LORC_EWORKSPACE;
  if (n == 0) return LORC_OK;
  if (!parents || !children || !lens || !copy_src || !copy_dst || !status) return LORC_EINVAL;
  ForkParams p;
  p.block_table = block_table;
  p.page_refs = page_refs;
  p.parents = parents;
  p.children = children;
  p.lens = lens;
  p.copy_src = copy_src;
  p.copy_dst = copy_dst;
  p.status = status;
  p.owner = static_cast<int32_t*>(workspace);
  p.asks = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + align256((size_t)n_seqs * 4));
  p.n = n;
  p.n_seqs = n_seqs;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  return launch_fork(p, static_cast<hipStream_t>(stream));
}

int lorc_free_sequences(int32_t* block_table, int32_t n_seqs, int32_t max_pages, int32_t* page_refs, int32_t n_pages,
                        const int32_t* seqs, int32_t n, void* stream) {
  if (int rc = table_args(block_table, n_seqs, max_pages, page_refs, n_pages)) return rc;
  if (!list_ok(n)) return LORC_EINVAL;
  if (n == 0) return LORC_OK;
  if (!seqs) return LORC_EINVAL;
  return launch_free(block_table, n_seqs, max_pages, page_refs, n_pages, seqs, n, static_cast<hipStream_t>(stream));
}

int lorc_compact_pages(int32_t* block_table, int32_t n_seqs, int32_t max_pages, int32_t* page_refs, int32_t n_pages,
                       int32_t* move_src, int32_t* move_dst, int32_t max_moves, int32_t* page_map, void* stream) {
  if (int rc = table_args(block_table, n_seqs, max_pages, page_refs, n_pages)) return rc;
  if (!page_map || !list_ok(max_moves) || (max_moves > 0 && (!move_src || !move_dst))) return LORC_EINVAL;
  CompactParams p;
  p.block_table = block_table;
  p.page_refs = page_refs;
  p.move_src = move_src;
  p.move_dst = move_dst;
  p.page_map = page_map;
  p.max_moves = max_moves;
  p.n_seqs = n_seqs;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  return launch_compact(p, static_cast<hipStream_t>(stream));
}

int lorc_reserve_pages(int32_t* block_table, int32_t n_seqs, int32_t max_pages, int32_t* page_refs, int32_t n_pages,
                       const int32_t* seqs, const int32_t* lens, int32_t n, int32_t* status, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (int rc = table_args(block_table, n_seqs, max_pages, page_refs, n_pages)) return rc;
  if (!workspace || !list_ok(n)) return LORC_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return LORC_EINVAL;
  if (workspace_bytes < lorc_pages_workspace_bytes(n_seqs, n_pages)) return LORC_EWORKSPACE;
  if (n == 0) return LORC_OK;
  if (!seqs || !lens || !status) return LORC_EINVAL;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  ReserveParams p;
  p.block_table = block_table;
  p.page_refs = page_refs;
  p.seqs = seqs;
  p.lens = lens;
  p.status = status;
  p.owner = reinterpret_cast<int32_t*>(ws);
  p.first = reinterpret_cast<int32_t*>(ws + align256((size_t)n_seqs * 4));
  p.pages = reinterpret_cast<int32_t*>(ws + 2 * align256((size_t)n_seqs * 4));
  p.n = n;
  p.n_seqs = n_seqs;
  p.max_pages = max_pages;
  p.n_pages = n_pages;
  return launch_reserve(p, static_cast<hipStream_t>(stream));
}

// ---- 8-bit cache
int lorc_quantize_latents(const lorc_layer_desc* desc, const void* cache, const int32_t* block_table, int32_t max_pages, int32_t n_pages,
                          const int32_t* pos_begin, const int32_t* pos_end, int32_t b, int32_t max_tokens, void* cache_q8,
                          const int32_t* block_table_q8, int32_t max_pages_q8, int32_t n_pages_q8, void* stream) {
  if (!desc || !cache || !block_table || !pos_begin || !pos_end || !cache_q8 || !block_table_q8) return LORC_EINVAL;
  if (int rc = check_desc(*desc)) return rc;
  if (b <= 0 || max_tokens < 0 || max_pages <= 0 || n_pages <= 0 || max_pages_q8 <= 0 || n_pages_q8 <= 0) return LORC_EINVAL;
  if (max_pages > INT32_MAX / kPage || max_pages_q8 > INT32_MAX / kPage) return LORC_EINVAL;
  if (!aligned16(cache) || !aligned16(cache_q8)) return LORC_EINVAL;
  if (max_tokens == 0) return LORC_OK;
  QuantizeParams p;
  p.src = static_cast<const uint16_t*>(cache);
  p.dst = static_cast<unsigned char*>(cache_q8);
  p.src_table = block_table;
  p.dst_table = block_table_q8;
  p.pos_begin = pos_begin;
  p.pos_end = pos_end;
  p.b = b;
  p.src_max_pages = max_pages;
  p.src_pages = n_pages;
  p.dst_max_pages = max_pages_q8;
  p.dst_pages = n_pages_q8;
  const int least = max_pages < max_pages_q8 ? max_pages : max_pages_q8;
  p.max_tokens = max_tokens;
  p.span = (int)(((long)max_tokens + 2 * kPage - 2) / kPage);  // pages that max_tokens positions touch at most
  if (p.span > least) p.span = least;
  p.r_k = desc->rank_k;
  p.r_v = desc->rank_v;
  return launch_quantize(p, static_cast<hipStream_t>(stream));
}

namespace {
size_t q8_workspace(const lorc_layer_desc* desc, Q8Form form, int32_t b, int32_t max_ctx) {
  if (!desc || check_desc(*desc) != LORC_OK || b <= 0 || max_ctx < 0) return 0;
  return make_q8_plan(*desc, form, b, max_ctx, cu_count_or_default(), kAnySplits).total_bytes;
}

int decode_q8(const lorc_layer_desc* desc, Q8Form form, const void* q, const int32_t* q_pos, const int32_t* ctx_len, int32_t b,
              int32_t max_ctx, const void* packed, const void* cache, const int32_t* block_table, int32_t max_pages, int32_t n_pages,
              void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const bool rotary = form != Q8Form::kAbsorbed;
  if (int rc = decode_args(desc, q, q_pos, rotary, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out, workspace))
    return rc;
  if (!q8_shape_ok(*desc, form, max_ctx)) return LORC_EUNSUPPORTED;
  int n_cus = 0;
  if (int rc = device_ready(&n_cus)) return rc;
  const DecodePlan plan = make_q8_plan_within(*desc, form, b, max_ctx, n_cus, workspace_bytes);
  DecodeParams p;
  if (int rc = decode_params(p, desc, q, q_pos, rotary, ctx_len, b, max_ctx, packed, cache, block_table, max_pages, n_pages, out,
                             workspace, workspace_bytes, plan, 0, n_cus))
    return rc;
  p.page_elems = q8_page_bytes(desc->rank_k, desc->rank_v) / 2;
  p.coded = static_cast<const unsigned char*>(packed) +
            packed_off_coded_bytes(desc->d_model, desc->rank_k, desc->rank_v, desc->n_kv_heads * desc->head_dim);
  return launch_decode_q8(*desc, form, p, plan, static_cast<hipStream_t>(stream));
}
}  // namespace

size_t lorc_decode_quantized_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  return q8_workspace(desc, Q8Form::kRotary, b, max_ctx);
}

int lorc_decode_attention_quantized(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos, const int32_t* ctx_len, int32_t b,
                                    int32_t max_ctx, const void* packed, const void* cache_q8, const int32_t* block_table,
                                    int32_t max_pages, int32_t n_pages, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return decode_q8(desc, Q8Form::kRotary, q, q_pos, ctx_len, b, max_ctx, packed, cache_q8, block_table, max_pages, n_pages, out, workspace,
                   workspace_bytes, stream);
}

size_t lorc_decode_plain_quantized_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  return q8_workspace(desc, Q8Form::kPlain, b, max_ctx);
}

int lorc_decode_attention_plain_quantized(const lorc_layer_desc* desc, const void* q, const int32_t* q_pos, const int32_t* ctx_len,
                                          int32_t b, int32_t max_ctx, const void* packed, const void* cache_q8, const int32_t* block_table,
                                          int32_t max_pages, int32_t n_pages, void* out, void* workspace, size_t workspace_bytes,
                                          void* stream) {
  return decode_q8(desc, Q8Form::kPlain, q, q_pos, ctx_len, b, max_ctx, packed, cache_q8, block_table, max_pages, n_pages, out, workspace,
                   workspace_bytes, stream);
}

size_t lorc_decode_absorbed_quantized_workspace_bytes(const lorc_layer_desc* desc, int32_t b, int32_t max_ctx) {
  return q8_workspace(desc, Q8Form::kAbsorbed, b, max_ctx);
}

int lorc_decode_attention_absorbed_quantized(const lorc_layer_desc* desc, const void* q_lat, const int32_t* ctx_len, int32_t b,
                                             int32_t max_ctx, const void* packed, const void* cache_q8, const int32_t* block_table,
                                             int32_t max_pages, int32_t n_pages, void* out, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  return decode_q8(desc, Q8Form::kAbsorbed, q_lat, nullptr, ctx_len, b, max_ctx, packed, cache_q8, block_table, max_pages, n_pages, out,
                   workspace, workspace_bytes, stream);
}

int lorc_stream_read_probe(const void* src, size_t bytes, void* sink, void* stream) {
  if (!src || !sink || bytes == 0 || (bytes & 15) || !aligned16(src)) return LORC_EINVAL;
  return launch_stream_probe(src, bytes, sink, static_cast<hipStream_t>(stream));
}

int lorc_mfma_rate_probe(float* sink, size_t sink_floats, int32_t workgroups, int32_t iters, int32_t operands, void* stream) {
  if (!sink || workgroups <= 0 || workgroups > 65536 || iters <= 0 || iters > (1 << 24) || operands < 0 || operands > 2) return LORC_EINVAL;
  if (sink_floats < (size_t)workgroups * 256) return LORC_EINVAL;
  return launch_mfma_probe(sink, workgroups, iters, operands, static_cast<hipStream_t>(stream));
}

}  // extern "C"
