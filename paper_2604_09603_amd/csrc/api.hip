// C ABI entry points: host-side argument checks, workspace sizing, launch.
#include <hip/hip_runtime.h>

#include <math.h>

#include <mutex>
#include <vector>

#include "echo.h"
#include "echo_internal.h"

namespace echo {

int device_cu_count() {
  static std::mutex mu;
  static std::vector<int> cache;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  std::lock_guard<std::mutex> lock(mu);
  if (dev >= int(cache.size())) cache.resize(dev + 1, 0);
  if (cache[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
      n = 256;
    cache[dev] = n;
  }
  return cache[dev];
}

}  // namespace echo

namespace {
inline bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }
inline hipStream_t as_stream(echo_stream_t s) { return reinterpret_cast<hipStream_t>(s); }

// The softmax takes each row's maximum of the raw logits as its reference and
// scales it afterwards, which is only valid for a positive finite scale.
inline bool scale_ok(float s) { return s > 0.0f && s <= 3.4028234663852886e38f; }

// Host-side checks and argument packing of the contiguous-cache attention:
// ECHO_OK with *a filled, or the error code.
int32_t attn_contiguous_args(const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                             const uint16_t* k_cache, const uint16_t* v_cache,
                             const int64_t* kv_offsets, int64_t kv_rows, const int32_t* q_offsets,
                             const uint32_t* tree_mask, int32_t mask_words, int32_t R,
                             int32_t max_rows, int32_t num_q_heads, int32_t num_kv_heads,
                             int32_t head_dim, float sm_scale, float* out, float* lse,
                             void* workspace, size_t workspace_bytes, int32_t* status,
                             hipEvent_t ev_start, hipEvent_t ev_stop, echo::AttnArgs* a_out) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || num_kv_heads < 1 || mask_words < 1 ||
      kv_rows < 0)
    return ECHO_ERR_INVALID_ARG;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(sm_scale)) return ECHO_ERR_INVALID_ARG;
  if (head_dim != ECHO_HEAD_DIM || R > ECHO_MAX_REQUESTS || kv_rows >= (int64_t(1) << 31))
    return ECHO_ERR_UNSUPPORTED;
  if (int64_t(max_rows) * num_q_heads >= (int64_t(1) << 26)) return ECHO_ERR_UNSUPPORTED;
  if (!q || !k_new || !v_new || !kv_offsets || !q_offsets || !tree_mask || !out || !workspace)
    return ECHO_ERR_INVALID_ARG;
  if (kv_rows > 0 && (!k_cache || !v_cache)) return ECHO_ERR_INVALID_ARG;
  if ((ev_start == nullptr) != (ev_stop == nullptr)) return ECHO_ERR_INVALID_ARG;
  if (!aligned256(workspace) ||
      workspace_bytes < echo::attn_workspace_bytes(R, max_rows, num_q_heads, num_kv_heads))
    return ECHO_ERR_WORKSPACE;
  // 16-byte vector loads of every bf16 row
  const uintptr_t mis = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) |
                        reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(k_cache) |
                        reinterpret_cast<uintptr_t>(v_cache) | reinterpret_cast<uintptr_t>(out);
  if (mis & 15u) return ECHO_ERR_INVALID_ARG;
  echo::AttnArgs& a = *a_out;
  a = echo::AttnArgs{};
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.kv_offsets = kv_offsets;
  a.kv_rows = kv_rows;
  a.q_offsets = q_offsets;
  a.tree_mask = tree_mask;
  a.mask_words = mask_words;
  a.R = R;
  a.max_rows = max_rows;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.sm_scale = sm_scale;
  a.out = out;
  a.lse = lse;
  a.workspace = workspace;
  a.status = status;
  a.ev_start = ev_start;
  a.ev_stop = ev_stop;
  return ECHO_OK;
}

int32_t attn_contiguous(const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                        const uint16_t* k_cache, const uint16_t* v_cache, const int64_t* kv_offsets,
                        int64_t kv_rows, const int32_t* q_offsets, const uint32_t* tree_mask,
                        int32_t mask_words, int32_t R, int32_t max_rows, int32_t num_q_heads,
                        int32_t num_kv_heads, int32_t head_dim, float sm_scale, float* out,
                        float* lse, void* workspace, size_t workspace_bytes, int32_t* status,
                        hipEvent_t ev_start, hipEvent_t ev_stop, hipStream_t stream) {
  echo::AttnArgs a;
  const int32_t rc = attn_contiguous_args(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows,
                                          q_offsets, tree_mask, mask_words, R, max_rows,
                                          num_q_heads, num_kv_heads, head_dim, sm_scale, out, lse,
                                          workspace, workspace_bytes, status, ev_start, ev_stop,
                                          &a);
  if (rc != ECHO_OK || max_rows == 0) return rc;
  return echo::launch_tree_verify_attn(a, stream);
}

// The same for a paged prefix.
int32_t attn_paged(const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                   const uint16_t* k_pages, const uint16_t* v_pages, int64_t num_pages,
                   int32_t page_size, const int32_t* block_table, int32_t max_pages_per_request,
                   const int32_t* prefix_len, const int32_t* q_offsets, const uint32_t* tree_mask,
                   int32_t mask_words, int32_t R, int32_t max_rows, int32_t num_q_heads,
                   int32_t num_kv_heads, int32_t head_dim, float sm_scale, float* out, float* lse,
                   void* workspace, size_t workspace_bytes, int32_t* status, hipEvent_t ev_start,
                   hipEvent_t ev_stop, hipStream_t stream) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || num_kv_heads < 1 || mask_words < 1 ||
      num_pages < 1 || max_pages_per_request < 1)
    return ECHO_ERR_INVALID_ARG;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(sm_scale)) return ECHO_ERR_INVALID_ARG;
  // a page holds whole 32-key tiles and a power-of-two number of rows
  if (page_size < 32 || (page_size & (page_size - 1)) != 0) return ECHO_ERR_UNSUPPORTED;
  if (head_dim != ECHO_HEAD_DIM || R > ECHO_MAX_REQUESTS) return ECHO_ERR_UNSUPPORTED;
  if (num_pages * int64_t(page_size) >= (int64_t(1) << 31)) return ECHO_ERR_UNSUPPORTED;
  if (int64_t(max_pages_per_request) * page_size >= (int64_t(1) << 31)) return ECHO_ERR_UNSUPPORTED;
  if (int64_t(max_rows) * num_q_heads >= (int64_t(1) << 26)) return ECHO_ERR_UNSUPPORTED;
  if (!q || !k_new || !v_new || !k_pages || !v_pages || !block_table || !prefix_len ||
      !q_offsets || !tree_mask || !out || !workspace)
    return ECHO_ERR_INVALID_ARG;
  if ((ev_start == nullptr) != (ev_stop == nullptr)) return ECHO_ERR_INVALID_ARG;
  if (!aligned256(workspace) ||
      workspace_bytes < echo::attn_workspace_bytes(R, max_rows, num_q_heads, num_kv_heads))
    return ECHO_ERR_WORKSPACE;
  const uintptr_t mis = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) |
                        reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(k_pages) |
                        reinterpret_cast<uintptr_t>(v_pages) | reinterpret_cast<uintptr_t>(out);
  if (mis & 15u) return ECHO_ERR_INVALID_ARG;
  if (max_rows == 0) return ECHO_OK;
  echo::AttnArgs a{};
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_cache = k_pages;
  a.v_cache = v_pages;
  a.kv_offsets = nullptr;
  a.kv_rows = 0;
  a.block_table = block_table;
  a.prefix_len = prefix_len;
  a.page_size = page_size;
  a.max_pages = max_pages_per_request;
  a.num_pages = num_pages;
  a.q_offsets = q_offsets;
  a.tree_mask = tree_mask;
  a.mask_words = mask_words;
  a.R = R;
  a.max_rows = max_rows;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.sm_scale = sm_scale;
  a.out = out;
  a.lse = lse;
  a.workspace = workspace;
  a.status = status;
  a.ev_start = ev_start;
  a.ev_stop = ev_stop;
  return echo::launch_tree_verify_attn(a, stream);
}
}  // namespace

extern "C" {

size_t echo_gate_workspace_size(int32_t R, int32_t N, int32_t budget) {
  if (R < 0 || N < 0 || budget < 0) return 0;
  return echo::gate_workspace_bytes(R, N, budget);
}

int32_t echo_gate(const int32_t* cand_offsets, const int32_t* parent, const float* logq,
                  int32_t R, int32_t N, int32_t budget, float* path_score, uint8_t* selected,
                  int32_t* num_selected, void* workspace, size_t workspace_bytes, int32_t* status,
                  echo_stream_t stream) {
  if (R < 1 || N < 0 || budget < 0) return ECHO_ERR_INVALID_ARG;
  if (R > ECHO_MAX_REQUESTS || budget > ECHO_MAX_BUDGET) return ECHO_ERR_UNSUPPORTED;
  if (!cand_offsets || !num_selected || !workspace) return ECHO_ERR_INVALID_ARG;
  if (N > 0 && (!parent || !logq || !selected)) return ECHO_ERR_INVALID_ARG;
  if (!aligned256(workspace) || workspace_bytes < echo::gate_workspace_bytes(R, N, budget))
    return ECHO_ERR_WORKSPACE;
  return echo::launch_gate(cand_offsets, parent, logq, R, N, budget, nullptr, nullptr, 0,
                           path_score, selected, num_selected, nullptr, workspace, status,
                           as_stream(stream));
}

size_t echo_gate_sparse_workspace_size(int32_t R, int32_t N, int32_t budget) {
  return echo_gate_workspace_size(R, N, budget);
}

int32_t echo_gate_sparse(const int32_t* cand_offsets, const int32_t* parent, const float* logq,
                         int32_t R, int32_t N, int32_t budget, const int32_t* sig_depth,
                         const float* log_tau, int32_t num_sig, float* path_score,
                         uint8_t* selected, int32_t* num_selected, int32_t* trunc_depth,
                         void* workspace, size_t workspace_bytes, int32_t* status,
                         echo_stream_t stream) {
  if (R < 1 || N < 0 || budget < 0) return ECHO_ERR_INVALID_ARG;
  if (R > ECHO_MAX_REQUESTS || budget > ECHO_MAX_BUDGET) return ECHO_ERR_UNSUPPORTED;
  if (!cand_offsets || !num_selected || !workspace) return ECHO_ERR_INVALID_ARG;
  if (N > 0 && (!parent || !logq || !selected)) return ECHO_ERR_INVALID_ARG;
  if (num_sig < 0 || num_sig > ECHO_MAX_CHECKPOINTS) return ECHO_ERR_INVALID_ARG;
  if (num_sig > 0 && (!sig_depth || !log_tau)) return ECHO_ERR_INVALID_ARG;
  for (int k = 0; k < num_sig; ++k) {
    if (sig_depth[k] < 1 || sig_depth[k] > ECHO_MAX_DEPTH) return ECHO_ERR_INVALID_ARG;
    if (log_tau[k] != log_tau[k]) return ECHO_ERR_INVALID_ARG;  // NaN
  }
  if (!aligned256(workspace) || workspace_bytes < echo::gate_workspace_bytes(R, N, budget))
    return ECHO_ERR_WORKSPACE;
  return echo::launch_gate(cand_offsets, parent, logq, R, N, budget, sig_depth, log_tau, num_sig,
                           path_score, selected, num_selected, trunc_depth, workspace, status,
                           as_stream(stream));
}

size_t echo_gate_elastic_workspace_size(int32_t R, int32_t N, int32_t budget) {
  if (R < 0 || N < 0 || budget < 0) return 0;
  return echo::gate_elastic_workspace_bytes(R, N, budget);
}

int32_t echo_gate_elastic(const int32_t* cand_offsets, const int32_t* parent, const float* logq,
                          int32_t R, int32_t N, int32_t budget, const int32_t* sig_depth,
                          const float* log_tau, int32_t num_sig, int32_t w_topk, int32_t w_max,
                          float* path_score, uint8_t* selected, int32_t* num_selected,
                          int32_t* trunc_depth, void* workspace, size_t workspace_bytes,
                          int32_t* status, echo_stream_t stream) {
  if (R < 1 || N < 0 || budget < 0 || w_topk < 1 || w_max < 0) return ECHO_ERR_INVALID_ARG;
  if (R > ECHO_MAX_REQUESTS || budget > ECHO_MAX_BUDGET) return ECHO_ERR_UNSUPPORTED;
  if (!cand_offsets || !num_selected || !workspace) return ECHO_ERR_INVALID_ARG;
  if (N > 0 && (!parent || !logq || !selected)) return ECHO_ERR_INVALID_ARG;
  if (num_sig < 0 || num_sig > ECHO_MAX_CHECKPOINTS) return ECHO_ERR_INVALID_ARG;
  if (num_sig > 0 && (!sig_depth || !log_tau)) return ECHO_ERR_INVALID_ARG;
  for (int k = 0; k < num_sig; ++k) {
    if (sig_depth[k] < 1 || sig_depth[k] > ECHO_MAX_DEPTH) return ECHO_ERR_INVALID_ARG;
    if (log_tau[k] != log_tau[k]) return ECHO_ERR_INVALID_ARG;  // NaN
  }
  if (!aligned256(workspace) ||
      workspace_bytes < echo::gate_elastic_workspace_bytes(R, N, budget))
    return ECHO_ERR_WORKSPACE;
  return echo::launch_gate_elastic(cand_offsets, parent, logq, R, N, budget, sig_depth, log_tau,
                                   num_sig, w_topk, w_max, path_score, selected, num_selected,
                                   trunc_depth, workspace, status, as_stream(stream));
}

size_t echo_build_tree_mask_workspace_size(int32_t R, int32_t N, int32_t budget) {
  (void)R;
  (void)N;
  (void)budget;
  return 0;  // everything lives in LDS
}

int32_t echo_build_tree_mask(const int32_t* cand_offsets, const int32_t* parent,
                             const int32_t* token, const uint8_t* selected,
                             const int32_t* root_token, const int32_t* prefix_len, int32_t R,
                             int32_t N, int32_t budget, int32_t* q_offsets, int32_t* slot_cand,
                             int32_t* slot_parent, int32_t* slot_token, int32_t* position_ids,
                             uint32_t* tree_mask, int32_t mask_words, void* workspace,
                             size_t workspace_bytes, int32_t* status, echo_stream_t stream) {
  (void)workspace;
  (void)workspace_bytes;
  if (R < 1 || N < 0 || budget < 0) return ECHO_ERR_INVALID_ARG;
  if (R > ECHO_MAX_REQUESTS || budget > ECHO_MAX_BUDGET) return ECHO_ERR_UNSUPPORTED;
  if (int64_t(mask_words) * 32 < int64_t(budget) + 1) return ECHO_ERR_INVALID_ARG;
  if (!cand_offsets || !root_token || !prefix_len || !q_offsets || !slot_cand || !slot_parent ||
      !slot_token || !position_ids || !tree_mask)
    return ECHO_ERR_INVALID_ARG;
  if (N > 0 && (!parent || !token || !selected)) return ECHO_ERR_INVALID_ARG;
  if (echo::mask_lds_bytes(R, budget) > 150 * 1024) return ECHO_ERR_UNSUPPORTED;
  return echo::launch_build_tree_mask(cand_offsets, parent, token, selected, root_token,
                                      prefix_len, R, N, budget, q_offsets, slot_cand, slot_parent,
                                      slot_token, position_ids, tree_mask, mask_words, status,
                                      as_stream(stream));
}

size_t echo_tree_verify_attn_workspace_size(int32_t R, int32_t max_rows, int32_t num_q_heads,
                                            int32_t num_kv_heads, int32_t head_dim) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || num_kv_heads < 1 || head_dim != ECHO_HEAD_DIM)
    return 0;
  return echo::attn_workspace_bytes(R, max_rows, num_q_heads, num_kv_heads);
}

int32_t echo_tree_verify_attn(const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                              const uint16_t* k_cache, const uint16_t* v_cache,
                              const int64_t* kv_offsets, int64_t kv_rows,
                              const int32_t* q_offsets, const uint32_t* tree_mask,
                              int32_t mask_words, int32_t R, int32_t max_rows,
                              int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                              float sm_scale, float* out, float* lse, void* workspace,
                              size_t workspace_bytes, int32_t* status, echo_stream_t stream) {
  return attn_contiguous(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows, q_offsets,
                         tree_mask, mask_words, R, max_rows, num_q_heads, num_kv_heads, head_dim,
                         sm_scale, out, lse, workspace, workspace_bytes, status, nullptr, nullptr,
                         as_stream(stream));
}

int32_t echo_tree_verify_attn_timed(const uint16_t* q, const uint16_t* k_new,
                                    const uint16_t* v_new, const uint16_t* k_cache,
                                    const uint16_t* v_cache, const int64_t* kv_offsets,
                                    int64_t kv_rows, const int32_t* q_offsets,
                                    const uint32_t* tree_mask, int32_t mask_words, int32_t R,
                                    int32_t max_rows, int32_t num_q_heads, int32_t num_kv_heads,
                                    int32_t head_dim, float sm_scale, float* out, float* lse,
                                    void* workspace, size_t workspace_bytes, int32_t* status,
                                    void* ev_start, void* ev_stop, echo_stream_t stream) {
  if (ev_start == nullptr || ev_stop == nullptr) return ECHO_ERR_INVALID_ARG;
  return attn_contiguous(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows, q_offsets,
                         tree_mask, mask_words, R, max_rows, num_q_heads, num_kv_heads, head_dim,
                         sm_scale, out, lse, workspace, workspace_bytes, status,
                         reinterpret_cast<hipEvent_t>(ev_start),
                         reinterpret_cast<hipEvent_t>(ev_stop), as_stream(stream));
}

int32_t echo_tree_verify_attn_paged(
    const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new, const uint16_t* k_pages,
    const uint16_t* v_pages, int64_t num_pages, int32_t page_size, const int32_t* block_table,
    int32_t max_pages_per_request, const int32_t* prefix_len, const int32_t* q_offsets,
    const uint32_t* tree_mask, int32_t mask_words, int32_t R, int32_t max_rows,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float sm_scale, float* out,
    float* lse, void* workspace, size_t workspace_bytes, int32_t* status, echo_stream_t stream) {
  return attn_paged(q, k_new, v_new, k_pages, v_pages, num_pages, page_size, block_table,
                    max_pages_per_request, prefix_len, q_offsets, tree_mask, mask_words, R,
                    max_rows, num_q_heads, num_kv_heads, head_dim, sm_scale, out, lse, workspace,
                    workspace_bytes, status, nullptr, nullptr, as_stream(stream));
}

int32_t echo_tree_verify_attn_paged_timed(
    const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new, const uint16_t* k_pages,
    const uint16_t* v_pages, int64_t num_pages, int32_t page_size, const int32_t* block_table,
    int32_t max_pages_per_request, const int32_t* prefix_len, const int32_t* q_offsets,
    const uint32_t* tree_mask, int32_t mask_words, int32_t R, int32_t max_rows,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float sm_scale, float* out,
    float* lse, void* workspace, size_t workspace_bytes, int32_t* status, void* ev_start,
    void* ev_stop, echo_stream_t stream) {
  if (ev_start == nullptr || ev_stop == nullptr) return ECHO_ERR_INVALID_ARG;
  return attn_paged(q, k_new, v_new, k_pages, v_pages, num_pages, page_size, block_table,
                    max_pages_per_request, prefix_len, q_offsets, tree_mask, mask_words, R,
                    max_rows, num_q_heads, num_kv_heads, head_dim, sm_scale, out, lse, workspace,
                    workspace_bytes, status, reinterpret_cast<hipEvent_t>(ev_start),
                    reinterpret_cast<hipEvent_t>(ev_stop), as_stream(stream));
}

int32_t echo_accept(const int32_t* q_offsets, const int32_t* slot_parent,
                    const int32_t* slot_token, const int32_t* target_token, int32_t R,
                    int32_t max_rows, int32_t max_depth, int32_t* accept_len,
                    int32_t* accept_slots, int32_t* bonus_token, int32_t* status,
                    echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || max_depth < 1) return ECHO_ERR_INVALID_ARG;
  if (max_depth > ECHO_MAX_DEPTH || R > ECHO_MAX_REQUESTS) return ECHO_ERR_UNSUPPORTED;
  if (!q_offsets || !accept_len || !accept_slots || !bonus_token) return ECHO_ERR_INVALID_ARG;
  if (max_rows > 0 && (!slot_parent || !slot_token || !target_token)) return ECHO_ERR_INVALID_ARG;
  return echo::launch_accept(q_offsets, slot_parent, slot_token, target_token, R, max_rows,
                             max_depth, accept_len, accept_slots, bonus_token, status,
                             as_stream(stream));
}

int32_t echo_verify_step(
    const int32_t* cand_offsets, const int32_t* parent, const float* logq, const int32_t* token,
    int32_t R, int32_t N, int32_t budget, float* path_score, uint8_t* selected,
    int32_t* num_selected, void* gate_workspace, size_t gate_workspace_bytes,
    const int32_t* root_token, const int32_t* prefix_len, int32_t* q_offsets, int32_t* slot_cand,
    int32_t* slot_parent, int32_t* slot_token, int32_t* position_ids, uint32_t* tree_mask,
    int32_t mask_words, const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
    const uint16_t* k_cache, const uint16_t* v_cache, const int64_t* kv_offsets, int64_t kv_rows,
    int32_t max_rows, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
    float sm_scale, float* out, float* lse, void* attn_workspace, size_t attn_workspace_bytes,
    const int32_t* target_token, int32_t max_depth, int32_t* accept_len, int32_t* accept_slots,
    int32_t* bonus_token, int32_t* status, echo_stream_t stream) {
  // every check of the four calls, before anything is launched
  if (R < 1 || N < 0 || budget < 0) return ECHO_ERR_INVALID_ARG;
  if (R > ECHO_MAX_REQUESTS || budget > ECHO_MAX_BUDGET) return ECHO_ERR_UNSUPPORTED;
  if (!cand_offsets || !num_selected || !gate_workspace) return ECHO_ERR_INVALID_ARG;
  if (N > 0 && (!parent || !logq || !selected || !token)) return ECHO_ERR_INVALID_ARG;
  if (!aligned256(gate_workspace) ||
      gate_workspace_bytes < echo::gate_workspace_bytes(R, N, budget))
    return ECHO_ERR_WORKSPACE;
  if (int64_t(mask_words) * 32 < int64_t(budget) + 1) return ECHO_ERR_INVALID_ARG;
  if (!root_token || !prefix_len || !q_offsets || !slot_cand || !slot_parent || !slot_token ||
      !position_ids || !tree_mask)
    return ECHO_ERR_INVALID_ARG;
  if (echo::mask_lds_bytes(R, budget) > 150 * 1024) return ECHO_ERR_UNSUPPORTED;
  echo::AttnArgs a;
  int32_t rc = attn_contiguous_args(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows,
                                    q_offsets, tree_mask, mask_words, R, max_rows, num_q_heads,
                                    num_kv_heads, head_dim, sm_scale, out, lse, attn_workspace,
                                    attn_workspace_bytes, status, nullptr, nullptr, &a);
  if (rc != ECHO_OK) return rc;
  if (max_depth < 1) return ECHO_ERR_INVALID_ARG;
  if (max_depth > ECHO_MAX_DEPTH) return ECHO_ERR_UNSUPPORTED;
  if (!accept_len || !accept_slots || !bonus_token) return ECHO_ERR_INVALID_ARG;
  if (max_rows > 0 && !target_token) return ECHO_ERR_INVALID_ARG;
  hipStream_t s = as_stream(stream);
  const int list = echo::front_gate_list(N, R, budget);
  if (list >= 0) {
    rc = echo::launch_gate_select_only(cand_offsets, parent, logq, R, N, budget, path_score,
                                       selected, num_selected, gate_workspace, status, list != 0,
                                       s);
    if (rc != ECHO_OK) return rc;
  }
  echo::FrontLaunch f;
  f.N = N;
  f.R = R;
  f.budget = budget;
  f.mask_words = mask_words;
  f.gate_workspace = gate_workspace;
  f.logq = logq;
  f.path_score = path_score;
  f.selected = selected;
  f.num_selected = num_selected;
  f.cand_offsets = cand_offsets;
  f.parent = parent;
  f.token = token;
  f.root_token = root_token;
  f.prefix_len = prefix_len;
  f.q_offsets = q_offsets;
  f.slot_cand = slot_cand;
  f.slot_parent = slot_parent;
  f.slot_token = slot_token;
  f.position_ids = position_ids;
  f.tree_mask = tree_mask;
  f.kv_offsets = kv_offsets;
  f.kv_rows = kv_rows;
  f.max_rows = max_rows;
  f.hq = num_q_heads;
  f.hkv = num_kv_heads;
  f.attn_workspace = attn_workspace;
  f.status = status;
  rc = echo::launch_front(f, s);
  if (rc != ECHO_OK) return rc;
  if (max_rows == 0)  // no attention rows: the acceptance alone
    return echo::launch_accept(q_offsets, slot_parent, slot_token, target_token, R, max_rows,
                               max_depth, accept_len, accept_slots, bonus_token, status, s);
  rc = echo::launch_tree_verify_attn_main(a, s);
  if (rc != ECHO_OK) return rc;
  return echo::launch_tail(a, slot_parent, slot_token, target_token, max_depth, accept_len,
                           accept_slots, bonus_token, s);
}

const char* echo_status_string(int32_t code) {
  switch (code) {
    case ECHO_OK: return "ok";
    case ECHO_ERR_INVALID_ARG: return "invalid argument";
    case ECHO_ERR_UNSUPPORTED: return "unsupported size or shape";
    case ECHO_ERR_WORKSPACE: return "workspace too small or not 256-byte aligned";
    case ECHO_ERR_HIP: return "HIP launch or runtime failure";
    default: return "unknown status";
  }
}

const char* echo_version(void) { return "echo-mi355x 0.1.0 (gfx950)"; }

}  // extern "C"

extern "C" {

int32_t echo_accept_logits(const int32_t* q_offsets, const int32_t* slot_parent,
                           const int32_t* slot_token, const uint16_t* logits, int64_t vocab,
                           int32_t R, int32_t max_rows, int32_t max_depth, int32_t* target_token,
                           int32_t* accept_len, int32_t* accept_slots, int32_t* bonus_token,
                           int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || vocab < 1 || vocab > 0x7FFFFFFF) return ECHO_ERR_INVALID_ARG;
  if (max_depth < 1 || max_depth > ECHO_MAX_DEPTH || R > ECHO_MAX_REQUESTS)
    return ECHO_ERR_UNSUPPORTED;
  if (!q_offsets || !accept_len || !accept_slots || !bonus_token || !target_token)
    return ECHO_ERR_INVALID_ARG;
  if (max_rows > 0 && (!slot_parent || !slot_token || !logits)) return ECHO_ERR_INVALID_ARG;
  return echo::launch_accept_logits(q_offsets, slot_parent, slot_token, logits, vocab, R,
                                    max_rows, max_depth, target_token, accept_len, accept_slots,
                                    bonus_token, status, as_stream(stream));
}

int32_t echo_commit_kv(const int32_t* q_offsets, const int32_t* accept_len,
                       const int32_t* accept_slots, int32_t max_depth, const uint16_t* k_new,
                       const uint16_t* v_new, int32_t R, int32_t max_rows, int32_t num_kv_heads,
                       uint16_t* k_pages, uint16_t* v_pages, int64_t num_pages, int32_t page_size,
                       const int32_t* block_table, int32_t max_pages_per_request,
                       int32_t* prefix_len, int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || num_kv_heads < 1 || num_pages < 1 || page_size < 1 ||
      max_pages_per_request < 1)
    return ECHO_ERR_INVALID_ARG;
  if (max_depth < 1 || max_depth > ECHO_MAX_DEPTH || R > ECHO_MAX_REQUESTS)
    return ECHO_ERR_UNSUPPORTED;
  if (!q_offsets || !accept_len || !accept_slots || !k_new || !v_new || !k_pages || !v_pages ||
      !block_table || !prefix_len)
    return ECHO_ERR_INVALID_ARG;
  const uintptr_t al = reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new) |
                       reinterpret_cast<uintptr_t>(k_pages) | reinterpret_cast<uintptr_t>(v_pages);
  if (al & 15) return ECHO_ERR_INVALID_ARG;
  return echo::launch_commit_kv(q_offsets, accept_len, accept_slots, max_depth, k_new, v_new, R,
                                max_rows, num_kv_heads, k_pages, v_pages, num_pages, page_size,
                                block_table, max_pages_per_request, prefix_len, status,
                                as_stream(stream));
}

}  // extern "C"

namespace {
// The 8-bit cache's arguments: ECHO_OK with *c filled, or the error code.
int32_t cache_q8_args(int32_t kv_format, uint8_t* k_pages, uint8_t* v_pages, float* k_scale,
                      float* v_scale, int64_t num_pages, int32_t page_size, int32_t num_kv_heads,
                      int32_t head_dim, echo::CacheQ8Args* c) {
  if (num_pages < 1 || num_kv_heads < 1 || page_size < 1) return ECHO_ERR_INVALID_ARG;
  if (kv_format != ECHO_KV_E4M3 && kv_format != ECHO_KV_E5M2) return ECHO_ERR_INVALID_ARG;
  if (page_size < ECHO_KV_BLOCK || (page_size & (page_size - 1)) != 0) return ECHO_ERR_UNSUPPORTED;
  if (head_dim != ECHO_HEAD_DIM || num_kv_heads > (1 << 20)) return ECHO_ERR_UNSUPPORTED;
  // (compared by division: num_pages is any 64-bit number)
  if (num_pages >= (int64_t(1) << 31) / page_size) return ECHO_ERR_UNSUPPORTED;
  if (!k_pages || !v_pages || !k_scale || !v_scale) return ECHO_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_pages) | reinterpret_cast<uintptr_t>(v_pages)) & 15u)
    return ECHO_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale)) & 3u)
    return ECHO_ERR_INVALID_ARG;
  *c = echo::CacheQ8Args{kv_format, k_pages, v_pages, k_scale, v_scale, num_pages, page_size,
                         num_kv_heads};
  return ECHO_OK;
}
}  // namespace

extern "C" {

size_t echo_tree_verify_attn_paged_q8_workspace_size(int32_t R, int32_t max_rows,
                                                     int32_t num_q_heads, int32_t num_kv_heads,
                                                     int32_t head_dim,
                                                     int32_t max_pages_per_request) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || num_kv_heads < 1 ||
      head_dim != ECHO_HEAD_DIM || max_pages_per_request < 1)
    return 0;
  return echo::attn_q8_workspace_bytes(R, max_pages_per_request);
}

int32_t echo_tree_verify_attn_paged_q8(
    const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new, int32_t kv_format,
    const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scale, const float* v_scale,
    int64_t num_pages, int32_t page_size, const int32_t* block_table,
    int32_t max_pages_per_request, const int32_t* prefix_len, const int32_t* q_offsets,
    const uint32_t* tree_mask, int32_t mask_words, int32_t R, int32_t max_rows,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float sm_scale, uint16_t* out,
    float* lse, void* workspace, size_t workspace_bytes, int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || num_kv_heads < 1 || mask_words < 1 ||
      max_pages_per_request < 1)
    return ECHO_ERR_INVALID_ARG;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(sm_scale)) return ECHO_ERR_INVALID_ARG;
  echo::AttnQ8Args a{};
  const int32_t rc = cache_q8_args(kv_format, const_cast<uint8_t*>(k_pages),
                                   const_cast<uint8_t*>(v_pages), const_cast<float*>(k_scale),
                                   const_cast<float*>(v_scale), num_pages, page_size, num_kv_heads,
                                   head_dim, &a.cache);
  if (rc != ECHO_OK) return rc;
  // (32 rows of the new values, of 256 bytes a head, are addressed with 32-bit offsets)
  if (R > ECHO_MAX_REQUESTS || num_kv_heads > (1 << 19)) return ECHO_ERR_UNSUPPORTED;
  if (int64_t(max_pages_per_request) * page_size >= (int64_t(1) << 31)) return ECHO_ERR_UNSUPPORTED;
  if (int64_t(max_rows) * num_q_heads >= (int64_t(1) << 26)) return ECHO_ERR_UNSUPPORTED;
  // (32-bit numbers of the cache's blocks and of the tables' entries)
  if (num_pages * (page_size / ECHO_KV_BLOCK) >= (int64_t(1) << 32) / num_kv_heads ||
      int64_t(R) * max_pages_per_request >= (int64_t(1) << 31))
    return ECHO_ERR_UNSUPPORTED;
  if (!q || !k_new || !v_new || !block_table || !prefix_len || !q_offsets || !tree_mask || !out ||
      !workspace)
    return ECHO_ERR_INVALID_ARG;
  if (!aligned256(workspace) ||
      workspace_bytes < echo::attn_q8_workspace_bytes(R, max_pages_per_request))
    return ECHO_ERR_WORKSPACE;
  const uintptr_t mis = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) |
                        reinterpret_cast<uintptr_t>(v_new) | reinterpret_cast<uintptr_t>(out);
  if (mis & 15u) return ECHO_ERR_INVALID_ARG;
  if (max_rows == 0) return ECHO_OK;
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.block_table = block_table;
  a.max_pages = max_pages_per_request;
  a.prefix_len = prefix_len;
  a.q_offsets = q_offsets;
  a.tree_mask = tree_mask;
  a.mask_words = mask_words;
  a.R = R;
  a.max_rows = max_rows;
  a.hq = num_q_heads;
  a.sm_scale = sm_scale;
  a.out = out;
  a.lse = lse;
  a.workspace = workspace;
  a.status = status;
  return echo::launch_tree_verify_attn_q8(a, as_stream(stream));
}

int32_t echo_store_kv_q8(const uint16_t* k, const uint16_t* v, int64_t k_stride, int64_t v_stride,
                         const int64_t* slot_map, int32_t num_rows, int32_t num_kv_heads,
                         int32_t head_dim, int32_t kv_format, uint8_t* k_pages, uint8_t* v_pages,
                         float* k_scale, float* v_scale, int64_t num_pages, int32_t page_size,
                         int32_t* status, echo_stream_t stream) {
  if (num_rows < 0) return ECHO_ERR_INVALID_ARG;
  echo::CacheQ8Args c;
  const int32_t rc = cache_q8_args(kv_format, k_pages, v_pages, k_scale, v_scale, num_pages,
                                   page_size, num_kv_heads, head_dim, &c);
  if (rc != ECHO_OK) return rc;
  if (num_rows == 0) return ECHO_OK;
  if (!k || !v || !slot_map) return ECHO_ERR_INVALID_ARG;
  const int64_t row = int64_t(num_kv_heads) * ECHO_HEAD_DIM;
  if (k_stride < row || v_stride < row || ((k_stride | v_stride) & 7) != 0)
    return ECHO_ERR_INVALID_ARG;
  if (k_stride >= (int64_t(1) << 31) || v_stride >= (int64_t(1) << 31)) return ECHO_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return ECHO_ERR_INVALID_ARG;
  return echo::launch_store_kv_q8(k, v, k_stride, v_stride, slot_map, num_rows, c, status,
                                  as_stream(stream));
}

int32_t echo_commit_kv_q8(const int32_t* q_offsets, const int32_t* accept_len,
                          const int32_t* accept_slots, int32_t max_depth, const uint16_t* k_new,
                          const uint16_t* v_new, int32_t R, int32_t max_rows,
                          int32_t num_kv_heads, int32_t head_dim, int32_t kv_format,
                          uint8_t* k_pages, uint8_t* v_pages, float* k_scale, float* v_scale,
                          int64_t num_pages, int32_t page_size, const int32_t* block_table,
                          int32_t max_pages_per_request, const int32_t* prefix_len,
                          int32_t* new_len, int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || max_pages_per_request < 1) return ECHO_ERR_INVALID_ARG;
  if (max_depth < 1 || max_depth > ECHO_MAX_DEPTH || R > ECHO_MAX_REQUESTS)
    return ECHO_ERR_UNSUPPORTED;
  echo::CacheQ8Args c;
  const int32_t rc = cache_q8_args(kv_format, k_pages, v_pages, k_scale, v_scale, num_pages,
                                   page_size, num_kv_heads, head_dim, &c);
  if (rc != ECHO_OK) return rc;
  if (!q_offsets || !accept_len || !accept_slots || !k_new || !v_new || !block_table ||
      !prefix_len || !new_len)
    return ECHO_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) & 15u)
    return ECHO_ERR_INVALID_ARG;
  return echo::launch_commit_kv_q8(q_offsets, accept_len, accept_slots, max_depth, k_new, v_new, R,
                                   max_rows, c, block_table, max_pages_per_request, prefix_len,
                                   new_len, status, as_stream(stream));
}

int32_t echo_build_block_tables(const int32_t* want_len, int32_t R, int32_t page_size,
                                int32_t* block_table, int32_t max_pages_per_request,
                                const int32_t* num_held, int32_t* num_held_out,
                                int32_t* free_pages, int32_t max_free, const int32_t* num_free,
                                int32_t* num_free_out, const int32_t* row_offsets,
                                const int32_t* row_start, int32_t max_rows, int64_t* slot_map,
                                int32_t* status, echo_stream_t stream) {
  if (R < 1 || page_size < 1 || max_pages_per_request < 1 || max_free < 1)
    return ECHO_ERR_INVALID_ARG;
  if ((page_size & (page_size - 1)) != 0 || R > ECHO_MAX_REQUESTS ||
      int64_t(R) * max_pages_per_request >= (int64_t(1) << 31))
    return ECHO_ERR_UNSUPPORTED;
  if (!want_len || !block_table || !num_held || !num_held_out || !free_pages || !num_free ||
      !num_free_out)
    return ECHO_ERR_INVALID_ARG;
  if (slot_map != nullptr && (max_rows < 0 || !row_offsets || !row_start))
    return ECHO_ERR_INVALID_ARG;
  const echo::TablesArgs a{want_len, R, page_size, block_table, max_pages_per_request, num_held,
                           num_held_out, free_pages, max_free, num_free, num_free_out,
                           row_offsets, row_start, max_rows, slot_map, status};
  return echo::launch_build_block_tables(a, as_stream(stream));
}

}  // extern "C"

extern "C" {

int32_t echo_rope(const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, uint16_t* q_out,
                  int64_t q_out_row_stride, int64_t q_out_head_stride, int32_t num_q_heads,
                  const uint16_t* k, int64_t k_row_stride, int64_t k_head_stride, uint16_t* k_out,
                  int64_t k_out_row_stride, int64_t k_out_head_stride, int32_t num_k_heads,
                  const int32_t* positions, int32_t num_rows, const int32_t* row_count,
                  int32_t rot_dim, int32_t layout, const double* inv_freq, float scale,
                  int32_t* status, echo_stream_t stream) {
  if (num_rows < 0 || num_q_heads < 0 || num_k_heads < 0 || rot_dim < 2 || rot_dim % 2 != 0)
    return ECHO_ERR_INVALID_ARG;
  if (layout != ECHO_ROPE_HALF && layout != ECHO_ROPE_INTERLEAVED) return ECHO_ERR_INVALID_ARG;
  if (!isfinite(scale)) return ECHO_ERR_INVALID_ARG;
  // (a workgroup numbers a row's pairs of all heads in 32 bits)
  const int64_t heads = int64_t(num_q_heads) + num_k_heads;
  if (rot_dim > ECHO_ROPE_MAX_DIM || heads > (1 << 16) || num_rows > ECHO_ROPE_MAX_ROWS)
    return ECHO_ERR_UNSUPPORTED;
  if (num_rows == 0 || heads == 0) return ECHO_OK;
  if (!positions || !inv_freq) return ECHO_ERR_INVALID_ARG;
  if ((num_q_heads > 0 && (!q || !q_out)) || (num_k_heads > 0 && (!k || !k_out)))
    return ECHO_ERR_INVALID_ARG;
  const int64_t most = int64_t(1) << 31;
  // inputs may repeat rows or heads (stride 0), outputs may not
  const auto side = [&](const uint16_t* x, int64_t row, int64_t head, const uint16_t* y,
                        int64_t out_row, int64_t out_head, int32_t n) -> int32_t {
    if (row < 0 || head < 0 || out_row < 0 || out_head < 0) return ECHO_ERR_INVALID_ARG;
    if (row >= most || head >= most || out_row >= most || out_head >= most)
      return ECHO_ERR_UNSUPPORTED;
    const bool apart = (n <= 1 || out_head >= rot_dim) && (num_rows <= 1 || out_row >= rot_dim);
    const bool nested = n <= 1 || num_rows <= 1 ||
                        out_row >= int64_t(n - 1) * out_head + rot_dim ||
                        out_head >= int64_t(num_rows - 1) * out_row + rot_dim;
    if (!apart || !nested) return ECHO_ERR_INVALID_ARG;
    if (x == y && ((num_rows > 1 && row != out_row) || (n > 1 && head != out_head)))
      return ECHO_ERR_INVALID_ARG;
    return ECHO_OK;
  };
  int32_t rc = ECHO_OK;
  if (num_q_heads > 0)
    rc = side(q, q_row_stride, q_head_stride, q_out, q_out_row_stride, q_out_head_stride,
              num_q_heads);
  if (rc == ECHO_OK && num_k_heads > 0)
    rc = side(k, k_row_stride, k_head_stride, k_out, k_out_row_stride, k_out_head_stride,
              num_k_heads);
  if (rc != ECHO_OK) return rc;
  const echo::RopeArgs a{q, q_out, q_row_stride, q_head_stride, q_out_row_stride, q_out_head_stride,
                         k, k_out, k_row_stride, k_head_stride, k_out_row_stride, k_out_head_stride,
                         num_q_heads, num_k_heads, positions, num_rows, row_count, rot_dim, layout,
                         inv_freq, scale, status};
  return echo::launch_rope(a, as_stream(stream));
}

int32_t echo_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                              double original_len, double low_turns, double high_turns,
                              double* inv_freq, float* scale) {
  if (rot_dim < 2 || rot_dim % 2 != 0 || !inv_freq || !scale) return ECHO_ERR_INVALID_ARG;
  if (rot_dim > ECHO_ROPE_MAX_DIM) return ECHO_ERR_UNSUPPORTED;
  if (!(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor))
    return ECHO_ERR_INVALID_ARG;
  if (scaling < ECHO_ROPE_PLAIN || scaling > ECHO_ROPE_SMOOTH) return ECHO_ERR_INVALID_ARG;
  if (scaling == ECHO_ROPE_BASE && rot_dim < 4) return ECHO_ERR_INVALID_ARG;
  const bool by_turns = scaling == ECHO_ROPE_BANDS || scaling == ECHO_ROPE_SMOOTH;
  if (by_turns && (!(original_len > 0.0) || !isfinite(original_len) || !(low_turns > 0.0) ||
                   !(high_turns > low_turns) || !isfinite(high_turns)))
    return ECHO_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586;
  const double n = rot_dim;
  if (scaling == ECHO_ROPE_BASE) base *= pow(factor, n / (n - 2.0));
  if (!isfinite(base)) return ECHO_ERR_INVALID_ARG;
  double lo = 0.0, hi = 0.0;  // ECHO_ROPE_BANDS: the ramp's first and last dims (of pairs)
  if (scaling == ECHO_ROPE_BANDS) {
    const auto dim_of = [&](double turns) {
      return n * log(original_len / (turns * two_pi)) / (2.0 * log(base));
    };
    lo = fmax(floor(dim_of(high_turns)), 0.0);
    hi = fmin(ceil(dim_of(low_turns)), n - 1.0);
  }
  for (int32_t i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / n);
    if (scaling == ECHO_ROPE_LINEAR) f /= factor;
    if (scaling == ECHO_ROPE_BANDS) {
      const double ramp = fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
      f = f / factor * ramp + f * (1.0 - ramp);
    }
    if (scaling == ECHO_ROPE_SMOOTH) {
      const double turns = original_len * f / two_pi;
      const double s = fmin(fmax((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0);
      f = f * s + f / factor * (1.0 - s);
    }
    inv_freq[i] = f;
  }
  *scale = scaling == ECHO_ROPE_BANDS ? float(0.1 * log(factor) + 1.0) : 1.0f;
  return ECHO_OK;
}

}  // extern "C"

namespace {
// The latent cache's arguments: ECHO_OK with *c filled, or the error code.
int32_t cache_latent_args(uint16_t* pages, int64_t num_pages, int32_t page_size,
                          echo::LatentCacheArgs* c) {
  if (num_pages < 1 || page_size < 1) return ECHO_ERR_INVALID_ARG;
  if (page_size < 32 || (page_size & (page_size - 1)) != 0) return ECHO_ERR_UNSUPPORTED;
  // (compared by division: num_pages is any 64-bit number)
  if (num_pages >= (int64_t(1) << 31) / page_size) return ECHO_ERR_UNSUPPORTED;
  if (!pages || (reinterpret_cast<uintptr_t>(pages) & 15u)) return ECHO_ERR_INVALID_ARG;
  *c = echo::LatentCacheArgs{pages, num_pages, page_size};
  return ECHO_OK;
}
bool latent_dims_ok(int32_t latent_dim, int32_t rope_dim) {
  return latent_dim == ECHO_LATENT_DIM && rope_dim == ECHO_LATENT_ROPE_DIM;
}
}  // namespace

extern "C" {

int32_t echo_store_latent(const uint16_t* kv, int64_t kv_stride, const uint16_t* norm_weight,
                          float eps, const int32_t* positions, const double* inv_freq,
                          float rope_scale, int32_t layout, int32_t num_rows,
                          const int32_t* row_count, int32_t latent_dim, int32_t rope_dim,
                          uint16_t* latent_new, const int64_t* slot_map, uint16_t* pages,
                          int64_t num_pages, int32_t page_size, int32_t* status,
                          echo_stream_t stream) {
  if (num_rows < 0) return ECHO_ERR_INVALID_ARG;
  if (!latent_dims_ok(latent_dim, rope_dim) || num_rows > ECHO_ROPE_MAX_ROWS)
    return ECHO_ERR_UNSUPPORTED;
  if (layout != ECHO_ROPE_HALF && layout != ECHO_ROPE_INTERLEAVED) return ECHO_ERR_INVALID_ARG;
  if (norm_weight != nullptr && !(eps >= 0.0f && isfinite(eps))) return ECHO_ERR_INVALID_ARG;
  if (inv_freq != nullptr && !isfinite(rope_scale)) return ECHO_ERR_INVALID_ARG;
  if (num_rows == 0) return ECHO_OK;
  if (!kv || (!latent_new && !slot_map) || (inv_freq != nullptr && !positions))
    return ECHO_ERR_INVALID_ARG;
  if (kv_stride < ECHO_LATENT_DIM + ECHO_LATENT_ROPE_DIM || (kv_stride & 7) != 0)
    return ECHO_ERR_INVALID_ARG;
  if (kv_stride >= (int64_t(1) << 31)) return ECHO_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(kv) | reinterpret_cast<uintptr_t>(norm_weight) |
       reinterpret_cast<uintptr_t>(latent_new)) & 15u)
    return ECHO_ERR_INVALID_ARG;
  // A row is read before it is written, but in no order with other rows: in place only where none moves.
  const bool in_place = latent_new == kv && (kv_stride == ECHO_LATENT_DIM + ECHO_LATENT_ROPE_DIM || num_rows == 1);
  if (latent_new != nullptr && !in_place) {
    const uintptr_t row = (ECHO_LATENT_DIM + ECHO_LATENT_ROPE_DIM) * sizeof(uint16_t);
    const uintptr_t x = reinterpret_cast<uintptr_t>(kv), y = reinterpret_cast<uintptr_t>(latent_new);
    const uintptr_t before = uintptr_t(num_rows - 1);
    if (x < y + before * row + row && y < x + before * uintptr_t(kv_stride) * sizeof(uint16_t) + row)
      return ECHO_ERR_INVALID_ARG;
  }
  echo::LatentCacheArgs c{nullptr, 0, 0};
  if (slot_map != nullptr) {
    const int32_t rc = cache_latent_args(pages, num_pages, page_size, &c);
    if (rc != ECHO_OK) return rc;
  }
  const echo::StoreLatentArgs a{kv, kv_stride, norm_weight, eps, positions, inv_freq, rope_scale,
                                layout, num_rows, row_count, latent_new, slot_map, c, status};
  return echo::launch_store_latent(a, as_stream(stream));
}

size_t echo_tree_verify_attn_latent_workspace_size(int32_t R, int32_t max_rows,
                                                   int32_t num_q_heads, int32_t latent_dim,
                                                   int32_t rope_dim,
                                                   int32_t max_pages_per_request) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || !latent_dims_ok(latent_dim, rope_dim) ||
      max_pages_per_request < 1)
    return 0;
  return echo::attn_latent_workspace_bytes(R, max_pages_per_request);
}

int32_t echo_tree_verify_attn_latent(
    const uint16_t* q, const uint16_t* latent_new, const uint16_t* pages, int64_t num_pages,
    int32_t page_size, const int32_t* block_table, int32_t max_pages_per_request,
    const int32_t* prefix_len, const int32_t* q_offsets, const uint32_t* tree_mask,
    int32_t mask_words, int32_t R, int32_t max_rows, int32_t num_q_heads, int32_t latent_dim,
    int32_t rope_dim, float sm_scale, uint16_t* out, float* lse, void* workspace,
    size_t workspace_bytes, int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || num_q_heads < 1 || mask_words < 1 || max_pages_per_request < 1)
    return ECHO_ERR_INVALID_ARG;
  if (!scale_ok(sm_scale)) return ECHO_ERR_INVALID_ARG;
  if (!latent_dims_ok(latent_dim, rope_dim) || R > ECHO_MAX_REQUESTS) return ECHO_ERR_UNSUPPORTED;
  echo::AttnLatentArgs a{};
  const int32_t rc =
      cache_latent_args(const_cast<uint16_t*>(pages), num_pages, page_size, &a.cache);
  if (rc != ECHO_OK) return rc;
  if (int64_t(max_pages_per_request) * page_size >= (int64_t(1) << 31) ||
      int64_t(max_rows) * num_q_heads >= (int64_t(1) << 26))
    return ECHO_ERR_UNSUPPORTED;
  if (!q || !latent_new || !block_table || !prefix_len || !q_offsets || !tree_mask || !out ||
      !workspace)
    return ECHO_ERR_INVALID_ARG;
  if (!aligned256(workspace) ||
      workspace_bytes < echo::attn_latent_workspace_bytes(R, max_pages_per_request))
    return ECHO_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(latent_new) |
       reinterpret_cast<uintptr_t>(out)) & 15u)
    return ECHO_ERR_INVALID_ARG;
  if (max_rows == 0) return ECHO_OK;
  a.q = q;
  a.latent_new = latent_new;
  a.block_table = block_table;
  a.max_pages = max_pages_per_request;
  a.prefix_len = prefix_len;
  a.q_offsets = q_offsets;
  a.tree_mask = tree_mask;
  a.mask_words = mask_words;
  a.R = R;
  a.max_rows = max_rows;
  a.hq = num_q_heads;
  a.sm_scale = sm_scale;
  a.out = out;
  a.lse = lse;
  a.workspace = workspace;
  a.status = status;
  return echo::launch_tree_verify_attn_latent(a, as_stream(stream));
}

int32_t echo_commit_latent(const int32_t* q_offsets, const int32_t* accept_len,
                           const int32_t* accept_slots, int32_t max_depth,
                           const uint16_t* latent_new, int32_t R, int32_t max_rows,
                           int32_t latent_dim, int32_t rope_dim, uint16_t* pages,
                           int64_t num_pages, int32_t page_size, const int32_t* block_table,
                           int32_t max_pages_per_request, const int32_t* prefix_len,
                           int32_t* new_len, int32_t* status, echo_stream_t stream) {
  if (R < 1 || max_rows < 0 || max_pages_per_request < 1) return ECHO_ERR_INVALID_ARG;
  if (max_depth < 1 || max_depth > ECHO_MAX_DEPTH || R > ECHO_MAX_REQUESTS ||
      !latent_dims_ok(latent_dim, rope_dim))
    return ECHO_ERR_UNSUPPORTED;
  echo::LatentCacheArgs c;
  const int32_t rc = cache_latent_args(pages, num_pages, page_size, &c);
  if (rc != ECHO_OK) return rc;
  if (!q_offsets || !accept_len || !accept_slots || !latent_new || !block_table || !prefix_len ||
      !new_len)
    return ECHO_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(latent_new) & 15u) return ECHO_ERR_INVALID_ARG;
  return echo::launch_commit_latent(q_offsets, accept_len, accept_slots, max_depth, latent_new, R,
                                    max_rows, c, block_table, max_pages_per_request, prefix_len,
                                    new_len, status, as_stream(stream));
}

}  // extern "C"
