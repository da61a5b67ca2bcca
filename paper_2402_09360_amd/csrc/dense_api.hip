// C ABI of the dense operators next to the sparse steps (declared in include/hire.h): argument validation, workspace
// layout and launches.
#include "../../include/hire.h"

#include "kernels.h"

namespace {

using namespace hire;

constexpr size_t kAlign = 256;
size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool given(const void* p, size_t a) { return p != nullptr && aligned(p, a); }
bool optional(const void* p, size_t a) { return p == nullptr || aligned(p, a); }

int launched(hipError_t e) {
  if (e == hipSuccess) return HIRE_OK;
  last_launch_error() = e;
  return HIRE_ELAUNCH;
}

int check_gated(const hire_gated_layer* L, int T) {
  static_assert(HIRE_ACT_RELU == kActRelu && HIRE_ACT_SILU == kActSilu && HIRE_ACT_GELU == kActGelu, "same numbers");
  if (!L || T < 1 || L->d_model < 8 || L->d_model % 8 != 0 || L->d_ff < 8 || L->d_ff % 8 != 0) return HIRE_EINVAL;
  if (L->act != HIRE_ACT_RELU && L->act != HIRE_ACT_SILU && L->act != HIRE_ACT_GELU) return HIRE_EINVAL;
  if (T > HIRE_GATED_MAX_TOKENS || L->d_model > HIRE_GATED_MAX_WIDTH || L->d_ff > HIRE_GATED_MAX_WIDTH)
    return HIRE_EUNSUPPORTED;
  return HIRE_OK;
}
bool gated_weights(const hire_gated_layer* L) { return given(L->wg, 256) && given(L->wu, 256) && given(L->w2u, 256); }
GatedLayer gated_layer(const hire_gated_layer* L) {
  return GatedLayer{L->d_model, L->d_ff, L->act, static_cast<const uint16_t*>(L->wg), static_cast<const uint16_t*>(L->wu),
                    static_cast<const uint16_t*>(L->w2u)};
}
uint16_t* bf16_at(void* base, size_t off) { return reinterpret_cast<uint16_t*>(static_cast<char*>(base) + off); }

int check_mx(int T, int rows, int cols) {
  if (T < 1 || rows < 1 || cols < 32 || cols % 32 != 0) return HIRE_EINVAL;
  if (T > HIRE_MXFP4_MAX_TOKENS || rows > HIRE_MXFP4_MAX_ROWS || cols > HIRE_MXFP4_MAX_COLS) return HIRE_EUNSUPPORTED;
  return HIRE_OK;
}
int mx_product(const void* x, const uint8_t* x_scales, int T, const void* w_codes, const void* w_scales, int rows, int cols,
               void* y, int y_type, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check_mx(T, rows, cols); rc != HIRE_OK) return rc;
  if (!given(w_codes, 16) || !w_scales || !given(y, 16) || !given(workspace, 256)) return HIRE_EINVAL;
  if (y_type != HIRE_F32 && y_type != HIRE_BF16) return HIRE_EINVAL;
  if (workspace_bytes < hire_mxfp4_product_workspace_bytes(T, rows, cols)) return HIRE_ENOSPC;
  return launched(launch_mx_product(MxProduct{x, x_scales, T, static_cast<const uint8_t*>(w_codes),
                                              static_cast<const uint8_t*>(w_scales), rows, cols, y, y_type == HIRE_BF16,
                                              workspace},
                                    static_cast<hipStream_t>(stream)));
}

int check_drafts(const hire_drafts* D) {
  static_assert(HIRE_MAX_DRAFT == kMaxDraft && HIRE_MAX_RANK_ORDER_K == kMaxDraftList, "same numbers");
  if (!D || D->B < 1 || D->n < 0 || D->vocab < 1) return HIRE_EINVAL;
  if (!given(D->target_prob, 4) || !optional(D->target_idx, 4) || !optional(D->draft_prob, 4) || !optional(D->draft_idx, 4))
    return HIRE_EINVAL;
  if (!optional(D->lengths, 4) || !given(D->sample_u, 4) || (D->draft_idx && !D->draft_prob)) return HIRE_EINVAL;
  if (D->n > 0 ? !given(D->tokens, 4) || !given(D->accept_u, 4) : D->draft_prob != nullptr) return HIRE_EINVAL;
  if ((D->target_idx && D->target_k < 1) || (D->draft_idx && D->draft_k < 1)) return HIRE_EINVAL;
  if (D->B > HIRE_MAX_DRAFT_BATCH || D->n > HIRE_MAX_DRAFT || D->vocab > HIRE_MAX_DRAFT_VOCAB) return HIRE_EUNSUPPORTED;
  if ((D->target_idx && D->target_k > HIRE_MAX_RANK_ORDER_K) || (D->draft_idx && D->draft_k > HIRE_MAX_RANK_ORDER_K))
    return HIRE_EUNSUPPORTED;
  return HIRE_OK;
}

DraftArgs draft_args(const hire_drafts* D) {
  DraftArgs a{};
  a.B = D->B, a.n = D->n, a.vocab = D->vocab;
  a.lengths = D->lengths, a.tokens = D->tokens;
  a.target = D->target_prob, a.target_idx = D->target_idx, a.target_k = D->target_k;
  a.draft = D->draft_prob, a.draft_idx = D->draft_idx, a.draft_k = D->draft_k;
  a.accept_u = D->accept_u, a.sample_u = D->sample_u;
  return a;
}

size_t hidden_bytes(const hire_gated_layer* L, int T) { return align_up((size_t)T * L->d_ff * 2); }
GatedKept kept_planes(const hire_gated_layer* L, int T, void* saved) {
  const size_t plane = hidden_bytes(L, T);
  return GatedKept{bf16_at(saved, 0), bf16_at(saved, plane), bf16_at(saved, 2 * plane), bf16_at(saved, 3 * plane)};
}
bool keeps_rest(int T) { return T <= kGatedRestTokens; }
// Planes at the front of a workspace: h and its rest; dg, du, their rests and that of h.
size_t forward_planes(const hire_gated_layer* L, int T) { return (keeps_rest(T) ? 2 : 1) * hidden_bytes(L, T); }
size_t backward_planes(const hire_gated_layer* L, int T) { return (keeps_rest(T) ? 5 : 2) * hidden_bytes(L, T); }

}  // namespace

extern "C" {

size_t hire_gated_ffn_workspace_bytes(const hire_gated_layer* L, int T) {
  if (check_gated(L, T) != HIRE_OK) return 0;
  return forward_planes(L, T) + align_up(gated_forward_part_bytes(T, L->d_model, L->d_ff));
}

size_t hire_gated_ffn_saved_bytes(const hire_gated_layer* L, int T) {
  return check_gated(L, T) != HIRE_OK ? 0 : 4 * hidden_bytes(L, T);
}

int hire_gated_ffn_step(const hire_gated_layer* L, const void* x, int T, void* y, void* saved, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (const int rc = check_gated(L, T); rc != HIRE_OK) return rc;
  if (!gated_weights(L) || !given(x, 16) || !given(y, 16) || !optional(saved, 256) || !given(workspace, 256))
    return HIRE_EINVAL;
  if (workspace_bytes < hire_gated_ffn_workspace_bytes(L, T)) return HIRE_ENOSPC;
  GatedKept kept = saved ? kept_planes(L, T, saved) : GatedKept{bf16_at(workspace, 0), nullptr, nullptr, nullptr};
  if (keeps_rest(T)) kept.rest = bf16_at(workspace, hidden_bytes(L, T));
  float* part = reinterpret_cast<float*>(bf16_at(workspace, forward_planes(L, T)));
  return launched(launch_gated_forward(gated_layer(L), static_cast<const uint16_t*>(x), T, static_cast<uint16_t*>(y), kept, part,
                                       static_cast<hipStream_t>(stream)));
}

size_t hire_gated_ffn_backward_workspace_bytes(const hire_gated_layer* L, int T) {
  if (check_gated(L, T) != HIRE_OK) return 0;
  return backward_planes(L, T) + align_up(gated_backward_part_bytes(T, L->d_model, L->d_ff));
}

int hire_gated_ffn_backward(const hire_gated_layer* L, const void* x, int T, const void* saved, const void* dy, void* dx,
                            void* dwg, void* dwu, void* dw2u, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check_gated(L, T); rc != HIRE_OK) return rc;
  if (!gated_weights(L) || !given(x, 16) || !given(saved, 256) || !given(dy, 16) || !given(workspace, 256)) return HIRE_EINVAL;
  if (!optional(dx, 16) || !optional(dwg, 16) || !optional(dwu, 16) || !optional(dw2u, 16) || !(dx || dwg || dwu || dw2u))
    return HIRE_EINVAL;
  if (workspace_bytes < hire_gated_ffn_backward_workspace_bytes(L, T)) return HIRE_ENOSPC;
  const size_t hidden = hidden_bytes(L, T);
  GatedSlopes slopes{bf16_at(workspace, 0), bf16_at(workspace, hidden)};
  if (keeps_rest(T)) {
    slopes.dg_rest = bf16_at(workspace, 2 * hidden);
    slopes.du_rest = bf16_at(workspace, 3 * hidden);
    slopes.h_rest = bf16_at(workspace, 4 * hidden);
  }
  return launched(launch_gated_backward(
      gated_layer(L), static_cast<const uint16_t*>(x), T, kept_planes(L, T, const_cast<void*>(saved)),
      static_cast<const uint16_t*>(dy), static_cast<uint16_t*>(dx), static_cast<uint16_t*>(dwg), static_cast<uint16_t*>(dwu),
      static_cast<uint16_t*>(dw2u), slopes, reinterpret_cast<float*>(bf16_at(workspace, backward_planes(L, T))),
      static_cast<hipStream_t>(stream)));
}

int hire_pack_mxfp4(const void* w_bf16, int rows, int cols, void* codes, void* scales, void* stream) {
  if (rows < 1 || cols < 32 || cols % 32 != 0 || !given(w_bf16, 16) || !given(codes, 16) || !scales) return HIRE_EINVAL;
  return launched(launch_pack_mxfp4(static_cast<const uint16_t*>(w_bf16), rows, cols, static_cast<uint8_t*>(codes),
                                    static_cast<uint8_t*>(scales), static_cast<hipStream_t>(stream)));
}

int hire_unpack_mxfp4(const void* codes, const void* scales, int rows, int cols, void* w_bf16, void* stream) {
  if (rows < 1 || cols < 32 || cols % 32 != 0 || !given(w_bf16, 16) || !given(codes, 16) || !scales) return HIRE_EINVAL;
  return launched(launch_unpack_mxfp4(static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), rows, cols,
                                      static_cast<uint16_t*>(w_bf16), static_cast<hipStream_t>(stream)));
}

size_t hire_mxfp4_product_workspace_bytes(int T, int rows, int cols) {
  if (check_mx(T, rows, cols) != HIRE_OK) return 0;
  return align_up(mx_workspace_bytes(T, rows, cols)) + kAlign;
}

int hire_mxfp4_product(const void* x_codes, const void* x_scales, int T, const void* w_codes, const void* w_scales, int rows,
                       int cols, void* y, int y_type, void* workspace, size_t workspace_bytes, void* stream) {
  if (!given(x_codes, 16) || !x_scales) return HIRE_EINVAL;
  return mx_product(x_codes, static_cast<const uint8_t*>(x_scales), T, w_codes, w_scales, rows, cols, y, y_type, workspace,
                    workspace_bytes, stream);
}

int hire_mxfp4_product_bf16(const void* x, int T, const void* w_codes, const void* w_scales, int rows, int cols, void* y,
                            int y_type, void* workspace, size_t workspace_bytes, void* stream) {
  static_assert(HIRE_MAX_BATCH == kMxFewTokens, "the tokens of a decode step");
  if (!given(x, 16)) return HIRE_EINVAL;
  if (T > HIRE_MAX_BATCH) return HIRE_EUNSUPPORTED;
  return mx_product(x, nullptr, T, w_codes, w_scales, rows, cols, y, y_type, workspace, workspace_bytes, stream);
}

size_t hire_verify_draft_workspace_bytes(const hire_drafts* D) {
  if (check_drafts(D) != HIRE_OK) return 0;
  return D->target_idx ? kAlign : align_up(draft_part_bytes(draft_args(D)));
}

int hire_verify_draft(const hire_drafts* D, int32_t* tokens_out, int32_t* accepted_out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  if (const int rc = check_drafts(D); rc != HIRE_OK) return rc;
  if (!given(tokens_out, 4) || !given(accepted_out, 4) || !given(workspace, 256)) return HIRE_EINVAL;
  if (workspace_bytes < hire_verify_draft_workspace_bytes(D)) return HIRE_ENOSPC;
  DraftArgs a = draft_args(D);
  a.out_tokens = tokens_out, a.accepted = accepted_out;
  a.part = static_cast<double*>(workspace);
  return launched(launch_verify(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
