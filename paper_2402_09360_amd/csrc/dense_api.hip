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
                                              static_cast<const uint8_t*>(w_scales), rows, cols, y, y_type == HIRE_BF16},
                                    static_cast<hipStream_t>(stream)));
}

size_t hidden_bytes(const hire_gated_layer* L, int T) { return align_up((size_t)T * L->d_ff * 2); }

}  // namespace

extern "C" {

size_t hire_gated_ffn_workspace_bytes(const hire_gated_layer* L, int T) {
  if (check_gated(L, T) != HIRE_OK) return 0;
  return hidden_bytes(L, T) + align_up(gated_part_bytes(T, L->d_model, L->d_ff, 1));
}

int hire_gated_ffn_step(const hire_gated_layer* L, const void* x, int T, void* y, void* g, void* u, void* h,
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check_gated(L, T); rc != HIRE_OK) return rc;
  if (!gated_weights(L) || !given(x, 16) || !given(y, 16) || !given(workspace, 256)) return HIRE_EINVAL;
  if (!optional(g, 16) || !optional(u, 16) || !optional(h, 16) || (!g != !u) || (!g != !h)) return HIRE_EINVAL;
  if (workspace_bytes < hire_gated_ffn_workspace_bytes(L, T)) return HIRE_ENOSPC;
  uint16_t* hidden = h ? static_cast<uint16_t*>(h) : bf16_at(workspace, 0);
  float* part = reinterpret_cast<float*>(bf16_at(workspace, hidden_bytes(L, T)));
  return launched(launch_gated_forward(gated_layer(L), static_cast<const uint16_t*>(x), T, static_cast<uint16_t*>(y), hidden,
                                       static_cast<uint16_t*>(g), static_cast<uint16_t*>(u), part,
                                       static_cast<hipStream_t>(stream)));
}

size_t hire_gated_ffn_backward_workspace_bytes(const hire_gated_layer* L, int T) {
  if (check_gated(L, T) != HIRE_OK) return 0;
  return 2 * hidden_bytes(L, T) + align_up(gated_part_bytes(T, L->d_model, L->d_ff, 2));
}

int hire_gated_ffn_backward(const hire_gated_layer* L, const void* x, int T, const void* g, const void* u, const void* h,
                            const void* dy, void* dx, void* dwg, void* dwu, void* dw2u, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (const int rc = check_gated(L, T); rc != HIRE_OK) return rc;
  if (!gated_weights(L) || !given(x, 16) || !given(g, 16) || !given(u, 16) || !given(h, 16) || !given(dy, 16) ||
      !given(workspace, 256))
    return HIRE_EINVAL;
  if (!optional(dx, 16) || !optional(dwg, 16) || !optional(dwu, 16) || !optional(dw2u, 16) || !(dx || dwg || dwu || dw2u))
    return HIRE_EINVAL;
  if (workspace_bytes < hire_gated_ffn_backward_workspace_bytes(L, T)) return HIRE_ENOSPC;
  const size_t hidden = hidden_bytes(L, T);
  return launched(launch_gated_backward(
      gated_layer(L), static_cast<const uint16_t*>(x), T, static_cast<const uint16_t*>(g), static_cast<const uint16_t*>(u),
      static_cast<const uint16_t*>(h), static_cast<const uint16_t*>(dy), static_cast<uint16_t*>(dx),
      static_cast<uint16_t*>(dwg), static_cast<uint16_t*>(dwu), static_cast<uint16_t*>(dw2u), bf16_at(workspace, 0),
      bf16_at(workspace, hidden), reinterpret_cast<float*>(bf16_at(workspace, 2 * hidden)),
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
  return kAlign;
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

}  // extern "C"
