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

}  // extern "C"
