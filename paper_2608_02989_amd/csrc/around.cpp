// C ABI of the operators around the layer (residual norm, sampling,
// accepted path): host-side argument checks (before any HIP call) and kernel
// launches.  See include/acceptmoe.h.
#include "acceptmoe.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "abi_util.hpp"
#include "launch.hpp"

using amoe::abi::aligned;
using amoe::abi::clear_err;
using amoe::abi::fail;
using amoe::abi::hip_fail;

namespace {

// [a, a + an) and [b, b + bn) share a byte
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const char* x = static_cast<const char*>(a);
  const char* y = static_cast<const char*>(b);
  return x < y + bn && y < x + an;
}

}  // namespace

extern "C" {

int32_t acceptmoe_residual_norm(const void* hidden, int32_t dtype, const float* y, const void* weight, int32_t T,
                                int32_t H, float eps, int32_t group, void* hidden_out, void* norm_out,
                                float* scale_out, void* stream) {
  clear_err();
  if (dtype != ACCEPTMOE_F32 && dtype != ACCEPTMOE_BF16)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: unknown dtype %d", dtype);
  if (T < 0 || H < 1) return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: bad sizes (T=%d H=%d)", T, H);
  if (H % 4 != 0 || H > amoe::kMaxNormWidth)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "residual_norm: H must be a multiple of 4 up to %d (got %d)",
                amoe::kMaxNormWidth, H);
  if (!std::isfinite(eps) || eps < 0.f)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: eps must be finite and >= 0");
  if (group != 0 && group != -1 && group != 32 && group != 64 && group != 128 && group != 256)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "residual_norm: group must be 0, -1 (the row), 32, 64, 128 or 256 (got %d)",
                group);
  if (group > 0 && H % group != 0)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "residual_norm: H must be a multiple of the group (H=%d group=%d)", H, group);
  if (T == 0) return ACCEPTMOE_OK;
  if (!hidden || !weight || !norm_out) return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: null pointer");
  if (y && !hidden_out) return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: an addend needs hidden_out");
  if (group != 0 && !scale_out) return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: 8-bit output needs scale_out");
  if (!aligned(hidden, 16) || !aligned(y, 16) || !aligned(weight, 16) || !aligned(hidden_out, 16) ||
      !aligned(norm_out, 16) || !aligned(scale_out, 4))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: pointers must be 16-byte aligned");
  const size_t n = static_cast<size_t>(T) * H, eb = dtype == ACCEPTMOE_BF16 ? 2 : 4;
  const size_t norm_bytes = n * (group != 0 ? 1 : eb);
  if (overlap(norm_out, norm_bytes, hidden, n * eb) || (y && overlap(norm_out, norm_bytes, y, n * 4)) ||
      overlap(norm_out, norm_bytes, weight, H * eb))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: norm_out overlaps an input");
  if (y && ((hidden_out != hidden && overlap(hidden_out, n * eb, hidden, n * eb)) ||
            overlap(hidden_out, n * eb, y, n * 4) || overlap(hidden_out, n * eb, weight, H * eb) ||
            overlap(hidden_out, n * eb, norm_out, norm_bytes)))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: hidden_out overlaps another argument");
  const amoe::NormParams p = {hidden, y, weight, hidden_out, norm_out, scale_out, T, H, dtype == ACCEPTMOE_BF16, group,
                              eps};
  hipError_t e = amoe::launch_residual_norm(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "residual_norm launch");
}

size_t acceptmoe_sample_workspace_size(int32_t R, int32_t V) {
  if (R < 0 || V < 1 || V > ACCEPTMOE_MAX_VOCAB) return 0;
  return amoe::sample_workspace_bytes(R, V);
}

int32_t acceptmoe_sample(const void* logits, int32_t dtype, int64_t row_stride, int32_t R, int32_t V,
                         const float* uniform, const float* temperature, const int32_t* top_k, const float* top_p,
                         const float* min_p, int32_t* token, float* prob, void* workspace, size_t workspace_bytes,
                         void* stream) {
  clear_err();
  if (dtype != ACCEPTMOE_F32 && dtype != ACCEPTMOE_BF16)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "sample: unknown dtype %d", dtype);
  if (R < 0 || V < 1) return fail(ACCEPTMOE_ERR_INVALID_ARG, "sample: bad sizes (R=%d V=%d)", R, V);
  if (V > ACCEPTMOE_MAX_VOCAB || R > ACCEPTMOE_MAX_SAMPLE_ROWS)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "sample: V must be <= %d and R <= %d (V=%d R=%d)", ACCEPTMOE_MAX_VOCAB,
                ACCEPTMOE_MAX_SAMPLE_ROWS, V, R);
  if (row_stride < V || row_stride > (1ll << 40))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "sample: row_stride must be >= V (got %lld)",
                static_cast<long long>(row_stride));
  if (R == 0) return ACCEPTMOE_OK;
  if (!logits || !uniform || !token || !prob) return fail(ACCEPTMOE_ERR_INVALID_ARG, "sample: null pointer");
  if (!aligned(logits, dtype == ACCEPTMOE_BF16 ? 2 : 4))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "sample: logits must be aligned to their element");
  const size_t need = amoe::sample_workspace_bytes(R, V);
  if (workspace == nullptr || workspace_bytes < need)
    return fail(ACCEPTMOE_ERR_WORKSPACE, "sample: workspace needs %zu bytes (got %zu)", need, workspace_bytes);
  if (!aligned(workspace, 256)) return fail(ACCEPTMOE_ERR_WORKSPACE, "sample: workspace must be 256-byte aligned");
  amoe::SampleParams p;
  std::memset(&p, 0, sizeof p);
  p.logits = logits;
  p.uniform = uniform;
  p.temperature = temperature;
  p.top_k = top_k;
  p.top_p = top_p;
  p.min_p = min_p;
  p.token = token;
  p.prob = prob;
  p.row_stride = static_cast<size_t>(row_stride);
  p.R = R;
  p.V = V;
  p.is_bf16 = dtype == ACCEPTMOE_BF16;
  hipError_t e = amoe::launch_sample(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "sample launch");
}

int32_t acceptmoe_accept(const int32_t* token, const int32_t* parent, const int32_t* target,
                         const int32_t* tree_offsets, int32_t B, int32_t T, uint8_t* on_path, int32_t* path,
                         int32_t path_len, int32_t* length, int32_t* bonus, void* stream) {
  clear_err();
  if (T < 0) return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: T must be >= 0 (got %d)", T);
  if (T == 0 && B == 0) return ACCEPTMOE_OK;
  if (B < 1 || B > ACCEPTMOE_MAX_TREES)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "accept: B must be in [1, %d] (got %d)", ACCEPTMOE_MAX_TREES, B);
  amoe::TreeOffsets offs;
  if (tree_offsets == nullptr) {
    if (B != 1) return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: tree_offsets is NULL but B = %d", B);
    offs.o[0] = 0;
    offs.o[1] = T;
  } else {
    if (tree_offsets[0] != 0) return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: tree_offsets[0] must be 0");
    for (int b = 0; b <= B; ++b) offs.o[b] = tree_offsets[b];
    if (offs.o[B] != T) return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: tree_offsets[B] must equal T");
  }
  int longest = 0;
  for (int b = 0; b < B; ++b) {
    if (offs.o[b + 1] < offs.o[b])
      return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: tree_offsets must be non-decreasing");
    const int n = offs.o[b + 1] - offs.o[b];
    if (n > ACCEPTMOE_MAX_TREE_NODES)
      return fail(ACCEPTMOE_ERR_UNSUPPORTED, "accept: tree %d has more than %d nodes", b, ACCEPTMOE_MAX_TREE_NODES);
    if (n > longest) longest = n;
  }
  if (path_len < longest)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: path_len must hold the largest tree's %d nodes (got %d)", longest,
                path_len);
  if (!length || !bonus || (path_len > 0 && !path) || (T > 0 && (!token || !parent || !target || !on_path)))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "accept: null pointer");
  const amoe::AcceptParams p = {token, parent, target, on_path, path, length, bonus, B, path_len};
  hipError_t e = amoe::launch_accept(p, offs, longest, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "accept launch");
}

}  // extern "C"
