// C ABI of the operators around the layer (residual norm, sampling,
// accepted path) and of the experts with 4-bit weights: host-side argument checks (before any HIP call) and kernel
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

static_assert(ACCEPTMOE_MAX_VOCAB == amoe::kMaxVocab, "the kernels' largest vocabulary");

constexpr int kQ4MaxSize = 65536;  // a quad's run over K stays addressable by 32 bits

bool q4_size(int32_t n) { return n >= 32 && n % 32 == 0 && n <= kQ4MaxSize; }

int32_t q4_check(const char* who, int32_t E, int32_t I, int32_t H) {
  if (E < 1 || E > ACCEPTMOE_MAX_EXPERTS)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "%s: E must be in [1, %d] (got %d)", who, ACCEPTMOE_MAX_EXPERTS, E);
  if (!q4_size(H) || !q4_size(I))
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "%s: H and I must be positive multiples of 32 up to %d (H=%d I=%d)", who,
                kQ4MaxSize, H, I);
  return ACCEPTMOE_OK;
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
  const size_t scale_bytes = group == 0 ? 0 : static_cast<size_t>(T) * (group > 0 ? H / group : 1) * 4;
  if (group != 0 && (overlap(scale_out, scale_bytes, hidden, n * eb) || (y && overlap(scale_out, scale_bytes, y, n * 4)) ||
                     overlap(scale_out, scale_bytes, weight, H * eb) || overlap(scale_out, scale_bytes, norm_out, norm_bytes) ||
                     (y && overlap(scale_out, scale_bytes, hidden_out, n * eb))))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "residual_norm: scale_out overlaps another argument");
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
  p.workspace = workspace;
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

// ---------------------------------------------------------------------------
size_t acceptmoe_q4_gate_up_bytes(int32_t E, int32_t I, int32_t H) {
  if (E < 1 || E > ACCEPTMOE_MAX_EXPERTS || !q4_size(I) || !q4_size(H)) return 0;
  return amoe::packed_gate_up_q4_bytes(E, I, H);
}

size_t acceptmoe_q4_down_bytes(int32_t E, int32_t H, int32_t I) {
  if (E < 1 || E > ACCEPTMOE_MAX_EXPERTS || !q4_size(I) || !q4_size(H)) return 0;
  return amoe::packed_down_q4_bytes(E, H, I);
}

int32_t acceptmoe_quantize_q4(const void* w, int32_t dtype, int64_t n, uint8_t* codes, uint8_t* scales, void* stream) {
  clear_err();
  if (dtype != ACCEPTMOE_F32 && dtype != ACCEPTMOE_BF16)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "quantize_q4: unknown dtype %d", dtype);
  if (n < 0 || n % 32 != 0)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "quantize_q4: n must be a multiple of 32 (got %lld)",
                static_cast<long long>(n));
  if (n == 0) return ACCEPTMOE_OK;
  if (!w || !codes || !scales) return fail(ACCEPTMOE_ERR_INVALID_ARG, "quantize_q4: null pointer");
  if (!aligned(w, 16) || !aligned(codes, 16))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "quantize_q4: w and codes must be 16-byte aligned");
  const size_t bytes = static_cast<size_t>(n) * (dtype == ACCEPTMOE_BF16 ? 2 : 4);
  if (overlap(w, bytes, codes, n / 2) || overlap(w, bytes, scales, n / 32) || overlap(codes, n / 2, scales, n / 32))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "quantize_q4: arguments overlap");
  hipError_t e = amoe::launch_quantize_q4(w, dtype == ACCEPTMOE_BF16, static_cast<size_t>(n) / 32, codes, scales,
                                          static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "quantize_q4 launch");
}

int32_t acceptmoe_pack_gate_up_q4(const uint8_t* gate, const uint8_t* gate_scale, const uint8_t* up,
                                  const uint8_t* up_scale, int32_t E, int32_t I, int32_t H, void* dst, void* stream) {
  clear_err();
  const int32_t rc = q4_check("pack_gate_up_q4", E, I, H);
  if (rc != ACCEPTMOE_OK) return rc;
  if (!gate || !gate_scale || !up || !up_scale || !dst)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_gate_up_q4: null pointer");
  if (!aligned(gate, 16) || !aligned(up, 16) || !aligned(dst, 16))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_gate_up_q4: codes and dst must be 16-byte aligned");
  const size_t n = static_cast<size_t>(E) * I * H, out = amoe::packed_gate_up_q4_bytes(E, I, H);
  if (overlap(dst, out, gate, n / 2) || overlap(dst, out, up, n / 2) || overlap(dst, out, gate_scale, n / 32) ||
      overlap(dst, out, up_scale, n / 32))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_gate_up_q4: a source overlaps dst");
  hipError_t e = amoe::launch_pack_gate_up_q4(gate, gate_scale, up, up_scale, E, I, H, dst,
                                              static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "pack_gate_up_q4 launch");
}

int32_t acceptmoe_pack_down_q4(const uint8_t* down, const uint8_t* down_scale, int32_t E, int32_t H, int32_t I,
                               void* dst, void* stream) {
  clear_err();
  const int32_t rc = q4_check("pack_down_q4", E, I, H);
  if (rc != ACCEPTMOE_OK) return rc;
  if (!down || !down_scale || !dst) return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_down_q4: null pointer");
  if (!aligned(down, 16) || !aligned(dst, 16))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_down_q4: codes and dst must be 16-byte aligned");
  const size_t n = static_cast<size_t>(E) * I * H, out = amoe::packed_down_q4_bytes(E, H, I);
  if (overlap(dst, out, down, n / 2) || overlap(dst, out, down_scale, n / 32))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "pack_down_q4: a source overlaps dst");
  hipError_t e = amoe::launch_pack_down_q4(down, down_scale, E, H, I, dst, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "pack_down_q4 launch");
}

size_t acceptmoe_moe_forward_q4_workspace_size(int32_t T, int32_t H, int32_t I, int32_t E, int32_t k) {
  if (T < 0 || H < 1 || I < 1 || E < 1 || k < 1) return 0;
  return amoe::forward_q4_workspace_bytes(T, H, I, E, k);
}

int32_t acceptmoe_moe_forward_q4(const void* hidden, const void* w_gate_up, const void* w_down, int32_t T, int32_t H,
                                 int32_t I, int32_t E, int32_t k, const int32_t* topk_idx, const float* topk_gate,
                                 float* out, void* workspace, size_t workspace_bytes, void* stream) {
  clear_err();
  if (T < 0) return fail(ACCEPTMOE_ERR_INVALID_ARG, "forward_q4: T must be >= 0 (got %d)", T);
  const int32_t rc = q4_check("forward_q4", E, I, H);
  if (rc != ACCEPTMOE_OK) return rc;
  if (k < 1 || k > ACCEPTMOE_MAX_TOPK)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "forward_q4: k must be in [1, %d] (got %d)", ACCEPTMOE_MAX_TOPK, k);
  if (T == 0) return ACCEPTMOE_OK;
  if (static_cast<long long>(T) * k > (1ll << 30) || static_cast<long long>(T) * H >= (1ll << 31) - 8)
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "forward_q4: T too large: hidden is addressed in 32 bits (T=%d k=%d H=%d)", T,
                k, H);
  if (!amoe::forward_q4_grids_fit(T, H, I, E, k))
    return fail(ACCEPTMOE_ERR_UNSUPPORTED, "forward_q4: T too large: a product takes fewer than 2^24 workgroups (T=%d k=%d I=%d H=%d)",
                T, k, I, H);
  if (!hidden || !w_gate_up || !w_down || !topk_idx || !topk_gate || !out)
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "forward_q4: null pointer");
  if (!aligned(hidden, 16) || !aligned(w_gate_up, 16) || !aligned(w_down, 16) || !aligned(out, 16))
    return fail(ACCEPTMOE_ERR_INVALID_ARG, "forward_q4: hidden, weights and out must be 16-byte aligned");
  const size_t need = amoe::forward_q4_workspace_bytes(T, H, I, E, k);
  if (workspace == nullptr || workspace_bytes < need)
    return fail(ACCEPTMOE_ERR_WORKSPACE, "forward_q4: workspace needs %zu bytes (got %zu)", need, workspace_bytes);
  if (!aligned(workspace, 256))
    return fail(ACCEPTMOE_ERR_WORKSPACE, "forward_q4: workspace must be 256-byte aligned");
  amoe::ForwardParams p;
  std::memset(&p, 0, sizeof p);
  p.hidden = hidden;
  p.w_gate_up = w_gate_up;
  p.w_down = w_down;
  p.topk_idx = topk_idx;
  p.topk_gate = topk_gate;
  p.out = out;
  p.T = T;
  p.H = H;
  p.I = I;
  p.E = E;
  p.k = k;
  p.is_bf16 = 1;
  amoe::forward_q4_carve(workspace, p);
  hipError_t e = amoe::launch_forward_q4(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ACCEPTMOE_OK : hip_fail(e, "forward_q4 launch");
}

}  // extern "C"
