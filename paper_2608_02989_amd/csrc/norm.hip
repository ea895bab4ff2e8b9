// Residual addition with the root-mean-square norm behind it, the step between
// two layers of a stack:
//   s = hidden + y (fp32),  hidden' = round(s),
//   n = s / sqrt(mean(s^2) + eps) * weight, rounded once to the layer's type,
// or held in 8 bits (e4m3, largest value 448): per group of columns
//   scale = max|n| / 448,  code = e4m3(n / scale).
//
// Bound by memory with many rows: every value is read and written once, 10 H bytes a row
// in bf16 with an addend (16384 rows of 4096: 671 MB in 130 us, 5.2 TB/s, the rate of a large
// copy).  1920 rows of 2048 to codes take 11.0 us a call (3.2 TB/s: 60 waves for
// the 32 places of a CU, latency), one row 2.5 us.  256 threads a row: no difference.
#include "common.hpp"
#include "launch.hpp"

namespace amoe {

namespace {

constexpr float kE4m3Max = 448.f;

enum class NormOut { Plain, Groups, Row };

// larger of two magnitudes; their bits are ordered like them, and a NaN's stand above all (fmaxf
// would drop it, and a broken row would leave as codes and scales of a sound one)
__device__ __forceinline__ float larger(float a, float b) {
  return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}

// sum (kMax: largest magnitude) over the workgroup's threads, in a fixed order
template <bool kMax>
__device__ __forceinline__ float block_reduce(float v, float* part) {
  auto op = [](float a, float b) { return kMax ? larger(a, b) : a + b; };
  v = dpp::reduce(v, 0.f, op);
  const int waves = blockDim.x / kWave;
  if (waves == 1) return v;
  if (lane_id() == 0) part[wave_id()] = v;
  __syncthreads();
  float s = part[0];
  for (int w = 1; w < waves; ++w) s = op(s, part[w]);
  return s;
}

// One workgroup per row; thread t holds the float4 columns t, t + threads, ... (NV of
// them) in registers, so every value is read once and the sum of squares, the
// largest value and the codes come from the same registers.
template <bool kBf16, bool kAdd, int NV, NormOut kOut>
__global__ __launch_bounds__(1024) void residual_norm_kernel(const void* __restrict__ hidden,
                                                             const float4* __restrict__ y,
                                                             const void* __restrict__ weight, int n4, float inv_h,
                                                             float eps, int lanes, void* __restrict__ hidden_out,
                                                             void* __restrict__ norm_out, float* __restrict__ scale) {
  __shared__ float part[2][16];
  const int tid = threadIdx.x, threads = blockDim.x;
  const size_t row = static_cast<size_t>(blockIdx.x) * n4;
  auto load4 = [](const void* p, size_t i) {
    if (kBf16) {
      const uint2 h = static_cast<const uint2*>(p)[i];
      return make_float4(__uint_as_float(h.x << 16), __uint_as_float(h.x & 0xffff0000u), __uint_as_float(h.y << 16),
                         __uint_as_float(h.y & 0xffff0000u));
    }
    return static_cast<const float4*>(p)[i];
  };
  auto store4 = [](void* p, size_t i, const float4& v) {
    if (kBf16)
      static_cast<uint2*>(p)[i] =
          make_uint2(float_to_bf16_bits(v.x) | (static_cast<uint32_t>(float_to_bf16_bits(v.y)) << 16),
                     float_to_bf16_bits(v.z) | (static_cast<uint32_t>(float_to_bf16_bits(v.w)) << 16));
    else
      static_cast<float4*>(p)[i] = v;
  };
  float4 s[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = tid + i * threads;
    s[i] = c < n4 ? load4(hidden, row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (kAdd) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = tid + i * threads;
      if (c < n4) {
        const float4 v = y[row + c];
        s[i] = make_float4(s[i].x + v.x, s[i].y + v.y, s[i].z + v.z, s[i].w + v.w);
        store4(hidden_out, row + c, s[i]);
      }
    }
  }
  float4 w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = tid + i * threads;
    w[i] = c < n4 ? load4(weight, c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) sq += s[i].x * s[i].x + s[i].y * s[i].y + s[i].z * s[i].z + s[i].w * s[i].w;
  const float inv = rsqrtf(block_reduce<false>(sq, part[0]) * inv_h + eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    s[i].x = s[i].x * inv * w[i].x;
    s[i].y = s[i].y * inv * w[i].y;
    s[i].z = s[i].z * inv * w[i].z;
    s[i].w = s[i].w * inv * w[i].w;
  }
  if constexpr (kOut == NormOut::Plain) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = tid + i * threads;
      if (c < n4) store4(norm_out, row + c, s[i]);
    }
  } else {
    auto largest = [&](int i) {
      return larger(larger(fabsf(s[i].x), fabsf(s[i].y)), larger(fabsf(s[i].z), fabsf(s[i].w)));
    };
    float row_max = 0.f;
    if constexpr (kOut == NormOut::Row) {
#pragma unroll
      for (int i = 0; i < NV; ++i) row_max = larger(row_max, largest(i));
      row_max = block_reduce<true>(row_max, part[1]);
      if (tid == 0) scale[blockIdx.x] = row_max / kE4m3Max;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = tid + i * threads;
      float m = row_max;
      if constexpr (kOut == NormOut::Groups) {
        // a group is `lanes` neighbouring lanes of one wave
        m = largest(i);
        for (int o = 1; o < lanes; o <<= 1) m = larger(m, __shfl_xor(m, o));
      }
      if (c >= n4) continue;
      const float sc = m / kE4m3Max;
      if (kOut == NormOut::Groups && c % lanes == 0) scale[(row + c) / lanes] = sc;
      auto code = [&](float v) {
        v = sc == 0.f ? 0.f : v / sc;
        return v != v ? v : fminf(fmaxf(v, -kE4m3Max), kE4m3Max);
      };
      int packed = __builtin_amdgcn_cvt_pk_fp8_f32(code(s[i].x), code(s[i].y), 0, false);
      packed = __builtin_amdgcn_cvt_pk_fp8_f32(code(s[i].z), code(s[i].w), packed, true);
      static_cast<int*>(norm_out)[row + c] = packed;
    }
  }
}

template <bool kBf16, bool kAdd, int NV>
hipError_t launch_norm(const NormParams& p, int threads, hipStream_t stream) {
  const int n4 = p.H / 4;
  const float inv_h = 1.f / static_cast<float>(p.H);
  auto go = [&](auto kern, int lanes) {
    const size_t eb = kBf16 ? 2 : 4, norm_eb = p.group == 0 ? eb : 1;
    const int scales = p.group > 0 ? p.H / p.group : 1, most = max_workgroups(threads);
    hipError_t err = hipSuccess;
    for (int t0 = 0; t0 < p.T && err == hipSuccess; t0 += most) {
      const size_t at = static_cast<size_t>(t0) * p.H;
      kern<<<p.T - t0 < most ? p.T - t0 : most, threads, 0, stream>>>(
          static_cast<const char*>(p.hidden) + at * eb, kAdd ? reinterpret_cast<const float4*>(p.y + at) : nullptr, p.weight,
          n4, inv_h, p.eps, lanes, kAdd ? static_cast<char*>(p.hidden_out) + at * eb : nullptr,
          static_cast<char*>(p.norm_out) + at * norm_eb,
          p.group != 0 ? p.scale + static_cast<size_t>(t0) * scales : nullptr);
      err = hipGetLastError();
      if (p.T - t0 <= most) break;
    }
    return err;
  };
  if (p.group == 0) return go(&residual_norm_kernel<kBf16, kAdd, NV, NormOut::Plain>, 0);
  if (p.group > 0) return go(&residual_norm_kernel<kBf16, kAdd, NV, NormOut::Groups>, p.group / 4);
  return go(&residual_norm_kernel<kBf16, kAdd, NV, NormOut::Row>, 0);
}

template <bool kBf16, bool kAdd>
hipError_t launch_norm_nv(const NormParams& p, hipStream_t stream) {
  const int n4 = p.H / 4;
  int nv = 1;
  while (nv < 16 && (n4 + nv - 1) / nv > 1024) nv *= 2;
  const int threads = ((n4 + nv - 1) / nv + kWave - 1) / kWave * kWave;
  switch (nv) {
    case 1: return launch_norm<kBf16, kAdd, 1>(p, threads, stream);
    case 2: return launch_norm<kBf16, kAdd, 2>(p, threads, stream);
    case 4: return launch_norm<kBf16, kAdd, 4>(p, threads, stream);
    case 8: return launch_norm<kBf16, kAdd, 8>(p, threads, stream);
    default: return launch_norm<kBf16, kAdd, 16>(p, threads, stream);
  }
}

}  // namespace

hipError_t launch_residual_norm(const NormParams& p, hipStream_t stream) {
  if (p.is_bf16) return p.y ? launch_norm_nv<true, true>(p, stream) : launch_norm_nv<true, false>(p, stream);
  return p.y ? launch_norm_nv<false, true>(p, stream) : launch_norm_nv<false, false>(p, stream);
}

}  // namespace amoe
