// A token per row of logits from a given random number u: temperature, top-k,
// top-p and min-p.
//
// The tokens of a row stand in the order (logit descending, index ascending).  With
// w_j = exp((z_j - max z) / temperature) and C_j the sum of the first j weights, the
// filters keep a prefix of that order, and the sample is the first j with
// C_j > u C_kept.  Every cut (the k-th token, the first C_j >= p C_k, the
// sample itself) is the first place where a running sum of counts or weights
// reaches a number, and equal logits have equal weights, so it is found as a key
// (the logit's order-preserving 32 bits) and a count of tokens with that key.
//
// Sums: the weights' exponentials are taken in 64 bits and held as whole numbers
// of 2^-43, so a sum of up to 2^20 of them fits 64 bits, has no rounding and does
// not depend on the order of the additions.  fp32 sums would move a border between
// two of 50,000 kept tokens past u in about one of 2000 rows.
#include "common.hpp"
#include "launch.hpp"

namespace amoe {

namespace {

constexpr uint32_t kKeyNegInf = 0x007fffffu;  // logit_key(-inf); NaN gets key 0
constexpr double kWeightOne = 8796093022208.0;  // 2^43

__device__ __forceinline__ uint32_t token_key(float z) { return z != z ? 0u : logit_key(z); }

__device__ __forceinline__ double key_logit(uint32_t key) {
  return static_cast<double>(__uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key));
}

// a row's settings and its largest key
struct RowRule {
  uint32_t top;  // largest key
  double zmax, tau;

  // exp((z - zmax) / tau); the row's largest logits weigh 1 also where they are infinite
  __device__ __forceinline__ double weight(uint32_t key) const {
    return key == top ? 1.0 : exp((key_logit(key) - zmax) / tau);
  }
  __device__ __forceinline__ uint64_t fixed(uint32_t key) const {
    return static_cast<uint64_t>(__double2ull_rn(weight(key) * kWeightOne));
  }
};

// sum over the workgroup, the same for every thread
template <class T>
__device__ __forceinline__ T block_sum(T v, T* part) {
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();  // the last call's parts are no longer read
  if (lane_id() == 0) part[wave_id()] = v;
  __syncthreads();
  T s = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) s += part[w];
  return s;
}

__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* part) {
  for (int o = 32; o >= 1; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(v, o)));
  __syncthreads();
  if (lane_id() == 0) part[wave_id()] = v;
  __syncthreads();
  uint32_t s = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) s = max(s, part[w]);
  return s;
}

// ---------------------------------------------------------------------------
// One workgroup per row, over the row in memory: a radix search by digits of 11,
// 11 and 10 bits of the key, with the weights (or counts) of each digit summed
// in LDS.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 1024;
constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;

struct RowShared {
  unsigned long long bin[kBins];
  unsigned long long part64[kRowThreads / kWave];
  uint32_t part32[kRowThreads / kWave];
  unsigned long long before;
  uint32_t digit;
  int index;
};

template <bool kBf16>
struct Row {
  const void* p;
  int V;
  __device__ __forceinline__ uint32_t key(int i) const {
    const float z = kBf16 ? bf16_bits_to_float(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
    return token_key(z);
  }
};

struct Place {
  uint32_t key;     // where the running sum reaches `need`
  uint64_t before;  // the sum over larger keys
};

// 1 <= need <= the sum over all finite keys
template <bool kBf16, bool kCount>
__device__ Place find_place(const Row<kBf16>& row, const RowRule& rule, uint64_t need, RowShared& sh) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t before = 0;
  for (int shift = 21, bits = 11, pass = 0; pass < 3; ++pass) {
    for (int i = tid; i < kBins; i += kRowThreads) sh.bin[i] = 0;
    __syncthreads();
    for (int i = tid; i < row.V; i += kRowThreads) {
      const uint32_t key = row.key(i);
      if (key <= kKeyNegInf || (pass > 0 && (key >> (shift + bits)) != prefix)) continue;
      const uint64_t w = kCount ? 1u : rule.fixed(key);
      if (w != 0) atomicAdd(&sh.bin[(key >> shift) & ((1u << bits) - 1u)], static_cast<unsigned long long>(w));
    }
    __syncthreads();
    // thread t holds bins top - 2 t and top - 2 t - 1: running sums from the largest digit on
    const int top = (1 << bits) - 1 - 2 * tid;
    const uint64_t a = top >= 0 ? sh.bin[top] : 0, b = top >= 1 ? sh.bin[top - 1] : 0;
    uint64_t incl = a + b;
    for (int o = 1; o < kWave; o <<= 1) {
      const uint64_t v = __shfl_up(incl, o);
      if (lane_id() >= o) incl += v;
    }
    if (lane_id() == kWave - 1) sh.part64[wave_id()] = incl;
    __syncthreads();
    uint64_t base = before + incl - a - b;
    for (int w = 0; w < wave_id(); ++w) base += sh.part64[w];
    if (base < need && base + a >= need) {
      sh.digit = top;
      sh.before = base;
    } else if (base + a < need && base + a + b >= need) {
      sh.digit = top - 1;
      sh.before = base + a;
    }
    __syncthreads();
    prefix = (prefix << bits) | sh.digit;
    before = sh.before;
    if (pass == 0) shift = 10;
    else if (pass == 1) shift = 0, bits = 10;
  }
  return {prefix, before};
}

// Index of the r-th token (r >= 1) whose key is `key`; at least r have it.
template <bool kBf16>
__device__ int find_index(const Row<kBf16>& row, uint32_t key, uint64_t r, RowShared& sh) {
  const int tid = threadIdx.x;
  uint64_t seen = 0;
  for (int i0 = 0; i0 < row.V; i0 += kRowThreads) {
    const int i = i0 + tid;
    const bool hit = i < row.V && row.key(i) == key;
    const uint64_t m = __ballot(hit);
    __syncthreads();
    if (lane_id() == 0) sh.part32[wave_id()] = popc64(m);
    __syncthreads();
    uint64_t at = seen + popc64(m & lanes_below(lane_id())) + 1;
    for (int w = 0; w < kRowThreads / kWave; ++w) {
      at += w < wave_id() ? sh.part32[w] : 0;
      seen += sh.part32[w];
    }
    if (hit && at == r) sh.index = i;
    if (seen >= r) break;
  }
  __syncthreads();
  return sh.index;
}

template <bool kBf16>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleParams p) {
  __shared__ RowShared sh;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Row<kBf16> row{static_cast<const char*>(p.logits) + r * p.row_stride * (kBf16 ? 2 : 4), p.V};
  uint32_t top = 0;
  for (int i = tid; i < p.V; i += kRowThreads) top = max(top, row.key(i));
  top = block_max(top, sh.part32);
  if (top <= kKeyNegInf) {  // no token left
    if (tid == 0) p.token[r] = -1, p.prob[r] = 0.f;
    return;
  }
  const float tau = p.temperature ? p.temperature[r] : 1.f;
  if (!(tau > 0.f)) {  // greedy
    const int i = find_index(row, top, 1, sh);
    if (tid == 0) p.token[r] = i, p.prob[r] = 1.f;
    return;
  }
  const RowRule rule{top, key_logit(top), tau};
  // top-k: tokens above (cut, ties of it)
  uint32_t cut = 0;
  uint64_t ties = 0;
  const int k = p.top_k ? p.top_k[r] : 0;
  if (k > 0 && k < p.V) {
    uint32_t live = 0;
    for (int i = tid; i < p.V; i += kRowThreads) live += row.key(i) > kKeyNegInf ? 1u : 0u;
    live = block_sum(live, sh.part32);
    if (static_cast<uint32_t>(k) < live) {
      const Place at = find_place<kBf16, true>(row, rule, k, sh);
      cut = at.key;
      ties = k - at.before;
    }
  }
  auto sum_above = [&](uint32_t limit) {
    unsigned long long s = 0;
    for (int i = tid; i < p.V; i += kRowThreads) {
      const uint32_t key = row.key(i);
      if (key > limit) s += rule.fixed(key);
    }
    return block_sum(s, sh.part64);
  };
  uint64_t total = sum_above(max(cut, kKeyNegInf)) + (cut != 0 ? ties * rule.fixed(cut) : 0);
  const float top_p = p.top_p ? p.top_p[r] : 1.f;
  if (!(top_p >= 1.f)) {
    const double want = ceil(static_cast<double>(top_p > 0.f ? top_p : 0.f) * static_cast<double>(total));
    const uint64_t need = min(max(static_cast<uint64_t>(want), static_cast<uint64_t>(1)), total);
    const Place at = find_place<kBf16, false>(row, rule, need, sh);
    const uint64_t w = rule.fixed(at.key);
    cut = at.key;
    total = at.before + (need - at.before + w - 1) / w * w;
  }
  const double min_p = p.min_p ? fmin(static_cast<double>(p.min_p[r]), 1.0) : 0.0;
  if (min_p > 0.0 && (cut == 0 || rule.weight(cut) < min_p)) {
    // tokens that weigh less come behind all others
    unsigned long long s = 0;
    for (int i = tid; i < p.V; i += kRowThreads) {
      const uint32_t key = row.key(i);
      if (key > max(cut, kKeyNegInf) && rule.weight(key) >= min_p) s += rule.fixed(key);
    }
    total = block_sum(s, sh.part64);
  }
  const double u = fmax(static_cast<double>(p.uniform[r]), 0.0);
  const uint64_t need = min(static_cast<uint64_t>(u * static_cast<double>(total)) + 1, total);
  const Place at = find_place<kBf16, false>(row, rule, need, sh);
  const uint64_t w = rule.fixed(at.key);
  const int i = find_index(row, at.key, (need - at.before + w - 1) / w, sh);
  if (tid == 0) {
    p.token[r] = i;
    p.prob[r] = static_cast<float>(rule.weight(at.key) * kWeightOne / static_cast<double>(total));
  }
}

}  // namespace

size_t sample_workspace_bytes(int, int) { return 256; }

hipError_t launch_sample(const SampleParams& p, hipStream_t stream) {
  if (p.is_bf16) sample_row_kernel<true><<<p.R, kRowThreads, 0, stream>>>(p);
  else sample_row_kernel<false><<<p.R, kRowThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace amoe
