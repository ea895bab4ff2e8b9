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
// not depend on the order of the additions.  Bins of weights (below) are added up as
// 64-bit floats, in a fixed order.
//
// Bound: with many rows the first pass over the logits (512 rows of 100003 in bf16, 102 MB:
// 35.2 us of the call's 58, 2.9 TB/s; vector instructions take half of the SIMDs' cycles, and the
// waves wait for loads and for the search's barriers 47 % of their time); with few the
// latency of three or four launches of short dependent steps (one row of 32000: 6.3 us
// for the pass, 9.8 for cutting and ordering its top 64, 2.6 for the launch that has
// nothing left to do; 64 fp32 rows of 131072 with top-p alone: 14.6, 10.6, then 13.8 for the
// second pass and 13.5 for the order within two bins).
#include "common.hpp"
#include "launch.hpp"

namespace amoe {

namespace {

constexpr uint32_t kKeyNegInf = 0x007fffffu;  // logit_key(-inf); NaN gets key 0
constexpr double kWeightOne = 8796093022208.0;  // 2^43
static_assert(kMaxVocab <= 1 << 20, "a row's sum of weights of 2^43 fits 64 bits");

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

constexpr int kFastK = 1000;  // largest top_k taken by candidate lists

enum class Mode { Greedy, TopK, Full, Slow };

// A row's settings.  Absent ones are read from `uniform` and replaced, so that all loads
// go out together and no branch waits for one.
struct Rules {
  float tau;
  int k;
  double top_p, min_p, u;  // top_p >= 1, min_p <= 0: off
  Mode mode;
  __device__ __forceinline__ bool by_p() const { return !(top_p >= 1.0); }
  __device__ __forceinline__ bool by_m() const { return min_p > 0.0; }
};
__device__ __forceinline__ Rules row_rules(const SampleParams& p, int r) {
  const float tau = (p.temperature ? p.temperature : p.uniform)[r];
  const int k = (p.top_k ? p.top_k : reinterpret_cast<const int32_t*>(p.uniform))[r];
  const float top_p = (p.top_p ? p.top_p : p.uniform)[r], min_p = (p.min_p ? p.min_p : p.uniform)[r];
  const float u = p.uniform[r];
  Rules s;
  s.tau = p.temperature ? tau : 1.f;
  s.k = p.top_k ? k : 0;
  s.top_p = p.top_p ? fmax(static_cast<double>(top_p), 0.0) : 1.0;
  s.min_p = p.min_p ? fmin(static_cast<double>(min_p), 1.0) : 0.0;
  s.u = fmin(fmax(static_cast<double>(u), 0.0), 1.0 - 1.0 / 16777216.0);
  s.mode = !(s.tau > 0.f) ? Mode::Greedy : s.k <= 0 || s.k >= p.V ? Mode::Full : s.k <= kFastK ? Mode::TopK : Mode::Slow;
  return s;
}

// the workgroup's largest `high` and smallest `low`
__device__ __forceinline__ void block_range(uint32_t& high, uint32_t& low, uint32_t* part) {
  const int waves = static_cast<int>(blockDim.x) / kWave;
  for (int o = 32; o >= 1; o >>= 1) {
    high = max(high, static_cast<uint32_t>(__shfl_xor(high, o)));
    low = min(low, static_cast<uint32_t>(__shfl_xor(low, o)));
  }
  __syncthreads();
  if (lane_id() == 0) {
    part[wave_id()] = high;
    part[waves + wave_id()] = low;
  }
  __syncthreads();
  for (int w = 0; w < waves; ++w) {
    high = max(high, part[w]);
    low = min(low, part[waves + w]);
  }
}

// ---------------------------------------------------------------------------
// Any row but a greedy one, by one workgroup over the row in memory: a radix search by digits of 11,
// 11 and 10 bits of the key, with the weights (or counts) of each digit summed
// in LDS.  (For all rows: 148 / 647 / 1221 us where the spread form below takes 17 / 51 / 58.)
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 512;
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
    // a thread holds neighbouring bins, the largest digits first: running sums from there on
    constexpr int kMine = kBins / kRowThreads;
    const int top = (1 << bits) - 1 - kMine * tid;
    uint64_t own = 0;
    for (int e = 0; e < kMine; ++e) own += top >= e ? sh.bin[top - e] : 0;
    uint64_t incl = own;
    for (int o = 1; o < kWave; o <<= 1) {
      const uint64_t v = __shfl_up(incl, o);
      if (lane_id() >= o) incl += v;
    }
    if (lane_id() == kWave - 1) sh.part64[wave_id()] = incl;
    __syncthreads();
    uint64_t base = before + incl - own;
    for (int w = 0; w < wave_id(); ++w) base += sh.part64[w];
    for (int e = 0; e < kMine; ++e) {
      const uint64_t w = top >= e ? sh.bin[top - e] : 0;
      if (base < need && base + w >= need) {
        sh.digit = top - e;
        sh.before = base;
      }
      base += w;
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
__device__ void sample_row(const SampleParams& p, int r, const Rules& rules, RowShared& sh) {
  const int tid = threadIdx.x;
  const Row<kBf16> row{static_cast<const char*>(p.logits) + r * p.row_stride * (kBf16 ? 2 : 4), p.V};
  uint32_t top = 0;
  for (int i = tid; i < p.V; i += kRowThreads) top = max(top, row.key(i));
  top = block_max(top, sh.part32);
  if (top <= kKeyNegInf) {  // no token left
    if (tid == 0) p.token[r] = -1, p.prob[r] = 0.f;
    return;
  }
  const RowRule rule{top, key_logit(top), rules.tau};
  // top-k: tokens above (cut, ties of it)
  uint32_t cut = 0;
  uint64_t ties = 0;
  const int k = rules.k;
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
  if (rules.by_p()) {
    const double want = ceil(rules.top_p * static_cast<double>(total));
    const uint64_t need = min(max(static_cast<uint64_t>(want), static_cast<uint64_t>(1)), total);
    const Place at = find_place<kBf16, false>(row, rule, need, sh);
    const uint64_t w = rule.fixed(at.key);
    cut = at.key;
    total = at.before + (need - at.before + w - 1) / w * w;
  }
  if (rules.by_m() && (cut == 0 || rule.weight(cut) < rules.min_p)) {
    // tokens that weigh less come behind all others
    unsigned long long s = 0;
    for (int i = tid; i < p.V; i += kRowThreads) {
      const uint32_t key = row.key(i);
      if (key > max(cut, kKeyNegInf) && rule.weight(key) >= rules.min_p) s += rule.fixed(key);
    }
    total = block_sum(s, sh.part64);
  }
  const uint64_t need = min(static_cast<uint64_t>(rules.u * static_cast<double>(total)) + 1, total);
  const Place at = find_place<kBf16, false>(row, rule, need, sh);
  const uint64_t w = rule.fixed(at.key);
  const int i = find_index(row, at.key, (need - at.before + w - 1) / w, sh);
  if (tid == 0) {
    p.token[r] = i;
    p.prob[r] = static_cast<float>(rule.weight(at.key) * kWeightOne / static_cast<double>(total));
  }
}


// ---------------------------------------------------------------------------
// The common cases, rows spread over R x splits workgroups.  What a launch does depends on
// the row's settings:
//   greedy, or 0 < top_k <= kFastK: `scan` lists each split's candidates (the largest
//     logits, at least top_k of them), `place` cuts them to the top_k, sorts those and
//     picks.  One read of the row.
//   no top_k: `scan` sums weights per bin of 1/32 in z / temperature, `place` finds the
//     bins in which the kept prefix ends and in which the sample lies, `filter` lists
//     the tokens of those (the second read), `finish` orders them and picks.
//   other top_k, more candidates or tokens in a bin than the lists hold (many
//     equal logits): `finish` runs sample_row.
// ---------------------------------------------------------------------------
constexpr int kScanThreads = 512;
constexpr int kCandCap = 1280;      // candidates of a split
constexpr int kGridBins = 1024;     // 32 nats below the largest logit; weights beyond sum to less than 2^20 e^-31
constexpr int kCopies = 4;          // of each bin, by lane, against LDS atomics on one address
constexpr int kListCap = 4096;      // tokens of the listed bins
constexpr int kRowsPerLaunch = 1024;
constexpr int kMaxSplits = 64;
constexpr double kPerNat = 32.0;

// a token as one number: larger logit, then lower index, is larger
__device__ __forceinline__ unsigned long long token_order(uint32_t key, int index) {
  return (static_cast<unsigned long long>(key) << 32) | (0xffffffffu - static_cast<uint32_t>(index));
}
__device__ __forceinline__ uint32_t order_key(unsigned long long v) { return static_cast<uint32_t>(v >> 32); }
__device__ __forceinline__ int order_index(unsigned long long v) {
  return static_cast<int>(0xffffffffu - static_cast<uint32_t>(v));
}

struct SplitPart {
  uint32_t top;  // largest key of the split
  uint32_t cut;  // its candidates are the tokens from this key on
  int n;         // candidates (may exceed kCandCap: not all are here)
  unsigned long long data[kCandCap];  // candidates, or the sums of kGridBins bins
};
static_assert(kGridBins <= kCandCap, "bins fit");

struct RowHead {
  int n_cut, n_pick;     // tokens listed (may exceed kListCap)
  int t_cut;             // bin in which the kept prefix ends, -1: everything is kept
  int t_pick0, t_pick1;  // bins in which the sample lies
  int slow;              // finish with sample_row
  uint32_t top;
  double before_cut, before_pick, total, grid_top;
};
struct RowPart : RowHead {
  unsigned long long cut[kListCap], pick[kListCap];
};

__host__ __device__ inline size_t sample_part_bytes(int splits) {
  return (sizeof(RowPart) + splits * sizeof(SplitPart) + 255) / 256 * 256;
}

struct RowView {
  RowPart* row;
  SplitPart* split;
  __device__ RowView(const SampleParams& p, int local, int splits) {
    char* base = static_cast<char*>(p.workspace) + local * sample_part_bytes(splits);
    row = reinterpret_cast<RowPart*>(base);
    split = reinterpret_cast<SplitPart*>(base + sizeof(RowPart));
  }
};

// z / temperature in bins of 1/32: the whole part names the bin, the rest gives the
// weight within it, exp(rest / 32) in [1, 1.032).  A bin's sum of these does not depend
// on the row's largest logit, so splits are added without knowing it.
struct Grid {
  double scale;
  __device__ __forceinline__ double at(uint32_t key) const { return key_logit(key) * scale; }
  static __device__ __forceinline__ double weight(double rest) {
    // y = rest / 32 < 2^-5: the series up to y^6 / 720 is off by less than 6e-15
    const double y = rest * (1.0 / kPerNat);
    double v = fma(y, 1.0 / 720, 1.0 / 120);
    v = fma(y, v, 1.0 / 24);
    v = fma(y, v, 1.0 / 6);
    v = fma(y, v, 0.5);
    v = fma(y, v, 1.0);
    return fma(y, v, 1.0);
  }
};

// the pieces of 16 bytes that hold a split of a row, in registers; places outside the row are -inf
template <bool kBf16, int NV, int kThreads>
struct Pieces {
  static constexpr int kPer = kBf16 ? 8 : 4;  // tokens of a piece
  uint4 v[NV];
  int first;  // token index of this thread's first piece's first place

  __device__ __forceinline__ void load(const SampleParams& p, int r, int s) {
    const char* row = static_cast<const char*>(p.logits) + r * p.row_stride * (kBf16 ? 2 : 4);
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row) % 16) / (kBf16 ? 2 : 4);
    const uint4* base = reinterpret_cast<const uint4*>(row - skew * (kBf16 ? 2 : 4));
    const int q0 = s * kThreads * NV + static_cast<int>(threadIdx.x);
    first = q0 * kPer - skew;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e0 = first + i * kThreads * kPer;
      v[i] = kBf16 ? make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u)
                   : make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
      if (e0 >= 0 && e0 + kPer <= p.V) {
        v[i] = base[q0 + i * kThreads];
      } else if (e0 + kPer > 0 && e0 < p.V) {  // the row's first or last piece
        uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          if (e0 + j < 0 || e0 + j >= p.V) continue;
          if (kBf16) {
            const uint32_t h = reinterpret_cast<const uint16_t*>(row)[e0 + j];
            w[j / 2] = j % 2 ? (w[j / 2] & 0xffffu) | (h << 16) : (w[j / 2] & 0xffff0000u) | h;
          } else {
            w[j] = reinterpret_cast<const uint32_t*>(row)[e0 + j];
          }
        }
        v[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  __device__ __forceinline__ float logit(int i, int j) const {
    const uint32_t w = (kBf16 ? j / 2 : j) == 0 ? v[i].x : (kBf16 ? j / 2 : j) == 1 ? v[i].y : (kBf16 ? j / 2 : j) == 2 ? v[i].z : v[i].w;
    return __uint_as_float(kBf16 ? (j % 2 ? w & 0xffff0000u : w << 16) : w);
  }
  __device__ __forceinline__ int index(int i, int j) const { return first + i * kThreads * kPer + j; }
  // largest logit of a piece; NaN never wins
  __device__ __forceinline__ float largest(int i) const {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPer; ++j) m = fmaxf(m, logit(i, j));
    return m;
  }
};

// Workgroup-wide number of the values a thread counts by ballot; one barrier a call,
// calls in a row alternate between two halves of `part`.
template <int kThreads>
__device__ __forceinline__ int block_count(int wave_count, int* part, int turn) {
  constexpr int kWaves = kThreads / kWave;
  int* half = part + (turn & 1) * kWaves;
  if (lane_id() == 0) half[wave_id()] = wave_count;
  __syncthreads();
  const int v = half[lane_id() % kWaves];
  return wave_sum_i32(v) / (kWave / kWaves);
}

// The largest cut, at least `lo`, with count(cut) >= need, or one before it whose count is
// at most `enough`; count() falls from count(lo) >= need on and is 0 above hi.
template <class T, class Count>
__device__ __forceinline__ T bisect(T lo, T hi, int need, int enough, Count count) {
  while (lo < hi) {
    const T mid = hi - (hi - lo) / 2;
    const int c = count(mid);
    if (c >= need) {
      lo = mid;
      if (c <= enough) break;
    } else {
      hi = mid - 1;
    }
  }
  return lo;
}

// Six waves per SIMD: registers that hold all pieces, and three workgroups per CU (a call on 512
// bf16 rows of 100003, top-100: 61.4 us; cut to eight, with registers spilled, 60.6, without a
// bound 70.9; on 64 fp32 rows of 131072, top-64: 27.6, 31.4, 27.5).
template <bool kBf16, int NV>
__global__ __launch_bounds__(kScanThreads) __attribute__((amdgpu_waves_per_eu(6))) void sample_scan_kernel(
    SampleParams p, int row0, int splits) {
  __shared__ unsigned long long s_bin[kGridBins * kCopies];
  __shared__ uint32_t s_max[2 * kScanThreads / kWave];
  __shared__ int s_part[2 * kScanThreads / kWave];
  __shared__ int s_n, s_queued;
  const int local = blockIdx.x / splits, r = row0 + local, s = blockIdx.x % splits, tid = threadIdx.x;
  Pieces<kBf16, NV, kScanThreads> z;
  z.load(p, r, s);  // ahead of the settings
  const Rules rules = row_rules(p, r);
  const Mode mode = rules.mode;
  const RowView ws(p, local, splits);
  SplitPart& out = ws.split[s];
  if (s == 0 && tid == 0) {
    ws.row->n_cut = ws.row->n_pick = 0;
    ws.row->t_cut = -1;
    ws.row->slow = mode == Mode::Slow;
  }
  if (mode == Mode::Slow) return;
  if (tid == 0) s_n = s_queued = 0;
  if (mode == Mode::Full)
    for (int i = tid; i < kGridBins * kCopies; i += kScanThreads) s_bin[i] = 0;
  uint32_t most[NV], top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    most[i] = token_key(z.largest(i));
    top = max(top, most[i]);
  }
  uint32_t low = top;  // the smallest of the threads' largest
  block_range(top, low, s_max);  // orders the clearing above, too
  if (tid == 0) out.top = top;
  if (top <= kKeyNegInf) {
    if (tid == 0) out.n = 0;
    return;
  }
  if (mode == Mode::Full) {
    const Grid grid{kPerNat / static_cast<double>(rules.tau)};
    const double grid_top = floor(grid.at(top));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < Pieces<kBf16, NV, kScanThreads>::kPer; ++j) {
        const double g = static_cast<double>(z.logit(i, j)) * grid.scale, b = floor(g);
        const double t = grid_top - b;
        if (t >= 0.0 && t < kGridBins) {
          // weight 2^43 rounded to a whole number in the low bits of the sum
          const double w = fma(Grid::weight(g - b), kWeightOne, 4503599627370496.0);
          atomicAdd(&s_bin[static_cast<int>(t) * kCopies + (tid & (kCopies - 1))],
                    static_cast<unsigned long long>(__double_as_longlong(w)) & 0xfffffffffffffull);
        }
      }
    }
    __syncthreads();
    for (int b = tid; b < kGridBins; b += kScanThreads) {
      unsigned long long sum = 0;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) sum += s_bin[b * kCopies + c];
      out.data[b] = sum;
    }
    return;
  }
  uint32_t cut = top;
  int turn = 0;
  if (mode == Mode::TopK) {
    // At least k pieces reach the k-th largest of the pieces' largest logits, so at
    // least k tokens do, and few more while there are many more pieces than k.
    const int k = rules.k;
    auto pieces = [&](uint32_t least) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) c += popc64(__ballot(most[i] >= least));
      return block_count<kScanThreads>(c, s_part, turn++);
    };
    // every thread's largest logit is at least the smallest of them
    cut = max(low, kKeyNegInf + 1);
    int c = pieces(cut);
    if (c < k && cut > kKeyNegInf + 1) {
      cut = kKeyNegInf + 1;
      c = pieces(cut);
    }
    if (c > k) cut = bisect<uint32_t>(cut, top, k, k + k / 8 + 8, pieces);
  }
  if (mode == Mode::Greedy) {
    // the lowest index of the largest logit
    uint32_t best = 0;
#pragma unroll
    for (int i = NV - 1; i >= 0; --i) {
      if (most[i] != top) continue;
#pragma unroll
      for (int j = Pieces<kBf16, NV, kScanThreads>::kPer - 1; j >= 0; --j)
        if (token_key(z.logit(i, j)) == top) best = 0xffffffffu - static_cast<uint32_t>(z.index(i, j));
    }
    best = block_max(best, s_max);
    if (tid == 0) {
      out.n = 1;
      out.data[0] = (static_cast<unsigned long long>(top) << 32) | best;
    }
    return;
  }
  // The pieces that reach the cut, a few of each wave, are queued in LDS and their tokens
  // looked at one per thread.  More pieces than the queue holds: more candidates than
  // the list holds, too.
  uint4* queue = reinterpret_cast<uint4*>(s_bin);
  int* first = reinterpret_cast<int*>(queue + kCandCap);
  static_assert(sizeof(s_bin) >= kCandCap * (sizeof(uint4) + sizeof(int)), "the queue fits");
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (most[i] < cut) continue;
    const int at = atomicAdd(&s_queued, 1);
    if (at < kCandCap) {
      queue[at] = z.v[i];
      first[at] = z.index(i, 0);
    }
  }
  __syncthreads();
  constexpr int kPer = Pieces<kBf16, NV, kScanThreads>::kPer;
  const int queued = s_queued, waiting = min(queued, kCandCap) * kPer;
  auto queued_key = [&](int i) {
    const int j = i % kPer;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(queue + i / kPer);
    return token_key(__uint_as_float(kBf16 ? (j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16) : w[j]));
  };
  auto list = [&]() {
    for (int i = tid; i < waiting; i += kScanThreads) {
      const uint32_t key = queued_key(i);
      if (key < cut) continue;
      const int at = atomicAdd(&s_n, 1);
      if (at < kCandCap) out.data[at] = token_order(key, first[i / kPer] + i % kPer);
    }
    __syncthreads();
  };
  list();
  if (mode == Mode::TopK && s_n > kCandCap && queued <= kCandCap) {
    // a top_k of a good part of the pieces: cut by tokens
    cut = bisect<uint32_t>(cut, top, rules.k, kCandCap, [&](uint32_t least) {
      int c = 0;
      for (int i = 0; i < waiting; i += kScanThreads)
        c += popc64(__ballot(i + tid < waiting && queued_key(i + tid) >= least));
      return block_count<kScanThreads>(c, s_part, turn++);
    });
    __syncthreads();
    if (tid == 0) s_n = 0;
    __syncthreads();
    list();
  }
  if (tid == 0) {
    out.n = queued > kCandCap ? queued : s_n;
    out.cut = cut;
  }
}

// ---------------------------------------------------------------------------
// From here on a workgroup works on one row, once, so its time is latency and, with
// code that runs once, the fetching of instructions: short loops over LDS instead of
// unrolled code over registers (an unrolled sort and search took 25 us for 64 rows, 6 us
// where all rows were done already).
// ---------------------------------------------------------------------------
// inclusive running sum over the workgroup, in thread order
__device__ __forceinline__ double block_scan(double v, double* part) {
  for (int o = 1; o < kWave; o <<= 1) {
    const double u = __shfl_up(v, o);
    if (lane_id() >= o) v += u;
  }
  __syncthreads();
  if (lane_id() == kWave - 1) part[wave_id()] = v;
  __syncthreads();
  double before = 0.0;
  for (int w = 0; w < wave_id(); ++w) before += part[w];
  return before + v;
}

__device__ __forceinline__ unsigned long long wave_sum_u64(unsigned long long v) {
  auto add = [](double a, double b) {
    return __longlong_as_double(__double_as_longlong(a) + __double_as_longlong(b));
  };
  return static_cast<unsigned long long>(__double_as_longlong(dpp::reduce(__longlong_as_double(v), 0.0, add)));
}

constexpr int kPlaceThreads = 256;
constexpr int kPlaceMine = kGridBins / kPlaceThreads;  // neighbouring bins (or sorted tokens) of a thread
constexpr int kDirect = 128;
constexpr int kNearMax = 2048;                         // candidates that reach the cut known so far
static_assert(kFastK <= kGridBins, "a sorted top-k fits the places");

struct PlaceShared {
  unsigned long long near[kNearMax];
  unsigned long long token[kGridBins], weight[kGridBins], sum[kGridBins];
  double part[kPlaceThreads / kWave];
  double value;
  unsigned long long most;
  int4 counts[2 * kPlaceThreads / kWave];
  int offset[kMaxSplits + 1];  // candidates in front of each split's
  int n, at;
};

// smallest bin at which `hit` holds, n if none
__device__ __forceinline__ int first_bin(const bool (&hit)[kPlaceMine], int n, PlaceShared& sh) {
  int mine = n;
#pragma unroll
  for (int e = kPlaceMine - 1; e >= 0; --e) mine = hit[e] ? static_cast<int>(threadIdx.x) * kPlaceMine + e : mine;
  const uint64_t m = __ballot(mine < n);
  __syncthreads();
  if (threadIdx.x == 0) sh.at = n;
  __syncthreads();
  if (m != 0 && lane_id() == __builtin_ctzll(m)) atomicMin(&sh.at, mine);
  __syncthreads();
  return sh.at;
}

__device__ __forceinline__ double bin_value(const double (&v)[kPlaceMine], int bin, PlaceShared& sh) {
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kPlaceMine; ++e)
    if (static_cast<int>(threadIdx.x) * kPlaceMine + e == bin) sh.value = v[e];
  __syncthreads();
  return sh.value;
}

// The i-th candidate of a row; offsets hold the counts in front of each split's.
__device__ __forceinline__ unsigned long long candidate(const RowView& ws, const int* offset, int i) {
  int s = 0;
  while (i >= offset[s + 1]) ++s;
  return ws.split[s].data[i - offset[s]];
}

// bisect() with three cuts a round, whose counts come back together: a round is a barrier and a
// trip through LDS, whatever it counts.
template <class T, class Count>
__device__ __forceinline__ T quarter(T lo, T hi, int need, Count count) {
  while (lo < hi) {
    const T span = hi - lo, c1 = lo + span / 4 + 1, c2 = max(c1, lo + span / 2 + 1), c3 = max(c2, hi - span / 4);
    const int4 c = count(c1, c2, c3);
    if (c.z >= need) lo = c3;
    else if (c.y >= need) lo = c2, hi = c3 - 1;
    else if (c.x >= need) lo = c1, hi = c2 - 1;
    else hi = c1 - 1;
    if (c.x == need || c.y == need || c.z == need) return c.z == need ? c3 : c.y == need ? c2 : c1;
  }
  return lo;
}

// The cut that leaves exactly k of the candidates; at least k have a key >= least.  Keys of
// bf16 logits differ in their upper half only (below it zeros, or ones if negative).
template <class CountKeys, class CountTokens>
__device__ __forceinline__ unsigned long long cut_to(const SampleParams& p, int k, uint32_t least, uint32_t top,
                                                     CountKeys keys, CountTokens tokens) {
  const int shift = p.is_bf16 ? 16 : 0;
  uint32_t key = quarter<uint32_t>(least >> shift, top >> shift, k,
                                   [&](uint32_t a, uint32_t b, uint32_t c) { return keys(a << shift, b << shift, c << shift); })
                 << shift;
  if (p.is_bf16 && !(key & 0x80000000u)) key |= 0xffffu;
  return quarter<unsigned long long>(token_order(key, p.V - 1), token_order(key, 0), k, tokens);
}

// sh.token[0, n) in descending order (n <= kGridBins)
__device__ __forceinline__ void sort_tokens(int n, PlaceShared& sh) {
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += kPlaceThreads) sh.token[i] = 0;
  for (int run = 2; run <= size; run *= 2) {
    for (int j = run / 2; j > 0; j /= 2) {
      __syncthreads();
      for (int q = threadIdx.x; q < size / 2; q += kPlaceThreads) {
        const int i = 2 * q - (q & (j - 1));
        const unsigned long long a = sh.token[i], b = sh.token[i + j];
        if (((i & run) == 0) == (a < b)) {
          sh.token[i] = b;
          sh.token[i + j] = a;
        }
      }
    }
  }
  __syncthreads();
}

// Candidates of a greedy or top-k row -> token.  False: the lists do not hold them all.
__device__ __forceinline__ bool pick_candidates(const SampleParams& p, int r, const Rules& rules, const RowView& ws,
                                                int splits, PlaceShared& sh) {
  const int tid = threadIdx.x, lane = lane_id();
  // every wave reads the splits' heads, one per lane
  const int ns = lane < splits ? ws.split[lane].n : 0;
  uint32_t top = lane < splits && ns > 0 ? ws.split[lane].top : 0;
  const uint32_t split_cut = lane < splits ? ws.split[lane].cut : 0;
  auto larger = [](uint32_t a, uint32_t b) { return max(a, b); };
  top = dpp::reduce(top, 0u, larger);
  const int upto = wave_incl_scan_i32(ns);
  const int n = lane_value(upto, kWave - 1);
  if (__ballot(ns > kCandCap) != 0) return false;
  if (n == 0) {
    if (tid == 0) p.token[r] = -1, p.prob[r] = 0.f;
    return true;
  }
  if (rules.mode == Mode::Greedy) {
    if (tid < kWave) {
      unsigned long long best = ns > 0 ? ws.split[lane].data[0] : 0;
      for (int o = 32; o >= 1; o >>= 1) best = max(best, __shfl_xor(best, o));
      if (tid == 0) p.token[r] = order_index(best), p.prob[r] = 1.f;
    }
    return true;
  }
  const int k = min(rules.k, n);
  // a split with k candidates of its own: at least k of the row reach its cut
  uint32_t least = dpp::reduce(ns >= k ? split_cut : 0u, 0u, larger);
  if (wave_id() == 0) {
    if (lane < splits) sh.offset[lane + 1] = upto;
    if (lane == 0) sh.offset[0] = sh.n = 0;
  }
  // all candidates, eight of a thread's requested at a time
  auto each_candidate = [&](auto take) {
    constexpr int kLoads = 8;
    for (int i0 = tid; i0 < n; i0 += kLoads * kPlaceThreads) {
      unsigned long long v[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int i = i0 + u * kPlaceThreads;
        v[u] = i < n ? candidate(ws, sh.offset, i) : 0;
      }
#pragma unroll
      for (int u = 0; u < kLoads; ++u)
        if (v[u] != 0) take(v[u]);
    }
  };
  if (n > kNearMax) {
    // raise that bound: counts of 1024 equal ranges of keys
    int* count = reinterpret_cast<int*>(sh.sum);
    for (int i = tid; i < kGridBins; i += kPlaceThreads) count[i] = 0;
    __syncthreads();
    const int shift = max(0, 32 - __clz(static_cast<int>(top - least)) - 10);
    each_candidate([&](unsigned long long v) {
      if (order_key(v) >= least) atomicAdd(&count[(order_key(v) - least) >> shift], 1);
    });
    __syncthreads();
    int mine = 0, incl[kPlaceMine];
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e) {
      mine += count[kGridBins - 1 - (tid * kPlaceMine + e)];
      incl[e] = mine;
    }
    const int front = static_cast<int>(block_scan(mine, sh.part)) - mine;
    bool hit[kPlaceMine];
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e) hit[e] = front + incl[e] >= k;
    least += static_cast<uint32_t>(kGridBins - 1 - first_bin(hit, kGridBins - 1, sh)) << shift;
  }
  __syncthreads();
  each_candidate([&](unsigned long long v) {
    if (order_key(v) < least) return;
    const int at = atomicAdd(&sh.n, 1);
    if (at < kNearMax) sh.near[at] = v;
  });
  __syncthreads();
  const int m = sh.n;
  if (m > kNearMax) return false;
  constexpr int kMine = kNearMax / kPlaceThreads;
  unsigned long long mine[kMine];  // empty places are 0, which no cut above 0 reaches
#pragma unroll
  for (int i = 0; i < kMine; ++i) mine[i] = tid + i * kPlaceThreads < m ? sh.near[tid + i * kPlaceThreads] : 0;
  unsigned long long cut = 1;
  if (m > k) {
    int turn = 0;
    auto counts = [&](auto value, auto a, auto b, auto c) {
      int4 n3 = make_int4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (i * kPlaceThreads >= m) continue;
        n3.x += popc64(__ballot(value(mine[i]) >= a));
        n3.y += popc64(__ballot(value(mine[i]) >= b));
        n3.z += popc64(__ballot(value(mine[i]) >= c));
      }
      int4* half = sh.counts + (turn++ & 1) * (kPlaceThreads / kWave);
      if (lane == 0) half[wave_id()] = n3;
      __syncthreads();
      n3 = half[0];
#pragma unroll
      for (int w = 1; w < kPlaceThreads / kWave; ++w) {
        n3.x += half[w].x;
        n3.y += half[w].y;
        n3.z += half[w].z;
      }
      return n3;
    };
    cut = cut_to(
        p, k, least, top,
        [&](uint32_t a, uint32_t b, uint32_t c) { return counts([](unsigned long long v) { return order_key(v); }, a, b, c); },
        [&](unsigned long long a, unsigned long long b, unsigned long long c) {
          return counts([](unsigned long long v) { return v; }, a, b, c);
        });
  }
  __syncthreads();
  if (tid == 0) sh.n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMine; ++i)
    if (mine[i] >= cut) sh.token[atomicAdd(&sh.n, 1)] = mine[i];  // k in all
  __syncthreads();
  // Weights as whole numbers, and each token's sum through it: up to kDirect tokens by adding
  // up all that are larger, shared by the 256 / k threads of a token, more by sorting (the
  // whole call, 96 of 32000: 23.0 / 26.0 us, 128: 26.2 / 28.1, 256: 36.0 / 29.7).
  const RowRule rule{top, key_logit(top), rules.tau};
  const bool direct = k <= kDirect;
  if (!direct) sort_tokens(k, sh);
  ulonglong2* pair = reinterpret_cast<ulonglong2*>(sh.near);  // token and weight: one read of LDS
  for (int t = tid; t < k; t += kPlaceThreads) {
    const unsigned long long w = rule.fixed(order_key(sh.token[t]));
    sh.weight[t] = w;
    if (direct) pair[t] = make_ulonglong2(sh.token[t], w);
  }
  if (tid == 0) sh.most = 0;
  __syncthreads();
  unsigned long long total = 0;
  if (direct) {
    int share = 1;
    while (2 * share * k <= kPlaceThreads && share < kWave) share *= 2;
    const int t = tid / share;
    unsigned long long s = 0;
    if (t < k) {
      const unsigned long long own = sh.token[t];
#pragma unroll 8
      for (int j = tid & (share - 1); j < k; j += share) s += pair[j].x >= own ? pair[j].y : 0;
    }
    for (int o = 1; o < share; o *= 2) s += __shfl_xor(s, o);
    if (t < k && (tid & (share - 1)) == 0) sh.sum[t] = s;
  } else {
    unsigned long long run[kPlaceMine], s = 0;
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e) {
      const int t = tid * kPlaceMine + e;
      s += t < k ? sh.weight[t] : 0;
      run[e] = s;
    }
    unsigned long long upto64 = s;
    for (int o = 1; o < kWave; o <<= 1) {
      const unsigned long long u = __shfl_up(upto64, o);
      if (lane >= o) upto64 += u;
    }
    if (lane == kWave - 1) sh.near[wave_id()] = upto64;
    __syncthreads();
    unsigned long long front = upto64 - s;
    for (int w = 0; w < wave_id(); ++w) front += sh.near[w];
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e)
      if (tid * kPlaceMine + e < k) sh.sum[tid * kPlaceMine + e] = front + run[e];
  }
  __syncthreads();
  // C of the top_k is the largest sum, C of what the other filters keep the largest one kept:
  // each keeps a prefix, and always the first token (whose sum is its weight)
  for (int t = tid; t < k; t += kPlaceThreads) total = max(total, sh.sum[t]);
  if (total != 0) atomicMax(&sh.most, total);
  __syncthreads();
  const double want = rules.by_p() ? rules.top_p * static_cast<double>(sh.most) : INFINITY;
  __syncthreads();
  if (tid == 0) sh.most = 0;
  __syncthreads();
  unsigned long long kept = 0;
  for (int t = tid; t < k; t += kPlaceThreads) {
    const unsigned long long w = sh.weight[t], before = sh.sum[t] - w;
    const bool keep = static_cast<double>(before) < want &&
                      (!rules.by_m() || rule.weight(order_key(sh.token[t])) >= rules.min_p);
    if (keep || before == 0) kept = max(kept, sh.sum[t]);
  }
  if (kept != 0) atomicMax(&sh.most, kept);
  __syncthreads();
  const double c = static_cast<double>(sh.most);
  const unsigned long long at = min(static_cast<unsigned long long>(rules.u * c), sh.most - 1);
  for (int t = tid; t < k; t += kPlaceThreads) {
    if (sh.sum[t] <= at || sh.sum[t] - sh.weight[t] > at) continue;  // one token's sum passes u C
    p.token[r] = order_index(sh.token[t]);
    p.prob[r] = static_cast<float>(rule.weight(order_key(sh.token[t])) * kWeightOne / c);
  }
  return true;
}

// One workgroup per row: a greedy or top-k row's token from its candidates, else the bins in
// which the kept prefix ends and in which the sample lies.
__global__ __launch_bounds__(kPlaceThreads) void sample_place_kernel(SampleParams p, int row0, int splits) {
  __shared__ PlaceShared sh;
  const int local = blockIdx.x, r = row0 + local, tid = threadIdx.x;
  const RowView ws(p, local, splits);
  const Rules rules = row_rules(p, r);
  if (rules.mode == Mode::Slow) return;
  if (rules.mode != Mode::Full) {
    if (!pick_candidates(p, r, rules, ws, splits, sh) && tid == 0) ws.row->slow = 1;
    return;
  }
  uint32_t top = lane_id() < splits ? ws.split[lane_id()].top : 0;
  top = dpp::reduce(top, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
  const Grid grid{kPerNat / static_cast<double>(rules.tau)};
  const double grid_top = floor(grid.at(top));
  // far from 0 the grid's 64 bits no longer hold the weights' digits
  const bool slow = !(fabs(grid.at(top)) < 33554432.0);
  if (tid == 0) {
    ws.row->top = top;
    ws.row->slow = slow && top > kKeyNegInf;
    ws.row->grid_top = grid_top;
  }
  if (top <= kKeyNegInf || slow) return;
  // the row's sums in this thread's bins below its largest logit
  unsigned long long sum[kPlaceMine] = {};
  for (int i = 0; i < splits; ++i) {
    const uint32_t part_top = ws.split[i].top;
    if (part_top <= kKeyNegInf) continue;
    const double lower = grid_top - floor(grid.at(part_top));
    if (lower >= kGridBins) continue;
    const int at = tid * kPlaceMine - static_cast<int>(lower);
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e)
      if (at + e >= 0) sum[e] += ws.split[i].data[at + e];
  }
  double incl[kPlaceMine], excl[kPlaceMine], mine = 0.0;
  constexpr double kStep = 0.96923323447634413;  // exp(-1 / 32)
  double factor = exp(-tid * kPlaceMine / kPerNat) / kWeightOne;
#pragma unroll
  for (int e = 0; e < kPlaceMine; ++e) {
    excl[e] = mine;
    mine += static_cast<double>(sum[e]) * factor;
    incl[e] = mine;
    factor *= kStep;
  }
  const double front = block_scan(mine, sh.part) - mine;
#pragma unroll
  for (int e = 0; e < kPlaceMine; ++e) {
    excl[e] += front;
    incl[e] += front;
  }
  const double total = bin_value(incl, kGridBins - 1, sh);
  bool hit[kPlaceMine];
  auto first = [&](auto passes, int n) {
#pragma unroll
    for (int e = 0; e < kPlaceMine; ++e) hit[e] = passes(incl[e]);
    return min(first_bin(hit, n, sh), n);
  };
  int cut = -1;
  double kept = total, least = total;  // the kept sum lies between
  if (rules.by_p()) {
    const double want = rules.top_p * total;
    cut = first([&](double v) { return v >= want; }, kGridBins - 1);
  }
  if (rules.by_m()) {
    // Where the border meets a bin's lower edge within rounding the next bin is looked at: its first
    // tokens may weigh min_p in 64 bits (a temperature of 1e20 with min_p = 1: all weigh 1).
    const double below = kPerNat * log(rules.min_p);
    const double slack = (fabs(grid.at(top)) - below + 1.0) * 0x1p-50;
    const double t = grid_top - floor(grid.at(top) + below - slack);
    if (t < (cut < 0 ? kGridBins : cut)) cut = static_cast<int>(t);
  }
  if (cut >= 0) {
    kept = bin_value(incl, cut, sh);
    least = bin_value(excl, cut, sh);
  }
  // the last bin that holds a kept weight, for roundings at the end
  const int last = cut >= 0 ? cut : first([&](double v) { return v >= total; }, kGridBins - 1);
  const int pick0 = first([&](double v) { return v > rules.u * least; }, last);
  const int pick1 = kept > least ? first([&](double v) { return v > rules.u * kept; }, last) : pick0;
#pragma unroll
  for (int e = 0; e < kPlaceMine; ++e) {
    if (tid * kPlaceMine + e == pick0) ws.row->before_pick = excl[e];
    if (tid * kPlaceMine + e == cut) ws.row->before_cut = excl[e];
  }
  if (tid == 0) {
    ws.row->t_cut = cut;
    ws.row->t_pick0 = pick0;
    ws.row->t_pick1 = pick1;
    ws.row->total = total;
  }
}

struct FilterCounts {
  int n_cut, n_pick, cut0, pick0;
};

// Lists the tokens of part s of a row that lie in the named bins: a bit per token of this
// thread, then one counter per list in LDS and one addition to the row's per workgroup.
template <bool kBf16, int NV, int kThreads>
__device__ __forceinline__ void list_tokens(const Pieces<kBf16, NV, kThreads>& z, const Grid& grid, RowPart& row,
                                            FilterCounts& sh) {
  constexpr int kPer = Pieces<kBf16, NV, kThreads>::kPer;
  static_assert(NV * kPer <= 32, "a bit per token");
  const double grid_top = row.grid_top, cut = row.t_cut, pick0 = row.t_pick0, pick1 = row.t_pick1;
  uint32_t in_cut = 0, in_pick = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const double t = grid_top - floor(static_cast<double>(z.logit(i, j)) * grid.scale);
      in_cut |= t == cut ? 1u << (i * kPer + j) : 0u;
      in_pick |= t >= pick0 && t <= pick1 ? 1u << (i * kPer + j) : 0u;
    }
  }
  if (threadIdx.x == 0) sh.n_cut = sh.n_pick = 0;
  __syncthreads();
  int at_cut = in_cut ? atomicAdd(&sh.n_cut, __popc(in_cut)) : 0;
  int at_pick = in_pick ? atomicAdd(&sh.n_pick, __popc(in_pick)) : 0;
  __syncthreads();
  if (threadIdx.x == 0) {
    sh.cut0 = sh.n_cut ? atomicAdd(&row.n_cut, sh.n_cut) : 0;
    sh.pick0 = sh.n_pick ? atomicAdd(&row.n_pick, sh.n_pick) : 0;
  }
  __syncthreads();
  at_cut += sh.cut0;
  at_pick += sh.pick0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t bit = 1u << (i * kPer + j);
      if (((in_cut | in_pick) & bit) == 0) continue;
      const unsigned long long token = token_order(token_key(z.logit(i, j)), z.index(i, j));
      if (in_cut & bit) {
        if (at_cut < kListCap) row.cut[at_cut] = token;
        ++at_cut;
      }
      if (in_pick & bit) {
        if (at_pick < kListCap) row.pick[at_pick] = token;
        ++at_pick;
      }
    }
  }
}

template <bool kBf16, int NV>
__global__ __launch_bounds__(kPlaceThreads) void sample_filter_kernel(SampleParams p, int row0, int rows, int splits) {
  __shared__ FilterCounts sh;
  const int local = blockIdx.x % rows, r = row0 + local, s = blockIdx.x / rows;
  Pieces<kBf16, NV, kPlaceThreads> z;
  z.load(p, r, s);
  const RowView ws(p, local, splits);
  const Rules rules = row_rules(p, r);
  if (rules.mode != Mode::Full || ws.row->slow || ws.row->top <= kKeyNegInf) return;
  list_tokens(z, Grid{kPerNat / static_cast<double>(rules.tau)}, *ws.row, sh);
}

constexpr int kFinishMine = kListCap / kRowThreads;
constexpr int kWindow = 64;  // tokens around a place, ordered by adding up all larger ones

struct FinishShared {
  ulonglong2 near[kWindow];  // token and weight
  double step[kGridBins];    // exp(-b / 32)
  unsigned long long part64[2 * kRowThreads / kWave];
  int part32[2 * kRowThreads / kWave];
  uint32_t range[2 * kRowThreads / kWave];
  unsigned long long found;
  double sum;
  int n, hit;
};

union FinishUnion {
  RowShared row;
  FinishShared fin;
};

// A listed range of bins in the registers of the workgroup: token and weight, in 2^-43 of
// the range's first bin (whole numbers: sums in any order are the same).
struct Listed {
  unsigned long long token[kFinishMine], weight[kFinishMine];
  int n;
};

struct PlaceInList {
  unsigned long long token;
  double sum;
};

// The token of a list, from bin t0 on, at which passes(before + sum up to it) turns true, and that
// sum; the list's last one if it never does, its first one where `before` passes by itself (a
// border of 0, or one that a rounding puts in front of the list).  The order is searched by
// halves until at most kWindow tokens are left around the place.
template <class Passes>
__device__ __forceinline__ PlaceInList place_in_list(const Listed& l, int t0, double before, FinishShared& sh,
                                                     Passes passes) {
  constexpr int kWaves = kRowThreads / kWave;
  const int tid = threadIdx.x, lane = lane_id();
  const double unit = sh.step[t0] / kWeightOne;
  // an empty sum reaches nothing
  auto reached = [&](unsigned long long sum) { return (sum != 0) & passes(before + static_cast<double>(sum) * unit); };
  // every token lies in [lo, hi): a list's keys share their upper bits
  uint32_t least = ~0u, most = 0;
#pragma unroll
  for (int i = 0; i < kFinishMine; ++i) {
    least = min(least, l.token[i] != 0 ? order_key(l.token[i]) : ~0u);
    most = max(most, order_key(l.token[i]));
  }
  block_range(most, least, sh.range);
  unsigned long long lo = static_cast<unsigned long long>(least) << 32;
  unsigned long long hi = (static_cast<unsigned long long>(most) + 1) << 32;
  unsigned long long above = 0;  // weight of tokens from hi on
  int inside = l.n, count_above = 0;
  for (int turn = 0; inside > kWindow && hi - lo > 1; ++turn) {
    const unsigned long long mid = lo + (hi - lo) / 2;
    unsigned long long w = 0;
    int c = 0;
#pragma unroll
    for (int i = 0; i < kFinishMine; ++i) {
      if (i * kRowThreads >= l.n) continue;
      w += l.token[i] >= mid ? l.weight[i] : 0;
      c += popc64(__ballot(l.token[i] >= mid));
    }
    w = wave_sum_u64(w);
    const int half = (turn & 1) * kWaves;
    if (lane == 0) {
      sh.part64[half + wave_id()] = w;
      sh.part32[half + wave_id()] = c;
    }
    __syncthreads();
    w = 0;
    c = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      w += sh.part64[half + i];
      c += sh.part32[half + i];
    }
    if (reached(w)) {
      lo = mid;
      inside = c - count_above;
    } else {
      hi = mid;
      inside -= c - count_above;
      above = w;
      count_above = c;
    }
  }
  __syncthreads();
  if (tid == 0) {
    sh.n = 0;
    sh.hit = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kFinishMine; ++i) {
    if (l.token[i] == 0 || l.token[i] < lo || l.token[i] >= hi) continue;
    const int at = atomicAdd(&sh.n, 1);  // kWindow at most
    sh.near[at] = make_ulonglong2(l.token[i], l.weight[i]);
  }
  __syncthreads();
  // the sum up to each token, by kShare threads (with one thread each the kernel took 17.8 us instead of 13.3)
  constexpr int kShare = kRowThreads / kWindow;
  const int m = sh.n, t = tid / kShare;
  const unsigned long long v = t < m ? sh.near[t].x : ~0ull, w = t < m ? sh.near[t].y : 0;
  unsigned long long s = 0;
  int c = 0;
#pragma unroll
  for (int j = 0; j < kWindow / kShare; ++j) {
    const int at = j * kShare + tid % kShare;
    const ulonglong2 other = sh.near[at];
    const bool up = at < m && other.x >= v;
    s += up ? other.y : 0;
    c += up ? 1 : 0;
  }
  for (int o = 1; o < kShare; o *= 2) {
    s += __shfl_xor(s, o);
    c += __shfl_xor(c, o);
  }
  s += above;
  const double sum = before + static_cast<double>(s) * unit;
  const bool mine = t < m && tid % kShare == 0;
  if (mine && reached(s) && !reached(s - w)) {
    sh.hit = 1;
    sh.found = v;
    sh.sum = sum;
  }
  __syncthreads();
  if (sh.hit == 0 && ((mine && c == m) || (m == 0 && tid == 0))) {  // none: the smallest
    sh.found = m == 0 ? 0 : v;
    sh.sum = m == 0 ? before : sum;
  }
  __syncthreads();
  return {sh.found, sh.sum};
}

__device__ __forceinline__ int bin_index(double t) { return static_cast<int>(fmin(fmax(t, 0.0), kGridBins - 1.0)); }

// The token of a row whose bins are listed.
__device__ __forceinline__ void finish_row(const SampleParams& p, int r, const Rules& rules, const RowPart& in,
                                           const RowHead& head, int n_cut, int n_pick, FinishShared& sh) {
  const int tid = threadIdx.x;
  const Grid grid{kPerNat / static_cast<double>(rules.tau)};
#pragma unroll 1
  for (int b = tid; b < kGridBins; b += kRowThreads) sh.step[b] = exp(-b / kPerNat);
  __syncthreads();
  double total = head.total;
  unsigned long long token = 0;
  // first the list in which the kept prefix ends, then that in which the sample lies
#pragma unroll 1
  for (int step = head.t_cut >= 0 ? 0 : 1; step < 2; ++step) {
    const unsigned long long* list = step == 0 ? in.cut : in.pick;
    const int t0 = step == 0 ? head.t_cut : head.t_pick0;
    const double before = step == 0 ? head.before_cut : head.before_pick;
    Listed l;
    l.n = step == 0 ? n_cut : n_pick;
#pragma unroll
    for (int i = 0; i < kFinishMine; ++i)
      l.token[i] = tid + i * kRowThreads < l.n ? list[tid + i * kRowThreads] : 0;
#pragma unroll
    for (int i = 0; i < kFinishMine; ++i) {
      l.weight[i] = 0;
      if (l.token[i] == 0) continue;
      const double g = grid.at(order_key(l.token[i])), b = floor(g);
      l.weight[i] = __double2ull_rn(Grid::weight(g - b) * sh.step[bin_index(head.grid_top - t0 - b)] * kWeightOne);
    }
    // both filters keep a prefix: the shorter one
    const double want = step == 1 ? rules.u * total : rules.by_p() ? rules.top_p * total : INFINITY;
    const PlaceInList at = place_in_list(l, t0, before, sh, [&](double sum) { return step == 1 ? sum > want : sum >= want; });
    if (step == 1) {
      token = at.token;
      break;
    }
    double kept = at.sum >= want ? at.sum : INFINITY;
    if (rules.by_m()) {
      const RowRule rule{head.top, key_logit(head.top), rules.tau};
      unsigned long long w = 0;
#pragma unroll 1
      for (int i = 0; i < l.n; i += kRowThreads) {
        unsigned long long v = 0, own = 0;
#pragma unroll
        for (int q = 0; q < kFinishMine; ++q) {
          v = q * kRowThreads == i ? l.token[q] : v;
          own = q * kRowThreads == i ? l.weight[q] : own;
        }
        if (v != 0 && rule.weight(order_key(v)) >= rules.min_p) w += own;
      }
      w = wave_sum_u64(w);
      __syncthreads();
      if (lane_id() == 0) sh.part64[wave_id()] = w;
      __syncthreads();
      w = 0;
      for (int i = 0; i < kRowThreads / kWave; ++i) w += sh.part64[i];
      kept = fmin(kept, before + static_cast<double>(w) * (sh.step[t0] / kWeightOne));
      __syncthreads();
    }
    total = fmin(kept, total);
  }
  if (tid == 0) {
    const double g = grid.at(order_key(token)), b = floor(g);
    p.token[r] = order_index(token);
    p.prob[r] = static_cast<float>(Grid::weight(g - b) * sh.step[bin_index(head.grid_top - b)] / total);
  }
}

// A row that is not done yet, by a workgroup.  kList: lists the bins' tokens itself, part after
// part; used beside top_k, where few rows need it.
template <bool kBf16, int NV, bool kList>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(4))) void sample_finish_kernel(SampleParams p, int row0, int splits) {
  __shared__ FinishUnion un;
  __shared__ FilterCounts counts;
  const int local = blockIdx.x, r = row0 + local, tid = threadIdx.x;
  const RowView ws(p, local, splits);
  RowPart& in = *ws.row;
  const RowHead head = in;
  const Rules rules = row_rules(p, r);
  if (head.slow == 0) {
    if (rules.mode != Mode::Full) return;
    if (head.top <= kKeyNegInf) {
      if (tid == 0) p.token[r] = -1, p.prob[r] = 0.f;
      return;
    }
    int n_cut = head.n_cut, n_pick = head.n_pick;
    if constexpr (kList) {
      const Grid grid{kPerNat / static_cast<double>(rules.tau)};
      for (int s = 0; s < splits; ++s) {
        Pieces<kBf16, NV, kScanThreads> z;
        z.load(p, r, s);
        __syncthreads();
        list_tokens(z, grid, in, counts);
      }
      __syncthreads();
      n_cut = __hip_atomic_load(&in.n_cut, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      n_pick = __hip_atomic_load(&in.n_pick, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (n_cut <= kListCap && n_pick <= kListCap) {
      finish_row(p, r, rules, in, head, n_cut, n_pick, un.fin);
      return;
    }
  }
  sample_row<kBf16>(p, r, rules, un.row);
}

// 16-byte pieces per thread: 32 tokens' worth; without top_k fewer while that spreads a row over
// more workgroups of an otherwise idle device (a row of 32000 fp32 logits, top-p: 27.0 us, else
// 28.7; beside top_k every split lists candidates: top-256 44.3 us, else 36.3)
struct Shape {
  int nv, splits;
};
Shape sample_shape(int R, int V, int is_bf16, int skew, bool spread) {
  const int per = is_bf16 ? 8 : 4;
  const int pieces = (skew + V + per - 1) / per;
  auto splits = [&](int nv) { return (pieces + kScanThreads * nv - 1) / (kScanThreads * nv); };
  int nv = 32 / per;
  while (spread && nv > 1 && splits(nv / 2) > splits(nv) && splits(nv / 2) <= 8 && R * splits(nv / 2) <= 1024) nv /= 2;
  return {nv, splits(nv)};
}

// the most tokens by which a row starts behind a 16-byte boundary
int row_skew(const SampleParams& p) {
  const size_t eb = p.is_bf16 ? 2 : 4;
  const size_t base = reinterpret_cast<uintptr_t>(p.logits) % 16;
  if (p.R == 1 || p.row_stride * eb % 16 == 0) return static_cast<int>(base / eb);
  return static_cast<int>(16 / eb) - 1;
}

template <bool kBf16, int NV>
hipError_t launch_sample_nv(const SampleParams& p, int splits, hipStream_t stream) {
  for (int row0 = 0; row0 < p.R; row0 += kRowsPerLaunch) {
    const int rows = p.R - row0 < kRowsPerLaunch ? p.R - row0 : kRowsPerLaunch;
    sample_scan_kernel<kBf16, NV><<<rows * splits, kScanThreads, 0, stream>>>(p, row0, splits);
    sample_place_kernel<<<rows, kPlaceThreads, 0, stream>>>(p, row0, splits);
    if (p.top_k) {
      sample_finish_kernel<kBf16, NV, true><<<rows, kRowThreads, 0, stream>>>(p, row0, splits);
    } else {
      sample_filter_kernel<kBf16, NV>
          <<<rows * splits * (kScanThreads / kPlaceThreads), kPlaceThreads, 0, stream>>>(p, row0, rows, splits);
      sample_finish_kernel<kBf16, NV, false><<<rows, kRowThreads, 0, stream>>>(p, row0, splits);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <bool kBf16>
hipError_t launch_sample_type(const SampleParams& p, hipStream_t stream) {
  const Shape sh = sample_shape(p.R, p.V, kBf16, row_skew(p), p.top_k == nullptr);
  switch (sh.nv) {
    case 1: return launch_sample_nv<kBf16, 1>(p, sh.splits, stream);
    case 2: return launch_sample_nv<kBf16, 2>(p, sh.splits, stream);
    case 4: return launch_sample_nv<kBf16, 4>(p, sh.splits, stream);
    default: break;
  }
  if constexpr (kBf16) return hipErrorInvalidValue;  // 32 tokens are four pieces
  else return launch_sample_nv<false, 8>(p, sh.splits, stream);
}

}  // namespace

// One size for both types: an fp32 row has more splits.  Grows with R: a row is spread
// over at most 8 workgroups or takes the splits of 32 tokens per thread.
static constexpr int most_splits(int V) { return (V + 6) / 4 / (kScanThreads * 8) + 1; }
static_assert(most_splits(kMaxVocab) <= kMaxSplits, "a row's splits: one per lane of a wave");

size_t sample_workspace_bytes(int R, int V) {
  const size_t rows = R < kRowsPerLaunch ? R : kRowsPerLaunch;
  const size_t whole = most_splits(V);
  return rows * sample_part_bytes(static_cast<int>(whole > 8 ? whole : 8));
}

hipError_t launch_sample(const SampleParams& p, hipStream_t stream) {
  return p.is_bf16 ? launch_sample_type<true>(p, stream) : launch_sample_type<false>(p, stream);
}

}  // namespace amoe
