// The grouped SwiGLU expert FFN with weights in 4 bits: a weight is an e2m1 code
// (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times a power of two shared by
// 32 columns of its row, W = code 2^(s - 127).
//   out_t = sum_j g_{t,j} W_d (silu(W_g x_t) * W_u x_t)
//
// Bound: with few rows per expert the weights' bytes (64 tokens in 26 experts, H = 4096,
// I = 1536: gate/up 174 MB in 41 us, 4.3 TB/s, down 87 MB in 27 us), with many the matrix cores
// and the expansion of the codes in front of them (1920 tokens, top-8, H = 2048, I = 768: 97
// and, with the second plane, 97 GFLOP in 107 to 128 us each, 760 to 900 TFLOP/s of the 1248 that a large
// bf16 product reaches), for a few tokens latency (one token: 6.2 and 6.0 us).
//
// Both factors of the gate and up products are exact in bf16 (a code has 2
// significant bits, its scale is a power of two), so they run on the bf16 MFMA
// with the weights expanded in registers.  The activation goes to the down
// product as two bf16 planes, hi = bf16(a) and lo = bf16(a - hi), 16 bits of it
// in all, which costs a second MFMA but no weight traffic: with hi alone every output
// would carry up to 2^-8 from that one rounding, more than from all else together.  A third
// plane would bring the error against 64 bits from 2.3e-6 .. 2.8e-6 to fp32's 0.6e-6 .. 1.2e-6, for
// half of the down product's MFMAs again where these bound it; the blocks that latency or the weights'
// bytes bound take the same two, so that precision does not depend on a block's size.
//
// Weights (pack_q4_kernel): per expert and quad of 16-row tiles one run over K;
// per 128 columns four fragments of 64 lanes x 16 B and 64 lanes x 4 B of scales.
// Lane (r, g) holds row r of each tile, columns 32 g .. + 31 of the chunk: one
// group, so one scale per fragment and lane, and four MFMA steps of 8 columns.
#include <type_traits>

#include "ffn_common.hpp"
#include "q4_plan.hpp"

namespace amoe {

namespace {

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// ---------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------
// One thread per lane of a quad's chunk.  kGateUp: tiles 0, 1 from a, 2, 3 from b
// (N = I rows); else four tiles of a (N = H rows).  Rows and columns past the
// stacks are zero codes.
template <bool kGateUp>
__global__ void pack_q4_kernel(const uint8_t* __restrict__ a, const uint8_t* __restrict__ a_scale,
                               const uint8_t* __restrict__ b, const uint8_t* __restrict__ b_scale,
                               uint8_t* __restrict__ dst, size_t total, int quads, int N, int K) {
  const int KC = q4_chunks(K);
  for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < total;
       i += static_cast<size_t>(gridDim.x) * blockDim.x) {
    const int lane = static_cast<int>(i % kWave), r = lane & 15, g = lane >> 4;
    const size_t qc = i / kWave;  // (e * quads + quad) * KC + chunk
    const int kc = static_cast<int>(qc % KC);
    const int quad = static_cast<int>(qc / KC % quads);
    const size_t e = qc / KC / quads;
    const int k0 = kc * kQ4Chunk + g * kQ4Group;
    uint8_t* out = dst + qc * kQ4QuadBytes;
    uint32_t scales = 0x7f7f7f7fu;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
      const int row = kGateUp ? quad * 32 + (f & 1) * 16 + r : quad * 64 + f * 16 + r;
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (row < N && k0 < K) {
        const bool second = kGateUp && f >= 2;
        const size_t at = (e * N + row) * K + k0;
        v = *reinterpret_cast<const uint4*>((second ? b : a) + at / 2);
        const uint32_t s = (second ? b_scale : a_scale)[at / kQ4Group];
        scales = (scales & ~(0xffu << (8 * f))) | (s << (8 * f));
      }
      reinterpret_cast<uint4*>(out)[f * kWave + lane] = v;
    }
    reinterpret_cast<uint32_t*>(out + 4 * 1024)[lane] = scales;
  }
}

// Codes and scales of 32 neighbouring values: the smallest power of two with
// max|w| <= 6 of it (scale byte 2 .. 252), each value to the nearest code, ties to the even one.
template <bool kBf16>
__global__ void quantize_q4_kernel(const void* __restrict__ w, size_t groups, uint4* __restrict__ codes,
                                   uint8_t* __restrict__ scales) {
  for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < groups;
       i += static_cast<size_t>(gridDim.x) * blockDim.x) {
    float v[32];
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < (kBf16 ? 4 : 8); ++j) {
      const uint4 q = static_cast<const uint4*>(w)[i * (kBf16 ? 4 : 8) + j];
      const uint32_t d[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (kBf16) {
          v[8 * j + 2 * c] = __uint_as_float(d[c] << 16);
          v[8 * j + 2 * c + 1] = __uint_as_float(d[c] & 0xffff0000u);
        } else {
          v[4 * j + c] = __uint_as_float(d[c]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) m = fmaxf(m, fabsf(v[j]));
    // m = 1.f 2^(e - 127): 6 2^(s - 127) holds it from s = e - 2 on, for .f above .5 from e - 1
    const uint32_t bits = __float_as_uint(m);
    int s = static_cast<int>(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x400000u ? 1 : 0);
    s = min(max(s, 2), 252);
    const float inv = __uint_as_float(static_cast<uint32_t>(254 - s) << 23);  // 2^(127 - s)
    uint32_t out[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float a = fabsf(v[j]) * inv;
      const uint32_t mag = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
      const uint32_t sign = (__float_as_uint(v[j]) >> 31) << 3;
      out[j / 8] |= (mag | sign) << (4 * (j % 8));
    }
    codes[i] = make_uint4(out[0], out[1], out[2], out[3]);
    scales[i] = static_cast<uint8_t>(s);
  }
}

// ---------------------------------------------------------------------------
// Dispatch: workgroup e counts every expert's slots in LDS, so it knows where expert
// e's list and items begin without waiting for another, and writes them: the slots
// that are routed to e in node order (deterministic) and one item (expert, first row,
// rows) per run of its rows.
// ---------------------------------------------------------------------------
constexpr int kDispatchSlots = 16384;  // routing entries of a chunk in LDS
constexpr uint16_t kNoExpert = 0xffff;

template <int KMAX, int kThreads>
__global__ __launch_bounds__(kThreads) void q4_dispatch_kernel(ForwardParams p) {
  __shared__ int s_cnt[kMaxExperts];
  __shared__ uint16_t s_idx[kDispatchSlots];
  __shared__ int s_wave[kThreads / kWave];
  __shared__ int s_off, s_item;
  const int tid = threadIdx.x, E = p.E, k = p.k, T = p.T, e = blockIdx.x;
  const int per_chunk = kDispatchSlots / k;  // rows
  // entries outside [0, E), and repeats within a row, as kNoExpert
  auto load = [&](int t0, int rows) {
    const int n = rows * k;
    const int32_t* idx = p.topk_idx + static_cast<size_t>(t0) * k;
    for (int i0 = tid; i0 < n; i0 += 4 * kThreads) {
      int v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i0 + u * kThreads < n ? idx[i0 + u * kThreads] : -1;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * kThreads < n)
          s_idx[i0 + u * kThreads] = v[u] >= 0 && v[u] < E ? static_cast<uint16_t>(v[u]) : kNoExpert;
    }
    __syncthreads();
    for (int r = tid; r < rows; r += kThreads) {
      uint16_t v[KMAX];
#pragma unroll
      for (int j = 0; j < KMAX; ++j) v[j] = s_idx[r * k + min(j, k - 1)];
#pragma unroll
      for (int j = 1; j < KMAX; ++j) {
        bool again = false;
#pragma unroll
        for (int d = 0; d < j; ++d) again = again | (v[d] == v[j]);
        if (again && j < k) s_idx[r * k + j] = kNoExpert;
      }
    }
    __syncthreads();
  };
  for (int i = tid; i < E; i += kThreads) s_cnt[i] = 0;
  for (int t0 = 0; t0 < T; t0 += per_chunk) {
    const int rows = min(per_chunk, T - t0);
    load(t0, rows);
    // Counted along the rows: neighbouring lanes hold one row's experts, which differ, where
    // the same slot of 64 rows is often one popular expert (64 LDS atomics in a row).
    for (int i = tid; i < rows * k; i += kThreads)
      if (s_idx[i] != kNoExpert) atomicAdd(&s_cnt[s_idx[i]], 1);
    __syncthreads();
  }
  if (tid < kWave) {
    int off = 0, items = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int c = e0 + tid < E ? s_cnt[e0 + tid] : 0;
      const int n = q4_items(c, p.item_rows);
      const int c_incl = wave_incl_scan_i32(c), n_incl = wave_incl_scan_i32(n);
      if (e0 + tid == e) {
        s_off = off + c_incl - c;
        s_item = items + n_incl - n;
      }
      off += lane_value(c_incl, kWave - 1);
      items += lane_value(n_incl, kWave - 1);
    }
    if (e == 0 && tid == 0) *p.n_items = items;
  }
  __syncthreads();
  const int count = s_cnt[e], off = s_off;
  if (count == 0) return;
  const int rows = q4_item_rows(count, p.item_rows);
  for (int m = tid; m < q4_items(count, p.item_rows); m += kThreads)
    p.items[s_item + m] = make_int4(e, off + rows * m, min(rows, count - rows * m), 0);
  int seen = 0;
  for (int t0 = 0; t0 < T && seen < count; t0 += per_chunk) {
    const int n_rows = min(per_chunk, T - t0);
    if (T > per_chunk) load(t0, n_rows);
    for (int r0 = 0; r0 < n_rows && seen < count; r0 += kThreads) {
      const int r = r0 + tid;
      int slot = -1;
      if (r < n_rows)
        for (int j = k - 1; j >= 0; --j) slot = s_idx[r * k + j] == e ? (t0 + r) * k + j : slot;
      const uint64_t m = __ballot(slot >= 0);
      if (lane_id() == 0) s_wave[wave_id()] = popc64(m);
      __syncthreads();
      int before = seen + popc64(m & lanes_below(lane_id()));
#pragma unroll
      for (int w = 0; w < kThreads / kWave; ++w) {
        before += w < wave_id() ? s_wave[w] : 0;
        seen += s_wave[w];
      }
      if (slot >= 0) p.ent_slot[off + before] = slot;
      __syncthreads();
    }
  }
}

// out[t] = sum of the token's slot rows, in slot order
template <int KMAX>
__global__ __launch_bounds__(256) void q4_combine_kernel(ForwardParams p, int hblocks, int t0) {
  const int t = t0 + blockIdx.x / hblocks;
  const int c = (blockIdx.x % hblocks) * 256 + threadIdx.x, H4 = p.H / 4;
  if (c >= H4) return;
  int ev[KMAX];
  const uint32_t valid = load_route_row<KMAX>(p.topk_idx + static_cast<size_t>(t) * p.k, p.k, p.E, ev);
  const float4* ys = reinterpret_cast<const float4*>(p.ys) + static_cast<size_t>(t) * p.k * H4 + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    if (valid & (1u << j)) {
      const float4 v = ys[static_cast<size_t>(j) * H4];
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  }
  reinterpret_cast<float4*>(p.out)[static_cast<size_t>(t) * H4 + c] = s;
}

// ---------------------------------------------------------------------------
// weights of a quad's chunk in registers
// ---------------------------------------------------------------------------
struct Q4Chunk {
  uint4 code[4];
  uint32_t scale;
};

template <int kPolicy = kPolicyStream>
__device__ __forceinline__ uint32_t load_scales(const uint4* base, int bytes, int offset) {
  __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint4*>(base), static_cast<short>(0), bytes, kBufferWord3);
  return __builtin_amdgcn_raw_buffer_load_b32(r, offset, 0, kPolicy);
}

template <int kPolicy>
__device__ __forceinline__ Q4Chunk load_q4(const uint4* base, int bytes, int kc, int lane) {
  Q4Chunk c;
#pragma unroll
  for (int f = 0; f < 4; ++f)
    c.code[f] = load_weight<kPolicy>(base, bytes, kc * (kQ4QuadBytes / 16) + f * kWave + lane);
  c.scale = load_scales<kPolicy>(base, bytes, kc * kQ4QuadBytes + 4096 + lane * 4);
  return c;
}

// 16 bytes at byte `offset` of [base, base + bytes), zeros outside
__device__ __forceinline__ uint4 load_piece(const void* base, uint32_t bytes, uint32_t offset) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0),
                                                               static_cast<int>(bytes), kBufferWord3);
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, static_cast<int>(offset), 0, kPolicyPlain);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// Eight codes (low nibble first) times the scale, in bf16: exact (infinite past the largest
// number).  The instruction takes the scale's exponent bits alone: byte 0, a scale of 0.0 as a
// float, stands for 2^-127, byte 255 for NaN.
__device__ __forceinline__ bf16x8 expand_q4(uint32_t codes, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float scale_of(uint32_t scales, int f) {
  return __uint_as_float(((scales >> (8 * f)) & 0xffu) << 23);
}

__device__ __forceinline__ uint32_t word(const uint4& v, int s) { return s == 0 ? v.x : s == 1 ? v.y : s == 2 ? v.z : v.w; }

// ---------------------------------------------------------------------------
// Grouped products.  A workgroup of four waves takes one item (expert, up to kRows of its
// rows) and four quads, one per wave.  Weights stream straight into the registers of the
// one wave that uses them; the item's rows are staged in LDS, once for the waves.  (K
// shared by two or four waves per quad, for blocks of few items: 92 -> 117 us on 64
// tokens of the wide layer, every workgroup stages the rows again.)
// ---------------------------------------------------------------------------
constexpr int kQ4Waves = 4;
constexpr int kQ4MaxRows = 64;
// LDS pieces of 16 B: two stages of an item's rows (down: in two planes)
template <bool kDown, int kRows>
constexpr int kQ4LdsPieces = 2 * (kDown ? 2 : 1) * kRows * 16;

// Waves per SIMD that the registers are cut for.
template <bool kDown, int kRows>
constexpr int kQ4WavesPerSimd = kDown ? 2 : 3;

struct Q4Rows {
  int slot[kQ4MaxRows];
  float gate[kQ4MaxRows];
};

template <bool kDown, int MT>
__device__ __forceinline__ void q4_rows(const ForwardParams& p, int e, int row0, int rows, int run, uint4* lds,
                                        const Q4Rows& qr) {
  constexpr int kPlanes = kDown ? 2 : 1;
  constexpr int kBuf = kPlanes * MT * 256;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // keeps address arithmetic of one tile count out of the others
  const int wave = wave_id(), lane = lane_id();
  const int r = lane & 15, g = lane >> 4;
  const int K = kDown ? p.I : p.H;
  const int KC = q4_chunks(K);
  const int quads = kDown ? q4_down_quads(p.H) : q4_gate_up_quads(p.I);
  const int quad = run * kQ4Waves + wave;
  const bool in = quad < quads;
  const size_t run_bytes = q4_quad_run(K);
  const uint4* w = uniform_ptr(reinterpret_cast<const uint4*>(static_cast<const char*>(kDown ? p.w_down : p.w_gate_up) +
                                                              (static_cast<size_t>(e) * quads + (in ? quad : 0)) * run_bytes));
  const int wbytes = in ? static_cast<int>(run_bytes) : 0;
  // thread tid loads piece tid % 16 (8 columns) of rows tid / 16 + 16 s
  constexpr int kPass = 4 * kQ4Waves, kPasses = 16 * MT / kPass;
  const int piece = tid & 15, srow = tid >> 4;
  const uint32_t plane_bytes = KC * (kQ4Chunk * 2);
  // Rows past the item's last read its first; their outputs are dropped.  Offsets into hidden fit
  // 32 bits (checked by the caller), those into the activations start at the item's first row.
  const void* xbase = kDown ? static_cast<const char*>(p.act) + static_cast<size_t>(row0) * 2 * plane_bytes
                            : static_cast<const char*>(p.hidden);
  const uint32_t xbytes = kDown ? static_cast<uint32_t>(rows) * 2 * plane_bytes
                                : static_cast<uint32_t>(p.T) * static_cast<uint32_t>(p.H) * 2;
  uint32_t xrow[kPasses];
#pragma unroll
  for (int s = 0; s < kPasses; ++s) {
    const int m = s * kPass + srow, row = m < rows ? m : 0;
    xrow[s] = (kDown ? static_cast<uint32_t>(row) * 2 * plane_bytes
                     : static_cast<uint32_t>(p.ent_slot[row0 + row] / p.k) * static_cast<uint32_t>(p.H) * 2) +
              piece * 16;
  }
  // Weights and rows are requested kAhead stages ahead: with few rows the stages are shorter
  // than the memory's latency and registers are left.
  constexpr int kAhead = MT == 1 ? 3 : 1;
  constexpr int kRing = kAhead == 1 ? 1 : kAhead + 1;  // rows in flight, and the stage being stored
  uint4 ra[kRing][kPlanes][kPasses], first[1][kPlanes][kPasses];
  // Columns past K lie outside the resource and read as zeros (a select behind the load would
  // be moved up to it, with a wait).
  auto load_rows = [&](int st, int slot, auto& to) {
    const bool valid = st * kQ4Chunk + piece * 8 < K;
#pragma unroll
    for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
      for (int s = 0; s < kPasses; ++s)
        to[slot % (sizeof(to) / sizeof(to[0]))][pl][s] =
            load_piece(xbase, xbytes, valid ? xrow[s] + (pl * plane_bytes + st * (kQ4Chunk * 2)) : ~15u);
  };
  // a row's piece sits at piece ^ row, so the 16 pieces of a row, and the 16
  // rows that a fragment reads at one piece, fall into different banks
  auto store_rows = [&](int slot, int buf, const auto& from) {
#pragma unroll
    for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
      for (int s = 0; s < kPasses; ++s) {
        const int row = s * kPass + srow;
        lds[buf * kBuf + (pl * MT * 16 + row) * 16 + (piece ^ (row & 15))] =
            from[slot % (sizeof(from) / sizeof(from[0]))][pl][s];
      }
  };
  floatx4 acc[4][MT];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[f][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int buf, const Q4Chunk& wc) {
    const uint4* x0 = lds + buf * kBuf + r * 16;
    float sc[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) sc[f] = scale_of(wc.scale, f);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      bf16x8 x[kPlanes][MT];
#pragma unroll
      for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          x[pl][mt] = __builtin_bit_cast(bf16x8, x0[(pl * MT + mt) * 256 + ((4 * g + s) ^ r)]);
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const bf16x8 b = expand_q4(word(wc.code[f], s), sc[f]);
#pragma unroll
        for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            acc[f][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[pl][mt], b, acc[f][mt], 0, 0, 0);
      }
    }
  };
  // Stage i: the rows of stage i + 1 go to the other LDS buffer, then the rows of stage
  // i + 1 + kAhead and the weights of stage i + kAhead are requested, then stage i is multiplied.
  Q4Chunk wb[kAhead + 1];
  load_rows(0, 0, first);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {  // in the loop's order: its first waits have to hold for both
    load_rows(i + 1, i + 1, ra);
    wb[i] = load_q4<kPolicyPlain>(w, wbytes, i, lane);
  }
  store_rows(0, 0, first);
  __syncthreads();
  auto stage = [&](int i, auto cur) {
    constexpr int c = decltype(cur)::value;
    store_rows(c + 1, (c & 1) ^ 1, ra);
    load_rows(i + 1 + kAhead, c + 1 + kAhead, ra);
    wb[(c + kAhead) % (kAhead + 1)] = load_q4<kPolicyPlain>(w, wbytes, i + kAhead, lane);  // past the run: zeros
    __builtin_amdgcn_sched_barrier(0);
    multiply(c & 1, wb[c]);
    __syncthreads();
  };
  // whole rounds of the ring without an exit between the stages: with one the compiler moves
  // values still being loaded from register to register and waits for them
  constexpr int kRound = kAhead + 1;
  int i = 0;
  for (; i + kRound <= KC; i += kRound) {
    stage(i, std::integral_constant<int, 0>{});
    stage(i + 1, std::integral_constant<int, 1>{});
    if constexpr (kRound == 4) {
      stage(i + 2, std::integral_constant<int, 2>{});
      stage(i + 3, std::integral_constant<int, 3>{});
    }
  }
  if (i < KC) stage(i, std::integral_constant<int, 0>{});
  if constexpr (kRound == 4) {
    if (i + 1 < KC) stage(i + 1, std::integral_constant<int, 1>{});
    if (i + 2 < KC) stage(i + 2, std::integral_constant<int, 2>{});
  }

  // Lane (r, g) holds rows 4 g .. 4 g + 3 of column r of each tile.  Each M-tile goes
  // through this wave's part of the LDS, so rows leave in 16-byte pieces.
  if (in) {
    constexpr int kRowBytes = kDown ? 64 * 4 : 2 * 32 * 2;  // gate/up: 32 columns, hi then lo
    constexpr int kRowPieces = kRowBytes / 16;
    constexpr int kStride = kRowBytes + 16;
    constexpr int kRowsPerStore = kWave / kRowPieces;
    char* mine = reinterpret_cast<char*>(lds) + wave * 16 * kStride;
    const int pc = lane % kRowPieces;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int mb = mt * 16;
      if (mb >= rows) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        char* row = mine + (4 * g + i) * kStride;
        if constexpr (kDown) {
          const float gate = qr.gate[min(mb + 4 * g + i, rows - 1)];
#pragma unroll
          for (int f = 0; f < 4; ++f) reinterpret_cast<float*>(row)[16 * f + r] = gate * acc[f][mt][i];
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float v = silu_mul(acc[j][mt][i], acc[2 + j][mt][i]);
            const uint16_t hi = float_to_bf16_bits(v);
            reinterpret_cast<uint16_t*>(row)[16 * j + r] = hi;
            reinterpret_cast<uint16_t*>(row)[32 + 16 * j + r] = float_to_bf16_bits(v - bf16_bits_to_float(hi));
          }
        }
      }
      wave_lds_sync();
#pragma unroll
      for (int q = 0; q < 16 / kRowsPerStore; ++q) {
        const int lr = q * kRowsPerStore + lane / kRowPieces;
        const int m = mb + lr;
        const uint4 v = *reinterpret_cast<const uint4*>(mine + lr * kStride + pc * 16);
        if (m < rows) {
          if constexpr (kDown) {
            if (quad * 64 + pc * 4 < p.H)
              reinterpret_cast<uint4*>(p.ys + static_cast<size_t>(qr.slot[m]) * p.H + quad * 64)[pc] = v;
          } else {
            const int Ipad = q4_chunks(p.I) * kQ4Chunk;
            reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.act) + (static_cast<size_t>(row0 + m) * 2 + pc / 4) * Ipad +
                                     quad * 32)[pc % 4] = v;
          }
        }
      }
      wave_lds_sync();
    }
  }
}

// Workgroup b runs on XCD b % 8.  Two neighbouring items, mostly of one expert, share an
// XCD and take the same run at the same time, so the second one's weights come from its L2;
// an item's runs follow each other there, so its rows do.
struct Q4Share {
  int item, run;
};
__device__ __forceinline__ Q4Share q4_share(int b, int runs) {
  const int slot = b / 8;
  return {(slot / 2 / runs * 8 + b % 8) * 2 + (slot & 1), slot / 2 % runs};
}
constexpr int q4_runs(int quads) { return (quads + kQ4Waves - 1) / kQ4Waves; }
long long q4_grid(int max_items, int runs) { return 16ll * ((max_items + 15) / 16) * runs; }

template <bool kDown, int kRows>
__global__ __launch_bounds__(kQ4Waves* kWave) __attribute__((amdgpu_waves_per_eu(kQ4WavesPerSimd<kDown, kRows>))) void q4_kernel(
    ForwardParams p, int quads) {
  __shared__ uint4 lds[kQ4LdsPieces<kDown, kRows>];
  __shared__ Q4Rows qr;
  const Q4Share sh = q4_share(blockIdx.x, q4_runs(quads));
  if (sh.item >= *p.n_items) return;
  const int4 d = p.items[sh.item];
  const int e = __builtin_amdgcn_readfirstlane(d.x);
  const int row0 = __builtin_amdgcn_readfirstlane(d.y);
  const int rows = __builtin_amdgcn_readfirstlane(d.z);
  if (kDown && static_cast<int>(threadIdx.x) < rows) {  // read behind the stages' barriers
    const int s = p.ent_slot[row0 + threadIdx.x];
    qr.slot[threadIdx.x] = s;
    qr.gate[threadIdx.x] = p.topk_gate[s];
  }
  if (rows <= 16) q4_rows<kDown, 1>(p, e, row0, rows, sh.run, lds, qr);
  else if (kRows == 32 || rows <= 32) q4_rows<kDown, 2>(p, e, row0, rows, sh.run, lds, qr);
  else if constexpr (kRows == 64) {
    if (rows <= 48) q4_rows<kDown, 3>(p, e, row0, rows, sh.run, lds, qr);
    else q4_rows<kDown, 4>(p, e, row0, rows, sh.run, lds, qr);
  }
}

template <bool kDown, int kRows>
hipError_t launch_q4_pass(const ForwardParams& p, hipStream_t stream) {
  const int quads = kDown ? q4_down_quads(p.H) : q4_gate_up_quads(p.I);
  const long long grid = q4_grid(q4_max_items(p.T * p.k, p.E, p.item_rows), q4_runs(quads));
  q4_kernel<kDown, kRows><<<static_cast<unsigned>(grid), kQ4Waves * kWave, 0, stream>>>(p, quads);
  return hipGetLastError();
}

template <int kRows>
hipError_t launch_q4_passes(const ForwardParams& p, hipStream_t stream) {
  const hipError_t err = launch_q4_pass<false, kRows>(p, stream);
  return err != hipSuccess ? err : launch_q4_pass<true, kRows>(p, stream);
}

// ---------------------------------------------------------------------------
// A few tokens (q4_few): latency is what counts, so two launches and no lists.  One
// routing entry per lane; the experts are the entries that no earlier one repeats, in
// that order, and the M side of the MFMA is the tokens themselves.
//   gate/up   a workgroup per (expert, quad), K shared by its waves; for every token
//             gate * silu(g) * u (zeros where the token is not routed there) in two planes
//   down      two workgroups per 16 columns over all experts: the chunks of all experts'
//             K are dealt to their waves, and the sum over the experts happens in the MFMA's
//             accumulators (zeros where a token is not routed: a weight that is not finite enters
//             every token's sum) and then over the waves, in wave order; each adds its half onto the
//             zeros that gate/up left in out (two additions onto zero commute: deterministic)
// ---------------------------------------------------------------------------
struct FewEntries {
  int e;           // this lane's expert, -1: none, out of range or repeated within its row
  uint64_t heads;  // lanes that hold an expert for the first time
};
__device__ __forceinline__ FewEntries few_entries(const ForwardParams& p) {
  const int lane = lane_id(), n = p.T * p.k;
  const int v = lane < n ? p.topk_idx[lane] : -1;
  const bool in = v >= 0 && v < p.E;
  uint32_t same = 0;  // entries with this lane's expert
  for (int i = 0; i < n; ++i) same |= lane_value(v, i) == v ? 1u << i : 0u;
  const uint32_t before = same & ((1u << (lane & 31)) - 1u);
  const int row0 = lane / p.k * p.k;  // this row's first entry
  const bool again = (before >> (row0 & 31)) != 0;
  return {in && !again ? v : -1, __ballot(in && before == 0)};
}
__device__ __forceinline__ int nth_lane(uint64_t m, int n) {
  for (int i = 0; i < n; ++i) m &= m - 1;
  return __builtin_ctzll(m);
}

constexpr int kFewUpWaves = 8, kFewDownWaves = 16;

__global__ __launch_bounds__(kFewUpWaves * kWave) __attribute__((amdgpu_waves_per_eu(4))) void q4_few_up_kernel(ForwardParams p, int quads) {
  __shared__ floatx4 s_sum[kFewUpWaves][4][kWave];
  __shared__ float s_gate[16];
  const int wave = wave_id(), lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int item = blockIdx.x / quads, quad = blockIdx.x % quads;
  const int K = p.H, KC = q4_chunks(K);
  const uint32_t xbytes = static_cast<uint32_t>(p.T) * p.H * 2;
  constexpr int kAhead = 2;  // chunks of this wave in flight behind the one multiplied
  uint4 xb[kAhead][4];
  auto load_x = [&](int kc, uint4 (&xv)[4]) {
    const int col = kc * kQ4Chunk + g * kQ4Group;
    const uint32_t at = col < K && r < p.T ? (static_cast<uint32_t>(r) * K + col) * 2 : ~63u;
#pragma unroll
    for (int s = 0; s < 4; ++s) xv[s] = load_piece(p.hidden, xbytes, (at & ~63u) | (16 * s));
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load_x(wave + i * kFewUpWaves, xb[i]);  // needs no expert
  const FewEntries en = few_entries(p);
  {
    float4* out = reinterpret_cast<float4*>(p.out);
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.T * p.H / 4; i += gridDim.x * blockDim.x)
      out[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (item >= popc64(en.heads)) return;
  const int e = lane_value(en.e, nth_lane(en.heads, item));
  const size_t run_bytes = q4_quad_run(K);
  const uint4* w = uniform_ptr(reinterpret_cast<const uint4*>(
      static_cast<const char*>(p.w_gate_up) + (static_cast<size_t>(e) * quads + quad) * run_bytes));
  const int wbytes = static_cast<int>(run_bytes);
  floatx4 acc[4] = {};
  Q4Chunk wb[kAhead];
  auto multiply = [&](const Q4Chunk& wv, const uint4 (&xv)[4]) {
#pragma unroll
    for (int f = 0; f < 4; ++f) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
        acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[s]),
                                                         expand_q4(word(wv.code[f], s), scale_of(wv.scale, f)), acc[f],
                                                         0, 0, 0);
    }
  };
  // chunks wave, wave + waves, ...; past the last one zeros
#pragma unroll
  for (int i = 0; i < kAhead; ++i) wb[i] = load_q4<kPolicyStream>(w, wbytes, wave + i * kFewUpWaves, lane);
  for (int kc = wave; kc < KC; kc += kAhead * kFewUpWaves) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      multiply(wb[i], xb[i]);
      const int next = kc + (i + kAhead) * kFewUpWaves;
      if (kc + kAhead * kFewUpWaves >= KC) continue;  // no round follows
      wb[i] = load_q4<kPolicyStream>(w, wbytes, next, lane);
      load_x(next, xb[i]);
    }
  }
#pragma unroll
  for (int f = 0; f < 4; ++f) s_sum[wave][f][lane] = acc[f];
  if (wave == 0) {
    // the tokens' gates for this expert
    if (en.e == e) s_gate[lane / p.k] = p.topk_gate[lane];
  }
  __syncthreads();
  if (wave > 1) return;
  // wave j: 16 columns, gate tile j and up tile 2 + j
  floatx4 z = {}, u = {};
#pragma unroll
  for (int c = 0; c < kFewUpWaves; ++c) {
    const floatx4 a = s_sum[c][wave][lane], b = s_sum[c][2 + wave][lane];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      z[q] += a[q];
      u[q] += b[q];
    }
  }
  uint64_t routed = __ballot(en.e == e);  // entries; a bit per token below
  const int Ipad = q4_chunks(p.I) * kQ4Chunk;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = 4 * g + i;
    if (t >= p.T) continue;
    const bool here = ((routed >> (t * p.k)) & ((1ull << p.k) - 1)) != 0;
    const float v = here ? s_gate[t] * silu_mul(z[i], u[i]) : 0.f;
    const uint16_t hi = float_to_bf16_bits(v);
    uint16_t* out = static_cast<uint16_t*>(p.act) + (static_cast<size_t>(item) * p.T + t) * 2 * Ipad + quad * 32 + 16 * wave + r;
    out[0] = hi;
    out[Ipad] = float_to_bf16_bits(v - bf16_bits_to_float(hi));
  }
}

__global__ __launch_bounds__(kFewDownWaves * kWave) __attribute__((amdgpu_waves_per_eu(8))) void q4_few_down_kernel(ForwardParams p, int quads) {
  __shared__ floatx4 s_sum[kFewDownWaves][kWave];
  const int wave = wave_id(), lane = lane_id(), r = lane & 15, g = lane >> 4;
  const FewEntries en = few_entries(p);
  const int n_items = popc64(en.heads);
  const int half = blockIdx.x % 2, f = blockIdx.x / 2 % 4, quad = blockIdx.x / 8;
  const int KC = q4_chunks(p.I), pairs = n_items * KC;
  const int first = half ? (pairs + 1) / 2 : 0, last = half ? pairs : (pairs + 1) / 2;
  const size_t run_bytes = q4_quad_run(p.I);
  const uint32_t plane = KC * (kQ4Chunk * 2);  // bytes
  const uint32_t abytes = static_cast<uint32_t>(n_items) * p.T * 2 * plane;
  floatx4 acc = {};
  // This half's (expert, chunk) pairs wave, wave + waves, ..., the weights of the next one requested
  // before this one is multiplied; past the last one zeros.  One ahead: at most 64 registers keep
  // two workgroups on a CU.
  struct Pair {
    uint4 codes;
    uint32_t scales;
  };
  auto load_pair = [&](int q) {
    const int at = min(q, last - 1), item = at / KC, kc = at - item * KC;
    const int e = lane_value(en.e, nth_lane(en.heads, item));
    const uint4* base = uniform_ptr(reinterpret_cast<const uint4*>(
        static_cast<const char*>(p.w_down) + (static_cast<size_t>(e) * quads + quad) * run_bytes +
        static_cast<size_t>(kc) * kQ4QuadBytes));
    const int bytes = q < last ? kQ4QuadBytes : 0;
    return Pair{load_weight<kPolicyStream>(base, bytes, f * kWave + lane), load_scales(base, bytes, 4096 + lane * 4)};
  };
  auto turn = [&](int q, const Pair& w, Pair& next) {
    const int item = q / KC, kc = q - item * KC;
    const bool in = q < last && kc * kQ4Chunk + g * kQ4Group < p.I && r < p.T;
    const uint32_t at = in ? (static_cast<uint32_t>(item) * p.T + r) * 2 * plane + (kc * kQ4Chunk + g * kQ4Group) * 2 : ~63u;
    const uint32_t at_lo = in ? at + plane : at;
    uint4 hi[4], lo[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      hi[s] = load_piece(p.act, abytes, (at & ~63u) | (16 * s));
      lo[s] = load_piece(p.act, abytes, (at_lo & ~63u) | (16 * s));
    }
    next = load_pair(q + kFewDownWaves);
    __builtin_amdgcn_sched_barrier(0);
    const float scale = scale_of(w.scales, f);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bf16x8 b = expand_q4(word(w.codes, s), scale);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi[s]), b, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo[s]), b, acc, 0, 0, 0);
    }
  };
  if (first + wave < last) {
    Pair even = load_pair(first + wave), odd;
    for (int q = first + wave;; q += 2 * kFewDownWaves) {
      turn(q, even, odd);
      if (q + kFewDownWaves >= last) break;
      turn(q + kFewDownWaves, odd, even);
      if (q + 2 * kFewDownWaves >= last) break;
    }
  }
  s_sum[wave][lane] = acc;
  __syncthreads();
  // wave i: row i of every lane's four
  const int t = 4 * g + wave, col = quad * 64 + f * 16 + r;
  if (wave > 3 || t >= p.T || col >= p.H) return;
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < kFewDownWaves; ++c) sum += reinterpret_cast<const float*>(&s_sum[c][lane])[wave];
  atomicAdd(p.out + static_cast<size_t>(t) * p.H + col, sum);
}

hipError_t launch_q4_few(const ForwardParams& p, hipStream_t stream) {
  const int slots = p.T * p.k, items = p.E < slots ? p.E : slots;
  const int up = q4_gate_up_quads(p.I), down = q4_down_quads(p.H);
  q4_few_up_kernel<<<items * up, kFewUpWaves * kWave, 0, stream>>>(p, up);
  q4_few_down_kernel<<<down * 8, kFewDownWaves * kWave, 0, stream>>>(p, down);
  return hipGetLastError();
}

template <int KMAX>
hipError_t launch_q4_dispatch(const ForwardParams& p, hipStream_t stream) {
  // (512 tokens top-8: 1024 threads 89 us for the whole forward, 256 threads 92; 64 tokens: 73.7, 72.4)
  if (p.T <= 256) q4_dispatch_kernel<KMAX, 256><<<p.E, 256, 0, stream>>>(p);
  else q4_dispatch_kernel<KMAX, 1024><<<p.E, 1024, 0, stream>>>(p);
  return hipGetLastError();
}

template <int KMAX>
hipError_t launch_q4_combine(const ForwardParams& p, hipStream_t stream) {
  const int hblocks = (p.H / 4 + 255) / 256, most = max_workgroups(256) / hblocks;  // tokens of a launch
  hipError_t err = hipSuccess;
  for (int t0 = 0; t0 < p.T && err == hipSuccess; t0 += most) {
    q4_combine_kernel<KMAX><<<hblocks * (p.T - t0 < most ? p.T - t0 : most), 256, 0, stream>>>(p, hblocks, t0);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace

size_t packed_gate_up_q4_bytes(int E, int I, int H) {
  return static_cast<size_t>(E) * q4_gate_up_quads(I) * q4_quad_run(H);
}

size_t packed_down_q4_bytes(int E, int H, int I) { return static_cast<size_t>(E) * q4_down_quads(H) * q4_quad_run(I); }

static int stride_grid(size_t threads) {
  const size_t want = (threads + 255) / 256;
  return static_cast<int>(want < 65536 ? want : 65536);
}

hipError_t launch_pack_gate_up_q4(const uint8_t* gate, const uint8_t* gate_scale, const uint8_t* up,
                                  const uint8_t* up_scale, int E, int I, int H, void* dst, hipStream_t stream) {
  const int quads = q4_gate_up_quads(I);
  const size_t total = static_cast<size_t>(E) * quads * q4_chunks(H) * kWave;
  pack_q4_kernel<true><<<stride_grid(total), 256, 0, stream>>>(gate, gate_scale, up, up_scale,
                                                               static_cast<uint8_t*>(dst), total, quads, I, H);
  return hipGetLastError();
}

hipError_t launch_pack_down_q4(const uint8_t* down, const uint8_t* down_scale, int E, int H, int I, void* dst,
                               hipStream_t stream) {
  const int quads = q4_down_quads(H);
  const size_t total = static_cast<size_t>(E) * quads * q4_chunks(I) * kWave;
  pack_q4_kernel<false><<<stride_grid(total), 256, 0, stream>>>(down, down_scale, nullptr, nullptr,
                                                                static_cast<uint8_t*>(dst), total, quads, H, I);
  return hipGetLastError();
}

hipError_t launch_quantize_q4(const void* w, int is_bf16, size_t groups, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream) {
  if (is_bf16)
    quantize_q4_kernel<true><<<stride_grid(groups), 256, 0, stream>>>(w, groups, reinterpret_cast<uint4*>(codes), scales);
  else
    quantize_q4_kernel<false><<<stride_grid(groups), 256, 0, stream>>>(w, groups, reinterpret_cast<uint4*>(codes), scales);
  return hipGetLastError();
}

// Activation rows: one per routing entry; a few tokens: one per expert and token.  (At least kQ4FewRows:
// a workspace serves smaller blocks, too.)
static size_t q4_act_rows(int T, int k) {
  const size_t slots = static_cast<size_t>(T) * k;
  return slots > kQ4FewRows ? slots : kQ4FewRows;
}

// workspace: [n_items], CSR slot ids, activations (two planes,
// rows padded to whole chunks), items, per-slot output rows
static size_t q4_carve(char* c, int T, int H, int I, int E, int k, ForwardParams* p) {
  const char* start = c;
  const size_t slots = static_cast<size_t>(T) * k;
  if (p) p->n_items = reinterpret_cast<int32_t*>(c);
  c += align256(sizeof(int32_t));
  if (p) p->ent_slot = reinterpret_cast<int32_t*>(c);
  c += align256(sizeof(int32_t) * slots);
  if (p) p->act = c;
  c += align256(q4_act_rows(T, k) * 2 * q4_chunks(I) * kQ4Chunk * 2);
  if (p) p->items = reinterpret_cast<int4*>(c);
  c += align256(static_cast<size_t>(q4_max_items(static_cast<int>(slots), E, kQ4LeastLimit)) * sizeof(int4));
  if (p) p->ys = reinterpret_cast<float*>(c);
  c += align256(slots * H * sizeof(float));
  return c - start;
}

size_t forward_q4_workspace_bytes(int T, int H, int I, int E, int k) { return q4_carve(nullptr, T, H, I, E, k, nullptr); }

// The products' launches take the block (far beyond one device's memory they do not).
bool forward_q4_grids_fit(int T, int H, int I, int E, int k) {
  const int items = q4_max_items(T * k, E, q4_item_limit(T, k)), most = max_workgroups(kQ4Waves * kWave);
  return q4_grid(items, q4_runs(q4_gate_up_quads(I))) <= most && q4_grid(items, q4_runs(q4_down_quads(H))) <= most;
}

void forward_q4_carve(void* ws, ForwardParams& p) { q4_carve(static_cast<char*>(ws), p.T, p.H, p.I, p.E, p.k, &p); }

hipError_t launch_forward_q4(ForwardParams p, hipStream_t stream) {
  if (q4_few(p.T, p.k)) return launch_q4_few(p, stream);
  p.item_rows = q4_item_limit(p.T, p.k);
  hipError_t err = p.k <= 8 ? launch_q4_dispatch<8>(p, stream) : launch_q4_dispatch<kMaxTopK>(p, stream);
  if (err != hipSuccess) return err;
  err = p.item_rows == 32 ? launch_q4_passes<32>(p, stream) : launch_q4_passes<64>(p, stream);
  if (err != hipSuccess) return err;
  return p.k <= 8 ? launch_q4_combine<8>(p, stream) : launch_q4_combine<kMaxTopK>(p, stream);
}

}  // namespace amoe
