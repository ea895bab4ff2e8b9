// The grouped SwiGLU expert FFN with weights in 4 bits: a weight is an e2m1 code
// (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times a power of two shared by
// 32 columns of its row, W = code 2^(s - 127).
//   out_t = sum_j g_{t,j} W_d (silu(W_g x_t) * W_u x_t)
//
// Both factors of the gate and up products are exact in bf16 (a code has 2
// significant bits, its scale is a power of two), so they run on the bf16 MFMA
// with the weights expanded in registers.  The activation goes to the down
// product as two bf16 planes, hi = bf16(a) and lo = bf16(a - hi), 16 bits of it
// in all, which costs a second MFMA but no weight traffic: with hi alone every output
// would carry up to 2^-8 from that one rounding, more than from all else together.
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
template <int KMAX, int kThreads>
__global__ __launch_bounds__(kThreads) void q4_dispatch_kernel(ForwardParams p) {
  __shared__ int s_cnt[kMaxExperts];
  __shared__ int s_wave[kThreads / kWave];
  __shared__ int s_off, s_item;
  const int tid = threadIdx.x, E = p.E, k = p.k, T = p.T, e = blockIdx.x;
  for (int i = tid; i < E; i += kThreads) s_cnt[i] = 0;
  __syncthreads();
  for (int t = tid; t < T; t += kThreads) {
    int ev[KMAX];
    const uint32_t valid = load_route_row<KMAX>(p.topk_idx + static_cast<size_t>(t) * k, k, E, ev);
#pragma unroll
    for (int j = 0; j < KMAX; ++j)
      if (valid & (1u << j)) atomicAdd(&s_cnt[ev[j]], 1);
  }
  __syncthreads();
  if (tid < kWave) {
    int off = 0, items = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int c = e0 + tid < E ? s_cnt[e0 + tid] : 0;
      const int n = q4_items(c);
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
  const int rows = q4_item_rows(count);
  for (int m = tid; m < q4_items(count); m += kThreads)
    p.items[s_item + m] = make_int4(e, off + rows * m, min(rows, count - rows * m), 0);
  int seen = 0;
  for (int t0 = 0; seen < count; t0 += kThreads) {  // ends at T at the latest: `count` rows hold e
    const int t = t0 + tid;
    int slot = -1;
    if (t < T) {
      int ev[KMAX];
      load_route_row<KMAX>(p.topk_idx + static_cast<size_t>(t) * k, k, E, ev);
#pragma unroll
      for (int j = KMAX - 1; j >= 0; --j) slot = ev[j] == e ? t * k + j : slot;
    }
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

// out[t] = sum of the token's slot rows, in slot order
template <int KMAX>
__global__ __launch_bounds__(256) void q4_combine_kernel(ForwardParams p, int hblocks) {
  const int t = blockIdx.x / hblocks;
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

template <int kPolicy>
__device__ __forceinline__ Q4Chunk load_q4(const uint4* base, int bytes, int kc, int lane) {
  Q4Chunk c;
#pragma unroll
  for (int f = 0; f < 4; ++f)
    c.code[f] = load_weight<kPolicy>(base, bytes, kc * (kQ4QuadBytes / 16) + f * kWave + lane);
  __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint4*>(base), static_cast<short>(0), bytes, kBufferWord3);
  c.scale = __builtin_amdgcn_raw_buffer_load_b32(r, kc * kQ4QuadBytes + 4096 + lane * 4, 0, kPolicy);
  return c;
}

// eight codes (low nibble first) times the scale, in bf16: exact for scale bytes 2 .. 252
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
// Grouped products.  A workgroup of 4 waves takes one item (expert, up to
// kQ4ItemRows of its rows) and 4 / KS quads; KS waves share a quad, each over
// every KS-th chunk of K.  Weights stream straight into the registers of the one
// wave that uses them; the item's rows are staged in LDS, KS chunks a stage, for
// the four waves.
// ---------------------------------------------------------------------------
// LDS pieces of 16 B: two stages of 64 rows; gate/up 32 KiB, four workgroups' worth per CU, down (two planes) 64
template <bool kDown>
constexpr int kQ4LdsPieces = kDown ? 4096 : 2048;

struct Q4Rows {
  int slot[kQ4ItemRows];
  float gate[kQ4ItemRows];
};

// most M-tiles of a pass: rows of KS chunks and their planes in half of the LDS
template <bool kDown, int KS>
constexpr int kQ4MaxTiles = 4 / KS;

template <bool kDown, int MT, int KS>
__device__ __forceinline__ void q4_rows(const ForwardParams& p, int e, int row0, int rows, int m0, int run, uint4* lds,
                                        const Q4Rows& qr) {
  constexpr int kPlanes = kDown ? 2 : 1;
  constexpr int kLoads = KS * kPlanes * MT;  // 16-byte row pieces per thread and stage
  constexpr int kBuf = kLoads * 256;
  static_assert(2 * kBuf <= kQ4LdsPieces<kDown>, "two stages fit");
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // keeps address arithmetic of one tile count out of the others
  const int wave = wave_id(), lane = lane_id();
  const int r = lane & 15, g = lane >> 4;
  const int ks = wave % KS;
  const int K = kDown ? p.I : p.H;
  const int KC = q4_chunks(K);
  const int quads = kDown ? q4_down_quads(p.H) : q4_gate_up_quads(p.I);
  const int quad = run * (4 / KS) + wave / KS;
  const bool in = quad < quads;
  const size_t run_bytes = q4_quad_run(K);
  const uint4* w = uniform_ptr(reinterpret_cast<const uint4*>(static_cast<const char*>(kDown ? p.w_down : p.w_gate_up) +
                                                              (static_cast<size_t>(e) * quads + (in ? quad : 0)) * run_bytes));
  const int wbytes = in ? static_cast<int>(run_bytes) : 0;
  // thread tid loads piece tid % 16 (8 columns) of rows tid / 16 + 16 mt
  const int piece = tid & 15, srow = tid >> 4;
  const int plane_pieces = KC * (kQ4Chunk / 8);
  const uint4* xbase = static_cast<const uint4*>(kDown ? p.act : p.hidden);
  uint32_t xrow[MT];  // pieces: fewer than 2^32 (checked by the caller)
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = m0 + mt * 16 + srow;
    const int row = row0 + (m < rows ? m : 0);  // rows past the item's last read its first; their outputs are dropped
    xrow[mt] = kDown ? static_cast<uint32_t>(row) * (2 * plane_pieces)
                     : static_cast<uint32_t>(p.ent_slot[row] / p.k) * (p.H / 8);
  }
  const int nst = (KC + KS - 1) / KS;
  uint4 ra[KS][kPlanes][MT];
  auto load_rows = [&](int st) {
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      int at = (st * KS + c) * 16 + piece;
      at = at * 8 < K ? at : piece * 8 < K ? piece : 0;  // past K: any piece of the row, see store_rows
#pragma unroll
      for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ra[c][pl][mt] = xbase[xrow[mt] + (pl * plane_pieces + at)];
    }
  };
  // row `srow`'s piece sits at piece ^ row, so the 16 pieces of a row, and the 16
  // rows that a fragment reads at one piece, fall into different banks
  auto store_rows = [&](int st, int buf) {
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      const bool valid = ((st * KS + c) * 16 + piece) * 8 < K;
#pragma unroll
      for (int pl = 0; pl < kPlanes; ++pl)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          lds[buf * kBuf + (((c * kPlanes + pl) * MT + mt) * 16 + srow) * 16 + (piece ^ srow)] =
              valid ? ra[c][pl][mt] : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  floatx4 acc[4][MT];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[f][mt] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int buf, const Q4Chunk& wc) {
    const uint4* x0 = lds + buf * kBuf + ks * kPlanes * MT * 256 + r * 16;
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
  // Stage i: the rows of stage i + 1, loaded one stage earlier, go to the other LDS
  // buffer, then the rows of stage i + 2 and the weights of stage i + 1 are
  // requested, then stage i is multiplied.
  Q4Chunk wb[2];
  load_rows(0);
  wb[0] = load_q4<kPolicyPlain>(w, wbytes, ks, lane);
  store_rows(0, 0);
  load_rows(1);
  __syncthreads();
  auto stage = [&](int i, auto cur) {
    constexpr int c = decltype(cur)::value;
    store_rows(i + 1, c ^ 1);
    load_rows(i + 2);
    wb[c ^ 1] = load_q4<kPolicyPlain>(w, wbytes, (i + 1) * KS + ks, lane);  // past the run: zeros
    __builtin_amdgcn_sched_barrier(0);
    multiply(c, wb[c]);
    __syncthreads();
  };
  for (int i = 0;;) {
    stage(i, std::integral_constant<int, 0>{});
    if (++i == nst) break;
    stage(i, std::integral_constant<int, 1>{});
    if (++i == nst) break;
  }
  if constexpr (KS > 1) {
    static_assert((KS - 1) * (4 / KS) * 4 * MT * kWave <= kQ4LdsPieces<kDown>, "the other waves' sums fit");
    floatx4* red = reinterpret_cast<floatx4*>(lds) + (wave / KS) * (KS - 1) * 4 * MT * kWave + lane;
    if (ks > 0) {
#pragma unroll
      for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) red[((ks - 1) * 4 * MT + f * MT + mt) * kWave] = acc[f][mt];
    }
    __syncthreads();
    if (ks == 0) {
#pragma unroll
      for (int c = 0; c < KS - 1; ++c)
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const floatx4 v = red[(c * 4 * MT + f * MT + mt) * kWave];
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[f][mt][q] += v[q];
          }
    }
    __syncthreads();
  }

  // Lane (r, g) holds rows 4 g .. 4 g + 3 of column r of each tile.  Each M-tile goes
  // through this wave's part of the LDS, so rows leave in 16-byte pieces.
  if (ks == 0 && in) {
    constexpr int kRowBytes = kDown ? 64 * 4 : 2 * 32 * 2;  // gate/up: 32 columns, hi then lo
    constexpr int kRowPieces = kRowBytes / 16;
    constexpr int kStride = kRowBytes + 16;
    constexpr int kRowsPerStore = kWave / kRowPieces;
    char* mine = reinterpret_cast<char*>(lds) + (wave / KS) * 16 * kStride;
    const int pc = lane % kRowPieces;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int mb = m0 + mt * 16;
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
template <bool kDown, int KS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kDown ? 2 : 3))) void q4_kernel(ForwardParams p,
                                                                                                    int runs) {
  __shared__ uint4 lds[kQ4LdsPieces<kDown>];
  __shared__ Q4Rows qr;
  const int n_items = *p.n_items;
  const int slot = blockIdx.x / 8;
  const int item = (slot / 2 / runs * 8 + blockIdx.x % 8) * 2 + (slot & 1);
  if (item >= n_items) return;
  const int run = slot / 2 % runs;
  const int4 d = p.items[item];
  const int e = __builtin_amdgcn_readfirstlane(d.x);
  const int row0 = __builtin_amdgcn_readfirstlane(d.y);
  const int rows = __builtin_amdgcn_readfirstlane(d.z);
  if (kDown && static_cast<int>(threadIdx.x) < rows) {  // read behind the stages' barriers
    const int s = p.ent_slot[row0 + threadIdx.x];
    qr.slot[threadIdx.x] = s;
    qr.gate[threadIdx.x] = p.topk_gate[s];
  }
  constexpr int kMax = kQ4MaxTiles<kDown, KS>;
  for (int m0 = 0; m0 < rows; m0 += 16 * kMax) {
    const int mt = (rows - m0 + 15) / 16;
    if (m0 > 0) __syncthreads();  // the rows before have left the LDS
    if (mt == 1) q4_rows<kDown, 1, KS>(p, e, row0, rows, m0, run, lds, qr);
    else if (kMax <= 2 || mt == 2) q4_rows<kDown, (kMax < 2 ? kMax : 2), KS>(p, e, row0, rows, m0, run, lds, qr);
    else if (kMax == 3 || mt == 3) q4_rows<kDown, (kMax < 3 ? kMax : 3), KS>(p, e, row0, rows, m0, run, lds, qr);
    else q4_rows<kDown, kMax, KS>(p, e, row0, rows, m0, run, lds, qr);
  }
}

template <bool kDown>
hipError_t launch_q4_pass(const ForwardParams& p, int max_items, hipStream_t stream) {
  const int quads = kDown ? q4_down_quads(p.H) : q4_gate_up_quads(p.I);
  const int runs = (quads + 3) / 4;
  const long long grid = 16ll * ((max_items + 15) / 16) * runs;
  if (grid > 0x7fffffffll) return hipErrorInvalidValue;  // far beyond one device's memory
  q4_kernel<kDown, 1><<<static_cast<unsigned>(grid), 256, 0, stream>>>(p, runs);
  return hipGetLastError();
}

template <int KMAX>
hipError_t launch_q4_dispatch(const ForwardParams& p, hipStream_t stream) {
  if (p.T <= 256) q4_dispatch_kernel<KMAX, 256><<<p.E, 256, 0, stream>>>(p);
  else q4_dispatch_kernel<KMAX, 1024><<<p.E, 1024, 0, stream>>>(p);
  return hipGetLastError();
}

template <int KMAX>
hipError_t launch_q4_combine(const ForwardParams& p, hipStream_t stream) {
  const int hblocks = (p.H / 4 + 255) / 256;
  q4_combine_kernel<KMAX><<<static_cast<unsigned>(hblocks) * static_cast<unsigned>(p.T), 256, 0, stream>>>(p, hblocks);
  return hipGetLastError();
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
  c += align256(slots * 2 * q4_chunks(I) * kQ4Chunk * 2);
  if (p) p->items = reinterpret_cast<int4*>(c);
  c += align256(static_cast<size_t>(q4_max_items(static_cast<int>(slots), E)) * sizeof(int4));
  if (p) p->ys = reinterpret_cast<float*>(c);
  c += align256(slots * H * sizeof(float));
  return c - start;
}

size_t forward_q4_workspace_bytes(int T, int H, int I, int E, int k) { return q4_carve(nullptr, T, H, I, E, k, nullptr); }

void forward_q4_carve(void* ws, ForwardParams& p) { q4_carve(static_cast<char*>(ws), p.T, p.H, p.I, p.E, p.k, &p); }

hipError_t launch_forward_q4(const ForwardParams& p, hipStream_t stream) {
  hipError_t err = p.k <= 8 ? launch_q4_dispatch<8>(p, stream) : launch_q4_dispatch<kMaxTopK>(p, stream);
  if (err != hipSuccess) return err;
  const int max_items = q4_max_items(p.T * p.k, p.E);
  err = launch_q4_pass<false>(p, max_items, stream);
  if (err != hipSuccess) return err;
  err = launch_q4_pass<true>(p, max_items, stream);
  if (err != hipSuccess) return err;
  return p.k <= 8 ? launch_q4_combine<8>(p, stream) : launch_q4_combine<kMaxTopK>(p, stream);
}

}  // namespace amoe
