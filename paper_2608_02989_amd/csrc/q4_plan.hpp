// Sizes shared by the 4-bit expert kernels and the host code around them.
#pragma once

#include <cstddef>

namespace amoe {

constexpr int kQ4Group = 32;    // K columns per scale
constexpr int kQ4Chunk = 128;   // K columns of a weight fragment (16 rows): 64 lanes x 16 B of codes
constexpr int kQ4QuadBytes = 4 * 1024 + 256;  // four fragments of a chunk and their scales

constexpr int q4_chunks(int K) { return (K + kQ4Chunk - 1) / kQ4Chunk; }
// quads of 16-row tiles: gate 2p, gate 2p + 1, up 2p, up 2p + 1; four tiles of the down projection
constexpr int q4_gate_up_quads(int I) { return (I + 31) / 32; }
constexpr int q4_down_quads(int H) { return (H + 63) / 64; }
constexpr size_t q4_quad_run(int K) { return static_cast<size_t>(q4_chunks(K)) * kQ4QuadBytes; }

// Most rows of an item: fewer for smaller blocks, whose items are few for 256 CUs, while an expert's
// second item reads its weights again, mostly from L2.  H = 2048, I = 768, top-8 in us with 32 /
// 48 / 64 rows: 320 tokens in 40 experts 63 / 67 / 71, 512 in 64 88 / 84 / 93, 1024 in 128 157 /
// 154 / 163, 1920 in 128 245 / 249 / 239.
constexpr int q4_item_limit(int T, int k) { return T * k <= 2560 ? 32 : T * k <= 8192 ? 48 : 64; }
constexpr int kQ4LeastLimit = 32;

// An expert's `count` rows in equal runs of whole M-tiles, at most `limit` each.
constexpr int q4_item_rows(int count, int limit) {
  const int items = (count + limit - 1) / limit;
  return items > 0 ? 16 * (((count + 15) / 16 + items - 1) / items) : 16;
}
constexpr int q4_items(int count, int limit) {
  return (count + q4_item_rows(count, limit) - 1) / q4_item_rows(count, limit);
}

// Blocks of up to kQ4FewSlots routing entries take two launches without a dispatch: every
// workgroup finds its expert in the entries itself.  The second one reads a row of activations
// per expert and token, kQ4FewRows at most.  128 experts, H = 2048, I = 768, in us, so and by
// dispatch: 1 token top-8 9.9 / 24.7, 2 top-8 16.5 / 25.5, 3 top-8 24.6 / 31, 4 top-8 32 / 29,
// 16 top-1 25 / 23; H = 4096, I = 1536: 1 top-8 26 / 43, 2 top-8 47 / 44.
constexpr int kQ4FewSlots = 32;
constexpr int kQ4FewRows = 96;
constexpr bool q4_few(int T, int k) { return T <= 16 && T * k <= kQ4FewSlots && T * T * k <= kQ4FewRows; }

// most items of a block of `slots` routing entries: one per active expert and one
// more per full item
constexpr int q4_max_items(int slots, int E, int limit) { return (E < slots ? E : slots) + slots / limit; }

}  // namespace amoe
