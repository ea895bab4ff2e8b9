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

// Most rows of an item.  Blocks of up to kQ4SmallT tokens, with few items for the device's
// CUs, take items of 32 rows and workgroups of two waves (64 tokens in 26 experts, H = 4096,
// I = 1536: 312 workgroups of four waves on 256 CUs took as long as 512).
constexpr int kQ4SmallT = 256;
constexpr int q4_item_limit(int T) { return T <= kQ4SmallT ? 32 : 64; }

// An expert's `count` rows in equal runs of whole M-tiles, at most `limit` each.
constexpr int q4_item_rows(int count, int limit) {
  const int items = (count + limit - 1) / limit;
  return items > 0 ? 16 * (((count + 15) / 16 + items - 1) / items) : 16;
}
constexpr int q4_items(int count, int limit) {
  return (count + q4_item_rows(count, limit) - 1) / q4_item_rows(count, limit);
}

// Blocks of up to this many routing entries (and 16 tokens) take two launches without a
// dispatch: every workgroup finds its expert in the entries itself.
constexpr int kQ4FewSlots = 32;
constexpr int kQ4FewT = 16;
constexpr bool q4_few(int T, int k) { return T <= kQ4FewT && T * k <= kQ4FewSlots; }

// most items of a block of `slots` routing entries: one per active expert and one
// more per full item
constexpr int q4_max_items(int slots, int E, int limit) { return (E < slots ? E : slots) + slots / limit; }

}  // namespace amoe
