// Sizes shared by the 4-bit expert kernels and the host code around them.
#pragma once

#include <cstddef>

namespace amoe {

constexpr int kQ4Group = 32;    // K columns per scale
constexpr int kQ4Chunk = 128;   // K columns of a weight fragment (16 rows): 64 lanes x 16 B of codes
constexpr int kQ4QuadBytes = 4 * 1024 + 256;  // four fragments of a chunk and their scales
constexpr int kQ4ItemRows = 64;

constexpr int q4_chunks(int K) { return (K + kQ4Chunk - 1) / kQ4Chunk; }
// quads of 16-row tiles: gate 2p, gate 2p + 1, up 2p, up 2p + 1; four tiles of the down projection
constexpr int q4_gate_up_quads(int I) { return (I + 31) / 32; }
constexpr int q4_down_quads(int H) { return (H + 63) / 64; }
constexpr size_t q4_quad_run(int K) { return static_cast<size_t>(q4_chunks(K)) * kQ4QuadBytes; }

// An expert's `count` rows in equal runs of whole M-tiles, at most kQ4ItemRows each.
constexpr int q4_item_rows(int count) {
  const int items = (count + kQ4ItemRows - 1) / kQ4ItemRows;
  return items > 0 ? 16 * (((count + 15) / 16 + items - 1) / items) : 16;
}
constexpr int q4_items(int count) { return (count + q4_item_rows(count) - 1) / q4_item_rows(count); }

// most items of a block of `slots` routing entries: one per active expert and one
// more per full item
constexpr int q4_max_items(int slots, int E) { return (E < slots ? E : slots) + slots / kQ4ItemRows; }

}  // namespace amoe
