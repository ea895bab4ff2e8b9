// The accepted path of each draft tree: from the root on, a node is accepted
// when its parent is and its token is the target's choice at the parent; of
// siblings with that token the first counts, so the accepted nodes are one path.
//
// A node's place is found by doubling: `up` first holds the parent of a node whose
// token fits, the root for the root and a dead end for all others; after i rounds
// up = up[up] it holds the ancestor 2^i steps above, so ceil(log2 n) rounds tell
// whether a node hangs on the root, also for a chain of 1024 nodes (1023
// steps one after the other otherwise).  Nodes come behind their parents, so
// an accepted node's place is the count of accepted nodes before it.
//
// Bound by latency: one workgroup per tree, three words a node (one tree of 64 nodes 2.4 us,
// 32 of 60 3.6 us).
#include "common.hpp"
#include "launch.hpp"

namespace amoe {

namespace {

__global__ __launch_bounds__(kMaxTreeNodes) void accept_kernel(AcceptParams p, TreeOffsets offs) {
  __shared__ int s_target[kMaxTreeNodes];
  __shared__ int s_first[kMaxTreeNodes];   // first child with the target's token
  __shared__ int s_up[kMaxTreeNodes + 1];  // entry n: the dead end
  __shared__ int s_cnt[kMaxTreeNodes / kWave];
  const int b = blockIdx.x, t = threadIdx.x;
  const int first = offs.o[b], n = offs.o[b + 1] - first;
  int32_t* path = p.path + static_cast<size_t>(b) * p.path_len;
  int par = -1, tok = 0;
  if (t < n) {
    const int global = p.parent[first + t];
    par = global >= first ? global - first : -1;
    tok = p.token[first + t];
    s_target[t] = p.target[first + t];
    s_first[t] = kMaxTreeNodes;
  }
  if (t == 0) s_up[n] = n;
  __syncthreads();
  // a parent outside the tree or behind its child links nothing
  const bool fits = t > 0 && t < n && par >= 0 && par < t && tok == s_target[par];
  if (fits) atomicMin(&s_first[par], t);
  __syncthreads();
  int up = t == 0 ? 0 : fits && s_first[par] == t ? par : n;
  if (t < n) s_up[t] = up;
  for (int reach = 1; reach < n; reach *= 2) {
    __syncthreads();
    const int next = t < n ? s_up[up] : n;
    __syncthreads();
    up = next;
    if (t < n) s_up[t] = up;
  }
  const bool on = t < n && up == 0;
  const uint64_t m = __ballot(on);
  if (lane_id() == 0) s_cnt[wave_id()] = popc64(m);
  __syncthreads();
  int before = popc64(m & lanes_below(lane_id())), length = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) {
    before += w < wave_id() ? s_cnt[w] : 0;
    length += s_cnt[w];
  }
  if (t < n) p.on_path[first + t] = on;
  if (on) {
    path[before] = first + t;
    if (before == length - 1) p.bonus[b] = s_target[t];
  }
  for (int i = length + t; i < p.path_len; i += blockDim.x) path[i] = -1;
  if (t == 0) {
    p.length[b] = length;
    if (n == 0) p.bonus[b] = -1;
  }
}

}  // namespace

hipError_t launch_accept(const AcceptParams& p, const TreeOffsets& offs, int max_nodes, hipStream_t stream) {
  const int threads = max_nodes > kWave ? (max_nodes + kWave - 1) / kWave * kWave : kWave;
  accept_kernel<<<p.B, threads, 0, stream>>>(p, offs);
  return hipGetLastError();
}

}  // namespace amoe
