// The paged cache's row movers for gfx950: appended rows, accepted tree paths,
// copied pages.  All are bound by HBM where they are large (each row read once
// and written once, 16 bytes a lane) and by a launch and a few dependent loads
// where they are small, so what the host knows travels in the kernel
// arguments and a wave finds its request with one round of loads.
#include "sv_chunk.h"

namespace sv {
namespace {

__device__ __forceinline__ int64_t readlane64(int64_t x, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Byte offset of 16-byte unit u of a token row.
__device__ __forceinline__ int64_t unit_at(int u, int row_units, int64_t sh_bytes) {
  const int h = u / row_units;
  return h * sh_bytes + (int64_t)(u - h * row_units) * 16;
}

// A wave a new row, layer and matrix: blockIdx.y = 2 layer + (1 for V).
__global__ __launch_bounds__(256) void cache_append(AppendParams p) {
  const int lane = threadIdx.x & 63;
  const int row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
  if (row >= p.rows) return;
  // requests whose rows end at or before this one
  int req = 0;
  for (int b = 0; b < p.n_req; b += 64) {
    const int i = b + lane;
    const bool before = i < p.n_req && p.end[min(i, kMoveRequests - 1)] <= row;
    req += __builtin_popcountll(__ballot(before));
  }
  req = __builtin_amdgcn_readfirstlane(min(req, p.n_req - 1));
  const int first = req > 0 ? p.end[req - 1] : 0;
  const int t = p.ctx[req] + (row - first);
  const int pg = p.bt[req * p.bt_stride + t / p.c.page_tokens];
  if (pg < 0 || pg >= p.c.num_pages) return;
  const int layer = (int)blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  char* dst = (isv ? p.c.v : p.c.k) + layer * p.c.layer_bytes + pg * p.c.page_bytes +
              (int64_t)(t % p.c.page_tokens) * p.c.st_bytes;
  const char* src = (isv ? p.v_new : p.k_new) + layer * p.new_sl + (int64_t)(p.row0 + row) * p.new_st;
  const int units = p.c.heads * p.c.row_units;
  for (int u0 = lane; u0 < units; u0 += 256) {
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (u0 + 64 * i < units) x[i] = *reinterpret_cast<const uint4*>(src + unit_at(u0 + 64 * i, p.c.row_units, p.new_sh));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (u0 + 64 * i < units) *reinterpret_cast<uint4*>(dst + unit_at(u0 + 64 * i, p.c.row_units, p.c.sh_bytes)) = x[i];
  }
}

// A wave 64 units of a request's rows in one layer and matrix.  The path's
// node at depth t is read into lane t; rows move in the order of their depth.
// A node's index is at least its depth, so a row's new place is never the old
// place of a deeper one: batches of loads ahead of their stores, ascending,
// are safe, and no two waves touch the same bytes.
__global__ __launch_bounds__(64) void cache_commit(CommitParams p) {
  const int lane = threadIdx.x;
  const int req = blockIdx.x;
  const int topo = p.shared ? 0 : req;
  const int nodes = p.nodes[topo];
  const int node = __builtin_amdgcn_readfirstlane(p.accepted[req]);
  if (node <= 0 || node >= nodes) return;
  const int par = p.parent[topo][lane & 31];
  // the path from the node up, then turned round: lane t holds the node at depth t
  int depth = 0;
  for (int n = node; n > 0 && depth < 32; n = __builtin_amdgcn_readlane(par, n)) ++depth;
  int mine = 0;
  {
    int n = node;
    for (int t = depth; t > 0; --t) {
      mine = lane == t ? n : mine;
      n = __builtin_amdgcn_readlane(par, n);
    }
  }
  const int32_t* bt = p.bt + req * p.bt_stride;
  const int P = p.c.page_tokens;
  int64_t from = 0, to = 0;
  int bad = 0;
  if (lane >= 1 && lane <= depth) {
    const int ts = p.ctx[req] + mine, td = p.ctx[req] + lane;
    const int ps = bt[ts / P], pd = bt[td / P];
    bad = pd < 0 || pd >= p.c.num_pages || mine == lane;
    from = min(max(ps, 0), p.c.num_pages - 1) * p.c.page_bytes + (int64_t)(ts % P) * p.c.st_bytes;
    to = bad ? 0 : pd * p.c.page_bytes + (int64_t)(td % P) * p.c.st_bytes;
  }
  const uint64_t moves = __ballot(lane >= 1 && lane <= depth && !bad);
  const int layer = (int)blockIdx.y >> 1;
  char* base = ((blockIdx.y & 1) ? p.c.v : p.c.k) + layer * p.c.layer_bytes;
  const int u = (int)blockIdx.z * 64 + lane;
  const bool on = u < p.c.heads * p.c.row_units;
  base += on ? unit_at(u, p.c.row_units, p.c.sh_bytes) : 0;
  for (int t0 = 1; t0 <= depth; t0 += 4) {
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4*>(base + readlane64(from, min(t0 + i, depth)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (on && ((moves >> (t0 + i)) & 1)) *reinterpret_cast<uint4*>(base + readlane64(to, t0 + i)) = x[i];
  }
}

constexpr int kCopyUnits = 4;          // 16-byte units a thread

// blockIdx.x: pair; y: 2 layer + (1 for V); z: part of the page.
__global__ __launch_bounds__(256) void cache_copy_pages(PageCopyParams p) {
  const int i = blockIdx.x;
  const int row_units = p.c.heads * p.c.row_units;
  const int units = p.tokens[i] * row_units;
  const int u0 = (int)blockIdx.z * (256 * kCopyUnits) + (int)threadIdx.x;
  if ((int)blockIdx.z * (256 * kCopyUnits) >= units) return;
  const int layer = (int)blockIdx.y >> 1;
  char* base = ((blockIdx.y & 1) ? p.c.v : p.c.k) + layer * p.c.layer_bytes;
  const char* src = base + p.src[i] * p.c.page_bytes;
  char* dst = base + p.dst[i] * p.c.page_bytes;
  uint4 x[kCopyUnits];
  int64_t at[kCopyUnits];
#pragma unroll
  for (int j = 0; j < kCopyUnits; ++j) {
    const int u = u0 + 256 * j;
    const int t = u / row_units;
    at[j] = (int64_t)t * p.c.st_bytes + unit_at(u - t * row_units, p.c.row_units, p.c.sh_bytes);
    if (u < units) x[j] = *reinterpret_cast<const uint4*>(src + at[j]);
  }
#pragma unroll
  for (int j = 0; j < kCopyUnits; ++j)
    if (u0 + 256 * j < units) *reinterpret_cast<uint4*>(dst + at[j]) = x[j];
}

}  // namespace

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  cache_append<<<dim3((p.rows + 3) / 4, 2 * p.c.layers), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_commit(const CommitParams& p, hipStream_t s) {
  cache_commit<<<dim3(p.n_req, 2 * p.c.layers, (p.c.heads * p.c.row_units + 63) / 64), dim3(64), 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageCopyParams& p, hipStream_t s) {
  int most = 0;
  for (int i = 0; i < p.n; ++i) most = p.tokens[i] > most ? p.tokens[i] : most;
  const int units = most * p.c.heads * p.c.row_units;
  cache_copy_pages<<<dim3(p.n, 2 * p.c.layers, (units + 256 * kCopyUnits - 1) / (256 * kCopyUnits)), dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace sv
