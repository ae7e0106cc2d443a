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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Byte offset of 16-byte unit u of a token row (RUN: its heads follow each
// other without a gap).
template <bool RUN>
__device__ __forceinline__ int64_t unit_at(int u, int row_units, int64_t sh_bytes) {
  if constexpr (RUN) return (int64_t)u * 16;
  const int h = u / row_units;
  return h * sh_bytes + (int64_t)(u - h * row_units) * 16;
}

// A unit's store: with the streaming hint in calls that write more than the
// Infinity Cache would keep for whoever reads it next (kMoveStream).
template <bool STREAM>
__device__ __forceinline__ void store(char* to, u32x4 x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to));
  else *reinterpret_cast<u32x4*>(to) = x;
}

// blockIdx: (block of 16 rows, segment, 2 layer + (1 for V)).  Blocks are
// 16-aligned, so one lies in one page.  A wave takes every fourth row of the
// block, up to four rows' units in flight.
template <bool RUN, bool STREAM>
__global__ __launch_bounds__(256) void cache_append(AppendParams p) {
  const AppendSegment sg = p.seg[blockIdx.y];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b0 = (sg.pos & ~(kMoveRows - 1)) + kMoveRows * (int)blockIdx.x;
  const int lo = max(b0, sg.pos), n = min(b0 + kMoveRows, sg.pos + sg.n) - lo;
  if (w >= n) return;
  const int pg = p.bt[sg.req * p.bt_stride + lo / p.c.page_tokens];
  const int layer = (int)blockIdx.z >> 1;
  const bool isv = blockIdx.z & 1;
  const char* src = (isv ? p.v_new : p.k_new) + layer * p.new_sl + (int64_t)(sg.row + (lo - sg.pos)) * p.new_st;
  char* dst = (isv ? p.c.v : p.c.k) + layer * p.c.layer_bytes + pg * p.c.page_bytes +
              (int64_t)(lo % p.c.page_tokens) * p.c.st_bytes;
  if (pg < 0 || pg >= p.c.num_pages) return;
  const int units = p.c.heads * p.c.row_units;
  for (int u = lane; u < units; u += 64) {
    const char* from = src + unit_at<RUN>(u, p.c.row_units, p.new_sh);
    char* to = dst + unit_at<RUN>(u, p.c.row_units, p.c.sh_bytes);
    u32x4 x[kMoveRows / 4];
#pragma unroll
    for (int i = 0; i < kMoveRows / 4; ++i)              // rows past the end: the wave's first again
      x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + (w + 4 * i < n ? w + 4 * i : w) * p.new_st));
#pragma unroll
    for (int i = 0; i < kMoveRows / 4; ++i)
      if (w + 4 * i < n) store<STREAM>(to + (w + 4 * i) * (int64_t)p.c.st_bytes, x[i]);
  }
}

// A wave 64 units of a request's rows in one layer and matrix.  The path's
// node at depth t is read into lane t; rows move in the order of their depth.
// A node's index is at least its depth, so a row's new place is never the old
// place of a deeper one: batches of loads ahead of their stores, ascending,
// are safe, and no two waves touch the same bytes.
template <bool RUN>
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
  base += on ? unit_at<RUN>(u, p.c.row_units, p.c.sh_bytes) : 0;
  for (int t0 = 1; t0 <= depth; t0 += 4) {
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4*>(base + readlane64(from, min(t0 + i, depth)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (on && ((moves >> (t0 + i)) & 1)) *reinterpret_cast<u32x4*>(base + readlane64(to, t0 + i)) = x[i];
  }
}

constexpr int kCopyUnits = 4;          // 16-byte units a thread

// blockIdx: (part of the page, pair, 2 layer + (1 for V)).
template <bool RUN, bool STREAM>
__global__ __launch_bounds__(256) void cache_copy_pages(PageCopyParams p) {
  const int i = blockIdx.y;
  const int row_units = p.c.heads * p.c.row_units;
  const int units = p.tokens[i] * row_units;
  const int u0 = (int)blockIdx.x * (256 * kCopyUnits);
  if (u0 >= units) return;
  const int layer = (int)blockIdx.z >> 1;
  char* base = ((blockIdx.z & 1) ? p.c.v : p.c.k) + layer * p.c.layer_bytes;
  const char* src = base + p.src[i] * p.c.page_bytes;
  char* dst = base + p.dst[i] * p.c.page_bytes;
  u32x4 x[kCopyUnits];
  int64_t at[kCopyUnits];
#pragma unroll
  for (int j = 0; j < kCopyUnits; ++j) {
    const int u = min(u0 + (int)threadIdx.x + 256 * j, units - 1);
    const int t = u / row_units;
    at[j] = (int64_t)t * p.c.st_bytes + unit_at<RUN>(u - t * row_units, p.c.row_units, p.c.sh_bytes);
    x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + at[j]));
  }
#pragma unroll
  for (int j = 0; j < kCopyUnits; ++j)
    if (u0 + (int)threadIdx.x + 256 * j < units) store<STREAM>(dst + at[j], x[j]);
}

}  // namespace

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  const dim3 g(p.parts, p.n_seg, 2 * p.c.layers);
  const bool run = p.c.heads == 1;
  if (p.c.stream) (run ? cache_append<true, true> : cache_append<false, true>)<<<g, dim3(256), 0, s>>>(p);
  else (run ? cache_append<true, false> : cache_append<false, false>)<<<g, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_commit(const CommitParams& p, hipStream_t s) {
  const dim3 g(p.n_req, 2 * p.c.layers, (p.c.heads * p.c.row_units + 63) / 64);
  if (p.c.heads == 1) cache_commit<true><<<g, dim3(64), 0, s>>>(p);
  else cache_commit<false><<<g, dim3(64), 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageCopyParams& p, hipStream_t s) {
  int most = 0;
  for (int i = 0; i < p.n; ++i) most = p.tokens[i] > most ? p.tokens[i] : most;
  const int units = most * p.c.heads * p.c.row_units;
  const dim3 g((units + 256 * kCopyUnits - 1) / (256 * kCopyUnits), p.n, 2 * p.c.layers);
  const bool run = p.c.heads == 1;
  if (p.c.stream) (run ? cache_copy_pages<true, true> : cache_copy_pages<false, true>)<<<g, dim3(256), 0, s>>>(p);
  else (run ? cache_copy_pages<true, false> : cache_copy_pages<false, false>)<<<g, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace sv
