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

__device__ __forceinline__ int64_t page_bytes(const CachePools& c) { return (int64_t)c.page_tokens * c.st_bytes; }

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
// block, up to four rows' units in flight.  2-9 rows of 128 requests (5.8 MB
// moved): 3.9 us, the launch; 300-700 rows of 4 requests in 32 layers (553 MB): 93
// us, 5.9 TB/s (torch's copy 4.9).
template <bool RUN, bool STREAM, int N>
__global__ __launch_bounds__(256) void cache_append(AppendParams<N> p) {
  const AppendSegment sg = p.seg[N > 1 ? blockIdx.y : 0];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b0 = (sg.pos & ~(kMoveRows - 1)) + kMoveRows * (int)blockIdx.x;
  const int lo = max(b0, sg.pos), n = min(b0 + kMoveRows, sg.pos + sg.n) - lo;
  if (w >= n) return;
  const int pg = p.bt[(int64_t)sg.req * p.bt_stride + lo / p.c.page_tokens];
  const int layer = (int)blockIdx.z >> 1;
  const bool isv = blockIdx.z & 1;
  const char* src = (isv ? p.v_new : p.k_new) + layer * p.new_sl + (int64_t)(sg.row + (lo - sg.pos)) * p.new_st;
  char* dst = (isv ? p.c.v : p.c.k) + layer * p.c.layer_bytes + pg * page_bytes(p.c) +
              (int64_t)(lo % p.c.page_tokens) * p.c.st_bytes;
  if (pg < 0 || pg >= p.c.num_pages) return;
  const int units = p.c.heads * p.c.row_units;
  for (int u = lane; u < units; u += 64) {
    const char* from = src + unit_at<RUN>(u, p.c.row_units, (int64_t)p.new_sh * 16);
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
// are safe, and no two waves touch the same bytes.  One tree of 15 nodes in 32
// layers 3.8 us (the launch and its dependent loads), 64 of them 8.4 us for
// about 29 MB moved, which the append before left in the caches.
template <bool RUN, int N>
__global__ __launch_bounds__(64) void cache_commit(CommitParams<N> p) {
  const int lane = threadIdx.x;
  const int req = N > 1 ? blockIdx.x : 0;
  const int topo = N == 1 || p.shared ? 0 : req;
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
  const int32_t* bt = p.bt + (int64_t)req * p.bt_stride;
  const int P = p.c.page_tokens;
  int64_t from = 0, to = 0;
  int bad = 0;
  if (lane >= 1 && lane <= depth) {
    const int ts = p.ctx[req] + mine, td = p.ctx[req] + lane;
    const int ps = bt[ts / P], pd = bt[td / P];
    bad = pd < 0 || pd >= p.c.num_pages || mine == lane;
    from = min(max(ps, 0), p.c.num_pages - 1) * page_bytes(p.c) + (int64_t)(ts % P) * p.c.st_bytes;
    to = bad ? 0 : pd * page_bytes(p.c) + (int64_t)(td % P) * p.c.st_bytes;
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

// blockIdx: (part of the page, pair, 2 layer + (1 for V)).  One page of 64 rows
// in 32 layers (2 x 8 heads of 128) 3.2 us, the launch; 96 of them (1.61 GB) 284
// us, 5.7 TB/s.
template <bool RUN, bool STREAM, int N>
__global__ __launch_bounds__(256) void cache_copy_pages(PageCopyParams<N> p) {
  const PagePair pair = p.pair[blockIdx.y];
  const int row_units = p.c.heads * p.c.row_units;
  const int units = pair.tokens * row_units;
  const int u0 = (int)blockIdx.x * (256 * kCopyUnits);
  if (u0 >= units) return;
  const int layer = (int)blockIdx.z >> 1;
  char* base = ((blockIdx.z & 1) ? p.c.v : p.c.k) + layer * p.c.layer_bytes;
  const char* src = base + pair.src * page_bytes(p.c);
  char* dst = base + pair.dst * page_bytes(p.c);
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

// The first M entries of a table.
template <int M, int N>
static AppendParams<M> small(const AppendParams<N>& p) {
  AppendParams<M> q{p.c, p.k_new, p.v_new, p.bt, p.new_sl, p.new_st, p.new_sh, p.bt_stride, {}};
  for (int i = 0; i < M; ++i) q.seg[i] = p.seg[i];
  return q;
}
template <int M, int N>
static CommitParams<M> small(const CommitParams<N>& p) {
  CommitParams<M> q{p.c, p.bt, p.accepted, p.bt_stride, p.shared, {}, {}, {}};
  for (int i = 0; i < M; ++i) {
    q.ctx[i] = p.ctx[i];
    q.nodes[i] = p.nodes[i];
    for (int x = 0; x < 32; ++x) q.parent[i][x] = p.parent[i][x];
  }
  return q;
}
template <int M, int N>
static PageCopyParams<M> small(const PageCopyParams<N>& p) {
  PageCopyParams<M> q{p.c, {}};
  for (int i = 0; i < M; ++i) q.pair[i] = p.pair[i];
  return q;
}

template <int N>
static hipError_t append(const AppendParams<N>& p, dim3 g, bool stream, hipStream_t s) {
  const bool run = p.c.heads == 1;
  if (stream) (run ? cache_append<true, true, N> : cache_append<false, true, N>)<<<g, dim3(256), 0, s>>>(p);
  else (run ? cache_append<true, false, N> : cache_append<false, false, N>)<<<g, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}
hipError_t launch_append(const AppendParams<kMoveSegments>& p, int n, int parts, const MoveLaunch& l, hipStream_t s) {
  const dim3 g(parts, n, 2 * l.layers);
  return n == 1 ? append(small<1>(p), g, l.stream, s) : append(p, g, l.stream, s);
}

template <int N>
static hipError_t commit(const CommitParams<N>& p, dim3 g, hipStream_t s) {
  (p.c.heads == 1 ? cache_commit<true, N> : cache_commit<false, N>)<<<g, dim3(64), 0, s>>>(p);
  return hipGetLastError();
}
hipError_t launch_commit(const CommitParams<kMoveTrees>& p, int n, const MoveLaunch& l, hipStream_t s) {
  const dim3 g(n, 2 * l.layers, (p.c.heads * p.c.row_units + 63) / 64);
  return n == 1 ? commit(small<1>(p), g, s) : commit(p, g, s);
}

template <int N>
static hipError_t page_copy(const PageCopyParams<N>& p, dim3 g, bool stream, hipStream_t s) {
  const bool run = p.c.heads == 1;
  if (stream) (run ? cache_copy_pages<true, true, N> : cache_copy_pages<false, true, N>)<<<g, dim3(256), 0, s>>>(p);
  else (run ? cache_copy_pages<true, false, N> : cache_copy_pages<false, false, N>)<<<g, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}
hipError_t launch_page_copy(const PageCopyParams<kMovePages>& p, int n, const MoveLaunch& l, hipStream_t s) {
  int most = 0;
  for (int i = 0; i < n; ++i) most = p.pair[i].tokens > most ? p.pair[i].tokens : most;
  const int units = most * p.c.heads * p.c.row_units;
  const dim3 g((units + 256 * kCopyUnits - 1) / (256 * kCopyUnits), n, 2 * l.layers);
  return n <= kMovePagesSmall ? page_copy(small<kMovePagesSmall>(p), g, l.stream, s) : page_copy(p, g, l.stream, s);
}

}  // namespace sv
