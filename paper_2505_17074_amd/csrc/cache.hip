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
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

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

// cos and sin of p f, an angle in radians, for a whole number p and an fp32 f:
// off by 2^-23 at most up to 2^45 radians (2^31 times an f of 2^14).  The product,
// of up to 55 bits, is two 64-bit numbers and so is 2 / pi, so that what is left
// of a quarter turn is off by 2^-53 of one, and by the angle's 2^-106; the rest
// within an eighth of a turn by the series, whose next terms are below 2^-28.
__device__ __forceinline__ float2 cos_sin(int32_t p, float f) {
  constexpr double kQuarters = 0.63661977236758134308, kQuartersLow = -3.9357353350364970e-17;      // 2 / pi
  const double angle = (double)p * (double)f, low = __builtin_fma((double)p, (double)f, -angle);
  const double whole = __builtin_rint(angle * kQuarters);
  const double part = __builtin_fma(angle, kQuarters, -whole) + __builtin_fma(angle, kQuartersLow, low * kQuarters);
  const float x = (float)(part * 1.57079632679489661923);
  const float y = x * x;
  const float s = x + x * y * fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  // the quadrant: whole mod 4 (whole / 4 may have more than 32 bits)
  const int q = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

template <bool F32>
struct Turned {                        // a 16-byte unit's elements in fp32
  static constexpr int VEC = F32 ? 4 : 8;
  float x[VEC];
  __device__ __forceinline__ explicit Turned(u32x4 u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F32) {
        x[i] = __uint_as_float(u[i]);
      } else {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ u32x4 pack() const {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F32) u[i] = __float_as_uint(x[i]);
      else u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, bf16x2));
    }
    return u;
  }
};

// Appended rows, K and the queries rotated on the way: for pair i of a head's
// first 2 `pairs` elements and angle p f_i,
//   (x, y) -> (x cos - y sin, y cos + x sin),
// in fp32, each result rounded once.  Pairs are elements i and i + pairs, or 2 i
// and 2 i + 1 (INTER).
// blockIdx: (block of two or four rows, segment, layer).  The block's angles are
// computed once, into LDS, beside the first loads; a thread keeps its columns of a head
// (two units, INTER or without a partner one) and goes from head to head and
// row to row, the queries' heads first, then K's and V's.  Bound by HBM where it is
// large (6 prompts' 13300 rows of 32 + 2 x 8 heads of 128, 327 MB: 60 us, 5.5 TB/s
// with torch's copy at 5.1) and by the launch and one round of loads where it is
// small (one row 4.0 us, 64 trees of 15 nodes, 24 MB, 8; a call 8 and 9 on the
// host).
template <bool F32, bool INTER, bool STREAM, int N>
__global__ __launch_bounds__(256) void cache_append_rotated(RotateParams<N> p) {
  constexpr int VEC = Turned<F32>::VEC, AHEAD = 4;
  __shared__ float cs[kTurnRows][2][kMaxTurned];
  const AppendSegment sg = p.seg[N > 1 ? blockIdx.y : 0];
  const int b0 = (sg.pos & ~(p.rows - 1)) + p.rows * (int)blockIdx.x;
  const int lo = max(b0, sg.pos), n = min(b0 + p.rows, sg.pos + sg.n) - lo;
  if (n <= 0) return;
  const int pg = p.bt[(int64_t)sg.req * p.bt_stride + lo / p.c.page_tokens];
  const bool kept = pg >= 0 && pg < p.c.num_pages;
  const int layer = blockIdx.z;
  const int64_t at = layer * p.c.layer_bytes + (kept ? pg : 0) * page_bytes(p.c) +
                     (int64_t)(lo % p.c.page_tokens) * p.c.st_bytes;
  const int64_t row0 = sg.row + (lo - sg.pos);
  // columns of a head: its turned ones (a unit and its partner), then the rest
  const int turned = INTER ? p.pairs * 2 / VEC : p.pairs / VEC;
  const int cols = p.c.row_units - (INTER ? 0 : turned);
  const int heads = p.q_heads + 2 * p.c.heads;
  const int u0 = (int)threadIdx.x % cols, hstep = 256 / cols;

  struct Item {
    const char* from;
    char* to;
    int u, row;
    bool on, write, turn, two;
  };
  // a head narrower than 256 columns: hstep heads at a time; else the block walks the columns too
  const int wide = hstep ? 1 : (cols + 255) / 256;
  const int step = hstep ? hstep : 1;
  const int mine = hstep ? (int)threadIdx.x / cols : 0;
  const int items = n * heads * wide;
  auto item = [&](int i) {
    Item x;
    x.on = i < items && (hstep == 0 || mine < hstep);
    const int hw = i / wide, part = i - hw * wide;
    x.row = min(hw / heads, n - 1);
    const int h = min(hw - x.row * heads, heads - 1);
    x.u = hstep ? u0 : part * 256 + (int)threadIdx.x;
    x.on = x.on && x.u < cols;
    const int64_t r = row0 + x.row;
    const int hk = h - p.q_heads, hv = hk - p.c.heads;
    if (hk < 0) {
      x.from = p.q + r * p.q_st + (int64_t)h * p.q_sh * 16;
      x.to = p.q_out + r * p.out_st + (int64_t)h * p.out_sh * 16;
    } else {
      const int kh = hv < 0 ? hk : hv;
      x.from = (hv < 0 ? p.k_new : p.v_new) + layer * p.new_sl + r * p.new_st + (int64_t)kh * p.new_sh * 16;
      x.to = (hv < 0 ? p.c.k : p.c.v) + at + (int64_t)x.row * p.c.st_bytes + (int64_t)kh * p.c.sh_bytes;
    }
    x.write = x.on && (hk < 0 || kept);
    x.two = !INTER && x.u < turned;
    x.turn = x.u < turned && hv < 0;
    // behind the turned columns and their partners
    x.u += !INTER && x.u >= turned ? turned : 0;
    x.from += (int64_t)x.u * 16;
    x.to += (int64_t)x.u * 16;
    return x;
  };
  auto load = [&](const Item& x, u32x4& a, u32x4& b) {
    if (x.on) {
      a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x.from));
      if (x.two) b = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x.from) + turned);
    }
  };
  auto finish = [&](const Item& x, u32x4 a, u32x4 b) {
    if (!x.write) return;
    if (x.turn) {
      const float* c = &cs[x.row][0][0];
      const float* s = &cs[x.row][1][0];
      Turned<F32> y(a);
      if constexpr (INTER) {
        const int i0 = x.u * (VEC / 2);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
          const float u = y.x[i], v = y.x[i + 1], co = c[i0 + i / 2], si = s[i0 + i / 2];
          y.x[i] = fmaf(u, co, -(v * si));
          y.x[i + 1] = fmaf(v, co, u * si);
        }
      } else {
        const int i0 = x.u * VEC;
        Turned<F32> z(b);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float u = y.x[i], v = z.x[i], co = c[i0 + i], si = s[i0 + i];
          y.x[i] = fmaf(u, co, -(v * si));
          z.x[i] = fmaf(v, co, u * si);
        }
        b = z.pack();
      }
      a = y.pack();
    }
    store<STREAM>(x.to, a);
    if (x.two) store<STREAM>(x.to + (int64_t)turned * 16, b);
  };

  u32x4 a[AHEAD], b[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) load(item(mine + k * step), a[k], b[k]);
  for (int i = threadIdx.x; i < n * p.pairs; i += 256) {
    const int row = i / p.pairs, x = i - row * p.pairs;
    const int pos = p.positions ? p.positions[row0 + row] : lo + row;
    const float2 y = cos_sin(pos, p.freq[x]);
    cs[row][0][x] = y.x;
    cs[row][1][x] = y.y;
  }
  __syncthreads();
  for (int i = mine; i < items; i += AHEAD * step) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) finish(item(i + k * step), a[k], b[k]);
    if (i + AHEAD * step < items) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) load(item(i + (AHEAD + k) * step), a[k], b[k]);
    }
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
static RotateParams<M> small(const RotateParams<N>& p) {
  RotateParams<M> q{p.c,      p.k_new,  p.v_new, p.q,    p.q_out, p.bt,        p.freq,    p.positions, p.new_sl, p.new_st,
                    p.q_st,   p.out_st, p.new_sh, p.q_sh, p.out_sh, p.bt_stride, p.q_heads, p.pairs,     p.rows,  {}};
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

template <bool F32, bool INTER, int N>
static hipError_t rotate(const RotateParams<N>& p, dim3 g, bool stream, hipStream_t s) {
  if (stream) cache_append_rotated<F32, INTER, true, N><<<g, dim3(256), 0, s>>>(p);
  else cache_append_rotated<F32, INTER, false, N><<<g, dim3(256), 0, s>>>(p);
  return hipGetLastError();
}
hipError_t launch_rotate(const RotateParams<kMoveSegments>& p, int n, int parts, const MoveLaunch& l, bool f32,
                         bool interleaved, hipStream_t s) {
  const dim3 g(parts, n, l.layers);
  auto go = [&](const auto& x) {
    if (f32) return interleaved ? rotate<true, true>(x, g, l.stream, s) : rotate<true, false>(x, g, l.stream, s);
    return interleaved ? rotate<false, true>(x, g, l.stream, s) : rotate<false, false>(x, g, l.stream, s);
  };
  return n == 1 ? go(small<1>(p)) : go(p);
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
