// C ABI of the paged cache's operators (speccache.h): argument checks, the
// chunk attention's plan, and the row movers' launches.  Every check runs
// before the first HIP call.
#include "../../include/speccache.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <unordered_set>
#include <vector>

#include "sv_chunk.h"

namespace {

using sv::ChunkItem;
using sv::ChunkJoin;

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// No exception leaves the library: one from the standard containers is memory
// that the host does not have.
template <typename F>
spec_status_t guarded(F&& f) noexcept {
  try {
    return f();
  } catch (...) {
    return SPEC_ERR_WORKSPACE;
  }
}

int elem_bytes(spec_dtype_t t) { return t == SPEC_F32 ? 4 : 2; }

spec_status_t check_cache(const spec_cache_t* c, bool table) {
  if (!c) return SPEC_ERR_INVALID_ARG;
  if (c->dtype != SPEC_F32 && c->dtype != SPEC_BF16) return SPEC_ERR_INVALID_ARG;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->head_dim < 1 || c->num_pages < 1) return SPEC_ERR_INVALID_ARG;
  if (c->page_tokens < 32 || c->page_tokens % 32) return SPEC_ERR_INVALID_ARG;
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return SPEC_ERR_INVALID_ARG;
  const int64_t vec = 16 / elem_bytes(c->dtype);
  if (c->head_dim % vec) return SPEC_ERR_UNSUPPORTED;
  if (c->kv_stride_tok < 1 || c->kv_stride_head < 1 || c->kv_stride_tok % vec || c->kv_stride_head % vec)
    return SPEC_ERR_INVALID_ARG;
  if (c->num_layers > 1 && (c->layer_stride < 1 || c->layer_stride % vec)) return SPEC_ERR_INVALID_ARG;
  // a token row holds every head, heads apart
  if (c->num_kv_heads > 1 && c->kv_stride_head < c->head_dim) return SPEC_ERR_INVALID_ARG;
  if (c->kv_stride_head > INT32_MAX || c->kv_stride_tok > INT32_MAX ||
      c->kv_stride_head * (c->num_kv_heads - 1) + c->head_dim > c->kv_stride_tok)
    return SPEC_ERR_INVALID_ARG;
  // one page's rows are addressed with 32-bit offsets; a launch's second dimension holds K and V of every layer
  if ((int64_t)c->page_tokens * c->kv_stride_tok * elem_bytes(c->dtype) >= INT32_MAX || c->num_layers > 32767)
    return SPEC_ERR_UNSUPPORTED;
  if (table) {
    if (!c->block_table || reinterpret_cast<uintptr_t>(c->block_table) % 4 || c->block_stride < 1 ||
        c->block_width < 0 || c->block_width > c->block_stride)
      return SPEC_ERR_INVALID_ARG;
  }
  return SPEC_OK;
}

// The rows that a request's part of the block table has room for.
int64_t table_room(const spec_cache_t* c) {
  const int64_t pages = c->block_width ? c->block_width : c->block_stride;
  return std::min<int64_t>(pages * c->page_tokens, INT32_MAX / 2);
}

// Lengths that fit the block table; the number of new rows.
spec_status_t check_chunks(const spec_chunks_t* r, const spec_cache_t* c, int64_t* rows) {
  if (!r || r->num_requests < 1 || !r->ctx_len || !r->new_len) return SPEC_ERR_INVALID_ARG;
  const int64_t room = table_room(c);
  int64_t nq = 0;
  for (int i = 0; i < r->num_requests; ++i) {
    if (r->ctx_len[i] < 0 || r->new_len[i] < 0) return SPEC_ERR_INVALID_ARG;
    nq += r->new_len[i];
    if (r->new_len[i] > 0 && (int64_t)r->ctx_len[i] + r->new_len[i] > room) return SPEC_ERR_INVALID_ARG;
  }
  if (nq >= INT32_MAX / 2) return SPEC_ERR_INVALID_ARG;
  *rows = nq;
  return SPEC_OK;
}

int compute_units() {
  static std::atomic<int> cus[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
    (void)hipGetLastError();
    return 256;
  }
  if (const int known = cus[dev].load(std::memory_order_relaxed)) return known;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
    (void)hipGetLastError();
    n = 256;
  }
  cus[dev].store(n, std::memory_order_relaxed);
  return n;
}

struct ChunkPlan {
  std::vector<ChunkItem> items;
  std::vector<ChunkJoin> joins;
  bool tall = false;
  int32_t join_rows = 0, join_pieces = 0, turn0 = 0, turn1 = 0;
  int64_t parts = 0;
  size_t off_joins = 0, plan_bytes = 0;
  size_t off_part = 0, device_bytes = 0;
};

spec_status_t plan_chunk(const spec_chunks_t* r, const spec_cache_t* c, const spec_chunk_attn_args_t* a,
                         ChunkPlan& P) {
  spec_status_t st = check_cache(c, true);
  if (st != SPEC_OK) return st;
  if (!a || a->num_q_heads < 1 || a->num_q_heads % c->num_kv_heads) return SPEC_ERR_INVALID_ARG;
  if (a->layer < 0 || a->layer >= c->num_layers) return SPEC_ERR_INVALID_ARG;
  if (a->out_dtype != SPEC_F32 && a->out_dtype != SPEC_BF16) return SPEC_ERR_INVALID_ARG;
  if (c->dtype != SPEC_BF16 || (c->head_dim != 64 && c->head_dim != 128)) return SPEC_ERR_UNSUPPORTED;
  int64_t nq = 0;
  if ((st = check_chunks(r, c, &nq)) != SPEC_OK) return st;
  if (nq > 0 && (!a->q || !a->out)) return SPEC_ERR_INVALID_ARG;
  if (!aligned16(a->q) || !aligned16(a->out)) return SPEC_ERR_INVALID_ARG;
  if (a->q_stride_tok < 1 || a->q_stride_head < 1 || a->q_stride_tok % 8 || a->q_stride_head % 8)
    return SPEC_ERR_INVALID_ARG;
  const int Hkv = c->num_kv_heads, G = a->num_q_heads / Hkv;
  if (nq * G >= INT32_MAX / 2) return SPEC_ERR_UNSUPPORTED;

  // Row tiles of one height for the batch: 32 rows on one wave each where no
  // request has more (decoding), else 128 on a work-group of four.
  int64_t most = 0;
  for (int i = 0; i < r->num_requests; ++i) most = std::max<int64_t>(most, (int64_t)r->new_len[i] * G);
  P.tall = most > sv::kChunkLowRows;
  const int RT = P.tall ? sv::kChunkTallRows : sv::kChunkLowRows;
  struct RowTile { int32_t req, r0, rows, keys, q0, len, pieces; };
  std::vector<RowTile> tiles;
  int64_t q0 = 0, total = 0, longest = 0;
  for (int i = 0; i < r->num_requests; ++i) {
    const int n = r->new_len[i], rows = n * G;
    for (int r0 = 0; r0 < rows; r0 += RT) {
      const int nr = std::min(RT, rows - r0);
      tiles.push_back({i, r0, nr, r->ctx_len[i] + (r0 + nr - 1) / G + 1, (int32_t)q0, 0, 0});
      const int64_t kt = (tiles.back().keys + sv::kChunkTile - 1) / sv::kChunkTile;
      total += kt * Hkv;
      longest = std::max(longest, kt);
    }
    q0 += n;
  }
  const int cus = compute_units();
  // A row tile's keys in equal pieces of at most so many 64-key tiles.
  int64_t cap;
  if (!P.tall) {
    // Few rows: the keys stream past them at HBM's rate whatever the pieces, so
    // they are cut to 16 / 3 of them a compute unit, about what runs there at once
    // for d = 128 (five, by their 32 KB of LDS), where the last ones to end lose
    // least, down to 128 keys (64 where that leaves no compute unit two).  64
    // single tokens over 512-8192 rows: pieces of 1280 keys 190 us, 512 207, 4096
    // 214; one over 2000 rows of 8 KV heads: 64 keys 12.9, 128 14.9; over 4000:
    // 15.2 and 14.6.  All at d = 128; d = 64 goes by the same rule, though ten would
    // fit: 64 single tokens over 4000 rows of 8 KV heads (524 MB) 86 us, 6.1 TB/s.
    const int64_t slots = 4 * (int64_t)cus;
    cap = std::max<int64_t>(total <= cus ? 1 : 2, (3 * total + 4 * slots - 1) / (4 * slots));
  } else {
    // Many rows: a compute unit takes a 64-key tile in about a microsecond,
    // whether one work-group runs on it or two (1.1-1.2 and 0.94), so the longest
    // item bounds the kernel only where it is longer than a unit's mean share.
    // Only then is it cut, and where that saves more than the join costs (about
    // seven tiles).  Measured at d = 128 with a bf16 output, and used for d = 64
    // (three work-groups a unit) and fp32 outputs as it is; a tile of few rows
    // counts like a full one.  2048 new tokens, the longest 32 tiles of a mean of 33: whole
    // 48 us, pieces of 24 tiles 62, 16 64, 8 79; 1024, 16 of 9: whole 25, cut
    // 27; 64 over 2000 rows, 33 of 3: whole 40, pieces of 12 tiles 22, 8 20,
    // 4 17.  Decoding requests beside a chunk run in the same launch (beside 8
    // chunks of 33-700 tokens, 16 single ones: 181 us, in a launch of their own
    // before it 198).
    const int64_t mean = (total + cus - 1) / cus;
    cap = longest <= mean + 7 ? longest : std::max<int64_t>(4, mean);
  }
  int64_t n_items = 0;
  for (RowTile& t : tiles) {
    const int64_t kt = (t.keys + sv::kChunkTile - 1) / sv::kChunkTile;
    const int64_t pieces = (kt + cap - 1) / cap;
    t.len = (int32_t)((kt + pieces - 1) / pieces);
    t.pieces = (int32_t)((kt + t.len - 1) / t.len);
    n_items += t.pieces;
  }
  if (n_items * Hkv >= (int64_t)1 << 24) return SPEC_ERR_UNSUPPORTED;      // a launch's work-items are 32 bits
  // The longest first, so that the last to start are the shortest; after each,
  // its request's neighbouring row tiles down to 7 / 8 of its length, which
  // read the same keys at the same time.  With the heads innermost they also
  // run on the same XCD (work-group b on XCD b % 8) where the KV heads are a
  // multiple of eight (64 requests of 64 tokens over 4000 rows, 8 KV heads, 357
  // us, by length alone 419); four heads spread a head's tiles over two XCDs, one
  // over all.  Single tokens share nothing, and there a head's pieces follow
  // each other (64 of them 192 us, heads innermost 199).
  std::vector<int32_t> order, sorted(tiles.size());
  order.reserve(tiles.size());
  for (size_t i = 0; i < tiles.size(); ++i) sorted[i] = (int32_t)i;
  std::stable_sort(sorted.begin(), sorted.end(), [&](int32_t x, int32_t y) { return tiles[x].len > tiles[y].len; });
  std::vector<bool> placed(tiles.size(), false);
  for (const int32_t x : sorted) {
    if (placed[x]) continue;
    const RowTile& t = tiles[x];
    auto with = [&](int64_t y) {
      return y >= 0 && y < (int64_t)tiles.size() && !placed[y] && tiles[y].req == t.req &&
             8 * (int64_t)tiles[y].len >= 7 * (int64_t)t.len;
    };
    placed[x] = true;
    order.push_back(x);
    for (int step : {-1, 1})
      for (int64_t y = (int64_t)x + step; with(y); y += step) {
        placed[y] = true;
        order.push_back((int32_t)y);
      }
  }
  P.items.reserve((size_t)n_items);
  for (const int32_t x : order) {
    const RowTile& t = tiles[x];
    const int32_t len = t.len * sv::kChunkTile;
    for (int32_t s = 0; s < t.pieces; ++s)
      P.items.push_back({t.req, t.r0, t.rows, t.keys, len, s, t.pieces, r->ctx_len[t.req], P.parts, t.q0, 0});
    if (t.pieces > 1) {
      P.joins.push_back({t.r0, t.rows, t.pieces, t.q0, P.parts, 0});
      P.join_rows = std::max(P.join_rows, t.rows);
      P.join_pieces = std::max(P.join_pieces, t.pieces);
      P.parts += (int64_t)Hkv * t.pieces * t.rows;
    }
  }
  // work-groups b and b + cus of the tall kernel share a compute unit at first
  // (d = 128; with d = 64 a third joins them): the longest with the shortest of
  // the first two rounds
  if (P.tall && n_items * Hkv > cus) {
    P.turn0 = cus;
    P.turn1 = (int32_t)std::min<int64_t>(n_items * Hkv, 2 * (int64_t)cus);
  }

  P.off_joins = align_up(sizeof(ChunkItem) * P.items.size());
  P.plan_bytes = P.off_joins + align_up(sizeof(ChunkJoin) * P.joins.size());
  P.off_part = align_up(P.plan_bytes + sizeof(float2) * (size_t)P.parts);
  P.device_bytes = align_up(P.off_part + sizeof(float) * (size_t)P.parts * c->head_dim);
  return SPEC_OK;
}

// The row movers' view of the layers from `layer` on.  one_run: the heads
// follow each other without a gap on both sides, and move as one.
sv::CachePools pools(const spec_cache_t* c, int layer, bool one_run) {
  const int64_t eb = elem_bytes(c->dtype);
  sv::CachePools p;
  p.layer_bytes = c->num_layers > 1 ? c->layer_stride * eb : 0;
  p.k = static_cast<char*>(c->k) + layer * p.layer_bytes;
  p.v = static_cast<char*>(c->v) + layer * p.layer_bytes;
  p.st_bytes = (int32_t)(c->kv_stride_tok * eb);
  p.sh_bytes = (int32_t)(c->kv_stride_head * eb);
  p.num_pages = c->num_pages;
  p.page_tokens = c->page_tokens;
  p.heads = c->num_kv_heads;
  p.row_units = (int32_t)(c->head_dim * eb / 16);
  if (one_run) {
    p.row_units *= p.heads;
    p.heads = 1;
  }
  return p;
}
// `rows` token rows written in each of `layers` layers.
sv::MoveLaunch move_launch(const sv::CachePools& p, int layers, int64_t rows) {
  return {layers, rows * p.heads * p.row_units * 16 * 2 * layers >= sv::kMoveStream};
}
bool heads_touch(const spec_cache_t* c) { return c->num_kv_heads == 1 || c->kv_stride_head == c->head_dim; }

}  // namespace

extern "C" {

spec_status_t spec_chunk_workspace_bytes(const spec_chunks_t* chunks, const spec_cache_t* cache,
                                         const spec_chunk_attn_args_t* args, size_t* device_bytes,
                                         size_t* host_bytes) {
  return guarded([&]() -> spec_status_t {
    if (!device_bytes || !host_bytes) return SPEC_ERR_INVALID_ARG;
    ChunkPlan P;
    const spec_status_t st = plan_chunk(chunks, cache, args, P);
    if (st != SPEC_OK) return st;
    *device_bytes = P.device_bytes;
    *host_bytes = P.plan_bytes;
    return SPEC_OK;
  });
}

spec_status_t spec_chunk_attn(const spec_chunks_t* chunks, const spec_cache_t* cache,
                              const spec_chunk_attn_args_t* args, void* workspace, size_t workspace_bytes,
                              void* host_staging, size_t host_staging_bytes, void* stream) {
  return guarded([&]() -> spec_status_t {
    ChunkPlan P;
    const spec_status_t st = plan_chunk(chunks, cache, args, P);
    if (st != SPEC_OK) return st;
    if (P.items.empty()) return SPEC_OK;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign || workspace_bytes < P.device_bytes ||
        !host_staging || host_staging_bytes < P.plan_bytes)
      return SPEC_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* d = static_cast<char*>(workspace);
    char* h = static_cast<char*>(host_staging);
    std::memcpy(h, P.items.data(), sizeof(ChunkItem) * P.items.size());
    if (!P.joins.empty()) std::memcpy(h + P.off_joins, P.joins.data(), sizeof(ChunkJoin) * P.joins.size());
    // the kernels read the plan where it was staged when that is device-mapped
    // memory; otherwise it is copied into the workspace first
    const char* plan = d;
    void* mapped = nullptr;
    if (hipHostGetDevicePointer(&mapped, h, 0) == hipSuccess && mapped && aligned16(mapped)) {
      plan = static_cast<const char*>(mapped);
    } else {
      (void)hipGetLastError();
      if (hipMemcpyAsync(d, h, P.plan_bytes, hipMemcpyHostToDevice, s) != hipSuccess) return SPEC_ERR_HIP;
    }
    sv::ChunkParams p{};
    p.q = args->q;
    const int64_t lb = cache->num_layers > 1 ? args->layer * cache->layer_stride * 2 : 0;
    p.k = static_cast<const char*>(cache->k) + lb;
    p.v = static_cast<const char*>(cache->v) + lb;
    p.out = args->out;
    p.part = reinterpret_cast<float*>(d + P.off_part);
    p.items = reinterpret_cast<const ChunkItem*>(plan);
    p.bt = cache->block_table;
    p.q_st = args->q_stride_tok;
    p.q_sh = args->q_stride_head;
    p.kv_st = (int32_t)cache->kv_stride_tok;
    p.kv_sh = (int32_t)cache->kv_stride_head;
    p.bt_stride = cache->block_stride;
    p.page_tokens = cache->page_tokens;
    p.num_pages = cache->num_pages;
    p.Hkv = cache->num_kv_heads;
    p.G = args->num_q_heads / cache->num_kv_heads;
    p.turn0 = P.turn0;
    p.turn1 = P.turn1;
    const float scale = args->scale > 0.f ? args->scale : 1.f / std::sqrt((float)cache->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    sv::JoinParams j{};
    j.out = p.out;
    j.part = p.part;
    j.Hkv = p.Hkv;
    j.G = p.G;
    if (P.joins.size() == 1) j.one = P.joins[0];
    else j.joins = reinterpret_cast<const ChunkJoin*>(plan + P.off_joins);
    const sv::ChunkLaunch l = {(int32_t)P.items.size(), (int32_t)P.joins.size(), cache->head_dim,
                               args->out_dtype == SPEC_F32, P.tall, P.join_rows, P.join_pieces};
    return sv::launch_chunk(p, j, l, s) == hipSuccess ? SPEC_OK : SPEC_ERR_HIP;
  });
}

spec_status_t spec_cache_append(const spec_chunks_t* chunks, const spec_cache_t* cache, const spec_append_args_t* args,
                                void* stream) {
  spec_status_t st = check_cache(cache, true);
  if (st != SPEC_OK) return st;
  int64_t nq = 0;
  if ((st = check_chunks(chunks, cache, &nq)) != SPEC_OK) return st;
  if (!args || args->layer < 0 || args->num_layers < 1 || args->layer > cache->num_layers - args->num_layers)
    return SPEC_ERR_INVALID_ARG;
  if (nq > 0 && (!args->k_new || !args->v_new)) return SPEC_ERR_INVALID_ARG;
  if (!aligned16(args->k_new) || !aligned16(args->v_new)) return SPEC_ERR_INVALID_ARG;
  const int64_t eb = elem_bytes(cache->dtype), vec = 16 / eb;
  if (args->new_stride_tok < 1 || args->new_stride_head < 1 || args->new_stride_tok % vec ||
      args->new_stride_head % vec)
    return SPEC_ERR_INVALID_ARG;
  if (args->num_layers > 1 && (args->new_stride_layer < 1 || args->new_stride_layer % vec)) return SPEC_ERR_INVALID_ARG;

  const bool touch = heads_touch(cache) && (cache->num_kv_heads == 1 || args->new_stride_head == cache->head_dim);
  if (!touch && args->new_stride_head * eb / 16 > INT32_MAX) return SPEC_ERR_UNSUPPORTED;
  sv::AppendParams<sv::kMoveSegments> p{};
  p.c = pools(cache, args->layer, touch);
  const sv::MoveLaunch l = move_launch(p.c, args->num_layers, nq);
  p.k_new = static_cast<const char*>(args->k_new);
  p.v_new = static_cast<const char*>(args->v_new);
  p.new_sl = args->num_layers > 1 ? args->new_stride_layer * eb : 0;
  p.new_st = args->new_stride_tok * eb;
  p.new_sh = touch ? 0 : (int32_t)(args->new_stride_head * eb / 16);
  p.bt_stride = cache->block_stride;
  p.bt = cache->block_table;
  // Segments of at most `parts` blocks of 16 rows: as few blocks as keep the
  // batch in one launch's table, so that ragged batches leave few work-groups
  // without rows; a single request's rows are one segment.
  auto blocks = [&](int i) -> int64_t {
    const int64_t lo = chunks->ctx_len[i], n = chunks->new_len[i];
    return n ? (lo + n - 1) / sv::kMoveRows - lo / sv::kMoveRows + 1 : 0;
  };
  int64_t longest = 0, all = 0;
  for (int i = 0; i < chunks->num_requests; ++i) {
    longest = std::max(longest, blocks(i));
    all += blocks(i);
  }
  int64_t parts = longest == all && all < 1 << 16 ? std::max<int64_t>(longest, 1) : 1;
  for (;; parts *= 2) {
    int64_t segs = 0;
    for (int i = 0; i < chunks->num_requests; ++i) segs += (blocks(i) + parts - 1) / parts;
    if (segs <= sv::kMoveSegments || parts >= longest) break;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  int64_t row = 0;
  int n_seg = 0;
  for (int i = 0; i < chunks->num_requests; ++i) {
    int32_t pos = chunks->ctx_len[i];
    const int32_t end = pos + chunks->new_len[i];
    while (pos < end) {
      const int32_t stop = (int32_t)std::min<int64_t>(end, (pos / sv::kMoveRows + parts) * sv::kMoveRows);
      p.seg[n_seg++] = {i, pos, (int32_t)row, stop - pos};
      row += stop - pos;
      pos = stop;
      if (n_seg == sv::kMoveSegments) {
        if (sv::launch_append(p, n_seg, (int)parts, l, s) != hipSuccess) return SPEC_ERR_HIP;
        n_seg = 0;
      }
    }
  }
  if (n_seg > 0 && sv::launch_append(p, n_seg, (int)parts, l, s) != hipSuccess) return SPEC_ERR_HIP;
  return SPEC_OK;
}

spec_status_t spec_cache_commit(const spec_requests_t* req, const spec_cache_t* cache, const int32_t* accepted_node,
                                void* stream) {
  spec_status_t st = check_cache(cache, true);
  if (st != SPEC_OK) return st;
  if (!req || req->num_requests < 1 || !req->ctx_len || !accepted_node ||
      reinterpret_cast<uintptr_t>(accepted_node) % 4)
    return SPEC_ERR_INVALID_ARG;
  if (req->tree_nodes < 0 || req->tree_nodes > SPEC_MAX_TREE_NODES) return SPEC_ERR_INVALID_ARG;
  const bool per_req = req->node_count != nullptr;
  if (per_req && (req->tree_nodes != 0 || !req->tree_parents)) return SPEC_ERR_INVALID_ARG;
  if (!per_req && req->tree_nodes == 0 && !req->draft_len) return SPEC_ERR_INVALID_ARG;
  auto tree_ok = [](const int32_t* parent, int n) {
    if (n < 1 || n > SPEC_MAX_TREE_NODES || !parent || parent[0] != -1) return false;
    for (int x = 1; x < n; ++x)
      if (parent[x] < 0 || parent[x] >= x) return false;
    return true;
  };
  if (req->tree_nodes > 0 && !tree_ok(req->tree_parent, req->tree_nodes)) return SPEC_ERR_INVALID_ARG;
  const int64_t room = table_room(cache);
  int64_t o = 0;
  for (int i = 0; i < req->num_requests; ++i) {
    int n = req->tree_nodes;
    if (per_req) {
      n = req->node_count[i];
      if (!tree_ok(req->tree_parents + o, n)) return SPEC_ERR_INVALID_ARG;
      o += n;
    } else if (n == 0) {
      if (req->draft_len[i] < 0 || req->draft_len[i] > SPEC_MAX_DRAFT) return SPEC_ERR_INVALID_ARG;
      n = req->draft_len[i] + 1;
    }
    if (req->ctx_len[i] < 0 || (int64_t)req->ctx_len[i] + n > room) return SPEC_ERR_INVALID_ARG;
  }
  if (!per_req && req->tree_nodes == 0) return SPEC_OK;      // chains are in place
  if ((int64_t)cache->num_kv_heads * cache->head_dim * elem_bytes(cache->dtype) / 1024 >= 65535)
    return SPEC_ERR_UNSUPPORTED;

  sv::CommitParams<sv::kMoveTrees> p{};
  p.c = pools(cache, 0, heads_touch(cache));
  const sv::MoveLaunch l = move_launch(p.c, cache->num_layers, 0);
  p.bt_stride = cache->block_stride;
  p.shared = !per_req;
  o = 0;
  for (int i0 = 0; i0 < req->num_requests; i0 += sv::kMoveTrees) {
    const int n_req = std::min(sv::kMoveTrees, req->num_requests - i0);
    p.bt = cache->block_table + (int64_t)i0 * cache->block_stride;
    p.accepted = accepted_node + i0;
    for (int i = 0; i < n_req; ++i) {
      p.ctx[i] = req->ctx_len[i0 + i];
      if (i > 0 && !per_req) continue;
      const int n = per_req ? req->node_count[i0 + i] : req->tree_nodes;
      const int32_t* parent = per_req ? req->tree_parents + o : req->tree_parent;
      p.nodes[i] = (int8_t)n;
      for (int x = 0; x < n; ++x) p.parent[i][x] = (int8_t)std::max(parent[x], 0);
      o += n;
    }
    if (sv::launch_commit(p, n_req, l, static_cast<hipStream_t>(stream)) != hipSuccess) return SPEC_ERR_HIP;
  }
  return SPEC_OK;
}

spec_status_t spec_cache_copy_pages(const spec_cache_t* cache, const spec_page_copy_t* copies, int32_t num_copies,
                                    void* stream) {
  return guarded([&]() -> spec_status_t {
    spec_status_t st = check_cache(cache, false);
    if (st != SPEC_OK) return st;
    if (num_copies < 0 || (num_copies > 0 && !copies)) return SPEC_ERR_INVALID_ARG;
    if (num_copies > cache->num_pages) return SPEC_ERR_INVALID_ARG;      // some page is written twice
    std::unordered_set<int32_t> written;
    written.reserve(num_copies);
    for (int i = 0; i < num_copies; ++i) {
      const spec_page_copy_t& x = copies[i];
      if (x.src < 0 || x.src >= cache->num_pages || x.dst < 0 || x.dst >= cache->num_pages || x.tokens < 1 ||
          x.tokens > cache->page_tokens || !written.insert(x.dst).second)
        return SPEC_ERR_INVALID_ARG;
    }
    for (int i = 0; i < num_copies; ++i)
      if (written.count(copies[i].src)) return SPEC_ERR_INVALID_ARG;
    int64_t rows = 0;
    for (int i = 0; i < num_copies; ++i) rows += copies[i].tokens;
    sv::PageCopyParams<sv::kMovePages> p{};
    p.c = pools(cache, 0, heads_touch(cache));
    const sv::MoveLaunch l = move_launch(p.c, cache->num_layers, rows);
    for (int i0 = 0; i0 < num_copies; i0 += sv::kMovePages) {
      const int n = std::min(sv::kMovePages, num_copies - i0);
      for (int i = 0; i < n; ++i) p.pair[i] = {copies[i0 + i].src, copies[i0 + i].dst, copies[i0 + i].tokens};
      if (sv::launch_page_copy(p, n, l, static_cast<hipStream_t>(stream)) != hipSuccess) return SPEC_ERR_HIP;
    }
    return SPEC_OK;
  });
}

}  // extern "C"
