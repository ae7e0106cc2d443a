// Internal declarations of the paged cache's operators: chunk attention's
// plan items and kernel parameters, and the row movers' arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sv {

// One piece of the chunk attention's work, the same for every KV head: keys
// [piece * len, (piece + 1) * len) of the first `keys` keys of a request, for
// `rows` query rows from row r0 on.  Query row r of a request and KV head is new
// token r / G under the group's query head r % G, so that a run of rows sees a
// run of key ranges.  A row tile's pieces follow each other in the list.
struct ChunkItem {
  int32_t req;      // block table row
  int32_t r0, rows;
  int32_t keys;
  int32_t len;      // a multiple of kChunkTile
  int32_t piece, pieces;
  int32_t ctx;
  int64_t part;     // the tile's first partial row (pieces > 1): head h's piece s from (h pieces + s) rows on
  int32_t q0;       // the request's first row of q and out
  int32_t skip;     // keys left out behind the first ones (below), a multiple of 32
};
static_assert(sizeof(ChunkItem) == 48, "ChunkItem is read as 16-byte units");

// Items that leave out a run of keys: requests behind a shared prefix (kBehind),
// windows behind their sinks (kWindowed).  Their keys are counted without it: key t
// of an item is the request's row t where t < first, else t + skip, `first` the
// sinks rounded up to 32 (ChunkParams::sinks), and `keys` and `ctx` are in these
// counts (ctx may be negative).  New token j sees the keys t <= ctx + j, of a
// window those with t > ctx + j - window or t < sinks.  The run begins and ends on a
// 32-row border of the request, so that a 32-key block is of one page.  `part` is
// negative where the item writes out itself.
enum Keys { kEvery, kBehind, kWindowed };

// One query-row tile whose key range was cut: a head's pieces' partial rows
// follow each other, `rows` apart, the heads `pieces * rows` apart.
struct ChunkJoin {
  int32_t r0, rows;
  int32_t pieces;
  int32_t q0;
  int64_t part;
  int64_t pad;
};
static_assert(sizeof(ChunkJoin) == 32, "ChunkJoin is read as 16-byte units");

// Kernel arguments of 128 bytes and more cost the host 1.1 us a launch (2.8 us
// with less, 3.9 from there to 2 KB, 4.1 with 4 KB), which is what the smallest
// calls wait for: the arguments end below that where they can.
constexpr size_t kSmallArgs = 127;

struct ChunkParams {
  const void* q;
  const void* k;        // the layer's pools
  const void* v;
  void* out;
  float* part;          // partial row i, not normalised, at part + i d; its running maximum (log2
                        // units) and sum at (float2*)part - 1 - i
  const ChunkItem* items;
  const int32_t* bt;
  int64_t q_st, q_sh;
  int32_t kv_st, kv_sh;
  int32_t bt_stride;
  int32_t page_tokens, num_pages;
  int32_t Hkv, G;
  int32_t turn0, turn1; // work-groups [turn0, turn1) take their places from the end
  float scale_log2;
  int32_t window, sinks;               // kWindowed (sinks: 0 otherwise)
};

// Rows whose keys two tiles had, the prefix's and the request's own (a join of
// requests behind a shared prefix).  Row rr of the run is partial row part + (h
// pieces + s) stride + rr of each, h the KV head, s the piece.
struct ChunkMeet {
  int64_t part[2];
  int32_t pieces[2], stride[2];
  int32_t q0, r0, rows;                // the run's rows of the request that begins at row q0
  int32_t pad;
};
static_assert(sizeof(ChunkMeet) == 48, "ChunkMeet is read as 16-byte units");

struct MeetParams {
  void* out;
  const float* part;
  const ChunkMeet* meets;
  int32_t Hkv, G;
};

struct JoinParams {
  void* out;
  const float* part;
  const ChunkJoin* joins;              // null: `one` is all
  int32_t Hkv, G;
  ChunkJoin one;
};
static_assert(sizeof(ChunkParams) <= kSmallArgs && sizeof(JoinParams) <= kSmallArgs, "small arguments");

// What the launches go by.
struct ChunkLaunch {
  int32_t n_items, n_joins;            // of one KV head
  int32_t D;
  bool out_f32;
  bool tall;            // items of up to kChunkTallRows rows on four waves, else kChunkLowRows on one
  bool two_parts;       // a bf16 output: P in two bf16 parts, in tall items (kBehind) too
  int32_t join_rows;    // rows of the tallest joined tile
  int32_t join_pieces;  // pieces of the longest
  Keys keys;            // what the items leave out
  int32_t n_meets, meet_rows;
};

constexpr int kChunkLowRows = 32;
constexpr int kChunkTallRows = 128;
constexpr int kChunkTile = 64;         // pieces are cut at multiples of this many keys
constexpr int kNoWindow = 1 << 30;     // wider than any request is long

hipError_t launch_chunk(const ChunkParams& p, const JoinParams& j, const MeetParams& m, const ChunkLaunch& l,
                        hipStream_t s);

// The row movers' arguments hold what the host knows of a batch: N entries of a
// table that ends at 4 KB, or as many as stay under kSmallArgs.
struct CachePools {
  char* k;
  char* v;
  int64_t layer_bytes;
  int32_t st_bytes, sh_bytes;          // token and head strides inside a page
  int32_t num_pages, page_tokens;
  int32_t heads, row_units;            // a head's row in 16-byte units
};

// What the launches go by.
struct MoveLaunch {
  int32_t layers;                      // moved by this call, from k / v on
  bool stream;                         // the call writes kMoveStream bytes or more
};
// Where the streaming hint on the stores begins to pay (the Infinity Cache
// holds 256 MB): 276 MB of new rows 94 us with it against 107 without, 126 MB
// whose accepted paths are moved next 62 against 60.
constexpr int64_t kMoveStream = (int64_t)192 << 20;
// The same for rotated rows, queries among them (164 MB 62 us with it, 70 without).
constexpr int64_t kTurnStream = (int64_t)128 << 20;

// A run of one request's new rows: `n` rows from its logical row `pos` on,
// from row `row` of the new arrays on.
struct AppendSegment {
  int32_t req, pos, row, n;
};
constexpr int kMoveLog = 4, kMoveRows = 1 << kMoveLog;       // rows of one work-group (divides a page)
constexpr int kTurnLog = 2, kTurnRows = 1 << kTurnLog;       // of one that rotates them, at most (two in small batches)
// Where four rows a work-group begin to pay: 960 rows of 24 KB 7.6 us with two
// and 10.8 with four, 13300 of them 60.6 and 58.7.
constexpr int64_t kManyTurned = 4096;
constexpr int kMaxTurned = 256;        // pairs of a head that it rotates
constexpr int kMoveSegments = 240;

template <int N>
struct AppendParams {
  CachePools c;
  const char* k_new;
  const char* v_new;
  const int32_t* bt;
  int64_t new_sl, new_st;              // bytes
  int32_t new_sh;                      // 16-byte units
  int32_t bt_stride;
  AppendSegment seg[N];
};

// Appended rows with the rotation: the queries' rows beside them (null: none).
template <int N>
struct RotateParams {
  CachePools c;
  const char* k_new;
  const char* v_new;
  const char* q;
  char* q_out;
  const int32_t* bt;
  const float* freq;                   // [pairs]
  const int32_t* positions;            // of the packed rows; null: their logical rows
  int64_t new_sl, new_st, q_st, out_st;     // bytes
  int32_t new_sh, q_sh, out_sh;             // 16-byte units
  int32_t bt_stride;
  int32_t q_heads, pairs;
  int32_t rows;                        // of a work-group: 2 or 4
  AppendSegment seg[N];
};

constexpr int kMoveTrees = 64;

template <int N>
struct CommitParams {
  CachePools c;
  const int32_t* bt;
  const int32_t* accepted;             // of the block's first request
  int32_t bt_stride;
  int32_t shared;                      // one topology: parent[0], nodes[0] for every request
  int32_t ctx[N];
  int8_t parent[N][32];
  int8_t nodes[N];
};

struct PagePair {
  int32_t src, dst, tokens;
};
constexpr int kMovePages = 256, kMovePagesSmall = 5;

template <int N>
struct PageCopyParams {
  CachePools c;
  PagePair pair[N];
};

static_assert(sizeof(AppendParams<kMoveSegments>) <= 4096 && sizeof(RotateParams<kMoveSegments>) <= 4096 && sizeof(CommitParams<kMoveTrees>) <= 4096 &&
                  sizeof(PageCopyParams<kMovePages>) <= 4096, "kernel arguments");
static_assert(sizeof(AppendParams<1>) <= kSmallArgs && sizeof(CommitParams<1>) <= kSmallArgs &&
                  sizeof(PageCopyParams<kMovePagesSmall>) <= kSmallArgs, "small arguments");

// The first n entries of p's table; an append's segments have at most `parts`
// work-groups of kMoveRows (kTurnRows) rows.
hipError_t launch_append(const AppendParams<kMoveSegments>& p, int n, int parts, const MoveLaunch& l, hipStream_t s);
hipError_t launch_rotate(const RotateParams<kMoveSegments>& p, int n, int parts, const MoveLaunch& l, bool f32,
                         bool interleaved, hipStream_t s);
hipError_t launch_commit(const CommitParams<kMoveTrees>& p, int n, const MoveLaunch& l, hipStream_t s);
hipError_t launch_page_copy(const PageCopyParams<kMovePages>& p, int n, const MoveLaunch& l, hipStream_t s);

}  // namespace sv
