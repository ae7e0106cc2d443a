// Attention of a chunk of new tokens over a paged KV cache, for gfx950.
//
// With s_rt = scale q_r . k_t over the keys t that row r sees,
//   out_r = sum_t 2^(s_rt log2 e - m_r) v_t / sum_t 2^(s_rt log2 e - m_r),
// one pass over the keys with a running reference m_r and sum l_r (fp32).
//
// What bounds it, by the query rows that read a KV head's keys (d = 128; times
// of a whole call, those under 20 us in a row):
//   few: HBM.  64 single tokens over 512-8192 rows, 8 KV heads under 32 query
//     heads (1.16 GB): 191 us, 6.1 TB/s (a plain read stream reaches 6.5); one
//     over 1000 rows (4 MB): 11-15 us, two launches of 7.8 and 4.1.
//   many: the matrix cores, at the clock that their power leaves (1.67-1.75 GHz).
//     1024 tokens over 30011 rows, 8 heads a group (1.02 TFLOP): 902-975 us,
//     1.05-1.13 PFLOP/s, MFMA busy 61-64 % (the library's 8192^3 product 1.2).
//     2048 without a context, 4 heads a group (34 GFLOP): 46 us, 0.75 PFLOP/s: the
//     longest row tile's 32 key tiles, 1.1-1.2 us each on a compute unit that the
//     shorter ones have left (0.94 where two row tiles share it), and the start.
//   both: 8 chunks of 33-700 tokens and 16 single ones, 32 heads of their own
//     (671 MB, 73 GFLOP): 151 us, 4.5 TB/s; MFMA busy 33 %, a fifth of it for the
//     empty rows of partly filled tiles.
// An fp32 output has three products with V for one: 16 requests of 1-400 tokens
// over 0-1500 rows, d = 64: 38 us, MFMA busy 31 %, 1.2 waves a SIMD on average:
// the longest items' 28 key tiles (a unit's mean share is 25) outlast the rest.
#include "sv_chunk.h"

#include <type_traits>

namespace sv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(4))) const int32_t const_int32;

template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    static_for<B + 1, E>(f);
  }
}

// vmcnt(N), the other counters left alone
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// A barrier that leaves the tile transfers in flight (__syncthreads() would
// wait for them).
__device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A tile in LDS: K then V, TK rows of D bf16 each, 16-byte chunk c of row r at
// chunk slot c ^ swk(r) (K) or c ^ swv(r) (V).  K is read by rows, 16 lanes
// taking the same chunk of 16 rows (16 different slots); V by the transposing
// read, 32 lanes taking 64 bytes of 4 rows (4 different 64-byte slots).
template <int D, int TK>
struct Tile {
  static constexpr int ROWB = D * 2;
  static constexpr int CH = ROWB / 16;
  static constexpr int HALF = 32 * ROWB;      // 32 rows: what lies in one page
  static constexpr int MAT = TK * ROWB;
  static constexpr int STAGE = 2 * MAT;
  static constexpr int RPI = 1024 / ROWB;     // rows of one transfer (64 lanes x 16 bytes)
  static constexpr int T = 32 / RPI;          // transfers of a 32-row half
  static constexpr int NOFF = D == 128 ? 4 : 2;   // transfers after which K's swizzle comes round
};
template <int D>
__device__ __forceinline__ int swk(int r) {
  return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int swv(int r) {
  return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
}

// How a tile's transfers are dealt to NW waves: `UNITS` (matrix, half) pairs
// of T transfers, one or more whole units a wave.
template <int D, int TK, int NW>
struct Deal {
  static constexpr int UNITS = 2 * (TK / 32);
  static_assert(UNITS % NW == 0, "whole units per wave");
  static constexpr int U = UNITS / NW;
  static constexpr int PER = U * Tile<D, TK>::T;
};

// What a wave needs to fetch its units of any tile.
struct Fetch {
  const char* k;             // this KV head's rows of page 0
  const char* v;
  const int32_t* pages;      // the request's page ids
  int64_t page_bytes;
  int32_t page_tokens, num_pages, row_bytes;
  int32_t ke;
};

// Lane l's 32-key block b + l of the item (from key kb on): its page, and the
// place in it of its first key (those of the item's last block for blocks
// behind it).  kb and a page's tokens are multiples of 32, so a block's 32 rows
// lie in one page: whatever of them a transfer's bounds let through is memory of
// the pool.
// One load and one division serve 64 blocks; a step reads its block's by lane.
// (A scalar load a step had its latency in every step.)
struct Window {
  int b;
  int pg, place;
};
__device__ __forceinline__ void look(Window& x, const Fetch& f, int kb, int b, int lane) {
  const int t = min(kb + 32 * (b + lane), (f.ke - 1) & ~31);
  const int i = t / f.page_tokens;
  x.b = b;
  x.place = t - i * f.page_tokens;
  x.pg = min(max(f.pages[i], 0), f.num_pages - 1);
}

// The page of key t.
__device__ __forceinline__ int page_of(const Fetch& f, int t) {
  const int i = __builtin_amdgcn_readfirstlane(min(t, f.ke - 1) / f.page_tokens);
  const int pg = ((const const_int32*)f.pages)[i];
  return __builtin_amdgcn_readfirstlane(min(max(pg, 0), f.num_pages - 1));
}

// The query rows of one wave: 32 rows, lane l holding row l % 32 (both halves
// of the wave the same rows), the running softmax and O^T.
template <int D>
struct Rows {
  bf16x8 q[D / 16];          // q[ks]: elements 16 ks + 8 (l / 32) .. + 7
  f32x16 o[D / 32];          // o[eb][i]: column 32 eb + 8 (i / 4) + 4 (l / 32) + i % 4
  float m, l;                // reference (log2 units) and this half's sum
  int32_t last;              // the row's last visible key
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int eb = 0; eb < D / 32; ++eb)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[eb][i] = 0.f;
  }
};
template <int D>
__device__ __forceinline__ bool has_nan(const Rows<D>& S) {
  bool bad = false;
#pragma unroll
  for (int eb = 0; eb < D / 32; ++eb)
#pragma unroll
    for (int i = 0; i < 16; ++i) bad |= S.o[eb][i] != S.o[eb][i];
  return bad;
}

// Work-group b's work: keys [kb, ke) of one request and KV head, `rows` query
// rows from r0 on, the partial rows from `part` on (-1: it writes out itself).
struct Piece {
  int32_t req, kvh, r0, rows, kb, ke, ctx, q0;
  int64_t part;
};
// A row tile's work-groups are next to each other, those of a piece (HEADS: the
// XCDs read different heads) or of a head (a head's keys stream past in order).
template <bool HEADS>
__device__ __forceinline__ Piece piece_of(const ChunkParams& p, int b) {
  if (b >= p.turn0 && b < p.turn1) b = p.turn0 + p.turn1 - 1 - b;
  const int i = b / p.Hkv;
  const ChunkItem x = p.items[i];                        // some piece of the tile
  const int g = b - (i - x.piece) * p.Hkv;               // the work-group's place among the tile's
  const int h = HEADS ? b - i * p.Hkv : g / x.pieces;
  const int s = HEADS ? x.piece : g - h * x.pieces;
  const int kb = s * x.len;
  return {x.req, h, x.r0, x.rows, kb, min(x.keys, kb + x.len), x.ctx, x.q0,
          x.pieces > 1 ? x.part + ((int64_t)h * x.pieces + s) * x.rows : -1};
}

// Rows wr0 .. wr0 + 31 of the item (past its last: that one again).
template <int D>
__device__ __forceinline__ void load_rows(Rows<D>& S, const ChunkParams& p, const Piece& it, int wr0, int l32,
                                          int half) {
  const int r = it.r0 + min(wr0 + l32, it.rows - 1);
  const int j = r / p.G;
  const int h = it.kvh * p.G + (r - j * p.G);
  const char* src =
      static_cast<const char*>(p.q) + ((it.q0 + (int64_t)j) * p.q_st + (int64_t)h * p.q_sh) * 2 + half * 16;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) S.q[ks] = *reinterpret_cast<const bf16x8*>(src + ks * 32);
  S.last = min(it.ctx + j, it.ke - 1);
}
// The last key that one of them sees.
__device__ __forceinline__ int last_seen(const ChunkParams& p, const Piece& it, int wr0) {
  return min(it.ctx + (it.r0 + min(wr0 + 31, it.rows - 1)) / p.G, it.ke - 1);
}

template <int D, bool F32>
__device__ __forceinline__ void write_out(const ChunkParams& p, const Piece& it, const Rows<D>& S, int wr0, int l32,
                                          int half) {
  constexpr int ET = D / 32;
  const float l = S.l + __shfl_xor(S.l, 32);
  if (wr0 + l32 >= it.rows) return;
  const int r = it.r0 + wr0 + l32;
  if (it.part < 0) {
    const int j = r / p.G;
    const int64_t row = (it.q0 + (int64_t)j) * (p.Hkv * p.G) + it.kvh * p.G + (r - j * p.G);
    const float inv = 1.f / l;
#pragma unroll
    for (int eb = 0; eb < ET; ++eb)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int e = 32 * eb + 2 * i + 4 * half;
        const f32x4 y = {S.o[eb][i] * inv, S.o[eb][i + 1] * inv, S.o[eb][i + 2] * inv, S.o[eb][i + 3] * inv};
        if constexpr (F32) {
          *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row * D + e) = y;
        } else {
          *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + row * D + e) =
              __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
        }
      }
  } else {
    const int64_t row = it.part + wr0 + l32;
#pragma unroll
    for (int eb = 0; eb < ET; ++eb)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(p.part + row * D + 32 * eb + 2 * i + 4 * half) =
            f32x4{S.o[eb][i], S.o[eb][i + 1], S.o[eb][i + 2], S.o[eb][i + 3]};
    if (half == 0) reinterpret_cast<float2*>(p.part)[-1 - row] = make_float2(S.m, l);
  }
}

// What another wave has of the same rows, joined to this one's.
template <int D>
__device__ __forceinline__ void join_rows(Rows<D>& S, float m1, float l1, const f32x4* o1) {
  const float m = fmaxf(S.m, m1), ref = m == -INFINITY ? 0.f : m;
  const float a = __builtin_amdgcn_exp2f(S.m - ref), b = __builtin_amdgcn_exp2f(m1 - ref);
  S.m = m;
  S.l = S.l * a + l1 * b;
#pragma unroll
  for (int eb = 0; eb < D / 32; ++eb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 y = o1[(eb * 4 + i) * 64];
#pragma unroll
      for (int n = 0; n < 4; ++n) S.o[eb][4 * i + n] = S.o[eb][4 * i + n] * a + y[n] * b;
    }
}


// The wave's rows over keys [t, last] one at a time, by the rows' own
// visibility: a value of a key that a row does not see never meets the row, not
// even as a product with zero.
template <int D>
__device__ __forceinline__ void one_by_one(const Fetch& f, Rows<D>& S, int t, int last, float c, int half) {
  for (; t <= last; ++t) {
    const int64_t at = page_of(f, t) * f.page_bytes + (int64_t)(t % f.page_tokens) * f.row_bytes;
    const bf16x8* k = reinterpret_cast<const bf16x8*>(f.k + at) + half;
    const bf16x4* v = reinterpret_cast<const bf16x4*>(f.v + at) + half;
    float s = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const bf16x8 y = k[2 * ks];
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf((float)S.q[ks][i], (float)y[i], s);
    }
    s = (s + __shfl_xor(s, 32)) * c;
    const bool sees = t <= S.last;
    const float m = sees ? fmaxf(S.m, s) : S.m, ref = m == -INFINITY ? 0.f : m;
    const float alpha = __builtin_amdgcn_exp2f(S.m - ref), w = sees ? __builtin_amdgcn_exp2f(s - ref) : 0.f;
    S.m = m;
    S.l = S.l * alpha + (half ? 0.f : w);
#pragma unroll
    for (int eb = 0; eb < D / 32; ++eb)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const bf16x4 y = v[(32 * eb + 2 * i) / 4];
#pragma unroll
        for (int n = 0; n < 4; ++n) S.o[eb][i + n] = S.o[eb][i + n] * alpha + (sees ? w * (float)y[n] : 0.f);
      }
  }
}

}  // namespace

// ---------------------------------------------------------------------------
// One work-group of NW waves per item, 32 query rows a wave; TK-key tiles of K
// and V go HBM -> LDS through an NS-stage ring of direct transfers (no
// registers between), every wave reads every tile:
//   S^T[key, row] = K[key, :] . Q[row, :]     v_mfma_f32_32x32x16_bf16, K as A
//   softmax over the keys                      fp32
//   O^T[e, row] += V^T[e, key] . P^T[key, row] V^T by transposing LDS reads
// Rows are on the MFMA's columns in both products, so that a row's maximum, sum
// and factor are one lane's (and its partner's 32 lanes on), and the operand
// that all waves share is the one read from LDS.  Four waves a work-group and
// 64-key tiles (128 KB of LDS for the two on a compute unit) where a KV head has
// more than 32 query rows, else one wave, 32-key tiles and five work-groups a
// compute unit (d = 64: three and ten).  Long case above: 64 rows a wave 1197 us (the accumulators move
// between register files), eight waves 928 (a 2048-token prompt 71 for 46),
// 32-key tiles in four stages 1000, 64-row work-groups 1089.
// MFMA row m of S^T holds key 16 (m >> 4) + 8 ((m >> 2) & 1) + 4 ((m >> 3) & 1)
// + (m & 3) of its 32 keys: the C layout then leaves lane half h the keys 16 x
// + 8 h + 0 .. 7 of its row in registers 8 x .. 8 x + 7, which is the B operand
// of the second product as it is.
// Stage j of the ring holds K of tile j and V of tile j - 1: step t takes the
// scores of tile t + 1 (matrix cores) beside the softmax of tile t (vector
// units), then the product with V of tile t.
// PARTS: bf16 parts a probability is carried in, p = p1 + p2 + p3, each the
// rounding of what the ones before leave: half a step of bf16 is 2^-8, so one
// part is off by 2^-8 p at most, two by 2^-16 p, three by 2^-24 p.  An fp32
// output takes three.  A bf16 output rounds by 2^-8 itself.  With up to 32 rows
// a KV head (the keys' bytes are what the kernel waits for) it takes two parts,
// which add nothing to that and cost no time to speak of (64 single tokens over
// 512-8192 rows 190.0 -> 190.8 us, one over 1000 11.4 -> 11.5).  Beyond, where
// the matrix cores bound it, a second part is half as much work again (1024
// tokens over 30011 rows 887 -> 1197 us, 2048 without a context 46.4 -> 56.7, 8
// chunks beside 16 single tokens 150 -> 169), for an error of 0.0016 of the
// row's norm in place of 0.0021-0.0024, and it takes one: who needs the better
// product there asks for an fp32 output.
// ---------------------------------------------------------------------------
template <int D, int NW, int TK, int PARTS>
struct Chunk {
  using TL = Tile<D, TK>;
  using DL = Deal<D, TK, NW>;
  static constexpr int KS = D / 16, ET = D / 32, KB = TK / 32;
  // Cache policy of the transfers.  One wave's rows are all that read these keys:
  // nt, the streaming hint (64 single tokens over 512-8192 rows 217 -> 190 us);
  // larger tiles' keys are read again by the request's other tiles.
  static constexpr int CPOL = NW == 1 ? 2 : 0;
  static_assert(DL::U == 1 || KB == 1, "a wave's units are one, or K and V of a 32-key tile");
  template <int N>
  struct ScoresOf {            // N blocks of 32 keys
    f32x16 s[N];
  };
  using Scores = ScoresOf<KB>;
  // The addresses of a lane's reads and transfers.
  struct Lane {
    uint32_t koff[KS];         // K operand: chunk 2 ks + lane half of the lane's key row (keys 32.. : + HALF)
    uint32_t voff[ET];         // V operand: the transposing read's place (keys 16 kk ..: + 16 kk rows)
    uint32_t off[TL::NOFF];    // transfer x of a half: lane's row among its RPI and its swizzled chunk, by x % NOFF
    uint32_t offv;             // the same for V where a wave fetches both
  };

  // Unit u of wave w: V after K, the halves in order.
  static __device__ __forceinline__ bool unit_is_v(int w, int u) { return w * DL::U + u >= KB; }
  static __device__ __forceinline__ int unit_half(int w, int u) {
    const int x = w * DL::U + u;
    return x >= KB ? x - KB : x;
  }

  // The block (of 32 keys from the item's first on) that unit 0 fetches for
  // stage j; a second unit is V of the tile before.
  static __device__ __forceinline__ int block_of(int j, int w) {
    return KB * max(unit_is_v(w, 0) ? j - 1 : j, 0) + unit_half(w, 0);
  }

  // The wave's units of stage j: K of tile j, V of tile j - 1 (tiles begin at
  // key kb).  Rows past the item's end, and tiles that it does not have, are
  // past the buffer's records (a raw buffer's bounds check takes the scalar
  // offset in, measured on gfx950 by loads with the offset below, at and past the
  // records' end): they come as zeros.  Nothing rests on that but time: without
  // it they would be rows of the same block, which are masked, and a NaN among
  // them would send the rows through the fallback below.
  template <int POL = CPOL>
  static __device__ __forceinline__ void issue(lds_char* stage, const Fetch& f, int j, int kb, const Window& win,
                                               int2& before, int w, const Lane& A) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int bl = block_of(j, w) - win.b;
    const int2 now = make_int2(__builtin_amdgcn_readlane(win.pg, bl), __builtin_amdgcn_readlane(win.place, bl));
#pragma unroll
    for (int u = 0; u < DL::U; ++u) {
      const bool isv = unit_is_v(w, u);
      const int half = unit_half(w, u);
      const int tile = isv ? j - 1 : j;
      const int2 at_page = u == 0 ? now : before;
      const int rows = tile < 0 ? 0 : min(f.ke - (kb + TK * tile + 32 * half), 32);
      const char* src = (isv ? f.v : f.k) + (int64_t)at_page.x * f.page_bytes;
      const int soff = at_page.y * f.row_bytes;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          (void*)src, 0, rows > 0 ? soff + (rows - 1) * f.row_bytes + TL::ROWB : 0, 0x00020000);
      lds_char* dst = stage + (isv ? TL::MAT : 0) + half * TL::HALF;
#pragma unroll
      for (int x = 0; x < TL::T; ++x)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst + x * 1024), 16, at(A, u, x),
                                                 soff + x * TL::RPI * f.row_bytes, 0, POL);
    }
    before = now;
#endif
  }
  static __device__ __forceinline__ uint32_t at(const Lane& A, int u, int x) {
    if constexpr (DL::U > 1) return u > 0 ? A.offv : A.off[x % TL::NOFF];
    else return A.off[x % TL::NOFF];
  }

  template <int N = KB>
  static __device__ __forceinline__ ScoresOf<N> scores(const lds_char* cur, const Rows<D>& S, const Lane& A) {
    ScoresOf<N> r;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int kb = 0; kb < N; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) r.s[kb][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 a = *(lds_bf16x8*)(cur + A.koff[ks] + kb * TL::HALF);
        r.s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, S.q[ks], r.s[kb], 0, 0, 0);
      }
    }
#endif
    return r;
  }

  // Keys that the row does not see, of the tile starting at key t0.
  template <int N>
  static __device__ __forceinline__ void mask(ScoresOf<N>& x, const Rows<D>& S, int t0, int half) {
    const int lim = S.last - t0 - 8 * half;
#pragma unroll
    for (int kb = 0; kb < N; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) x.s[kb][i] = 32 * kb + 16 * (i >> 3) + (i & 7) <= lim ? x.s[kb][i] : -INFINITY;
  }

  template <int N>
  static __device__ __forceinline__ float largest(const ScoresOf<N>& x) {
    float top = x.s[0][0];
#pragma unroll
    for (int kb = 0; kb < N; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x.s[kb][i]);
    return top;
  }
  // The reference trails the running maximum by at most kLag (log2 units), so
  // p <= 2^kLag and most tiles leave O and l alone.  Returns what to subtract
  // for a tile whose largest score in this lane is `top`.
  static __device__ __forceinline__ float reference(float top, Rows<D>& S, float c) {
    constexpr float kLag = 8.f;
    top *= c;
    if (__any(top > S.m + kLag)) {                       // wave-uniform
      const float both = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(S.m, both);
      const float alpha = m_new == S.m ? 1.f : __builtin_amdgcn_exp2f(S.m - m_new);
      S.l *= alpha;
#pragma unroll
      for (int eb = 0; eb < ET; ++eb) S.o[eb] *= alpha;
      S.m = m_new;
    }
    return S.m == -INFINITY ? 0.f : S.m;
  }

  template <int N>
  struct Probs {
    uint32_t p[PARTS][N * 8];
  };
  template <int N>
  static __device__ __forceinline__ Probs<N> weights(const ScoresOf<N>& x, Rows<D>& S, float c, float ref) {
    Probs<N> P;
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int kb = 0; kb < N; ++kb)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        float x0 = __builtin_amdgcn_exp2f(fmaf(x.s[kb][i], c, -ref));
        float x1 = __builtin_amdgcn_exp2f(fmaf(x.s[kb][i + 1], c, -ref));
        sum0 += x0;
        sum1 += x1;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x0, x1}, bf16x2));
          P.p[part][kb * 8 + i / 2] = h;
          if (part + 1 < PARTS) {
            x0 -= __uint_as_float(h << 16);
            x1 -= __uint_as_float(h & 0xffff0000u);
          }
        }
      }
    S.l += sum0 + sum1;
    return P;
  }

  template <int N>
  static __device__ __forceinline__ bf16x8 p_operand(const uint32_t (&p)[N], int kk) {
    return __builtin_bit_cast(bf16x8, (u32x4){p[4 * kk], p[4 * kk + 1], p[4 * kk + 2], p[4 * kk + 3]});
  }

  // Eight keys of the lane's column: two transposing reads of four.
  static __device__ __forceinline__ bf16x8 v_operand(const lds_char* cur, uint32_t at) {
#if defined(__HIP_DEVICE_COMPILE__)
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(cur + at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(cur + at + 4 * TL::ROWB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#else
    (void)cur;
    (void)at;
    return bf16x8{};
#endif
  }

  template <int N>
  static __device__ __forceinline__ void product(const lds_char* cur, const Probs<N>& P, Rows<D>& S, const Lane& A) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int kk = 0; kk < 2 * N; ++kk)
#pragma unroll
      for (int eb = 0; eb < ET; ++eb) {
        const bf16x8 a = v_operand(cur, A.voff[eb] + kk * 16 * TL::ROWB);
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
          S.o[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p_operand(P.p[part], kk), S.o[eb], 0, 0, 0);
      }
#endif
  }

  // Step t of a wave whose rows see all of tile t: the transfers of stage
  // t + NS, the scores of tile t + 1 and their largest, the softmax and product
  // of tile t.  The stage written and the one read are different ones, which
  // the parameters say (restrict): without it the compiler waits for the
  // transfers before every read.
  static __device__ __forceinline__ void step(lds_char* __restrict__ nxt, const lds_char* __restrict__ cur,
                                              const Fetch& f, int jn, int kb, const Window& win, int2& before, int w,
                                              const Lane& A, Rows<D>& S, Scores& x, float& top, float c) {
    const float ref = reference(top, S, c);
    issue(nxt, f, jn, kb, win, before, w, A);
    const Scores y = scores(cur, S, A);
    const auto P = weights(x, S, c, ref);
    product(cur, P, S, A);
    top = largest(y);
    x = y;
  }
  // The same where they may not (see 0: none of its keys).
  static __device__ __forceinline__ void edge_step(lds_char* __restrict__ nxt, const lds_char* __restrict__ cur,
                                                   bool more, const Fetch& f, int jn, int kb, const Window& win,
                                                   int2& before, int w, const Lane& A, Rows<D>& S, Scores& x,
                                                   float& top, int t0, bool see, bool see_next, float c, int lane) {
    if (more) issue(nxt, f, jn, kb, win, before, w, A);
    __builtin_amdgcn_sched_barrier(0);
    if (see) {
      mask(x, S, t0, lane >> 5);
      const float ref = reference(largest(x), S, c);
      const auto P = weights(x, S, c, ref);
      product(cur, P, S, A);
    }
    if (see_next) x = scores(cur, S, A);
  }
  // The key of a 32-key block that lane l32 holds for the first product.
  static __device__ __forceinline__ int key_of(int l32) {
    return 16 * (l32 >> 4) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
  }
  // Where a lane reads its operands of both products (the layouts above).
  static __device__ __forceinline__ void places(Lane& A, int l32, int half, int lane) {
    const int key = key_of(l32);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) A.koff[ks] = (uint32_t)(key * TL::ROWB + (((2 * ks + half) ^ swk<D>(key)) * 16));
    const int s = lane & 15, row = 8 * half + (s >> 2);
#pragma unroll
    for (int eb = 0; eb < ET; ++eb) {
      const int ch = 4 * eb + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
      A.voff[eb] = (uint32_t)(TL::MAT + row * TL::ROWB + ((ch ^ swv<D>(row)) * 16) + (s & 1) * 8);
    }
  }
  // The wave's rows again, straight from the cache, where the products left a NaN
  // (a value of the item's V that is not finite, or a score that is NaN): an
  // unseen key's weight is zero, and zero times such a value is NaN.  Blocks that
  // all rows see whole (the first row does) have no unseen key and go through the
  // same products; only the rest, up to 31 keys of such a block, the rows' own
  // tokens and the last block, goes key by key.  1024 tokens over 30011 rows with
  // one NaN among the first keys, where every wave comes here: 3.9 ms for 0.94
  // (key by key over all of them 97 ms); 512 over 16000: 0.82 ms for 0.19 (23).
  static __device__ __forceinline__ void again(const Fetch& f, Rows<D>& S, int kb, int last, float c, int l32, int half) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int all = __builtin_amdgcn_readfirstlane(S.last);
    asm volatile("" : "+v"(l32), "+v"(half));          // none of the addresses below is held in the loops above
    S.clear();
    int t = kb;
    for (; t + 31 <= all; t += 32) {
      const int64_t at = page_of(f, t) * f.page_bytes + (int64_t)(t % f.page_tokens) * f.row_bytes;
      const char* k = f.k + at + (int64_t)key_of(l32) * f.row_bytes + half * 16;
      const char* v = f.v + at + (int64_t)(8 * half) * f.row_bytes + l32 * 2;
      ScoresOf<1> x;
#pragma unroll
      for (int i = 0; i < 16; ++i) x.s[0][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        x.s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(k + ks * 32), S.q[ks], x.s[0],
                                                         0, 0, 0);
      const float ref = reference(largest(x), S, c);
      const auto P = weights(x, S, c, ref);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        __builtin_amdgcn_sched_barrier(0);               // no more loads under way than there are registers
#pragma unroll
        for (int eb = 0; eb < ET; ++eb) {
          s16x8 a;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            a[i] = *reinterpret_cast<const short*>(v + (int64_t)(16 * kk + i) * f.row_bytes + eb * 64);
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
            S.o[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), p_operand(P.p[part], kk),
                                                              S.o[eb], 0, 0, 0);
        }
      }
    }
    one_by_one<D>(f, S, t, last, c, half);
#endif
  }
  // Step t of a wave that has 32 keys of every second tile, `cur` moved to them
  // (mine: of tile t, whose scores it has; else it takes the scores of tile t + 1).
  static __device__ __forceinline__ void shared_step(lds_char* __restrict__ nxt, const lds_char* __restrict__ cur,
                                                     bool more, const Fetch& f, int jn, int kb, const Window& win,
                                                     int2& before, int w, const Lane& A, Rows<D>& S, ScoresOf<1>& x,
                                                     bool mine, int t0, float c, int lane) {
    if (more) issue<2>(nxt, f, jn, kb, win, before, w, A);
    __builtin_amdgcn_sched_barrier(0);
    if (mine) {
      mask(x, S, t0, lane >> 5);
      const float ref = reference(largest(x), S, c);
      const auto P = weights(x, S, c, ref);
      product(cur, P, S, A);
    } else {
      x = scores<1>(cur, S, A);
    }
  }
  // A whole item of up to 32 rows, all that read its keys: every wave has the
  // rows, and 32 keys of every second tile, so that no wave idles and the step is
  // short beside the other work-group's; the streaming hint as for low tiles.  8
  // chunks of 33-700 tokens and 16 single ones, 32 heads of their own: 158 us
  // with wave 0 at all keys, 156 shared, 149 with the hint; 4 chunks of 512 and 44
  // single ones, 8 of 32 heads: 133, 127.
  template <int NS>
  static __device__ __forceinline__ bool shared_rows(const ChunkParams& p, const Piece& it, const Fetch& f, Lane& A,
                                                     Window& win, char* lds, int ntiles, int w, int lane, Rows<D>& S) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int ET = D / 32;
    const int l32 = lane & 31, half = lane >> 5;
    lds_char* ring = (lds_char*)lds;
    int2 before = make_int2(0, 0);
    load_rows(S, p, it, 0, l32, half);
#pragma unroll
    for (int j = 0; j < NS; ++j) issue<2>(ring + j * TL::STAGE, f, j, it.kb, win, before, w, A);
    S.clear();
    places(A, l32, half, lane);
    wait_vm<(NS - 1) * DL::PER>();
    tile_barrier();
    const int hb = w & 1, par = w >> 1;
    ScoresOf<1> x = scores<1>(ring + hb * TL::HALF, S, A);
    for (int t = 0; t < ntiles; ++t) {
      wait_vm<0>();
      tile_barrier();
      if (block_of(t + NS, w) >= win.b + 64) look(win, f, it.kb, block_of(t + NS, w), lane);
      shared_step(ring + (t % NS) * TL::STAGE, ring + ((t + 1) % NS) * TL::STAGE + hb * TL::HALF, t + NS <= ntiles, f,
                  t + NS, it.kb, win, before, w, A, S, x, (t & 1) == par, it.kb + TK * t + 32 * hb, p.scale_log2, lane);
    }
    wait_vm<0>();
    // The waves' shares meet in wave 0, the ring their place; a maximum that is NaN
    // tells that O has one.  (A vote of the work-group by __syncthreads_or has an
    // LDS variable of its own: with a second one the compiler no longer tells the
    // stages apart and waits for the transfers before every read, 49 -> 57 us for
    // a prompt of 2048.)
    bool bad = __any(has_nan(S));
    f32x4* at = reinterpret_cast<f32x4*>(lds) + lane;
    float2* ml = reinterpret_cast<float2*>(lds + (NW - 1) * D * 128) + lane;
    __syncthreads();
    if (w > 0) {
      at += (w - 1) * D * 8;
#pragma unroll
      for (int eb = 0; eb < ET; ++eb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          at[(eb * 4 + i) * 64] = f32x4{S.o[eb][4 * i], S.o[eb][4 * i + 1], S.o[eb][4 * i + 2], S.o[eb][4 * i + 3]};
      ml[(w - 1) * 64] = make_float2(bad ? NAN : S.m, S.l);
    }
    __syncthreads();
    if (w > 0) return false;
    for (int k = 0; k < NW - 1; ++k) {
      const float2 y = ml[k * 64];
      bad |= y.x != y.x;
      join_rows<D>(S, y.x, y.y, at + k * D * 8);
    }
    return bad;
#else
    return false;
#endif
  }
};

// (d = 64: three waves a SIMD.)
template <int D, int NW, int TK, int NS, int PARTS, bool F32>
__global__ __launch_bounds__(64 * NW, D == 64 ? 3 : 2) void chunk_attn(ChunkParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the host pass needs the signature only
  using C = Chunk<D, NW, TK, PARTS>;
  using TL = Tile<D, TK>;
  using DL = Deal<D, TK, NW>;
  __shared__ __attribute__((aligned(1024))) char lds[NS * TL::STAGE];

  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const Piece it = piece_of<NW != 1>(p, blockIdx.x);
  const int ntiles = (it.ke - it.kb + TK - 1) / TK;

  Fetch f;
  f.k = static_cast<const char*>(p.k) + (int64_t)it.kvh * p.kv_sh * 2;
  f.v = static_cast<const char*>(p.v) + (int64_t)it.kvh * p.kv_sh * 2;
  f.pages = p.bt + (int64_t)it.req * p.bt_stride;
  f.row_bytes = p.kv_st * 2;
  f.page_tokens = p.page_tokens;
  f.page_bytes = (int64_t)p.page_tokens * f.row_bytes;
  f.num_pages = p.num_pages;
  f.ke = it.ke;
  typename C::Lane A;
#pragma unroll
  for (int x = 0; x < TL::NOFF; ++x) {
    const int row = x * TL::RPI + lane / TL::CH, ch = lane % TL::CH;
    const int sw = C::unit_is_v(w, 0) ? swv<D>(row) : swk<D>(row);
    A.off[x] = (uint32_t)(lane / TL::CH * f.row_bytes + ((ch ^ sw) * 16));
    A.offv = (uint32_t)(lane / TL::CH * f.row_bytes + ((ch ^ swv<D>(row)) * 16));   // the same for every x
  }
  Window win;
  look(win, f, it.kb, 0, lane);
  int2 before = make_int2(0, 0);                         // a second unit's: what the first had last

  lds_char* ring = (lds_char*)lds;
  // A request of few rows in a batch of tall tiles: its rows on every wave.  (Not
  // for d = 64, where the registers of both ways leave two work-groups a compute
  // unit and not three: 16 requests of 1-400 tokens 44 us for 41.)
  const bool shared = NW == 4 && D == 128 && it.r0 == 0 && it.rows <= kChunkLowRows;
  const int wr0 = shared ? 0 : 32 * w;                   // the wave's first row of the item
  // the wave's last row's last key (none without rows)
  const int wave_sees = wr0 < it.rows ? last_seen(p, it, wr0) : -1;
  Rows<D> S;
  bool bad;
  if (!shared) {
    load_rows(S, p, it, wr0, l32, half);
#pragma unroll
    for (int j = 0; j < NS; ++j) C::issue(ring + j * TL::STAGE, f, j, it.kb, win, before, w, A);
    S.clear();
    C::places(A, l32, half, lane);
    const int all_see = min(it.ctx + it.r0 / p.G, it.ke - 1);    // the last key that the item's first row sees
    const int nfull = all_see + 1 >= it.kb ? (all_see + 1 - it.kb) / TK : 0;     // tiles that every row sees whole

    // stages 0 .. NS - 1 are under way: wait for stage 0 (K of tile 0)
    wait_vm<(NS - 1) * DL::PER>();
    tile_barrier();
    typename C::Scores x = C::scores(ring, S, A);
    float top = C::largest(x);
    // Step t: stage t + 1 has landed here and everywhere, and every wave has read
    // what it needs of stage t, where stage t + NS goes.
    int t = 0;
    if (wave_sees >= it.kb) {
      while (t + NS <= nfull) {
        if (C::block_of(t + 2 * NS - 1, w) >= win.b + 64) look(win, f, it.kb, C::block_of(t + NS, w), lane);
        static_for<0, NS>([&](auto st) {
          constexpr int ST = decltype(st)::value;
          wait_vm<(NS - 2) * DL::PER>();
          tile_barrier();
          C::step(ring + ST * TL::STAGE, ring + ((ST + 1) % NS) * TL::STAGE, f, t + ST + NS, it.kb, win, before, w, A,
                  S, x, top, p.scale_log2);
        });
        t += NS;
      }
    }
    for (; t < ntiles; ++t) {
      wait_vm<0>();
      tile_barrier();
      if (C::block_of(t + NS, w) >= win.b + 64) look(win, f, it.kb, C::block_of(t + NS, w), lane);
      const int t0 = it.kb + TK * t;
      C::edge_step(ring + (t % NS) * TL::STAGE, ring + ((t + 1) % NS) * TL::STAGE, t + NS <= ntiles, f, t + NS, it.kb,
                   win, before, w, A, S, x, top, t0, t0 <= wave_sees, t + 1 < ntiles && t0 + TK <= wave_sees,
                   p.scale_log2, lane);
    }
    wait_vm<0>();                                          // no transfer outlives the work-group's LDS
    bad = has_nan(S);
  } else {
    bad = C::template shared_rows<NS>(p, it, f, A, win, lds, ntiles, w, lane, S);
    if (w > 0) return;
  }
  if (__any(bad))
    C::again(f, S, it.kb, wave_sees, p.scale_log2, l32, half);
  write_out<D, F32>(p, it, S, wr0, l32, half);
#endif
}

// A running join of pieces: O = sum_s 2^(m_s - M) O_s, l alike, M = max_s m_s.
// A piece none of whose keys the row sees has m = -inf and adds nothing.
struct Joined {
  f32x4 o;
  float m, l;
  __device__ __forceinline__ void add(float m1, float l1, f32x4 o1) {
    const float M = fmaxf(m, m1), ref = M == -INFINITY ? 0.f : M;
    const float a = __builtin_amdgcn_exp2f(m - ref), b = __builtin_amdgcn_exp2f(m1 - ref);
    o = o * a + o1 * b;
    l = l * a + l1 * b;
    m = M;
  }
};

// The joins of cut row tiles, NG groups of D / 4 lanes a work-group: a row each
// where the tiles have few pieces (ROWS), else a row's pieces dealt to the
// groups, whose sums meet in LDS.  (A join by the last piece to end, in the
// kernel above, measured the same for one token over 1000 rows and 3 % slower
// for 64 of them: its stores and loads past the L2s cost what the launch does.)
template <int D, bool F32, bool ROWS>
__global__ __launch_bounds__(256) void chunk_join(JoinParams p) {
  constexpr int LPR = D / 4, NG = 256 / LPR;
  const int tile = (int)blockIdx.x / p.Hkv, kvh = (int)blockIdx.x - tile * p.Hkv;
  const ChunkJoin jn = p.joins ? p.joins[tile] : p.one;
  const int64_t part = jn.part + (int64_t)kvh * jn.pieces * jn.rows;
  const int g = threadIdx.x / LPR, x = threadIdx.x % LPR;
  const int rr = ROWS ? (int)blockIdx.y * NG + g : (int)blockIdx.y;
  if (!ROWS && rr >= jn.rows) return;
  Joined j = {f32x4{0.f, 0.f, 0.f, 0.f}, -INFINITY, 0.f};
  const int64_t first = part + min(rr, jn.rows - 1);
  const float2* ml = reinterpret_cast<const float2*>(p.part) - 1 - first;
  const float* po = p.part + first * D + 4 * x;
#pragma unroll 4
  for (int s = ROWS ? 0 : g; s < jn.pieces; s += ROWS ? 1 : NG) {
    const float2 y = ml[-(int64_t)s * jn.rows];
    j.add(y.x, y.y, *reinterpret_cast<const f32x4*>(po + (int64_t)s * jn.rows * D));
  }
  if constexpr (!ROWS) {
    __shared__ Joined lds[NG][LPR];
    lds[g][x] = j;
    __syncthreads();
    if (g > 0) return;
    for (int k = 1; k < NG; ++k) j.add(lds[k][x].m, lds[k][x].l, lds[k][x].o);
  } else if (rr >= jn.rows) {
    return;
  }
  const int r = jn.r0 + rr, tok = r / p.G;
  const int64_t at = ((jn.q0 + (int64_t)tok) * (p.Hkv * p.G) + kvh * p.G + (r - tok * p.G)) * D + 4 * x;
  const f32x4 y = j.o * (1.f / j.l);
  if constexpr (F32) *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = y;
  else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) =
      __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
}

template <int D, bool F32>
static hipError_t launch_d(const ChunkParams& p, const JoinParams& j, const ChunkLaunch& l, hipStream_t s) {
  if (l.tall) chunk_attn<D, 4, 64, 2, F32 ? 3 : 1, F32><<<dim3(l.n_items * p.Hkv), dim3(256), 0, s>>>(p);
  else chunk_attn<D, 1, 32, 2, F32 ? 3 : 2, F32><<<dim3(l.n_items * p.Hkv), dim3(64), 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || l.n_joins == 0) return e;
  constexpr int NG = 1024 / D;
  if (l.join_pieces <= 2 * NG)
    chunk_join<D, F32, true><<<dim3(l.n_joins * p.Hkv, (l.join_rows + NG - 1) / NG), dim3(256), 0, s>>>(j);
  else
    chunk_join<D, F32, false><<<dim3(l.n_joins * p.Hkv, l.join_rows), dim3(256), 0, s>>>(j);
  return hipGetLastError();
}

hipError_t launch_chunk(const ChunkParams& p, const JoinParams& j, const ChunkLaunch& l, hipStream_t s) {
  if (l.D == 128) return l.out_f32 ? launch_d<128, true>(p, j, l, s) : launch_d<128, false>(p, j, l, s);
  return l.out_f32 ? launch_d<64, true>(p, j, l, s) : launch_d<64, false>(p, j, l, s);
}

}  // namespace sv
