// Attention of a chunk of new tokens over a paged KV cache, for gfx950.
//
// With s_rt = scale q_r . k_t over the keys t that row r sees,
//   out_r = sum_t 2^(s_rt log2 e - m_r) v_t / sum_t 2^(s_rt log2 e - m_r),
// one pass over the keys with a running reference m_r and sum l_r (fp32).
#include "sv_chunk.h"

#include <type_traits>

namespace sv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
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
  const const_int32* table;  // the request's page ids
  int64_t page_bytes;
  int32_t page_tokens, num_pages, row_bytes;
  int32_t ke;
};

// The page of the 32-row half that starts at key t (clamped to the item).
__device__ __forceinline__ int page_of(const Fetch& f, int t) {
  const int i = __builtin_amdgcn_readfirstlane(min(t, f.ke - 1) / f.page_tokens);
  const int pg = f.table[i];
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
};

}  // namespace

// ---------------------------------------------------------------------------
// One work-group of NW waves per item, 32 query rows a wave; TK-key tiles of K
// and V go HBM -> LDS through an NS-stage ring of direct transfers (no
// registers between), every wave reads every tile:
//   S^T[key, row] = K[key, :] . Q[row, :]     v_mfma_f32_32x32x16_bf16, K as A
//   softmax over the keys                      fp32
//   O^T[e, row] += V^T[e, key] . P^T[key, row] V^T by transposing LDS reads
// MFMA row m of S^T holds key 16 (m >> 4) + 8 ((m >> 2) & 1) + 4 ((m >> 3) & 1)
// + (m & 3) of its 32 keys: the C layout then leaves lane half h the keys 16 x
// + 8 h + 0 .. 7 of its row in registers 8 x .. 8 x + 7, which is the B operand
// of the second product as it is.
// Stage j of the ring holds K of tile j and V of tile j - 1: step t takes the
// scores of tile t + 1 (matrix cores) beside the softmax of tile t (vector
// units), then the product with V of tile t.
// PARTS: bf16 parts a probability is carried in (1 for a bf16 output, 3 for
// an fp32 one: 24 bits).
// ---------------------------------------------------------------------------
template <int D, int NW, int TK, int PARTS>
struct Chunk {
  using TL = Tile<D, TK>;
  using DL = Deal<D, TK, NW>;
  static constexpr int KS = D / 16, ET = D / 32, KB = TK / 32;
  static_assert(DL::U == 1 || KB == 1, "a wave's units are one, or K and V of a 32-key tile");
  struct Scores {
    f32x16 s[KB];
  };
  // The addresses of a lane's reads and transfers.
  struct Lane {
    uint32_t koff[KS];         // K operand: chunk 2 ks + lane half of the lane's key row (keys 32.. : + HALF)
    uint32_t voff[ET];         // V operand: the transposing read's place (keys 16 kk ..: + 16 kk rows)
    uint32_t off[TL::T];       // transfers: row and swizzled chunk (one matrix a wave, or K and V by `flip`)
    uint32_t flip[DL::U > 1 ? TL::T : 1];
  };

  // Unit u of wave w: V after K, the halves in order.
  static __device__ __forceinline__ bool unit_is_v(int w, int u) { return w * DL::U + u >= KB; }
  static __device__ __forceinline__ int unit_half(int w, int u) {
    const int x = w * DL::U + u;
    return x >= KB ? x - KB : x;
  }

  // The wave's units of stage j: K of tile j, V of tile j - 1, whichever of
  // them the item has (tiles begin at key kb).
  static __device__ __forceinline__ void issue(lds_char* stage, const Fetch& f, int j, int kb, int ntiles,
                                               const int (&pg)[DL::U], int w, const Lane& A, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int u = 0; u < DL::U; ++u) {
      const bool isv = unit_is_v(w, u);
      const int half = unit_half(w, u);
      const int tile = isv ? j - 1 : j;
      if (tile < 0 || tile >= ntiles) continue;          // wave-uniform
      const int t = kb + TK * tile + 32 * half;
      const int tc = min(t, f.ke - 1);
      const int base = tc - tc % f.page_tokens;          // the page's first key
      const char* src = (isv ? f.v : f.k) + (int64_t)pg[u] * f.page_bytes;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          (void*)src, 0, (f.page_tokens - 1) * f.row_bytes + TL::ROWB, 0x00020000);
      lds_char* dst = stage + (isv ? TL::MAT : 0) + half * TL::HALF;
      if (t + 32 <= f.ke) {                              // wave-uniform
        const int soff = (t - base) * f.row_bytes;
#pragma unroll
        for (int x = 0; x < TL::T; ++x)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst + x * 1024), 16, at(A, u, x), soff, 0, 0);
      } else {                                           // rows past the end repeat the last one
#pragma unroll
        for (int x = 0; x < TL::T; ++x) {
          const int row = x * TL::RPI + lane / TL::CH;
          const uint32_t chunk = at(A, u, x) - (uint32_t)(row * f.row_bytes);
          const int key = min(t + row, f.ke - 1) - base;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst + x * 1024), 16,
                                                   (uint32_t)(key * f.row_bytes) + chunk, 0, 0, 0);
        }
      }
    }
#endif
  }
  static __device__ __forceinline__ uint32_t at(const Lane& A, int u, int x) {
    if constexpr (DL::U > 1) return u > 0 ? A.flip[x] : A.off[x];
    else return A.off[x];
  }

  static __device__ __forceinline__ Scores scores(const lds_char* cur, const Rows<D>& S, const Lane& A) {
    Scores r;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
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
  static __device__ __forceinline__ void mask(Scores& x, const Rows<D>& S, int t0, int half) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = t0 + 32 * kb + 16 * (i >> 3) + 8 * half + (i & 7);
        x.s[kb][i] = t <= S.last ? x.s[kb][i] : -INFINITY;
      }
  }

  // The reference trails the running maximum by at most kLag (log2 units), so
  // p <= 2^kLag and most tiles leave O and l alone.  Returns what to subtract.
  static __device__ __forceinline__ float reference(const Scores& x, Rows<D>& S, float c) {
    constexpr float kLag = 8.f;
    float top = x.s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, x.s[kb][i]);
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

  struct Probs {
    uint32_t p[PARTS][KB * 8];
  };
  static __device__ __forceinline__ Probs weights(const Scores& x, Rows<D>& S, float c, float ref) {
    Probs P;
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
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

  static __device__ __forceinline__ bf16x8 p_operand(const uint32_t (&p)[KB * 8], int kk) {
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

  static __device__ __forceinline__ void product(const lds_char* cur, const Probs& P, Rows<D>& S, const Lane& A) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int kk = 0; kk < 2 * KB; ++kk)
#pragma unroll
      for (int eb = 0; eb < ET; ++eb) {
        const bf16x8 a = v_operand(cur, A.voff[eb] + kk * 16 * TL::ROWB);
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
          S.o[eb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p_operand(P.p[part], kk), S.o[eb], 0, 0, 0);
      }
#endif
  }

  // Whether this lane's share of the tile's V holds an infinity or a NaN.
  static __device__ __forceinline__ bool bad_values(const lds_char* cur, const Lane& A) {
    uint32_t bad = 0;
#pragma unroll
    for (int kk = 0; kk < 2 * KB; ++kk)
#pragma unroll
      for (int eb = 0; eb < ET; ++eb) {
        const u32x4 a = __builtin_bit_cast(u32x4, v_operand(cur, A.voff[eb] + kk * 16 * TL::ROWB));
#pragma unroll
        for (int y = 0; y < 4; ++y)                      // exponents of all ones
          bad |= ((a[y] & 0x7f800000u) == 0x7f800000u) | ((a[y] & 0x7f80u) == 0x7f80u);
      }
    return bad != 0;
  }

  // The product where a value that is not finite stands in a tile of which
  // some row does not see all: key by key, so that a zero probability never
  // meets it.
  static __device__ __forceinline__ void careful_product(const lds_char* cur, const Probs& P, Rows<D>& S,
                                                         const Lane& A, int t0, int half) {
#if defined(__HIP_DEVICE_COMPILE__)
    for (int x = 0; x < TK; ++x) {
      const int kk = x >> 4;
      const bool mine = ((x >> 3) & 1) == half;
      u32x4 keep;
#pragma unroll
      for (int y = 0; y < 4; ++y) keep[y] = mine && ((x & 7) >> 1) == y ? ((x & 1) ? 0xffff0000u : 0xffffu) : 0u;
      const bool sees = t0 + x <= S.last;
#pragma unroll
      for (int eb = 0; eb < ET; ++eb) {
        const u32x4 a = __builtin_bit_cast(u32x4, v_operand(cur, A.voff[eb] + kk * 16 * TL::ROWB)) & keep;
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          u32x4 b = {0u, 0u, 0u, 0u};
#pragma unroll
          for (int k2 = 0; k2 < 2 * KB; ++k2)
#pragma unroll
            for (int y = 0; y < 4; ++y) b[y] = kk == k2 ? P.p[part][4 * k2 + y] : b[y];
          z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                      __builtin_bit_cast(bf16x8, b & keep), z, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) S.o[eb][i] += sees ? z[i] : 0.f;
      }
    }
#endif
  }

  // Step t of a wave whose rows see all of tile t: the transfers of stage
  // t + NS, the scores of tile t + 1, the softmax and product of tile t.  The
  // stage written and the one read are different ones, which the parameters
  // say (restrict): without it the compiler waits for the transfers before
  // every read.
  static __device__ __forceinline__ void step(lds_char* __restrict__ nxt, const lds_char* __restrict__ cur,
                                              const Fetch& f, int jn, int kb, int ntiles, const int (&pg)[DL::U],
                                              int w, const Lane& A, Rows<D>& S, Scores& x, float c, int lane) {
    issue(nxt, f, jn, kb, ntiles, pg, w, A, lane);
    __builtin_amdgcn_sched_barrier(0);
    const float ref = reference(x, S, c);
    const Scores y = scores(cur, S, A);
    const Probs P = weights(x, S, c, ref);
    product(cur, P, S, A);
    x = y;
  }
  // The same where they may not (see 0: none of its keys).
  static __device__ __forceinline__ void edge_step(lds_char* __restrict__ nxt, const lds_char* __restrict__ cur,
                                                   const Fetch& f, int jn, int kb, int ntiles,
                                                   const int (&pg)[DL::U], int w, const Lane& A, Rows<D>& S,
                                                   Scores& x, int t0, bool see, bool see_next, float c, int lane) {
    issue(nxt, f, jn, kb, ntiles, pg, w, A, lane);
    __builtin_amdgcn_sched_barrier(0);
    if (see) {
      const int half = lane >> 5;
      mask(x, S, t0, half);
      const float ref = reference(x, S, c);
      const Probs P = weights(x, S, c, ref);
      if (__any(bad_values(cur, A))) careful_product(cur, P, S, A, t0, half);
      else product(cur, P, S, A);
    }
    if (see_next) x = scores(cur, S, A);
  }
};

template <int D, int NW, int TK, int NS, int PARTS>
__global__ __launch_bounds__(64 * NW, NW == 1 ? 1 : 2) void chunk_attn(ChunkParams p) {
#if defined(__HIP_DEVICE_COMPILE__)   // the host pass needs the signature only
  using C = Chunk<D, NW, TK, PARTS>;
  using TL = Tile<D, TK>;
  using DL = Deal<D, TK, NW>;
  constexpr int KS = C::KS, ET = C::ET;
  __shared__ __attribute__((aligned(1024))) char lds[NS * TL::STAGE];

  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const ChunkItem it = p.items[blockIdx.x];
  const int ntiles = (it.ke - it.kb + TK - 1) / TK;

  Fetch f;
  f.k = static_cast<const char*>(p.k) + (int64_t)it.kvh * p.kv_sh * 2;
  f.v = static_cast<const char*>(p.v) + (int64_t)it.kvh * p.kv_sh * 2;
  f.table = (const const_int32*)(p.bt + (int64_t)it.req * p.bt_stride);
  f.row_bytes = (int)(p.kv_st * 2);
  f.page_tokens = p.page_tokens;
  f.page_bytes = (int64_t)p.page_tokens * f.row_bytes;
  f.num_pages = p.num_pages;
  f.ke = it.ke;
  typename C::Lane A;
#pragma unroll
  for (int x = 0; x < TL::T; ++x) {
    const int row = x * TL::RPI + lane / TL::CH, ch = lane % TL::CH;
    const bool v0 = C::unit_is_v(w, 0);
    A.off[x] = (uint32_t)(row * f.row_bytes + ((ch ^ (v0 ? swv<D>(row) : swk<D>(row))) * 16));
    if constexpr (DL::U > 1) A.flip[x] = (uint32_t)(row * f.row_bytes + ((ch ^ swv<D>(row)) * 16));
  }
  int pg[DL::U];
  auto pages = [&](int j) {
#pragma unroll
    for (int u = 0; u < DL::U; ++u) {
      const int tile = max(C::unit_is_v(w, u) ? j - 1 : j, 0);
      pg[u] = page_of(f, it.kb + TK * tile + 32 * C::unit_half(w, u));
    }
  };

  Rows<D> S;
  const int wr0 = 32 * w;                                // the wave's first row of the item
  {
    const int r = it.r0 + min(wr0 + l32, it.rows - 1);   // rows past the item's repeat its last
    const int j = r / p.G;
    const int h = it.kvh * p.G + (r - j * p.G);
    const char* src = static_cast<const char*>(p.q) + ((it.q0 + (int64_t)j) * p.q_st + (int64_t)h * p.q_sh) * 2 + half * 16;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) S.q[ks] = *reinterpret_cast<const bf16x8*>(src + ks * 32);
    S.last = min(it.ctx + j, it.ke - 1);
  }
  lds_char* ring = (lds_char*)lds;
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    pages(j);
    C::issue(ring + j * TL::STAGE, f, j, it.kb, ntiles, pg, w, A, lane);
  }
  pages(NS);
  S.m = -INFINITY;
  S.l = 0.f;
#pragma unroll
  for (int eb = 0; eb < ET; ++eb)
#pragma unroll
    for (int i = 0; i < 16; ++i) S.o[eb][i] = 0.f;
  {
    const int key = 16 * (l32 >> 4) + 8 * ((l32 >> 2) & 1) + 4 * ((l32 >> 3) & 1) + (l32 & 3);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) A.koff[ks] = (uint32_t)(key * TL::ROWB + (((2 * ks + half) ^ swk<D>(key)) * 16));
    const int s = lane & 15, row = 8 * half + (s >> 2);
#pragma unroll
    for (int eb = 0; eb < ET; ++eb) {
      const int ch = 4 * eb + 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
      A.voff[eb] = (uint32_t)(TL::MAT + row * TL::ROWB + ((ch ^ swv<D>(row)) * 16) + (s & 1) * 8);
    }
  }
  // the last key that the item's first row sees, and the wave's last row (none without rows)
  const int all_see = min(it.ctx + it.r0 / p.G, it.ke - 1);
  const int wave_sees = wr0 < it.rows ? min(it.ctx + (it.r0 + min(wr0 + 31, it.rows - 1)) / p.G, it.ke - 1) : -1;
  const int nfull = all_see + 1 >= it.kb ? (all_see + 1 - it.kb) / TK : 0;     // tiles that every row sees whole

  // stages 0 .. NS - 1 are under way: wait for stage 0 (K of tile 0)
  if (ntiles >= NS) {
    // V waves have nothing in stage 0; what is younger than it is NS - 1 stages
    wait_vm<(NS - 1) * DL::PER>();
  } else {
    wait_vm<0>();
  }
  tile_barrier();
  typename C::Scores x = C::scores(ring, S, A);
  // step t: stage t + 1 has landed here and everywhere, and every wave has
  // read what it needs of stage t, where stage t + NS goes
  auto turn = [&](int t) {
    if (t + NS - 1 < ntiles) wait_vm<(NS - 2) * DL::PER>();
    else wait_vm<0>();
    tile_barrier();
  };
  int t = 0;
  if (wave_sees >= it.kb) {
    while (t + NS <= nfull) {
      static_for<0, NS>([&](auto st) {
        constexpr int ST = decltype(st)::value;
        turn(t + ST);
        C::step(ring + ST * TL::STAGE, ring + ((ST + 1) % NS) * TL::STAGE, f, t + ST + NS, it.kb, ntiles, pg, w, A, S,
                x, p.scale_log2, lane);
        pages(t + ST + NS + 1);
      });
      t += NS;
    }
  }
  for (; t < ntiles; ++t) {
    turn(t);
    const int t0 = it.kb + TK * t;
    C::edge_step(ring + (t % NS) * TL::STAGE, ring + ((t + 1) % NS) * TL::STAGE, f, t + NS, it.kb, ntiles, pg, w, A, S,
                 x, t0, t0 <= wave_sees, t + 1 < ntiles && t0 + TK <= wave_sees, p.scale_log2, lane);
    pages(t + NS + 1);
  }

  const float l = S.l + __shfl_xor(S.l, 32);
  if (wr0 + l32 >= it.rows) return;
  const int r = it.r0 + wr0 + l32;
  if (it.part < 0) {
    const int j = r / p.G;
    const int64_t row = (it.q0 + (int64_t)j) * p.Hq + it.kvh * p.G + (r - j * p.G);
    const float inv = 1.f / l;
#pragma unroll
    for (int eb = 0; eb < ET; ++eb)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int e = 32 * eb + 2 * i + 4 * half;
        const f32x4 y = {S.o[eb][i] * inv, S.o[eb][i + 1] * inv, S.o[eb][i + 2] * inv, S.o[eb][i + 3] * inv};
        if constexpr (PARTS == 1) {
          typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
          *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + row * D + e) =
              __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
        } else {
          *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row * D + e) = y;
        }
      }
  } else {
    const int64_t row = it.part + wr0 + l32;
#pragma unroll
    for (int eb = 0; eb < ET; ++eb)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(p.part_o + row * D + 32 * eb + 2 * i + 4 * half) =
            f32x4{S.o[eb][i], S.o[eb][i + 1], S.o[eb][i + 2], S.o[eb][i + 3]};
    if (half == 0) p.part_ml[row] = make_float2(S.m, l);
  }
#endif
}

// The pieces of one cut row tile, a wave a row:
//   O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s,  M = max_s m_s,
// the pieces in order.  A piece none of whose keys the row sees has m = -inf.
template <int D, bool F32>
__global__ __launch_bounds__(256) void chunk_join(ChunkParams p, int groups) {
  const int x = (int)blockIdx.x / groups;
  const ChunkJoin jn = p.joins[x];
  const int lane = threadIdx.x & 63;
  const int rr = __builtin_amdgcn_readfirstlane(((int)blockIdx.x - x * groups) * 4 + (int)(threadIdx.x >> 6));
  if (rr >= jn.rows) return;
  constexpr int E = D / 64;                              // a lane's columns
  float M = -INFINITY;
  for (int s = 0; s < jn.pieces; ++s) M = fmaxf(M, p.part_ml[jn.part + (int64_t)s * jn.rows + rr].x);
  float L = 0.f, o[E] = {};
  for (int s = 0; s < jn.pieces; ++s) {
    const int64_t row = jn.part + (int64_t)s * jn.rows + rr;
    const float2 ml = p.part_ml[row];
    const float wgt = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    L += ml.y * wgt;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += wgt * p.part_o[row * D + lane * E + e];
  }
  const int r = jn.r0 + rr, j = r / p.G;
  const int64_t row = (jn.q0 + (int64_t)j) * p.Hq + jn.kvh * p.G + (r - j * p.G);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = o[e] / L;
    if constexpr (F32) static_cast<float*>(p.out)[row * D + lane * E + e] = y;
    else static_cast<__bf16*>(p.out)[row * D + lane * E + e] = (__bf16)y;
  }
}

template <int D, int PARTS>
static hipError_t launch_d(const ChunkParams& p, hipStream_t s) {
  if (p.tall == kChunkTallRows) chunk_attn<D, 4, 64, 2, PARTS><<<dim3(p.n_items), dim3(256), 0, s>>>(p);
  else chunk_attn<D, 1, 32, 4, PARTS><<<dim3(p.n_items), dim3(64), 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_joins == 0) return e;
  const int groups = (p.tall + 3) / 4;
  chunk_join<D, PARTS != 1><<<dim3(p.n_joins * groups), dim3(256), 0, s>>>(p, groups);
  return hipGetLastError();
}

hipError_t launch_chunk(const ChunkParams& p, hipStream_t s) {
  if (p.D == 128) return p.out_f32 ? launch_d<128, 3>(p, s) : launch_d<128, 1>(p, s);
  return p.out_f32 ? launch_d<64, 3>(p, s) : launch_d<64, 1>(p, s);
}

}  // namespace sv
