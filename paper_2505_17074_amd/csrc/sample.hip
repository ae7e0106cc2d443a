// Sampling for gfx950: a row's token by temperature, top-k, top-p and min-p.
//
// With w_v = exp((l_v - l_max) / T) and the order of the logits (descending, the
// lower id first), all three filters keep a run from the front of the order, so
// what stays is told by one token: the last of the shortest run, (cut, cut_id),
//   v stays iff l_v > cut, or l_v = cut and v <= cut_id, and w_v >= min_p.
// The cut is found without sorting: a histogram of the tokens' counts (top-k) or
// weights (top-p) over 2048 ranges of values, the range where the sum passes its
// mark, and again within that range until its tokens fit a list, whose order is
// taken by counting.  Weights are 64-bit, histograms of them in fixed point, so
// that no sum depends on the order of its terms.
//
// What bounds it (calls in a row): latency and launches where it is small, a wave's
// instructions and its waits for LDS and barriers, about half each, where it is
// large, never HBM.
//   one row of 32000 (fp32), top-k and top-p: 9-12 us by the logits; where 9.1 (10.9
//     with two barriers for each of the work-group's sums and searches), one kernel of
//     8.4: load and largest value 1.7, histogram 1.2, the list 2, its two orders and the
//     sums 3.
//   64 of them, all filters, the rows written (16 MB): 32 us, three kernels of 8, 11
//     and 15.5 with 3.5 between their first and last work-groups' ends and starts;
//     rows with top-p alone, and those of 400 tokens, are the last to end.
//   128 of 128256 (bf16), top-p (33 MB, 5 us at HBM's rate): 49 us, three kernels of
//     16, 21 and 13: 17 vector instructions and an LDS operation an element in the
//     first, 23 in the second (8.5 and 11 us at four cycles each), on one work-group a
//     compute unit (two of them with half the registers measured the same).
#include "sv_sample.h"

#include <type_traits>

namespace sv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;            // ranges of a histogram
constexpr int kRank = 768;             // tokens ranked by counting: one a thread
constexpr int kList = kSampleList;     // tokens of a sorted list
constexpr int kSlabs = kSampleSlabs;   // runs of ids whose weights are summed apart
constexpr int kGroups = kBins / 32;
static_assert(kBins == kSampleBins, "a slice's histogram in the workspace");

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// 2^t for t <= 0 in 64 bits, off by 1e-11 of it: e^(f ln 2) by its series up to
// the tenth power for |f| <= 1/2 (the next term is below 3e-13).
__device__ __forceinline__ double exp2_64(double t) {
  t = fmax(t, -2000.0);
  const double n = __builtin_rint(t), x = (t - n) * 0.69314718055994530942;
  double y = 1.0 / 3628800;
  y = __builtin_fma(y, x, 1.0 / 362880);
  y = __builtin_fma(y, x, 1.0 / 40320);
  y = __builtin_fma(y, x, 1.0 / 5040);
  y = __builtin_fma(y, x, 1.0 / 720);
  y = __builtin_fma(y, x, 1.0 / 120);
  y = __builtin_fma(y, x, 1.0 / 24);
  y = __builtin_fma(y, x, 1.0 / 6);
  y = __builtin_fma(y, x, 0.5);
  y = __builtin_fma(y, x, 1.0);
  y = __builtin_fma(y, x, 1.0);
  return __builtin_amdgcn_ldexp(y, (int)n);
}

// Descending order of values as ascending whole numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (int32_t)b < 0 ? b : ~b & 0x7fffffffu;
}

// x of another lane by a data-parallel move (CTRL, in the rows of ROWS), `none`
// where there is no such lane.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T moved(T x, T none) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(
        T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
  } else {
    const uint64_t a = __builtin_bit_cast(uint64_t, x), n = __builtin_bit_cast(uint64_t, none);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp((int)(uint32_t)n, (int)(uint32_t)a, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp((int)(uint32_t)(n >> 32), (int)(uint32_t)(a >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
  }
}
// f over the wave's lanes up to and including this one: within rows of 16 lanes by
// shifts, then the rows before by broadcasts of their last lanes.
template <typename T, typename F>
__device__ __forceinline__ T wave_scan(T x, T none, F&& f) {
  x = f(x, moved<0x111, 0xf>(x, none));
  x = f(x, moved<0x112, 0xf>(x, none));
  x = f(x, moved<0x114, 0xf>(x, none));
  x = f(x, moved<0x118, 0xf>(x, none));
  x = f(x, moved<0x142, 0xa>(x, none));
  x = f(x, moved<0x143, 0xc>(x, none));
  return x;
}
template <typename T>
__device__ __forceinline__ T last_lane(T x) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
  } else {
    const uint64_t a = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(T, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(a >> 32), 63) << 32 |
                                     (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)a, 63));
  }
}
struct Plus {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Least {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a < b ? a : b; }
};
struct Most {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; }
};
template <typename T>
__device__ __forceinline__ T wave_sum(T x) { return last_lane(wave_scan(x, T(0), Plus{})); }

// One row's elements, in 16-byte units on the memory's own 16-byte borders.
template <bool F32>
struct Row {
  static constexpr int VEC = F32 ? 4 : 8, EB = F32 ? 4 : 2;
  const char* base;          // of unit 0 (the row's first element is its `head`-th)
  int head, V, units;

  __device__ __forceinline__ Row(const void* p, int V_) : V(V_) {
    head = (int)(reinterpret_cast<uintptr_t>(p) % 16) / EB;
    base = static_cast<const char*>(p) - head * EB;
    units = (V + head + VEC - 1) / VEC;
  }
  __device__ __forceinline__ int first_id(int u) const { return u * VEC - head; }
  __device__ __forceinline__ bool whole(int u) const { return first_id(u) >= 0 && first_id(u) + VEC <= V; }
  __device__ __forceinline__ static float clean(uint32_t b) {
    // NaN as minus infinity, minus zero as zero
    const uint32_t m = b & 0x7fffffffu;
    return __uint_as_float(m > 0x7f800000u ? 0xff800000u : m == 0 ? 0 : b);
  }
  // Unit u as it is; elements outside the row are minus infinity.
  __device__ __forceinline__ u32x4 raw(int u) const {
    if (whole(u)) return *reinterpret_cast<const u32x4*>(base + (int64_t)u * 16);
    u32x4 r;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t b = F32 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
      for (int h = 0; h < VEC / 4; ++h) {
        const int i = w * (VEC / 4) + h, id = first_id(u) + i;
        if (u < units && id >= 0 && id < V) {
          const char* at = base + ((int64_t)u * VEC + i) * EB;
          if constexpr (F32) b = *reinterpret_cast<const uint32_t*>(at);
          else b = (b & ~(0xffffu << 16 * h)) | (uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16 * h;
        }
      }
      r[w] = b;
    }
    return r;
  }
  // Its values; a NaN among them fails every comparison below, as minus infinity does.
  __device__ __forceinline__ static void values(u32x4 r, float (&x)[VEC]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (F32) {
        x[w] = __uint_as_float(r[w]);
      } else {
        x[2 * w] = __uint_as_float(r[w] << 16);
        x[2 * w + 1] = __uint_as_float(r[w] & 0xffff0000u);
      }
    }
  }
  // Unit u's values; elements outside the row are minus infinity.
  __device__ __forceinline__ void load(int u, float (&x)[VEC]) const {
    if (whole(u)) {
      const u32x4 r = *reinterpret_cast<const u32x4*>(base + (int64_t)u * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
          x[i] = clean(r[i]);
        } else {
          x[2 * i] = clean(r[i] << 16);
          x[2 * i + 1] = clean(r[i] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int id = first_id(u) + i;
        x[i] = -INFINITY;
        if (u < units && id >= 0 && id < V) {
          const char* at = base + ((int64_t)u * VEC + i) * EB;
          if constexpr (F32) x[i] = clean(*reinterpret_cast<const uint32_t*>(at));
          else x[i] = clean((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
        }
      }
    }
  }
};

// bf16 values of magnitude 2^-13 to 2^5 by their bits: two signs of 18 powers of
// two of 128 values each, a place a sign for all others, one for the type's lowest
// value and one for what is masked out (both as masks have them; one for each lane, so
// that a row of them is not counted at one address).  A row's weights are those of
// so few values that they are counted, or looked up, in place of an exponential each.
constexpr int kOneSign = 18 * 128, kNegative = 2 * kOneSign + 1, kLowest = kNegative + 65, kMasked = kNegative + 130;
constexpr int kValues = kMasked + 127;
constexpr int kLeastValue = 114 << 7;
__device__ __forceinline__ bool value_in_table(float x) {
  const uint32_t h = __float_as_uint(x) >> 16;
  return (h & 0x7fffu) - kLeastValue < (uint32_t)kOneSign || h == 0xff7fu;
}
// Two values' places times SIZE, below 2^16 each; `most` reaches kOneSign where one is
// among a sign's others.
template <int SIZE>
__device__ __forceinline__ uint32_t value_places(uint32_t two, u16x2& most) {
  static_assert(kValues * SIZE <= 65536, "16 bits");
  const u16x2 h = __builtin_bit_cast(u16x2, two), one = {1, 1};
  const u16x2 m = __builtin_elementwise_min((u16x2)((h & one * (uint16_t)0x7fff) - one * (uint16_t)kLeastValue), one * (uint16_t)kOneSign);
  // 1 for the lowest, 2 for minus infinity and the NaNs behind it
  const u16x2 low = __builtin_elementwise_min(__builtin_elementwise_sub_sat(h, one * (uint16_t)0xff7e), one * (uint16_t)2);
  most = __builtin_elementwise_max(most, (u16x2)(m - low));
  // from the negative others' place 65 .. 128 on, or twice that
  const u16x2 on = low * (uint16_t)(65 + (threadIdx.x & 63)) + m;
  return __builtin_bit_cast(uint32_t, (u16x2)(((h >> 15) * (uint16_t)(kOneSign + 1) + on) * (uint16_t)SIZE));
}
// The value at a place; those of the others' places and the masked ones' are none of
// the table's.
__device__ __forceinline__ bool value_other(int i) { return i == kOneSign || i == kNegative || i >= kMasked; }
__device__ __forceinline__ float value_at(int i) {
  const int sign = i > kOneSign;
  const uint32_t h = i >= kLowest ? 0xff7fu : (uint32_t)(i - sign * (kOneSign + 1) + kLeastValue) | (uint32_t)sign << 15;
  return __uint_as_float(h << 16);
}

struct Shared {
  union {
    struct {
      union {
        uint32_t count[kBins];
        unsigned long long mass[kBins];
        unsigned long long by_id[kList];
        unsigned long long add[kSlabs];
      };
      union {
        struct {
          float x[kRank];
          int id[kRank];
          double w[kRank];
        } list;
        uint32_t values[kValues];      // how often a bf16 value comes
        unsigned long long runs[kThreads];       // of 64 keys in order
        int ids[kList];                // of the entries in by_id
      };
    };
    double weights[kValues];           // a bf16 value's weight
  };
  unsigned long long keys[kList];      // a list: order and id
  double slab[kSlabs];                 // weights that stay, by runs of ids
  unsigned long long group[kGroups];   // sums of 32 ranges
  int n;                               // of the list
  unsigned long long red[2][kWaves];   // taken in turn, so that one barrier an operation will do
  unsigned long long out[2];
};
static_assert(sizeof(Shared) <= 65536, "a work-group's LDS");

// What stays of a row.
struct Cut {
  float x;
  int id;
  __device__ __forceinline__ bool keeps(float y, int i) const { return y > x || (y == x && i <= id); }
};

// f over the work-group, the same for all threads.  `turn`: which of the places its
// waves meet at, not the last operation's.
template <typename T, typename F>
__device__ __forceinline__ T block_reduce(Shared& sh, int& turn, T x, T none, F&& f) {
  x = last_lane(wave_scan(x, none, f));
  T* at = reinterpret_cast<T*>(sh.red[turn]);
  turn ^= 1;
  if ((threadIdx.x & 63) == 0) at[threadIdx.x / 64] = x;
  __syncthreads();
  x = at[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) x = f(x, at[i]);
  return x;
}
// The sum over the threads up to and including this one.
template <typename T>
__device__ __forceinline__ T block_scan(Shared& sh, int& turn, T x) {
  x = wave_scan(x, T(0), Plus{});
  T* at = reinterpret_cast<T*>(sh.red[turn]);
  turn ^= 1;
  if ((threadIdx.x & 63) == 63) at[threadIdx.x / 64] = x;
  __syncthreads();
  T base = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) base += i < (int)threadIdx.x / 64 ? at[i] : T(0);
  return base + x;
}

template <bool F32>
struct Sampler {
  using R = Row<F32>;
  static constexpr int VEC = R::VEC;
  const R& row;
  Shared& sh;
  float top;
  double c;                            // log2(e) / T
  float bins;                          // kBins ranges to 32 T
  int fix;                             // fixed point: weights in units of 2^-fix
  mutable int turn = 0;

  __device__ __forceinline__ Sampler(const R& r, Shared& s) : row(r), sh(s) {}

  template <typename F>
  __device__ __forceinline__ void each_unit(F&& f) const {
    for (int u = threadIdx.x; u < row.units; u += kThreads) {
      float x[VEC];
      row.load(u, x);
      f(u, x);
    }
  }
  // f(value, id) of every token that is not masked out
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    each_unit([&](int u, const float (&x)[VEC]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (x[i] > -INFINITY) f(x[i], row.first_id(u) + i);
    });
  }
  __device__ __forceinline__ double weight(float x) const { return x == top ? 1.0 : exp2_64(((double)x - (double)top) * c); }
  __device__ __forceinline__ unsigned long long fixed(float x) const {
    return (unsigned long long)__builtin_amdgcn_ldexp(weight(x), fix);
  }

  // The range of the histogram where the running sum reaches `mark` (at least one,
  // at most the whole sum), and the sum before it.
  template <typename T>
  __device__ __forceinline__ int find_bin(const T* hist, unsigned long long mark, unsigned long long& before) const {
    static_assert(kBins == 2 * kThreads, "two ranges a thread");
    __syncthreads();
    const int t = threadIdx.x;
    const T a = hist[2 * t], b = hist[2 * t + 1];
    if (t == 0) sh.out[0] = 0;
    const unsigned long long s2 = block_scan(sh, turn, (unsigned long long)a + b), s1 = s2 - b, s0 = s1 - a;
    // the only range that begins below the mark and does not end below it
    if (s0 < mark && s1 >= mark) {
      sh.out[0] = 2 * t + 1;
      sh.out[1] = s0;
    }
    if (s1 < mark && s2 >= mark) {
      sh.out[0] = 2 * t + 2;
      sh.out[1] = s1;
    }
    __syncthreads();
    const int bin = (int)sh.out[0] - 1;
    before = sh.out[1];
    __syncthreads();
    return bin;
  }

  __device__ __forceinline__ int range_of(float x) const {
    return min((int)fminf((top - x) * bins, (float)(kBins - 1)), kBins - 1);
  }

  // The last token of the order's run whose sum (MASS: of fixed-point weights,
  // else of counts) first reaches `mark`, among the tokens that `in` keeps.  The
  // caller has filled the histogram of range_of over them.
  template <bool MASS>
  __device__ __forceinline__ Cut last_of(unsigned long long mark, const Cut& in) {
    using T = std::conditional_t<MASS, unsigned long long, uint32_t>;
    T* hist = reinterpret_cast<T*>(&sh.mass[0]);
    unsigned long long sum, before;
    const int bin = find_bin<T>(hist, mark, sum);
    // the range's tokens: their keys' range
    uint32_t lo = 0xffffffffu, hi = 0;
    int n = 0;
    each([&](float x, int id) {
      if (range_of(x) == bin && in.keeps(x, id)) {
        const uint32_t k = key_of(x);
        lo = min(lo, k);
        hi = max(hi, k);
        ++n;
      }
    });
    for (;;) {
      lo = block_reduce(sh, turn, lo, 0xffffffffu, Least{});
      hi = block_reduce(sh, turn, hi, 0u, Most{});
      n = block_reduce(sh, turn, n, 0, Plus{});
      if (n <= kRank || lo == hi) break;
      // again, over keys lo .. hi
      const int shift = max(0, 21 - __builtin_clz((hi - lo) | 1));
      const uint32_t first = lo, last = hi;
      __syncthreads();
      for (int i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
      __syncthreads();
      each([&](float x, int id) {
        const uint32_t k = key_of(x);
        if (k >= first && k <= last && in.keeps(x, id)) {
          if constexpr (MASS) atomicAdd(&sh.mass[(k - first) >> shift], fixed(x));
          else atomicAdd(&sh.count[(k - first) >> shift], 1u);
        }
      });
      const int b = find_bin<T>(hist, mark - sum, before);
      sum += before;
      lo = 0xffffffffu;
      hi = 0;
      n = 0;
      each([&](float x, int id) {
        const uint32_t k = key_of(x);
        if (k >= first && k <= last && (int)((k - first) >> shift) == b && in.keeps(x, id)) {
          lo = min(lo, k);
          hi = max(hi, k);
          ++n;
        }
      });
    }
    if (n > kRank) return tie<MASS>(lo, mark, sum, in);
    // the tokens as a list, and for each what comes before it in the order
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    each([&](float x, int id) {
      const uint32_t k = key_of(x);
      if (k >= lo && k <= hi && in.keeps(x, id)) {
        const int at = atomicAdd(&sh.n, 1);
        sh.list.x[at] = x;
        sh.list.id[at] = id;
      }
    });
    __syncthreads();
    const int t = threadIdx.x;
    float x = 0.f;
    int id = 0;
    if (t < n) {
      x = sh.list.x[t];
      id = sh.list.id[t];
      if constexpr (MASS) reinterpret_cast<unsigned long long*>(sh.list.w)[t] = fixed(x);
    }
    __syncthreads();
    if (t < n) {
      unsigned long long s = sum, own = 1;
      for (int i = 0; i < n; ++i) {
        const float y = sh.list.x[i];
        const bool ahead = y > x || (y == x && sh.list.id[i] < id);
        const unsigned long long w = MASS ? reinterpret_cast<unsigned long long*>(sh.list.w)[i] : 1ull;
        s += ahead ? w : 0;
        if (i == t) own = w;
      }
      // the first whose sum reaches the mark: those after it have it reached before
      if (s < mark && s + own >= mark) {
        sh.out[0] = __float_as_uint(x);
        sh.out[1] = (unsigned)id;
      }
    }
    __syncthreads();
    const Cut cut = {__uint_as_float((uint32_t)sh.out[0]), (int)sh.out[1]};
    __syncthreads();
    return cut;
  }

  // The same among many tokens of one value: so many of them, the lower ids first.
  template <bool MASS>
  __device__ __forceinline__ Cut tie(uint32_t key, unsigned long long mark, unsigned long long sum, const Cut& in) {
    const float x = __uint_as_float((int32_t)key < 0 ? key : ~key & 0x7fffffffu);
    const unsigned long long w = MASS ? fixed(x) : 1;
    // the smallest m with sum + m w >= mark
    const long long m = (long long)((mark - sum + w - 1) / w);
    // ids in rounds of the block: how many so far, then the thread that has the m-th
    long long so_far = 0;
    if (threadIdx.x == 0) sh.out[0] = 0x7fffffff;
    __syncthreads();
    for (int u0 = 0; u0 < row.units; u0 += kThreads) {
      const int u = u0 + threadIdx.x;
      float y[VEC];
      row.load(u, y);
      int mine = 0;
#pragma unroll
      for (int i = 0; i < VEC; ++i) mine += y[i] == x && in.keeps(y[i], row.first_id(u) + i);
      const int upto = block_scan(sh, turn, mine);
      long long at = so_far + upto - mine;
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (y[i] == x && in.keeps(y[i], row.first_id(u) + i) && ++at == m) sh.out[0] = row.first_id(u) + i;
      so_far += block_reduce(sh, turn, mine, 0, Plus{});
      if (so_far >= m) break;
    }
    const Cut cut = {x, (int)sh.out[0]};
    __syncthreads();
    return cut;
  }
};

// ---------------------------------------------------------------------------
// The same in slices, so that a few long rows fill the chip.  A row is cut into
// `slices` runs of units, one work-group each:
//   step 0          a slice's largest value and a histogram below it, of counts
//                   (top-k) or weights (top-p without it), over ranges of values
//                   that all slices have in common;
//   step 1          every slice's work-group adds the row's histograms and finds
//                   the range where the mark is reached; it lists its tokens of
//                   that range (and, for a small top-k, of all ranges before) and
//                   sums the weights of those before it, run of ids by run of ids;
//   step 2          one work-group a row sorts the list, cuts it, and finds the
//                   token;
//   step 3          writes the distribution.
// With one slice the four are one kernel, and where the rows are not the logits
// the last two are one (step 5): every slice's work-group finds the cut again.  A
// row that this does not suit (its mark past the 2048 ranges, more tokens in one
// range than a list holds, a top-p behind a large top-k) takes the way above in
// step 2.

enum Mode { kAll = 0, kFirst = 1, kEdge = 2, kHard = 3, kNone = 4 };

constexpr int kFew = 512;              // a top-k found by the threads' largest values
constexpr int kWindow = kBins - 32;    // ranges of a histogram below its largest value's (below)
constexpr double kListUnit = 281474976710656.0;      // 2^48: a list's weights in fixed point

// What a row asks for.
struct Rule {
  float T, top_p, min_p;
  int k;
  bool one, by_count, by_mass;         // a cut by top-k, by top-p alone
  bool few;                            // a top-k for which the threads' largest values tell the range
  float scale;                         // ranges a unit of value
  double c;                            // log2(e) / T

  __device__ __forceinline__ Rule(const SampleParams& p, int r) {
    // loads from some place in any case, so that none waits for another
    const float* any = reinterpret_cast<const float*>(p.work);
    const float t0 = *(p.temperature ? p.temperature + r : any), p0 = *(p.top_p ? p.top_p + r : any);
    const float m0 = *(p.min_p ? p.min_p + r : any);
    const int k0 = *(p.top_k ? p.top_k + r : reinterpret_cast<const int*>(any));
    T = p.temperature ? t0 : 1.f;
    k = p.top_k ? k0 : 0;
    top_p = p.top_p ? p0 : 1.f;
    min_p = p.min_p ? m0 : 0.f;
    one = !(T > 0.f) || !(top_p > 0.f) || !(min_p <= 1.f);
    if (k < 1 || k > p.V) k = p.V;
    if (one) k = 1, T = 1.f, top_p = 1.f, min_p = 0.f;
    c = 1.4426950408889634074 / (double)T;
    by_count = k < p.V;
    by_mass = !by_count && top_p < 1.f;
    few = by_count && k <= kFew;
    // counts: 64 units of value in all, logits' own scale; weights: 32 T, past
    // which e^-32 of the largest weight is left a token
    scale = by_count ? (float)kBins / 64.f : (float)kBins / (32.f * T);
  }
  // The range of a value, counted upwards (whole numbers in fp32: exact below 2^24).
  __device__ __forceinline__ float range(float x) const { return floorf(x * scale); }
};

// What step 1 leaves of a row, the same from all its slices.
struct RowState {
  int mode;
  float range;                         // the one where the mark is reached
  double before, mark;                 // sums ahead of it (counts or weights), the mark
};

struct RowView {
  SampleRow s;
  __device__ __forceinline__ RowView(const SampleParams& p, int r) {
    char* at = p.work + (int64_t)r * p.row_bytes;
    s.top = reinterpret_cast<float*>(at);
    s.n = reinterpret_cast<int32_t*>(at + 64);
    s.sum = reinterpret_cast<double*>(at + 128);
    s.state = at + 192;
    s.done = at + 256;
    s.slab = reinterpret_cast<double*>(at + kSampleHead);
    s.list = reinterpret_cast<unsigned long long*>(at + kSampleHead + sizeof(double) * kSlabs);
    s.hist = s.list + (int64_t)p.slices * kList;
    s.group = s.hist + (int64_t)p.slices * kBins;
  }
};
static_assert(sizeof(RowState) <= 64, "a row's state");

// What step 2 leaves for step 3.
struct RowDone {
  Cut cut;
  double total;
  float top;
  int kept;                            // none: all masked out
};
static_assert(sizeof(RowDone) <= 64, "a row's outcome");

// ONE: a row is one slice, and what the steps leave for each other stays in LDS.
template <bool F32, bool ONE>
struct Slices {
  using R = Row<F32>;
  static constexpr int VEC = R::VEC;
  static constexpr int kAhead = ONE ? 8 : 2;       // units that a thread loads at once
  const SampleParams& p;
  const R& row;
  Shared& sh;
  const Rule& rule;
  SampleRow ws;
  float top;
  double sum_all;                      // ONE: the histogram's
  mutable int turn = 0;

  __device__ __forceinline__ int begin(int slice) const { return slice * p.slice_units; }
  __device__ __forceinline__ int end(int slice) const { return min((slice + 1) * p.slice_units, row.units); }
  __device__ __forceinline__ double weight(float x) const { return x == top ? 1.0 : exp2_64(((double)x - (double)top) * rule.c); }
  // w in units of 1 / unit: the integer in the low bits of a double between 2^52 and 2^53
  __device__ __forceinline__ static unsigned long long fixed(double w, double unit) {
    return __builtin_bit_cast(unsigned long long, __builtin_fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull;
  }

  // The slice's units, kAhead of them a thread at once: f(unit as it is, which).
  // `held`: r holds the first of them (all, where they fit).
  __device__ __forceinline__ void load(int at, int u1, u32x4 (&r)[kAhead]) const {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int u = at + (int)threadIdx.x + j * kThreads;
      r[j] = u < u1 ? row.raw(u) : u32x4{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};     // NaN
    }
  }
  template <typename F>
  __device__ __forceinline__ void units(int slice, u32x4 (&r)[kAhead], bool held, F&& f) const {
    const int u0 = begin(slice), u1 = end(slice);
    for (int at = u0; at < u1; at += kAhead * kThreads) {
      if (!held || u0 + kAhead * kThreads < u1) load(at, u1, r);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (at + j * kThreads >= u1) break;
        f(r[j], at + (int)threadIdx.x + j * kThreads);
      }
    }
  }

  // How often each of the table's values comes in the slice (sh.values), which of the
  // thread's units hold others (the 64th and all after it by one bit), and the
  // thread's share of the search for the largest value.
  __device__ __forceinline__ float count_values(int slice, u32x4 (&r)[kAhead], uint64_t& others) const {
    const int t = threadIdx.x;
    for (int i = t; i < kValues; i += kThreads) sh.values[i] = 0;
    __syncthreads();
    int nth = 0;
    float m = -INFINITY;
    units(slice, r, false, [&](u32x4 y, int) {
      u16x2 most = {0, 0};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t at = value_places<4>(y[w], most);
        atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sh.values) + (at & 0xffffu)), 1u);
        atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(sh.values) + (at >> 16)), 1u);
      }
      if (max(most.x, most.y) >= kOneSign) {
        float x[VEC], z = -INFINITY;
        R::values(y, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) z = value_in_table(x[i]) ? z : fmaxf(z, x[i]);
        m = fmaxf(m, z);
        others |= (uint64_t)(z > -INFINITY) << min(nth, 63);
      }
      ++nth;
    });
    __syncthreads();
    for (int i = t; i < kValues; i += kThreads)
      if (!value_other(i) && sh.values[i]) m = fmaxf(m, value_at(i));
    return m;
  }
  // f(value) of the values that are none of the table's.
  template <typename F>
  __device__ __forceinline__ void each_other(int slice, uint64_t others, F&& f) const {
    const int u1 = end(slice);
    while (others) {
      const int k = __builtin_ctzll(others);
      others &= others - 1;
      for (int u = begin(slice) + threadIdx.x + k * kThreads; u < u1; u += kThreads) {
        float x[VEC];
        R::values(row.raw(u), x);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (x[i] > -INFINITY && !value_in_table(x[i])) f(x[i]);
        if (k < 63) break;
      }
    }
  }

  __device__ __forceinline__ void scan_slice(int slice, u32x4 (&r)[kAhead]) {
    const int t = threadIdx.x, u0 = begin(slice), u1 = end(slice);
    float m = -INFINITY;
    uint64_t others = 0;                                   // units with values that are none of the table's
    if (!F32 && rule.by_mass) {
      m = count_values(slice, r, others);
    } else {
      load(u0, u1, r);
      for (int at = u0;;) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          float x[VEC];
          R::values(r[j], x);
#pragma unroll
          for (int i = 0; i < VEC; ++i) m = fmaxf(m, x[i]);
        }
        at += kAhead * kThreads;
        if (at >= u1) break;
        load(at, u1, r);
      }
    }
    top = block_reduce(sh, turn, m, -INFINITY, Most{});
    if (!ONE && t == 0) ws.top[slice] = top;
    if (!rule.by_count && !rule.by_mass) return;
    for (int i = t; i < kBins; i += kThreads) sh.mass[i] = 0;
    __syncthreads();
    // Range g is at place g mod 2048, so that the slices' places agree; the window
    // ends 32 ranges short of the whole, so that a group of 32 ranges aligned to 32
    // never holds some from both of its ends.
    const float first = rule.range(top), lowest = first - (float)(kWindow - 1);
    const double unit = __builtin_amdgcn_ldexp(1.0, p.fix);
    unsigned long long all = 0;
    auto put = [&](float x, uint32_t n) {
      const float g = rule.range(x);
      const unsigned long long w = fixed(weight(x), unit) * n;
      if (g >= lowest) atomicAdd(&sh.mass[(int)g & (kBins - 1)], w);
      all += w;
    };
    auto tell = [&](float x) {
      if (!(x > -INFINITY)) return;
      const float g = rule.range(x);
      if (g >= lowest) atomicAdd(&sh.count[(int)g & (kBins - 1)], 1u);
      ++all;
    };
    // A few of them: k threads' largest values are as many tokens, so the k-th
    // largest of those is no larger than the k-th token, and few tokens lie between.
    if (rule.few) {
      tell(m);
    } else if (top > -INFINITY && rule.by_count) {
      units(slice, r, true, [&](u32x4 y, int) {
        float x[VEC];
        R::values(y, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) tell(x[i]);
      });
    } else if (top > -INFINITY) {
      if constexpr (F32) {
        units(slice, r, true, [&](u32x4 y, int) {
          float x[VEC];
          R::values(y, x);
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (x[i] > -INFINITY) put(x[i], 1);
        });
      } else {
        each_other(slice, others, [&](float x) { put(x, 1); });
        for (int i = t; i < kValues; i += kThreads)
          if (const uint32_t n = value_other(i) ? 0 : sh.values[i]) put(value_at(i), n);
      }
    }
    all = block_reduce(sh, turn, all, 0ull, Plus{});
    const double sum = rule.by_count ? (double)all : (double)all / unit;
    // groups of 32 ranges: 16 threads' pairs
    unsigned long long group = rule.by_count ? (unsigned long long)sh.count[2 * t] + sh.count[2 * t + 1]
                                             : sh.mass[2 * t] + sh.mass[2 * t + 1];
    group += moved<0x111, 0xf>(group, 0ull);
    group += moved<0x112, 0xf>(group, 0ull);
    group += moved<0x114, 0xf>(group, 0ull);
    group += moved<0x118, 0xf>(group, 0ull);
    if constexpr (ONE) {
      sum_all = sum;
      if (t % 16 == 15) sh.group[t / 16] = group;
      return;                                              // the histogram is where state() reads it
    }
    if (t == 0) ws.sum[slice] = sum;
    if (t % 16 == 15) ws.group[slice * kGroups + t / 16] = group;
    unsigned long long* to = ws.hist + (int64_t)slice * kBins;
    if (rule.by_count) {
      for (int i = t; i < kBins; i += kThreads) reinterpret_cast<uint32_t*>(to)[i] = sh.count[i];
    } else {
      for (int i = t; i < kBins; i += kThreads) to[i] = sh.mass[i];
    }
  }

  __device__ __forceinline__ void load_tops(float (&tops)[kSampleSlices]) {
    if constexpr (ONE) return;                             // as scan_slice left it
    top = -INFINITY;
#pragma unroll
    for (int s = 0; s < kSampleSlices; ++s) tops[s] = ws.top[min(s, p.slices - 1)];
#pragma unroll
    for (int s = 0; s < kSampleSlices; ++s) tops[s] = s < p.slices ? tops[s] : -INFINITY;
#pragma unroll
    for (int s = 0; s < kSampleSlices; ++s) top = fmaxf(top, tops[s]);
  }
  template <typename T>
  __device__ __forceinline__ static T of_lane(T x, int lane) {
    const uint64_t a = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(T, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(a >> 32), lane) << 32 |
                                     (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)a, lane));
  }

  // The row's largest value, and where its mark is reached: first among the groups
  // of 32 ranges, a wave adding each slice's, then among the group's ranges.  Every
  // wave finds it for itself.
  __device__ __forceinline__ RowState state() {
    // asked for before the row's largest value says which of them are first
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n = ONE ? 1 : p.slices;
    const unsigned long long ahead = ONE || w >= n ? 0ull : ws.group[w * kGroups + lane];
    const double sum = ONE || w >= n ? 0.0 : ws.sum[w];
    float tops[kSampleSlices];
    load_tops(tops);
    RowState st = {kAll, 0.f, 0.0, 0.0};
    if (!(top > -INFINITY)) st.mode = kNone;
    if (st.mode == kNone || (!rule.by_count && !rule.by_mass)) return st;
    st.mode = kHard;
    const float first = rule.range(top);
    // ranges that are not whole numbers apart, or all the same
    if (!(fabsf(first) < 8388608.f) || !(rule.scale > 0.f) || !(rule.scale < INFINITY)) return st;
    const int start = (int)first & ~31;                    // of the first group
    double* part = reinterpret_cast<double*>(sh.runs);     // [slices][64], sums, [slices][32]
    float own = top;                                       // of the wave's slice
    double f = 1.0;
    if constexpr (!ONE) {
#pragma unroll
      for (int s = 0; s < kSampleSlices; ++s) own = s == w ? tops[s] : own;
    }
    const float own_first = rule.range(own);
    const bool has = w < n && own > -INFINITY;
    if (w < n) {
      const int low = start - 32 * lane;
      double y = 0.0;
      if (has) {
        if (rule.by_mass) f = weight(own) * __builtin_amdgcn_ldexp(1.0, -p.fix);
        const int at = (low >> 5) & (kGroups - 1);
        unsigned long long x;
        if constexpr (ONE) x = sh.group[at];
        else x = __shfl(ahead, at);
        y = own_first >= (float)low ? (double)x * f : 0.0;
      }
      part[w * 64 + lane] = y;
      if (lane == 0) part[512 + w] = !has ? 0.0 : (ONE ? sum_all : sum) * (rule.by_mass ? weight(own) : 1.0);
    }
    __syncthreads();
    double y = 0.0, all = 0.0;
    for (int s = 0; s < n; ++s) {
      y += part[s * 64 + lane];
      all += part[512 + s];
    }
    if (rule.by_count && (double)rule.k >= all) {
      if (rule.few) {                                      // fewer threads with tokens than k: all tokens are listed
        st.mode = kFirst;
        st.range = -INFINITY;
      } else if (!(rule.top_p < 1.f)) {
        st.mode = kAll;                                    // nothing is cut
      }
      return st;
    }
    st.mark = rule.by_count ? (double)rule.k : (double)rule.top_p * all;
    double upto = wave_scan(y, 0.0, Plus{});
    uint64_t reached = __ballot(upto >= st.mark);
    if (!reached) return st;
    const int q = __builtin_ctzll(reached), low = start - 32 * q;
    if ((float)low < first - (float)(kWindow - 1)) return st;        // the group is not whole in the window
    st.before = of_lane(upto, q) - of_lane(y, q);
    if (w < n && lane < 32) {
      const int g = low + 31 - lane, at = g & (kBins - 1);
      double z = 0.0;
      if (has) {
        unsigned long long x;
        if constexpr (ONE) x = rule.by_count ? sh.count[at] : sh.mass[at];
        else x = rule.by_count ? reinterpret_cast<const uint32_t*>(ws.hist + (int64_t)w * kBins)[at]
                               : ws.hist[(int64_t)w * kBins + at];
        z = own_first >= (float)g ? (double)x * f : 0.0;
      }
      part[576 + w * 32 + lane] = z;
    }
    __syncthreads();
    y = 0.0;
    if (lane < 32)
      for (int s = 0; s < n; ++s) y += part[576 + s * 32 + lane];
    upto = st.before + wave_scan(y, 0.0, Plus{});
    reached = __ballot(upto >= st.mark);
    const int i = min(reached ? __builtin_ctzll(reached) : 31, 31);  // none, by the sums' rounding: the last
    st.before = of_lane(upto, i) - of_lane(y, i);
    st.range = (float)(low + 31 - i);
    if (rule.by_count && rule.k <= kSampleFirst) st.mode = kFirst;
    else if (!rule.by_count || !(rule.top_p < 1.f)) st.mode = kEdge;
    return st;
  }

  __device__ __forceinline__ void collect_slice(int slice, const RowState& st, u32x4 (&held)[kAhead]) {
    const int t = threadIdx.x, lane = t & 63;
    if (t == 0) sh.n = 0;
    __syncthreads();
    if (!ONE && slice == 0 && t == 0) *reinterpret_cast<RowState*>(ws.state) = st;
    if (st.mode == kHard || st.mode == kNone) return;
    unsigned long long* list = ONE ? sh.keys : ws.list + (int64_t)slice * kList;
    double* slab = ONE ? sh.slab : ws.slab;
    const double least = rule.min_p;
    // A value's range from a product alone: floor(x scale) >= g where x scale >= g.
    const float edge = st.range, past = st.range + 1.f;
    auto list_it = [&](float x, int id) {
      const int n = atomicAdd(&sh.n, 1);
      if (n < kList) list[n] = (unsigned long long)key_of(R::clean(__float_as_uint(x))) << 32 | (uint32_t)id;
    };
    if (st.mode == kFirst) {
      units(slice, held, ONE, [&](u32x4 y, int u) {
        float x[VEC];
        R::values(y, x);
        float most = x[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) most = fmaxf(most, x[i]);
        if (most * rule.scale >= edge && most > -INFINITY) {
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (x[i] * rule.scale >= edge && x[i] > -INFINITY) list_it(x[i], row.first_id(u) + i);
        }
      });
      __syncthreads();
      if (!ONE && t == 0) ws.n[slice] = sh.n;
      return;
    }
    auto in_edge = [&](float x) { return st.mode == kEdge && x * rule.scale >= edge && x * rule.scale < past; };
    auto ahead = [&](float x) { return st.mode == kAll || x * rule.scale >= past; };       // summed, not listed
    if constexpr (!F32) {
      // NaN where a value needs a closer look: listed, or none of the table's
      for (int i = t; i < kValues; i += kThreads) {
        const float v = value_at(i);
        double y = ahead(v) && i < kMasked ? weight(v) : 0.0;
        y = y >= least ? y : 0.0;
        sh.weights[i] = i < kMasked && (value_other(i) || in_edge(v)) ? NAN : y;
      }
      __syncthreads();
    }
    // a slice's units are whole runs of ids, a wave takes every sixteenth; so many
    // 64-unit parts of them at once
    constexpr int kAtOnce = ONE ? (F32 ? 8 : 4) : 2;
    const int per = p.slab_units, parts = per / 64, u1 = end(slice), w = t / 64;
    const int runs = (u1 - begin(slice) + per - 1) / per;
    const int steps = w < runs ? ((runs - w + kWaves - 1) / kWaves) * parts : 0;      // parts of this wave
    auto unit_of = [&](int k) { return begin(slice) + (w + k / parts * kWaves) * per + k % parts * 64 + lane; };
    double sum = 0.0;
    for (int k0 = 0; k0 < steps; k0 += kAtOnce) {
      u32x4 r[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int u = unit_of(k0 + j);
        r[j] = k0 + j < steps && u < u1 ? row.raw(u) : u32x4{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        if (k0 + j >= steps) break;
        auto take = [&](float x, int i) {
          if (in_edge(x)) {
            list_it(x, row.first_id(unit_of(k0 + j)) + i);
          } else if (x > -INFINITY && ahead(x)) {
            const double y = weight(x);
            if (y >= least) sum += y;
          }
        };
        if constexpr (F32) {
          float x[VEC];
          R::values(r[j], x);
          float most = x[0];
#pragma unroll
          for (int i = 1; i < VEC; ++i) most = fmaxf(most, x[i]);
          if (st.mode == kAll || most * rule.scale >= edge) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) take(x[i], i);
          }
        } else {
          double y[VEC], all = sum;
          u16x2 unused = {0, 0};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t at = value_places<8>(r[j][w], unused);
            y[2 * w] = *reinterpret_cast<const double*>(reinterpret_cast<const char*>(sh.weights) + (at & 0xffffu));
            y[2 * w + 1] = *reinterpret_cast<const double*>(reinterpret_cast<const char*>(sh.weights) + (at >> 16));
          }
#pragma unroll
          for (int i = 0; i < VEC; ++i) all += y[i];
          if (all == all) {
            sum = all;
          } else {
            uint32_t look = 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const bool in = y[i] == y[i];
              sum += in ? y[i] : 0.0;
              look |= (uint32_t)!in << i;
            }
            while (look) {
              const int i = __builtin_ctz(look);
              look &= look - 1;
              const uint32_t h = i < 4 ? (i < 2 ? r[j].x : r[j].y) : (i < 6 ? r[j].z : r[j].w);
              take(__uint_as_float(i & 1 ? h & 0xffff0000u : h << 16), i);
            }
          }
        }
        if ((k0 + j) % parts == parts - 1) {
          sum = wave_sum(sum);
          if (lane == 0) slab[begin(slice) / per + w + (k0 + j) / parts * kWaves] = sum;
          sum = 0.0;
        }
      }
    }
    __syncthreads();
    if (!ONE && t == 0) ws.n[slice] = sh.n;
  }

  // keys[0 .. n) ascending (n <= kList; all different).  Up to 64 by counting for each
  // how many are smaller.  Up to 1024: a wave puts 64 of them in order among its
  // lanes, then each finds its place in all runs of 64 by bisection, eight runs at
  // once, whose steps wait for memory together (450 of them 1.3 + 1.7 us; by counting
  // and one run after the other 1.8 + 1.9, by counting over all of them 6.5).  More
  // by a bitonic sort (entries up to the next power of two are written).
  __device__ __forceinline__ void sort(unsigned long long* keys, int n) const {
    const int t = threadIdx.x, lane = t & 63;
    if (n <= 64) {
      if (t < n) {
        const unsigned long long mine = keys[t];
        int at = 0;
#pragma unroll 16
        for (int j = 0; j < n; ++j) at += keys[j] < mine;
        keys[at] = mine;
      }
      __syncthreads();
      return;
    }
    if (n <= kThreads) {
      unsigned long long* runs = sh.runs;
      unsigned long long mine = ~0ull;
      constexpr int kAtOnce = 8;
      if (t - lane < n) {
        mine = t < n ? keys[t] : ~0ull;
#pragma unroll
        for (int k = 2; k <= 64; k *= 2)
#pragma unroll
          for (int j = k / 2; j > 0; j /= 2) {
            const unsigned long long y = __shfl_xor(mine, j);
            const bool least = (lane & j) == 0;
            mine = (y < mine) == (least == ((lane & k) == 0)) ? y : mine;
          }
        runs[t] = mine;
      }
      __syncthreads();
      if (t < n) {
        int at = 0;
        for (int r = 0; r < n; r += 64 * kAtOnce) {
          int k[kAtOnce];                                  // of the last run again where there are fewer
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j) k[j] = min(r + 64 * j, (n - 1) & ~63);
#pragma unroll
          for (int step = 32; step > 0; step /= 2)
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) k[j] += runs[k[j] + step - 1] < mine ? step : 0;
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j)
            if (r + 64 * j < n) at += k[j] - (r + 64 * j) + (runs[k[j]] < mine);
        }
        keys[at] = mine;
      }
      __syncthreads();
      return;
    }
    int N = 64;
    while (N < n) N *= 2;
    for (int i = n + threadIdx.x; i < N; i += kThreads) keys[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= N; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int i = threadIdx.x; i < N / 2; i += kThreads) {
          const int a = (i & ~(j - 1)) * 2 + (i & (j - 1)), b = a + j;
          const unsigned long long x = keys[a], y = keys[b];
          if ((x > y) == ((a & k) == 0)) {
            keys[a] = y;
            keys[b] = x;
          }
        }
        __syncthreads();
      }
  }
  __device__ __forceinline__ static float value_of(unsigned long long key) {
    const uint32_t k = (uint32_t)(key >> 32);
    return __uint_as_float((int32_t)k < 0 ? k : ~k & 0x7fffffffu);
  }
  // The weights of two neighbours of the list, and their sums from the list's start.
  struct Two {
    double w0, w1, s0, s1;
  };
  // Up to 128 entries, two a lane, every wave has all of them and needs no barrier.
  __device__ __forceinline__ static int entry_of(int n) { return 2 * (n <= 128 ? threadIdx.x & 63 : threadIdx.x); }
  template <typename T>
  __device__ __forceinline__ T scan(int n, T x) const {
    return n <= 128 ? wave_scan(x, T(0), Plus{}) : block_scan(sh, turn, x);
  }
  template <typename T, typename F>
  __device__ __forceinline__ T reduce(int n, T x, T none, F&& f) const {
    return n <= 128 ? last_lane(wave_scan(x, none, f)) : block_reduce(sh, turn, x, none, f);
  }
  // x of the thread whose first entry is 2 i.
  __device__ __forceinline__ double of_pair(int n, double x, int i) const {
    if (n <= 128) return of_lane(x, __builtin_amdgcn_readfirstlane(i));
    if ((int)threadIdx.x == i) reinterpret_cast<double*>(sh.out)[0] = x;
    __syncthreads();
    x = reinterpret_cast<double*>(sh.out)[0];
    __syncthreads();
    return x;
  }
  __device__ __forceinline__ Two weights(int n) const {
    const int i = entry_of(n);
    Two y;
    y.w0 = i < n ? weight(value_of(sh.keys[i])) : 0.0;
    y.w1 = i + 1 < n ? weight(value_of(sh.keys[i + 1])) : 0.0;
    y.s1 = scan(n, y.w0 + y.w1);
    y.s0 = y.s1 - y.w1;
    return y;
  }
  // The number of list entries that `f(entry, weight, sum)` holds for (a run from the front).
  template <typename F>
  __device__ __forceinline__ int count(const Two& y, int n, F&& f) const {
    const int i = entry_of(n);
    const int c = (i < n && f(i, y.w0, y.s0)) + (i + 1 < n && f(i + 1, y.w1, y.s1));
    return reduce(n, c, 0, Plus{});
  }

  // The token and what stays.  False: the row takes the other way.
  __device__ __forceinline__ bool finish(int r, const RowState& st, RowDone& done, int& token) {
    const int t = threadIdx.x;
    float tops[kSampleSlices];
    load_tops(tops);
    done = {{-INFINITY, 0x7fffffff}, 1.0, top, 1};
    token = -1;
    if (st.mode == kNone) {
      done.kept = 0;
      return true;
    }
    if (st.mode == kHard) return false;
    int n = 0;
    if (st.mode != kAll) {
      if constexpr (ONE) {
        n = sh.n;
        if (n > kList) return false;                       // the same for all threads
      } else {
        int m[kSampleSlices];
#pragma unroll
        for (int s = 0; s < kSampleSlices; ++s) m[s] = ws.n[min(s, p.slices - 1)];
#pragma unroll
        for (int s = 0; s < kSampleSlices; ++s) m[s] = s < p.slices ? min(m[s], kList + 1) : 0;
#pragma unroll
        for (int s = 0; s < kSampleSlices; ++s) n += m[s];
        if (n > kList) return false;                         // the same for all threads
        for (int i = t; i < n; i += kThreads) {
          int s = 0, at = i;
#pragma unroll
          for (int y = 0; y < kSampleSlices - 1; ++y)
            if (s == y && at >= m[y]) at -= m[y], ++s;
          sh.keys[i] = ws.list[(int64_t)s * kList + at];
        }
        __syncthreads();
      }
      sort(sh.keys, n);
    }
    const double u = p.tokens ? (double)p.uniforms[r] : 0.0, least = rule.min_p;
    if (st.mode == kFirst) {
      n = min(n, rule.k);
      Two y = weights(n);
      int stay = n;
      if (rule.top_p < 1.f) {
        const double mark = (double)rule.top_p * of_pair(n, n & 1 ? y.s0 : y.s1, (n - 1) / 2);
        stay = min(stay, 1 + count(y, n, [&](int, double, double s) { return s < mark; }));
      }
      if (least > 0.0) stay = min(stay, max(1, count(y, n, [&](int, double w, double) { return w >= least; })));
      done.cut = {value_of(sh.keys[stay - 1]), (int)(uint32_t)sh.keys[stay - 1]};
      if (stay > 128) {
        pick(y, stay, u, done, token);
        return true;
      }
      // ids ascending: (id, place in the list)
      for (int i = t; i < stay; i += kThreads) sh.by_id[i] = (sh.keys[i] << 32) | (uint32_t)i;
      __syncthreads();
      sort(sh.by_id, stay);
      const int i = entry_of(stay);
      const double w0 = i < stay ? weight(value_of(sh.keys[(uint32_t)sh.by_id[i]])) : 0.0;
      const double w1 = i + 1 < stay ? weight(value_of(sh.keys[(uint32_t)sh.by_id[i + 1]])) : 0.0;
      const double s1 = scan(stay, w0 + w1), s0 = s1 - w1;
      done.total = of_pair(stay, s1, (stay - 1) / 2);
      // the first whose sum exceeds the mark (none: the last that has weight)
      const double mark = u * done.total;
      int best = 0x7fffffff, last = 0;
      if (w1 > 0.0) last = i + 1;
      else if (w0 > 0.0) last = i;
      if (w1 > 0.0 && s1 > mark) best = i + 1;
      if (w0 > 0.0 && s0 > mark) best = i;
      best = reduce(stay, best, 0x7fffffff, Least{});
      last = reduce(stay, last, 0, Most{});
      token = (int)(sh.by_id[min(best, last)] >> 32);
      return true;
    }
    if (st.mode == kEdge) {
      if (n == 0) return false;
      const Two y = weights(n);
      // how many of the list stay: the first that reaches what is left of the mark is the last
      const double left = st.mark - st.before;
      const int stay = rule.by_count ? min(max((int)left, 1), n)
                                     : min(1 + count(y, n, [&](int, double, double s) { return s < left; }), n);
      done.cut = {value_of(sh.keys[stay - 1]), (int)(uint32_t)sh.keys[stay - 1]};
      for (int i = t; i < kSlabs; i += kThreads) sh.add[i] = 0;
      __syncthreads();
      // to the sums of their runs, in units of 2^-48 so that their order does not matter
      for (int k = 0; k < 2; ++k) {
        const int i = 2 * t + k;
        const double w = k ? y.w1 : y.w0;
        if (i < stay && w >= least)
          atomicAdd(&sh.add[((int)(uint32_t)sh.keys[i] + row.head) / VEC / p.slab_units], fixed(w, kListUnit));
      }
      __syncthreads();
    }
    by_runs(ONE ? sh.slab : ws.slab, st.mode == kEdge, u, done, token);
    return true;
  }

  // The total, and the token, of more than 128 list entries that stay, whose weights are
  // y's: which run of ids has it by the runs' sums (fixed point, whose order does not
  // matter), then which of the run's entries.  (Sorted by their ids instead, 400 of
  // them: 2 us longer.)
  __device__ __forceinline__ void pick(const Two& y, int stay, double u, RowDone& done, int& token) {
    const int t = threadIdx.x;
    auto run_of = [&](int id) { return (id + row.head) / VEC / p.slab_units; };
    static_assert(kSlabs == kThreads, "a run a thread");
    sh.add[t] = 0;
    if (t == 0) sh.n = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (2 * t + k < stay) atomicAdd(&sh.add[run_of((int)(uint32_t)sh.keys[2 * t + k])], fixed(k ? y.w1 : y.w0, kListUnit));
    __syncthreads();
    const unsigned long long mine = sh.add[t], upto = block_scan(sh, turn, mine);
    if (t == kThreads - 1) sh.out[0] = upto;
    __syncthreads();
    const double all = (double)sh.out[0], mark = u * all;
    done.total = all * (1.0 / kListUnit);
    // the first whose sum exceeds the mark (none: the last that has weight)
    int best = block_reduce(sh, turn, mine && (double)upto > mark ? t : 0x7fffffff, 0x7fffffff, Least{});
    best = min(best, block_reduce(sh, turn, mine ? t : 0, 0, Most{}));
    if (t == best) sh.out[0] = upto - mine;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (2 * t + k < stay) {
        const int id = (int)(uint32_t)sh.keys[2 * t + k];
        const unsigned long long w = fixed(k ? y.w1 : y.w0, kListUnit);
        if (w && run_of(id) == best) {
          const int at = atomicAdd(&sh.n, 1);
          sh.by_id[at] = w;
          sh.ids[at] = id;
        }
      }
    __syncthreads();
    const int m = sh.n;
    const unsigned long long before = sh.out[0];
    int first = 0x7fffffff, last = -1;
    for (int i = t; i < m; i += kThreads) {
      const int id = sh.ids[i];
      unsigned long long s = before;
      for (int j = 0; j < m; ++j) s += sh.ids[j] <= id ? sh.by_id[j] : 0;
      if ((double)s > mark) first = min(first, id);
      last = max(last, id);
    }
    first = block_reduce(sh, turn, first, 0x7fffffff, Least{});
    last = block_reduce(sh, turn, last, -1, Most{});
    token = min(first, last);
  }

  // The total, and the token, of what stays by the sums of its runs of ids (`list`: and
  // the listed ones').
  __device__ __forceinline__ void by_runs(const double* slab, bool list, double u, RowDone& done, int& token) {
    static_assert(kSlabs == kThreads, "a run a thread");
    const int t = threadIdx.x, slabs = (row.units + p.slab_units - 1) / p.slab_units;
    double mine = t < slabs ? slab[t] : 0.0;
    if (list && t < slabs) mine += (double)sh.add[t] * (1.0 / kListUnit);
    const double s1 = block_scan(sh, turn, mine);
    if (t == kThreads - 1) reinterpret_cast<double*>(sh.out)[0] = s1;
    __syncthreads();
    done.total = reinterpret_cast<double*>(sh.out)[0];
    if (!p.tokens) return;
    const double mark = u * done.total;
    int best = block_reduce(sh, turn, mine > 0.0 && s1 > mark ? t : 0x7fffffff, 0x7fffffff, Least{});
    best = min(best, block_reduce(sh, turn, mine > 0.0 ? t : 0, 0, Most{}));
    if (t == best) reinterpret_cast<double*>(sh.out)[0] = s1 - mine;
    __syncthreads();
    const double before = reinterpret_cast<double*>(sh.out)[0];
    if (t < 64)
      token = in_run(best * p.slab_units, min((best + 1) * p.slab_units, row.units), before, mark, done.cut, rule.min_p);
  }

  // The first token of units [u0, u1) where the sum of what stays, from `run` on, exceeds
  // `mark`, or the last that has weight; by one wave.
  __device__ __forceinline__ int in_run(int u0, int u1, double run, double mark, const Cut& cut, double least) const {
    const int lane = threadIdx.x;
    int best = 0x7fffffff, behind = -1;
    for (; u0 < u1 && best == 0x7fffffff; u0 += 64) {
      const int u = u0 + lane;
      float x[VEC];
      double y[VEC], mine = 0.0;
      if (u < u1) row.load(u, x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        y[i] = 0.0;
        if (u < u1 && x[i] > -INFINITY && cut.keeps(x[i], row.first_id(u) + i)) {
          y[i] = weight(x[i]);
          if (!(y[i] >= least)) y[i] = 0.0;
        }
        mine += y[i];
      }
      const double sum = wave_scan(mine, 0.0, Plus{});
      double at = run + sum - mine;
      int found = 0x7fffffff;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        at += y[i];
        if (y[i] > 0.0) behind = row.first_id(u) + i;
        if (y[i] > 0.0 && at > mark && found == 0x7fffffff) found = row.first_id(u) + i;
      }
      best = last_lane(wave_scan(found, 0x7fffffff, Least{}));
      run += last_lane(sum);
    }
    behind = last_lane(wave_scan(behind, -1, Most{}));
    return best == 0x7fffffff ? behind : best;
  }

  // The row by the histograms of the whole of it (the first half of this file).
  __device__ __forceinline__ void hard(int r, RowDone& done, int& token) {
    const int t = threadIdx.x;
    __syncthreads();
    Sampler<F32> S(row, sh);
    S.top = top;
    S.c = rule.c;
    S.bins = (float)kBins / (32.f * rule.T);
    S.fix = 62 - (32 - __builtin_clz(p.V));
    Cut cut = {-INFINITY, 0x7fffffff};
    auto clear = [&] {
      __syncthreads();
      for (int i = t; i < kBins; i += kThreads) sh.mass[i] = 0;
      __syncthreads();
    };
    if (rule.k < p.V) {
      clear();
      int n = 0;
      S.each([&](float x, int) {
        atomicAdd(&sh.count[S.range_of(x)], 1u);
        ++n;
      });
      n = block_reduce(sh, turn, n, 0, Plus{});
      if (rule.k < n) cut = S.template last_of<false>((unsigned long long)rule.k, cut);
    }
    if (rule.top_p < 1.f) {
      clear();
      unsigned long long all = 0;
      S.each([&](float x, int id) {
        if (!cut.keeps(x, id)) return;
        const unsigned long long w = S.fixed(x);
        atomicAdd(&sh.mass[S.range_of(x)], w);
        all += w;
      });
      all = block_reduce(sh, turn, all, 0ull, Plus{});
      const unsigned long long mark = (unsigned long long)ceil((double)rule.top_p * (double)all);
      cut = S.template last_of<true>(min(max(mark, 1ull), all), cut);
    }
    // sums of the weights over runs of ids, in the ids' order
    const double least = rule.min_p;
    const int lane = t & 63, per = p.slab_units, slabs = (row.units + per - 1) / per;
    for (int s = t / 64; s < slabs; s += kWaves) {
      double sum = 0.0;
      for (int u = s * per + lane; u < min((s + 1) * per, row.units); u += 64) {
        float x[VEC];
        row.load(u, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (x[i] > -INFINITY && cut.keeps(x[i], row.first_id(u) + i)) {
            const double y = weight(x[i]);
            if (y >= least) sum += y;
          }
      }
      sum = wave_sum(sum);
      if (lane == 0) sh.slab[s] = sum;
    }
    __syncthreads();
    done.cut = cut;
    by_runs(sh.slab, false, p.tokens ? (double)p.uniforms[r] : 0.0, done, token);
  }

  __device__ __forceinline__ void write_rows(int r, int slice, const RowDone& done) {
    top = done.top;
    char* out = static_cast<char*>(p.rows) + r * p.rows_stride * R::EB;
    const bool probs = p.kind == 1;
    const float none = probs ? 0.f : F32 ? -3.4028234663852886e38f : -3.3895313892515355e38f;
    const bool lines = (reinterpret_cast<uintptr_t>(out) - (uintptr_t)(row.head * R::EB)) % 16 == 0;
    const double least = rule.min_p, share = 1.0 / done.total;
    auto write = [&](int u, u32x4 in) {
      float x[VEC], y[VEC];
      R::values(in, x);
      uint32_t raw[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        y[i] = none;
        if (done.kept && x[i] > -INFINITY && done.cut.keeps(x[i], row.first_id(u) + i)) {
          const double q = weight(x[i]);
          if (q >= least) y[i] = probs ? (float)(q * share) : rule.one ? 0.f : (float)((double)x[i] / (double)rule.T);
        }
        raw[i] = F32 ? __float_as_uint(y[i]) : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[i]);
      }
      char* at = out + (int64_t)row.first_id(u) * R::EB;
      if (lines && row.whole(u)) {
        u32x4 z;
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = F32 ? raw[i] : raw[(2 * i) % VEC] | raw[(2 * i + 1) % VEC] << 16;
        *reinterpret_cast<u32x4*>(at) = z;
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int id = row.first_id(u) + i;
          if (id < 0 || id >= p.V) continue;
          if constexpr (F32) reinterpret_cast<uint32_t*>(at)[i] = raw[i];
          else reinterpret_cast<uint16_t*>(at)[i] = (uint16_t)raw[i];
        }
      }
    };
    for (int u = begin(slice) + threadIdx.x; u < end(slice); u += kThreads) write(u, row.raw(u));
  }
};

// STEP: 0 scan, 1 collect, 2 token, 3 rows; 4: all of them for one slice a row; 5:
// 2 and 3, the former again in every slice (the rows are not the logits).
template <bool F32, int STEP>
__global__ __launch_bounds__(kThreads) void sample_step(SampleParams p) {
  __shared__ Shared sh;
  constexpr bool ONE = STEP == 4;
  const int r = STEP == 2 || ONE ? blockIdx.x : blockIdx.x / p.slices;
  const int slice = STEP == 2 || ONE ? 0 : blockIdx.x - r * p.slices;
  const Row<F32> row(static_cast<const char*>(p.logits) + r * p.stride * Row<F32>::EB, p.V);
  const Rule rule(p, r);
  const RowView view(p, r);
  Slices<F32, ONE> S{p, row, sh, rule, view.s, 0.f, 0.0};
  RowState st;
  RowDone done;
  u32x4 units[S.kAhead];
  if constexpr (STEP == 0 || ONE) S.scan_slice(slice, units);
  if constexpr (ONE) __syncthreads();
  if constexpr (STEP == 1 || ONE) {
    st = S.state();
    S.collect_slice(slice, st, units);
  }
  if constexpr (STEP == 2 || STEP == 5) st = *reinterpret_cast<const RowState*>(view.s.state);
  if constexpr (ONE) __syncthreads();
  if constexpr (STEP == 2 || STEP == 5 || ONE) {
    int token;
    if (!S.finish(r, st, done, token)) S.hard(r, done, token);
    if (threadIdx.x == 0 && slice == 0) {
      if (p.tokens) p.tokens[r] = token;
      if (STEP == 2 && p.kind) *reinterpret_cast<RowDone*>(view.s.done) = done;
    }
  }
  if constexpr (STEP == 3) done = *reinterpret_cast<const RowDone*>(view.s.done);
  if constexpr (ONE) __syncthreads();                      // the rows may be the logits
  if constexpr (STEP == 3 || STEP == 5 || ONE) {
    if (p.kind) S.write_rows(r, slice, done);
  }
}

template <bool F32>
hipError_t steps(const SampleParams& p, int rows, hipStream_t s) {
  if (p.slices == 1) {
    sample_step<F32, 4><<<dim3(rows), dim3(kThreads), 0, s>>>(p);
    return hipGetLastError();
  }
  sample_step<F32, 0><<<dim3(rows * p.slices), dim3(kThreads), 0, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sample_step<F32, 1><<<dim3(rows * p.slices), dim3(kThreads), 0, s>>>(p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (p.kind != 0 && p.rows != p.logits) {
    sample_step<F32, 5><<<dim3(rows * p.slices), dim3(kThreads), 0, s>>>(p);
    return hipGetLastError();
  }
  sample_step<F32, 2><<<dim3(rows), dim3(kThreads), 0, s>>>(p);
  if ((e = hipGetLastError()) != hipSuccess || p.kind == 0) return e;
  sample_step<F32, 3><<<dim3(rows * p.slices), dim3(kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleParams& p, int num_rows, bool f32, hipStream_t s) {
  return f32 ? steps<true>(p, num_rows, s) : steps<false>(p, num_rows, s);
}

}  // namespace sv
