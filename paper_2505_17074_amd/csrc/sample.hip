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
#include "sv_sample.h"

#include <type_traits>

namespace sv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;            // ranges of a histogram
constexpr int kList = 1024;            // tokens of a list: one a thread
constexpr int kSlabs = 256;            // runs of ids whose weights are summed apart

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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

template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) x += __shfl_xor(x, i);
  return x;
}

// One row's elements, in 16-byte units on the memory's own 16-byte borders.
template <bool F32>
struct Row {
  static constexpr int VEC = F32 ? 4 : 8, EB = F32 ? 4 : 2;
  const char* base;          // of unit 0 (the row's first element is its `head`-th)
  int head, V, units;

  __device__ Row(const void* p, int V_) : V(V_) {
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

struct Shared {
  union {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
  };
  struct {
    float x[kList];
    int id[kList];
    double w[kList];
  } list;
  int n;                               // of the list
  unsigned long long red[kWaves];
  unsigned long long out[2];
  double slab[kSlabs];
};

// What stays of a row.
struct Cut {
  float x;
  int id;
  __device__ __forceinline__ bool keeps(float y, int i) const { return y > x || (y == x && i <= id); }
};

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

  __device__ Sampler(const R& r, Shared& s) : row(r), sh(s) {}

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

  template <typename T, typename F>
  __device__ __forceinline__ T block_reduce(T x, F&& f) const {
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x = f(x, __shfl_xor(x, i));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) reinterpret_cast<T*>(sh.red)[threadIdx.x / 64] = x;
    __syncthreads();
    x = reinterpret_cast<T*>(sh.red)[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x = f(x, reinterpret_cast<T*>(sh.red)[i]);
    return x;
  }

  // The range of the histogram where the running sum reaches `mark` (at least one,
  // at most the whole sum), and the sum before it.
  template <typename T>
  __device__ __forceinline__ int find_bin(const T* hist, unsigned long long mark, unsigned long long& before) const {
    static_assert(kBins == 2 * kThreads, "two ranges a thread");
    __syncthreads();
    const int t = threadIdx.x;
    const T a = hist[2 * t], b = hist[2 * t + 1];
    unsigned long long x = (unsigned long long)a + b;
    const unsigned long long own = x;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
      const unsigned long long y = __shfl_up(x, i);
      if ((t & 63) >= i) x += y;
    }
    if ((t & 63) == 63) sh.red[t / 64] = x;
    if (t == 0) sh.out[0] = 0;
    __syncthreads();
    unsigned long long base = 0;
    for (int i = 0; i < t / 64; ++i) base += sh.red[i];
    const unsigned long long s0 = base + x - own, s1 = s0 + a, s2 = s1 + b;
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
  __device__ Cut last_of(unsigned long long mark, const Cut& in) {
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
      lo = block_reduce(lo, [](uint32_t a, uint32_t b) { return min(a, b); });
      hi = block_reduce(hi, [](uint32_t a, uint32_t b) { return max(a, b); });
      n = block_reduce(n, [](int a, int b) { return a + b; });
      if (n <= kList || lo == hi) break;
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
    if (n > kList) return tie<MASS>(lo, mark, sum, in);
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
  __device__ Cut tie(uint32_t key, unsigned long long mark, unsigned long long sum, const Cut& in) {
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
      int s = mine;
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) {
        const int z = __shfl_up(s, i);
        if ((threadIdx.x & 63) >= i) s += z;
      }
      if ((threadIdx.x & 63) == 63) sh.red[threadIdx.x / 64] = s;
      __syncthreads();
      int base = 0, all = 0;
      for (int i = 0; i < kWaves; ++i) {
        base += i < (int)threadIdx.x / 64 ? (int)sh.red[i] : 0;
        all += (int)sh.red[i];
      }
      long long at = so_far + base + s - mine;
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (y[i] == x && in.keeps(y[i], row.first_id(u) + i) && ++at == m) sh.out[0] = row.first_id(u) + i;
      so_far += all;
      __syncthreads();
      if (so_far >= m) break;
    }
    const Cut cut = {x, (int)sh.out[0]};
    __syncthreads();
    return cut;
  }
};

// One work-group a row.
template <bool F32>
__global__ __launch_bounds__(kThreads) void sample_row(SampleParams p) {
  __shared__ Shared sh;
  const int r = blockIdx.x, t = threadIdx.x;
  const Row<F32> row(static_cast<const char*>(p.logits) + r * p.stride * Row<F32>::EB, p.V);
  constexpr int VEC = Row<F32>::VEC;
  Sampler<F32> S(row, sh);

  float top = -INFINITY;
  S.each([&](float x, int) { top = fmaxf(top, x); });
  top = S.block_reduce(top, [](float a, float b) { return fmaxf(a, b); });
  S.top = top;

  float T = p.temperature ? p.temperature[r] : 1.f;
  int k = p.top_k ? p.top_k[r] : 0;
  float tp = p.top_p ? p.top_p[r] : 1.f;
  float mp = p.min_p ? p.min_p[r] : 0.f;
  const bool one = !(T > 0.f) || !(tp > 0.f) || !(mp <= 1.f);
  if (k < 1 || k > p.V) k = p.V;
  if (one) k = 1;
  if (!(T > 0.f) || one) T = 1.f;
  if (one) tp = 1.f, mp = 0.f;
  S.c = 1.4426950408889634074 / (double)T;
  S.bins = (float)kBins / (32.f * T);
  S.fix = 62 - (32 - __builtin_clz(p.V));

  Cut cut = {-INFINITY, 0x7fffffff};
  if (top > -INFINITY) {
    auto clear = [&] {
      __syncthreads();
      for (int i = t; i < kBins; i += kThreads) sh.mass[i] = 0;
      __syncthreads();
    };
    if (k < p.V) {
      clear();
      int n = 0;
      S.each([&](float x, int) {
        atomicAdd(&sh.count[S.range_of(x)], 1u);
        ++n;
      });
      n = S.block_reduce(n, [](int a, int b) { return a + b; });
      if (k < n) cut = S.template last_of<false>((unsigned long long)k, cut);
    }
    if (tp < 1.f) {
      clear();
      unsigned long long all = 0;
      S.each([&](float x, int id) {
        if (!cut.keeps(x, id)) return;
        const unsigned long long w = S.fixed(x);
        atomicAdd(&sh.mass[S.range_of(x)], w);
        all += w;
      });
      all = S.block_reduce(all, [](unsigned long long a, unsigned long long b) { return a + b; });
      const unsigned long long mark = (unsigned long long)ceil((double)tp * (double)all);
      cut = S.template last_of<true>(min(max(mark, 1ull), all), cut);
    }
  }
  const double least = mp;
  auto kept = [&](float x, int id) { return x > -INFINITY && cut.keeps(x, id); };

  // sums of the weights over runs of ids, in the ids' order
  double total = 0.0;
  const int per = (row.units + kSlabs - 1) / kSlabs;       // units of a run
  const int w = t / 64, lane = t & 63;
  for (int s = w; s < kSlabs; s += kWaves) {
    double sum = 0.0;
    for (int u0 = s * per; u0 < min((s + 1) * per, row.units); u0 += 64) {
      const int u = u0 + lane;
      if (u < (s + 1) * per) {
        float x[VEC];
        row.load(u, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (kept(x[i], row.first_id(u) + i)) {
            const double y = S.weight(x[i]);
            if (y >= least) sum += y;
          }
        }
      }
    }
    sum = wave_sum(sum);
    if (lane == 0) sh.slab[s] = sum;
  }
  __syncthreads();
  for (int s = 0; s < kSlabs; ++s) total += sh.slab[s];

  if (p.tokens && w == 0) {
    int token = -1;
    if (top > -INFINITY) {
      const double mark = (double)p.uniforms[r] * total;
      double run = 0.0;
      int s = 0, last = 0;
      for (; s < kSlabs; ++s) {
        if (sh.slab[s] > 0.0) last = s;
        if (run + sh.slab[s] > mark) break;
        run += sh.slab[s];
      }
      if (s == kSlabs) {                                   // a uniform of one: the last token that has weight
        s = last;
        run = 0.0;
        for (int i = 0; i < s; ++i) run += sh.slab[i];
      }
      int best = 0x7fffffff, behind = -1;
      for (int u0 = s * per; u0 < min((s + 1) * per, row.units) && best == 0x7fffffff; u0 += 64) {
        const int u = u0 + lane;
        float x[VEC];
        double y[VEC], mine = 0.0;
        if (u < (s + 1) * per) row.load(u, x);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          y[i] = 0.0;
          if (u < (s + 1) * per && kept(x[i], row.first_id(u) + i)) {
            y[i] = S.weight(x[i]);
            if (!(y[i] >= least)) y[i] = 0.0;
          }
          mine += y[i];
        }
        double sum = mine;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
          const double z = __shfl_up(sum, i);
          if (lane >= i) sum += z;
        }
        double at = run + sum - mine;
        int found = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          at += y[i];
          if (y[i] > 0.0) behind = row.first_id(u) + i;
          if (y[i] > 0.0 && at > mark && found == 0x7fffffff) found = row.first_id(u) + i;
        }
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) found = min(found, __shfl_xor(found, i));
        best = found;
        run += __shfl(sum, 63);
      }
#pragma unroll
      for (int i = 32; i > 0; i >>= 1) behind = max(behind, __shfl_xor(behind, i));
      token = best == 0x7fffffff ? behind : best;
    }
    if (lane == 0) p.tokens[r] = token;
  }

  if (p.kind == 0) return;
  __syncthreads();                                         // the rows may be the logits
  char* out = static_cast<char*>(p.rows) + r * p.rows_stride * Row<F32>::EB;
  const float lowest = F32 ? -3.4028234663852886e38f : -3.3895313892515355e38f;
  const bool lines = (reinterpret_cast<uintptr_t>(out) - (uintptr_t)(row.head * Row<F32>::EB)) % 16 == 0;
  S.each_unit([&](int u, const float (&x)[VEC]) {
    float y[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      y[i] = p.kind == 1 ? 0.f : lowest;
      if (kept(x[i], row.first_id(u) + i)) {
        const double q = S.weight(x[i]);
        if (q >= least) y[i] = p.kind == 1 ? (float)(q / total) : one ? 0.f : (float)((double)x[i] / (double)T);
      }
    }
    uint32_t raw[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) raw[i] = F32 ? __float_as_uint(y[i]) : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y[i]);
    char* at = out + (int64_t)row.first_id(u) * Row<F32>::EB;
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
  });
}

}  // namespace

hipError_t launch_sample(const SampleParams& p, int num_rows, bool f32, hipStream_t s) {
  if (f32) sample_row<true><<<dim3(num_rows), dim3(kThreads), 0, s>>>(p);
  else sample_row<false><<<dim3(num_rows), dim3(kThreads), 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace sv
