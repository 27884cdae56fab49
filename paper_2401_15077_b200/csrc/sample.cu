// Sampling with temperature, top-k, top-p and min-p: a token per row of logits, and / or the distribution that it is drawn from.
//
// With w(v) = exp((z(v) - max z) / temperature), what the filters leave is the first tokens of the order (z descending, id ascending): all
// with a greater z than some z*, and the first few of those that equal it.  So nothing is sorted: each filter looks for its cut (z*, how many
// of z*) by a histogram over z and a ranking of the few values in the bin that the cut falls into.
//   top-k   counts; top-p: masses, after the mass of all that top-k left; min-p: w >= min_p, a comparison
// A cluster of C CTAs takes a row, each a slice of the vocabulary, which stays in shared memory (in the logits' own type) for all passes
// over it; histograms are merged and candidates exchanged through distributed shared memory.
//
// Weights are fp64 (argument, reduction by a table of sixteenths, polynomial) and are summed as integers of 2^-q, q = 43 .. 46 (the largest with which V
// of them fit 63 bits): sums then depend neither on the order of atomics nor on C.  A sum over V tokens is off by V * 2^-(q+1) at the most (10^5 tokens:
// 7e-10) and by 1e-13 * sqrt(V) or so of the largest weight as a rule; fp32 sums (relative 1e-6) would decide visibly otherwise.
//
// What top-p may cut off is bounded before its histogram is taken: n tokens of weights below (1 - p) Z / n sum to less than (1 - p) Z, so
// the cut is not among them.  Of a vocabulary's long tail nothing reaches the atomics then.
//
// What bounds it: instructions and their latencies (some 170 a token with top-p over a flat distribution, of which fp64 takes a third of the
// time that the SMs issue) and nine cluster barriers of about a microsecond, not the bytes.  From a graph, 64 rows of 129537 bf16 logits with
// all filters, tokens: 46 us (16.6 MB: 2.5 us); 656 rows of 32000 fp32 logits with top-p, distributions: 160 us (168 MB: 26 us; 45 of the 160 are the pass that
// writes).  Measured on the way: exponentials and histogram updates element by element, without picking what is left: 86 and 332 us; one CTA per SM: 216 us for the
// 656 rows; 512 candidates ranked at once: 53 us for the 64; positions of picked values by a scan over the lanes instead of a ballot per element: the same.
#include <cooperative_groups.h>

#include <type_traits>
#include <utility>

#include "sample.cuh"

namespace eagle {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kCountBins = 2048, kMassBins = 1024;
constexpr int kFew = 448;                    // (at least a tile's 32 x 8 and a carry of 31)
constexpr int kCandidates = 128;             // values that are ranked against one another, a thread each (more are cut finer first, which takes less)
constexpr size_t kSliceBytes = 160 * 1024;   // of a slice that stays in shared memory, at the most
constexpr size_t kPairBytes = 66 * 1024;     // and where two CTAs are to fit an SM

typedef unsigned long long u64;

// Shared memory behind the slice.
struct Shared {
  union {
    uint32_t count[kCountBins];      // top-k's histogram
    uint32_t mass[2][kMassBins];     // top-p's: low and high words
  } hist;
  u64 slot[2][kMaxCluster][2];       // exchanges, by turns
  u64 warp_sum[kWarps];
  double roots[16];                  // (sixteen 8-byte words: no two share a bank)
  float few[kWarps][kFew];           // a warp's values that are left of its part of the slice, or of a tile, side by side
  uint32_t list[kCandidates];        // this CTA's candidates
  uint32_t all[kCandidates];         // the cluster's
  u64 weight[kCandidates];
  uint32_t n, lo, hi;                // candidates found here, their range
  // a cut, found by one thread or by several with the same result
  uint32_t cut_key, cut_take, cut_ties;
  u64 cut_base;
  uint32_t bin;
  u64 base;
};

// Order-preserving number of a float (no NaN, no negative zero), and back.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// 2^(j / 16)
__constant__ double kRoots[16] = {1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927, 1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543, 1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};
// 2^(x / 16) for -16000 < x <= 0: the nearest whole number is taken off by adding and subtracting 1.5 * 2^52, its low four bits go through the table, the others
// to the exponent, and what is left, f in [-1/2, 1/2], through 1 + f times the polynomial that interpolates (2^(f / 16) - 1) / f at Chebyshev
// nodes (relative error 9e-15).
__device__ __forceinline__ double exp2_sixteenths(double x, const double* roots) {
  const double big = x + 6755399441055744.0, f = x - (big - 6755399441055744.0);
  const int n = __double2loint(big);
  double r = 1.2716049516906705e-09;
  r = fma(r, f, 1.4676387238435006e-07);
  r = fma(r, f, 1.3550807778387664e-05);
  r = fma(r, f, 0.0009383847926296646);
  r = fma(r, f, 0.04332169878499658);
  r = fma(r, f, 1.0) * roots[n & 15];
  return __hiloint2double(__double2hiint(r) + ((n >> 4) << 20), __double2loint(r));
}

struct Weigher {
  float top;             // the row's largest value
  double top_d, rate;    // 16 log2(e) / temperature
  double unit;           // 2^q
  const double* roots;
  __device__ __forceinline__ double real(float z) const {
    const double x = (static_cast<double>(z) - top_d) * rate;
    const double e = x > -16000.0 ? exp2_sixteenths(x, roots) : 0.0;      // -infinity, and NaN from infinities, are 0
    return z == top ? 1.0 : e;                            // (infinite ones too)
  }
  // A weight of at most 1 as an integer: adding 2^52 leaves it in the low bits of the sum.
  __device__ __forceinline__ u64 whole(double w) const { return __double_as_longlong(fma(w, unit, 4503599627370496.0)) & 0xfffffffffffffull; }
};

// Values of a row in their canonical form: NaN as -infinity, negative zero as zero.  (A maximum passes over NaN; one word: one value or two.)
__device__ __forceinline__ float clean(float z) { return fmaxf(z, -INFINITY) + 0.f; }
template <typename T>
__device__ __forceinline__ uint32_t clean_word(uint32_t w) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(clean(__uint_as_float(w)));
  else {
    const __nv_bfloat162 lowest = __floats2bfloat162_rn(-INFINITY, -INFINITY), zero = __floats2bfloat162_rn(0.f, 0.f);
    const __nv_bfloat162 z = __hadd2_rn(__hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w), lowest), zero);
    return *reinterpret_cast<const uint32_t*>(&z);
  }
}
// The larger one, of each half.
template <typename T>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  else {
    const __nv_bfloat162 z = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&z);
  }
}

template <typename T>
struct Vec {
  static constexpr int kLen = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ float at(int e) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
  }
  __device__ __forceinline__ void set(int e, float z) {
    uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(z);
    else w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | (__float_as_uint(z) & 0xffff0000u) : (w[e >> 1] & 0xffff0000u) | (__float_as_uint(z) >> 16);
    raw = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

__device__ __forceinline__ u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 warp_scan64(u64 v, int lane) {      // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// RESIDENT: the slice is in shared memory; else it is read again from the logits in each pass (vocabularies beyond 8 x 160 KB).
template <typename T, bool RESIDENT>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleParams p, int slice) {
  constexpr int kVec = Vec<T>::kLen, kTile = kThreads * kVec;
  extern __shared__ __align__(16) unsigned char dyn[];
  T* const held = reinterpret_cast<T*>(dyn);
  const int tiles = slice / kTile;
  u64* const part = reinterpret_cast<u64*>(dyn + (RESIDENT ? static_cast<size_t>(slice) * sizeof(T) : 0));      // [tiles][warps]
  uint32_t* const ties = reinterpret_cast<uint32_t*>(part + tiles * kWarps);                                      // [tiles][warps]
  uint16_t* const segment = reinterpret_cast<uint16_t*>(ties + tiles * kWarps);                                   // [tiles][warps]: where a tile's part of a list begins
  __shared__ Shared s;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x / C;
  const int b = static_cast<int>(row / p.R), r = static_cast<int>(row - static_cast<long long>(b) * p.R);
  if (p.num_rows && r >= p.num_rows[b]) return;           // (all of the cluster)

  // ---- the slice.  Positions count from the 16-byte boundary at or before the row's first element, so that vectors are aligned.
  if (tid < 16) s.roots[tid] = kRoots[tid];
  auto started = cluster.barrier_arrive();                // (shared memory of the others is there once all have started)
  const T* const src = static_cast<const T*>(p.logits) + row * p.V;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
  const int first = rank * slice - off;                   // id of the slice's position 0
  auto load = [&](int pos) {                              // canonical values of a vector; what is outside of the row is -infinity
    Vec<T> v;
    const int id = first + pos;
    if (id >= 0 && id + kVec <= p.V) {
      v.raw = __ldg(reinterpret_cast<const uint4*>(src + id));
      v.raw = make_uint4(clean_word<T>(v.raw.x), clean_word<T>(v.raw.y), clean_word<T>(v.raw.z), clean_word<T>(v.raw.w));
    } else {
      v.raw = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float z = -INFINITY;
        if (id + e >= 0 && id + e < p.V) z = clean(static_cast<float>(src[id + e]));
        v.set(e, z);
      }
    }
    return v;
  };
  auto fetch = [&](int pos) {
    if constexpr (RESIDENT) {
      Vec<T> v;
      v.raw = *reinterpret_cast<const uint4*>(held + pos);
      return v;
    } else {
      return load(pos);
    }
  };

  // Two numbers of each CTA to all of them; every thread gets them by rank from the returned slots.
  int turn = 0;
  auto exchange = [&](u64 a, u64 c) {                     // (a, c: of thread 0)
    if (warp == 0) {
      a = __shfl_sync(0xffffffffu, a, 0);
      c = __shfl_sync(0xffffffffu, c, 0);
      if (lane < C) {
        u64* to = cluster.map_shared_rank(&s.slot[turn][rank][0], lane);
        to[0] = a;
        to[1] = c;
      }
    }
    cluster.sync();
    const u64(*got)[2] = s.slot[turn];
    turn ^= 1;
    return got;
  };
  auto block_sum = [&](u64 v) {                           // of all threads, for all threads
    v = warp_sum64(v);
    __syncthreads();
    if (lane == 0) s.warp_sum[warp] = v;
    __syncthreads();
    u64 t = lane < kWarps ? s.warp_sum[lane] : 0;
    return warp_sum64(t);
  };
  auto cluster_sum = [&](u64 v) {
    const u64 mine = block_sum(v);
    const u64(*got)[2] = exchange(mine, 0);
    u64 t = 0;
    for (int c = 0; c < C; ++c) t += got[c][0];
    return t;
  };

  // The values of a warp's part of a tile that `stays(z)` picks, side by side in shared memory behind the `from` first, so that what is expensive (an
  // exponential in fp64) is done for 32 of them at a time however few there are in a vector.  at[e]: where element e is, -1: left out.
  // Returns their number.
  float* const few = s.few[warp];
  auto pick = [&](const Vec<T>& v, int from, auto stays, int* at) {
    int n = from;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const bool in = stays(v.at(e));
      const unsigned mask = __ballot_sync(0xffffffffu, in);
      at[e] = in ? n + __popc(mask & ((1u << lane) - 1u)) : -1;
      if (in) few[at[e]] = v.at(e);
      n += __popc(mask);
    }
    __syncwarp();
    return n;
  };
  // Once a bound is known below which nothing stays, each warp keeps the rest of its part of the slice in that way, if there is room for it in
  // all warps of the CTA: `listed`.  The passes from then on go over these lists.
  bool listed = false;
  int n_listed = 0;
  auto make_list = [&](auto stays) {
    __syncthreads();
    bool fits = true;
    int n = 0;
    for (int i = 0; i < tiles && fits; ++i) {
      int at[kVec];
      if (lane == 0) segment[i * kWarps + warp] = static_cast<uint16_t>(n);
      n = pick(fetch((i * kThreads + tid) * kVec), n, stays, at);
      fits = i + 1 >= tiles || n <= kFew - 32 * kVec;      // (room for another tile)
    }
    listed = !__syncthreads_or(!fits);
    n_listed = n;
  };
  auto in_segment = [&](int i, int* to) {                 // [returned, *to) of the list: tile i
    *to = i + 1 < tiles ? segment[(i + 1) * kWarps + warp] : n_listed;
    return static_cast<int>(segment[i * kWarps + warp]);
  };
  // `done(z)` for every value that may stay (those outside of the row too, unless there is a list).
  auto for_all = [&](auto done) {
    if (listed) {
      for (int j = lane; j < n_listed; j += 32) done(few[j]);
      return;
    }
    for (int i = 0; i < tiles; ++i) {
      const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
      for (int e = 0; e < kVec; ++e) done(v.at(e));
    }
  };
  // The same for those that `stays`, where `done` is expensive; without a list values are carried over from tile to tile until there are 32.
  auto for_few = [&](auto stays, auto done) {
    if (listed) {
      for (int j = lane; j < n_listed; j += 32)
        if (stays(few[j])) done(few[j]);
      return;
    }
    int n = 0;
    for (int i = 0; i < tiles; ++i) {
      int at[kVec];
      n = pick(fetch((i * kThreads + tid) * kVec), n, stays, at);
      int base = 0;
      for (; base + 32 <= n; base += 32) done(few[base + lane]);
      const float rest = base + lane < n ? few[base + lane] : 0.f;
      n -= base;
      __syncwarp();
      if (lane < n) few[lane] = rest;
      __syncwarp();
    }
    if (lane < n) done(few[lane]);
    __syncwarp();
  };

  // ---- the largest value
  uint32_t most = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;     // -infinity
#pragma unroll 4
  for (int i = 0; i < tiles; ++i) {
    const int pos = (i * kThreads + tid) * kVec;
    const Vec<T> v = load(pos);
    if constexpr (RESIDENT) *reinterpret_cast<uint4*>(held + pos) = v.raw;
    most = max_word<T>(most, max_word<T>(max_word<T>(v.raw.x, v.raw.y), max_word<T>(v.raw.z, v.raw.w)));
  }
  uint32_t top_key = sizeof(T) == 4 ? key_of(__uint_as_float(most)) : max(key_of(__uint_as_float(most << 16)), key_of(__uint_as_float(most & 0xffff0000u)));
  top_key = __reduce_max_sync(0xffffffffu, top_key);
  if (lane == 0) s.warp_sum[warp] = top_key;
  __syncthreads();
  top_key = __reduce_max_sync(0xffffffffu, lane < kWarps ? static_cast<uint32_t>(s.warp_sum[lane]) : 0u);
  cluster.barrier_wait(std::move(started));
  {
    const u64(*got)[2] = exchange(top_key, 0);
    for (int c = 0; c < C; ++c) top_key = max(top_key, static_cast<uint32_t>(got[c][0]));
  }
  Weigher w;
  w.top = value_of_key(top_key);
  const bool nothing = w.top == -INFINITY;
  if (nothing && rank == 0 && tid == 0) {
    report_status(p.status, EAGLE_ERR_ROW);
    if (p.tokens) p.tokens[row] = -1;
  }
  const float temperature = p.temperature ? p.temperature[b] : 1.f;
  const int k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f;
  const double least = p.min_p ? static_cast<double>(fminf(fmaxf(p.min_p[b], 0.f), 1.f)) : 0.0;      // (NaN: 0)
  const bool greedy = !(temperature > 0.f);
  w.rate = 16.0 * 1.4426950408889634 / (greedy ? 1.0 : static_cast<double>(temperature));
  w.top_d = w.top;
  w.roots = s.roots;
  const int q = min(46, 63 - (32 - __clz(p.V - 1)));
  w.unit = __hiloint2double((1023 + q) << 20, 0);

  // ---- the cut: tokens with a greater value stay, and the first `take` of those that equal it (`some`: these are not all of them).  `mass`: of
  // all that stay, where a search for the cut has found it.
  float cut = -INFINITY;
  uint32_t take = 0xffffffffu;
  bool some = false, known = false;
  u64 mass = 0;

  // Merged histogram -> the bin in which the prefix reaches the target, with what lies before it.  `reached(before, after)` is true in that
  // bin only.  Every CTA of the cluster does all of it.
  // (A histogram is cleared again only behind a further exchange, so that nobody reads it any more.)
  auto find_bin = [&](auto is_mass, auto reached) {
    constexpr bool MASS = decltype(is_mass)::value;
    constexpr int kPer = (MASS ? kMassBins : kCountBins) / kThreads;
    cluster.sync();                                       // all histograms are complete
    u64 v[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = 0;
    for (int c = 0; c < C; ++c) {
      const auto& hist = *cluster.map_shared_rank(&s.hist, c);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if constexpr (MASS) v[i] += hist.mass[0][tid * kPer + i] + (static_cast<u64>(hist.mass[1][tid * kPer + i]) << 32);
        else v[i] += hist.count[tid * kPer + i];
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += v[i];
    const u64 inc = warp_scan64(sum, lane);
    if (lane == 31) s.warp_sum[warp] = inc;
    __syncthreads();
    u64 before = inc - sum;
    {
      u64 t = lane < kWarps && lane < warp ? s.warp_sum[lane] : 0;
      before += warp_sum64(t);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (reached(before, before + v[i])) {
        s.bin = tid * kPer + i;
        s.base = before;
      }
      before += v[i];
    }
    __syncthreads();
  };
  // Exact 64-bit sums by 32-bit atomics: the carry goes along with the high word.
  auto add_mass = [&](int bin, u64 x) {
    const uint32_t lo = static_cast<uint32_t>(x), old = atomicAdd(&s.hist.mass[0][bin], lo);
    const uint32_t hi = static_cast<uint32_t>(x >> 32) + (old + lo < old ? 1u : 0u);
    if (hi) atomicAdd(&s.hist.mass[1][bin], hi);
  };
  auto clear = [&](uint32_t* words, int n) {
    for (int i = tid; i < n; i += kThreads) words[i] = 0;
    __syncthreads();
  };
  // Values of a bin are ranked against one another; a bin with too many of them is cut finer first, by their keys.  `member(z)`: lies in the bin;
  // MASS: before and target are masses, else counts.
  auto rank_in_bin = [&](auto member, auto is_mass, u64 base, double target) {
    constexpr bool MASS = decltype(is_mass)::value;
    uint32_t lo = 0, hi = 0xffffffffu;
    for (;;) {
      if (tid == 0) { s.n = 0; s.lo = 0xffffffffu; s.hi = 0; }
      __syncthreads();
      uint32_t least = 0xffffffffu, most = 0;
      for_all([&](float z) {
        const uint32_t key = key_of(z);
        if (member(z) && key >= lo && key <= hi) {
          least = min(least, key);
          most = max(most, key);
          const uint32_t at = atomicAdd(&s.n, 1u);
          if (at < kCandidates) s.list[at] = key;
        }
      });
      least = __reduce_min_sync(0xffffffffu, least);
      most = __reduce_max_sync(0xffffffffu, most);
      if (lane == 0) { atomicMin(&s.lo, least); atomicMax(&s.hi, most); }
      __syncthreads();
      const u64(*got)[2] = exchange(s.n, static_cast<u64>(s.lo) << 32 | s.hi);
      uint32_t n = 0, mine_at = 0;
      lo = 0xffffffffu;
      hi = 0;
      for (int c = 0; c < C; ++c) {
        n += static_cast<uint32_t>(got[c][0]);
        lo = min(lo, static_cast<uint32_t>(got[c][1] >> 32));
        hi = max(hi, static_cast<uint32_t>(got[c][1]));
      }
      if (lo == hi) {                                     // they are all equal
        if (tid == 0) {
          u64 need = n;
          const u64 one = MASS ? w.whole(w.real(value_of_key(lo))) : 1;
          const double x = ceil((target - static_cast<double>(base)) / static_cast<double>(one));
          if (x < static_cast<double>(n)) need = x > 1.0 ? static_cast<u64>(x) : 1;
          s.cut_key = lo;
          s.cut_take = static_cast<uint32_t>(need);
          s.cut_base = base;
          s.cut_ties = n;
        }
        break;
      }
      if (n <= kCandidates) {
        for (int c = 0; c < C; ++c) {
          const int m = static_cast<int>(got[c][0]);
          if (tid < m) s.all[mine_at + tid] = cluster.map_shared_rank(s.list, c)[tid];
          mine_at += m;
        }
        __syncthreads();
        if constexpr (MASS) {
          if (tid < n) s.weight[tid] = w.whole(w.real(value_of_key(s.all[tid])));
          __syncthreads();
        }
        if (tid < n) {
          const uint32_t key = s.all[tid];
          u64 before = base, one = 1;
          uint32_t equal = 0;
          for (uint32_t j = 0; j < n; ++j) {
            const uint32_t other = s.all[j];
            if (other > key) before += MASS ? s.weight[j] : 1;
            equal += other == key;
          }
          if constexpr (MASS) one = s.weight[tid];
          if (static_cast<double>(before) < target && !(static_cast<double>(before + equal * one) < target)) {
            const double x = ceil((target - static_cast<double>(before)) / static_cast<double>(one));
            s.cut_key = key;                              // (threads with this key all write the same)
            s.cut_take = x < static_cast<double>(equal) ? (x > 1.0 ? static_cast<uint32_t>(x) : 1u) : equal;
            s.cut_ties = equal;
            s.cut_base = before;
          }
        }
        break;
      }
      // finer bins over [lo, hi], from the top
      const uint32_t top = hi, span = hi - lo;
      const int shift = max(0, 32 - __clz(span) - 10);    // span >> shift is below kMassBins
      clear(reinterpret_cast<uint32_t*>(&s.hist), sizeof(s.hist) / 4);
      for_all([&](float z) {
        const uint32_t key = key_of(z);
        if (member(z) && key >= lo && key <= hi) add_mass((top - key) >> shift, MASS ? w.whole(w.real(z)) : 1ull);
      });
      const u64 base_now = base;
      find_bin(std::true_type{}, [&](u64 before, u64 after) {
        return static_cast<double>(base_now + before) < target && !(static_cast<double>(base_now + after) < target);
      });
      base += s.base;
      hi = top - (s.bin << shift);
      lo = max(lo, hi - ((1u << shift) - 1u));
    }
    __syncthreads();
    cut = value_of_key(s.cut_key);
    take = s.cut_take;
    some = take < s.cut_ties;
    mass = s.cut_base + take * (MASS ? w.whole(w.real(cut)) : 1);
    // (the others have read the candidates before the next exchange, and those are written again only behind one)
  };

  const bool by_k = !nothing && !greedy && k > 1 && k < p.V;
  if (nothing) {
    cut = INFINITY;                                       // nothing stays
    take = 0;
  } else if (greedy || k == 1 || top_p <= 0.f) {
    cut = w.top;
    take = 1;
    some = known = true;
    mass = w.whole(1.0);
  }
  if (by_k && !some) {
    // Bins of 1/64 from the top down, the last for all below, by a rounding that never turns an order around (which is all that is asked of it):
    // 64 (top - z) is rounded to a whole number in the low bits of its sum with 2^23.  Positions outside of the row are counted as -infinity: they
    // stand behind every token, and have no mass.
    constexpr float kWhole = 8388608.f;
    const float shift = fminf(w.top * 64.f + kWhole, 3.0e38f);
    auto place_of = [&](float z) { return fmaf(z, -64.f, shift); };
    auto bin_of = [&](float z) { return static_cast<int>(__float_as_uint(fminf(fmaxf(place_of(z), kWhole), kWhole + (kCountBins - 1.f))) & 0x7fffffu); };
    clear(s.hist.count, kCountBins);
    for (int i = 0; i < tiles; ++i) {
      const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
      for (int e = 0; e < kVec; ++e) atomicAdd(&s.hist.count[bin_of(v.at(e))], 1u);
    }
    const u64 want = static_cast<u64>(k);
    find_bin(std::false_type{}, [&](u64 before, u64 after) { return before < want && after >= want; });
    const int bin = static_cast<int>(s.bin);
    const float last = bin == kCountBins - 1 ? INFINITY : kWhole + bin;
    make_list([&](float z) { return place_of(z) <= last; });
    rank_in_bin([&](float z) { return bin_of(z) == bin; }, std::false_type{}, s.base, static_cast<double>(k));
  }
  if (!nothing && top_p < 1.f && !(cut == w.top && take == 1)) {
    u64 sum = 0;
    const bool whole_row = cut == -INFINITY && take == 0xffffffffu;
    if (whole_row) {
#pragma unroll 2
      for (int i = 0; i < tiles; ++i) {
        const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum += w.whole(w.real(v.at(e)));
      }
    } else {
      for_few([&](float z) { return z > cut; }, [&](float z) { sum += w.whole(w.real(z)); });
    }
    const u64 above = cluster_sum(sum);
    const u64 one = whole_row ? 0 : w.whole(w.real(cut));
    const u64 all = whole_row ? above : above + take * one;
    const double target = static_cast<double>(top_p) * static_cast<double>(all);
    if (!whole_row && static_cast<double>(above) < target) {      // among the last ones that top-k left
      const double x = ceil((target - static_cast<double>(above)) / static_cast<double>(one));
      if (x < static_cast<double>(take)) {
        take = x > 1.0 ? static_cast<uint32_t>(x) : 1u;
        some = true;
      }
      mass = above + take * one;
      known = true;
    } else {
      const double n = by_k ? k : p.V;
      // see above; the sums are of rounded weights, which are up to half a unit larger, and below half a unit 0
      const double half_unit = 0.5 / w.unit;
      const double tail = fmax((1.0 - static_cast<double>(top_p)) * static_cast<double>(all) / w.unit / n - half_unit, half_unit);
      const float depth = static_cast<float>((fmax(-log2(tail), 0.0) + 1e-3) * 16.0 / w.rate);
      const float scale = (kMassBins - 1.f) / depth;
      const float floor = cut;                            // (values of -infinity have no mass: nothing is lost where it is that)
      auto bin_of = [&](float z) { return z == w.top ? 0.f : (w.top - z) * scale; };
      auto member = [&](float z) { return z > floor && bin_of(z) < kMassBins; };
      if (!listed) make_list(member);
      clear(reinterpret_cast<uint32_t*>(&s.hist), sizeof(s.hist) / 4);
      for_few(member, [&](float z) { add_mass(static_cast<int>(bin_of(z)), w.whole(w.real(z))); });
      find_bin(std::true_type{}, [&](u64 before, u64 after) {
        return static_cast<double>(before) < target && !(static_cast<double>(after) < target);
      });
      const float bin = static_cast<float>(s.bin);
      rank_in_bin([&](float z) {
        const float x = bin_of(z);
        return x >= bin && x < bin + 1.f && z > floor;
      }, std::true_type{}, s.base, target);
      known = true;
    }
  }

  // ---- where only the first of equal values stay: how many there are before each warp's part of each tile
  u64 ties_before = 0;
  if (some) {
    uint32_t mine = 0;
    for (int i = 0; i < tiles; ++i) {
      uint32_t n = 0;
      if (listed) {
        int to;
        for (int j = in_segment(i, &to) + lane; j < to; j += 32) n += few[j] == cut;
      } else {
        const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
        for (int e = 0; e < kVec; ++e) n += v.at(e) == cut;
      }
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) ties[i * kWarps + warp] = n;
      mine += n;
    }
    const u64 here = block_sum(lane == 0 ? mine : 0);
    const u64(*got)[2] = exchange(here, 0);
    for (int c = 0; c < rank; ++c) ties_before += got[c][0];
    if (warp == 0) {                                      // exclusive prefix sums in place
      u64 carry = ties_before;
      for (int at = 0; at < tiles * kWarps; at += 32) {
        const u64 n = at + lane < tiles * kWarps ? ties[at + lane] : 0;
        const u64 inc = warp_scan64(n, lane);
        if (at + lane < tiles * kWarps) ties[at + lane] = static_cast<uint32_t>(carry + inc - n);
        carry += __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    __syncthreads();
  }
  // Of this warp's part of a tile: what stays, picked (see above); min-p takes out more when the weights are known.
  auto pick_left = [&](const Vec<T>& v, int group, int* at) {
    uint32_t rank_of = 0;
    if (some) {
      uint32_t n = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) n += v.at(e) == cut;
      uint32_t inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
      }
      rank_of = ties[group] + inc - n;
    }
    return pick(v, 0, [&](float z) { return z > cut || (z == cut && (some ? rank_of++ < take : take > 0)); }, at);
  };
  auto left = [&](float z) {
    const double x = w.real(z);
    return x < least ? 0.0 : x;
  };

  // ---- the mass of what stays; where a token is drawn, of each warp's part of each tile as well
  u64 before = 0, all = mass;
  u64 here = 0;
  if (p.tokens || !known || least > 0.0) {
    all = 0;
    u64 sum = 0;
    for (int i = 0; i < tiles; ++i) {
      u64 t = 0;
      if (listed) {
        int to;
        uint32_t seen = some ? ties[i * kWarps + warp] : 0;
        for (int j = in_segment(i, &to); j < to; j += 32) {
          const float z = j + lane < to ? few[j + lane] : -INFINITY;
          bool stays = j + lane < to && z >= cut;
          if (some) {
            const unsigned equal = __ballot_sync(0xffffffffu, stays && z == cut);
            if (z == cut) stays = stays && seen + __popc(equal & ((1u << lane) - 1u)) < take;
            seen += __popc(equal);
          } else if (z == cut) {
            stays = stays && take > 0;
          }
          if (stays) t += w.whole(left(z));
        }
      } else {
        int at[kVec];
        const int n = pick_left(fetch((i * kThreads + tid) * kVec), i * kWarps + warp, at);
        for (int x = lane; x < n; x += 32) t += w.whole(left(few[x]));
        __syncwarp();
      }
      if (p.tokens) {
        t = warp_sum64(t);
        if (lane == 0) part[i * kWarps + warp] = t;
        t = lane == 0 ? t : 0;
      }
      sum += t;
    }
    here = block_sum(sum);
    const u64(*got)[2] = exchange(here, 0);
    for (int c = 0; c < C; ++c) {
      if (c < rank) before += got[c][0];
      all += got[c][0];
    }
  }

  __syncthreads();                                        // (the lists are not needed any more: what follows picks from tiles again)

  // ---- the draw: the CTA, the warp's part of a tile, the lane and the element in which the prefix passes u times the sum
  if (p.tokens && !nothing && warp == 0) {
    const double total = static_cast<double>(all);
    double t = static_cast<double>(p.uniforms[row]) * total;
    t = t < total ? fmax(t, 0.0) : total * 0.9999999999999999;      // (u outside of [0, 1))
    if (here > 0 && !(static_cast<double>(before) > t) && static_cast<double>(before + here) > t) {
      u64 carry = before;
      int group = -1;
      for (int at = 0; at < tiles * kWarps; at += 32) {
        const u64 n = at + lane < tiles * kWarps ? part[at + lane] : 0;
        const u64 inc = warp_scan64(n, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, static_cast<double>(carry + inc) > t);
        if (hit) {
          const int l = __ffs(hit) - 1;
          group = at + l;
          carry += __shfl_sync(0xffffffffu, inc - n, l);
          break;
        }
        carry += __shfl_sync(0xffffffffu, inc, 31);
      }
      // (group >= 0: the CTA's sum passes t)
      const int pos = ((group / kWarps) * kThreads + (group % kWarps) * 32 + lane) * kVec;
      const Vec<T> v = fetch(pos);
      int at[kVec];
      pick_left(v, group, at);
      u64 e[kVec], mine = 0;
#pragma unroll
      for (int x = 0; x < kVec; ++x) {
        e[x] = at[x] >= 0 ? w.whole(left(v.at(x))) : 0;
        mine += e[x];
      }
      const u64 inc = warp_scan64(mine, lane);
      const unsigned hit = __ballot_sync(0xffffffffu, static_cast<double>(carry + inc) > t);
      if (lane == __ffs(hit) - 1) {
        u64 run = carry + inc - mine;
        int found = kVec - 1;
#pragma unroll
        for (int x = kVec - 1; x >= 0; --x) {
          u64 upto = run;
#pragma unroll
          for (int y = 0; y <= x; ++y) upto += e[y];
          if (static_cast<double>(upto) > t) found = x;
        }
        p.tokens[row] = first + pos + found;
      }
    }
  }

  // ---- the distribution
  if (p.probs) {
    float* const dst = p.probs + row * p.V;
    const double inv = nothing ? 0.0 : w.unit / static_cast<double>(all);
    const bool wide = ((reinterpret_cast<uintptr_t>(dst) - 4 * static_cast<uintptr_t>(off)) & 15) == 0;
    for (int i = 0; i < tiles; ++i) {
      const int pos = (i * kThreads + tid) * kVec, id = first + pos;
      int at[kVec];
      const int n = pick_left(fetch(pos), i * kWarps + warp, at);
      for (int x = lane; x < n; x += 32) few[x] = static_cast<float>(left(few[x]) * inv);
      __syncwarp();
      float out[kVec];
#pragma unroll
      for (int x = 0; x < kVec; ++x) out[x] = at[x] >= 0 ? few[at[x]] : 0.f;
      __syncwarp();
      if (wide && id >= 0 && id + kVec <= p.V) {
#pragma unroll
        for (int x = 0; x < kVec; x += 4) *reinterpret_cast<float4*>(dst + id + x) = make_float4(out[x], out[x + 1], out[x + 2], out[x + 3]);
      } else {
#pragma unroll
        for (int x = 0; x < kVec; ++x)
          if (id + x >= 0 && id + x < p.V) dst[id + x] = out[x];
      }
    }
  }
  cluster.sync();                                         // nobody leaves while another may still read or write here
}

template <typename T>
cudaError_t launch(const SampleParams& p, int sm_count, cudaStream_t stream) {
  constexpr int kTile = kThreads * Vec<T>::kLen;
  const long long rows = static_cast<long long>(p.B) * p.R, positions = static_cast<long long>(p.V) + Vec<T>::kLen;
  // Enough CTAs to a row to hold it in the shared memory of CTAs that are two to an SM, and more while all of them find a place at once and each has
  // more than a tile of the vocabulary.
  int C = 1;
  auto slice_of = [&](int c) { return static_cast<int>(((positions + c - 1) / c + kTile - 1) / kTile * kTile); };
  while (C < kMaxCluster && (slice_of(C) * sizeof(T) > kPairBytes || (rows * C <= sm_count && slice_of(C) > kTile))) C *= 2;
  const int slice = slice_of(C);
  const bool resident = slice * sizeof(T) <= kSliceBytes;
  const size_t bytes = (resident ? slice * sizeof(T) : 0) + static_cast<size_t>(slice / kTile) * kWarps * 14;
  auto kernel = resident ? sample_kernel<T, true> : sample_kernel<T, false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSliceBytes + 16384));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t config = {};
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = C;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.gridDim = dim3(static_cast<unsigned>(rows * C));
  config.blockDim = dim3(kThreads);
  config.dynamicSmemBytes = bytes;
  config.stream = stream;
  config.attrs = &attr;
  config.numAttrs = 1;
  e = cudaLaunchKernelEx(&config, kernel, p, slice);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_sample(const SampleParams& p, int sm_count, cudaStream_t stream) {
  return p.bf16 ? launch<__nv_bfloat16>(p, sm_count, stream) : launch<float>(p, sm_count, stream);
}

}  // namespace eagle
