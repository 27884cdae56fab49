// Sampling with temperature, top-k, top-p and min-p: a token per row of logits, and / or the distribution that it is drawn from.
//
// With w(v) = exp((z(v) - max z) / temperature), what the filters leave is the first tokens of the order (z descending, id ascending): all
// with a greater z than some z*, and the first few of those that equal it.  So nothing is sorted: each filter looks for its cut (z*, how many
// of z*) by a histogram over z and a ranking of the few values in the bin that the cut falls into.
//   top-k   counts; top-p: masses, after the mass of all that top-k left; min-p: w >= min_p, a comparison
// A cluster of C CTAs takes a row, each a slice of the vocabulary, which stays in shared memory (in the logits' own type) for all passes
// over it; histograms are merged and candidates exchanged through distributed shared memory.
//
// A small top-k (k <= 256) takes another way: the k-th largest of the threads' own largest values bounds the k-th value from below, what is above it is
// a few more than k tokens, these go to every CTA with their ids, and each CTA decides by itself, by ranks and prefix sums in that order.
//
// Weights are fp64 (argument, reduction by a table of sixteenths, polynomial) and are summed as integers of 2^-q, q = 43 .. 46 (the largest with which V
// of them fit 63 bits): sums then depend neither on the order of atomics nor on C.  A sum over V tokens is off by V * 2^-(q+1) at the most (10^5 tokens:
// 7e-10) and by 1e-13 * sqrt(V) or so of the largest weight as a rule; fp32 sums (relative 1e-6) would decide visibly otherwise.
//
// What top-p may cut off is bounded before its histogram is taken: n tokens of weights below (1 - p) Z / n sum to less than (1 - p) Z, so
// the cut is not among them.  For Z a lower bound will do, which is what the threads' largest values weigh.  Of a vocabulary's long tail nothing reaches
// the atomics then.
//
// What bounds it: the latency of its five to eight phases, each a pass over shared memory and a cluster barrier of 1 to 2 us, not the bytes (without any exponential
// and histogram update the 656 rows below take 110 us).  From a graph, 64 rows of 129537 bf16 logits, k log-uniform up to 12000, top-p, min-p, tokens: 46 us
// (16.6 MB: 2.5 us), with k = 50: 15 us (by the way of a large k: 37 us), k = 256: 25 us (38); 656 rows of 32000 fp32 logits with top-p, distributions: 132 us (168 MB: 26 us).
// Measured on the way: a pass for Z before the one for the histogram, lists of what can stay, 160 us for the 656 rows; every bin read from every CTA, 5 us more per
// search; a CTA to a row that reads its logits again from L2 in each pass, 148 us; four CTAs to a row, 225 us; four CTAs of 256 threads per SM, 141 us;
// candidates ranked in loops over all, 24 us for k = 50.
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
constexpr int kCandidates = 512;             // a small top-k's, a thread each
constexpr int kRanked = 256;                 // values of a bin that are ranked against one another (more are cut finer first)
constexpr int kKept = 4096;                  // of a large top-k's values, those that a CTA lists
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
  u64 coarse[kMaxCluster][kCountBins / 32];      // each CTA's histogram, 32 bins together
  double roots[16];                  // (sixteen 8-byte words: no two share a bank)
  uint32_t list[kCandidates];        // this CTA's candidates
  int list_id[kCandidates];
  uint32_t all[kRanked];             // the cluster's
  u64 weight[kCandidates];
  float kept[kKept];
  uint32_t n, lo, hi;                // candidates found here, their range
  uint32_t n_kept;
  // a cut, found by one thread or by several with the same result
  uint32_t cut_key, cut_take, cut_ties;
  u64 cut_base;
  uint32_t bin;
  u64 base, total;
  float warp_low[kWarps];
};

static_assert(kCandidates <= kThreads && kRanked <= kThreads && 2 * kCandidates * sizeof(u64) <= sizeof(Shared::hist), "a thread each; two tables of them in the histogram's room");

// Order-preserving number of a float (no NaN, no negative zero), and back.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// 2^(j / 16)
__constant__ double kRoots[16] = {1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927, 1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543, 1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};
// exp((z - top) / temperature) in parts: x = 16 log2(e) (z - top) / temperature goes to the nearest whole number n by adding and subtracting 1.5 * 2^52, whose
// low four bits go through the table, the others to the exponent, and what is left, f in [-1/2, 1/2], through 1 + f times the polynomial
// that interpolates (2^(f / 16) - 1) / f at Chebyshev nodes (relative error 9e-15).
struct Weigher {
  float top;             // the row's largest value
  float floor;           // values below it weigh less than 2^-980, or are -infinity, or beside +infinity: 0
  double top_d, rate;    // 16 log2(e) / temperature
  int q;                 // whole weights count 2^-q
  const double* roots;
  __device__ __forceinline__ bool any(float z) const { return z >= floor; }
  // (any(z) holds, or the result is not used; infinities, which are at the top, count as the largest number)
  __device__ __forceinline__ void parts(float z, int more, double* near, double* root) const {
    constexpr double kBig = 6755399441055744.0;
    const double d = static_cast<double>(fminf(z, 3.4028234663852886e38f)) - top_d;
    const double big = fma(d, rate, kBig), f = fma(d, rate, -(big - kBig));
    const int n = __double2loint(big);
    double r = 1.2716049516906705e-09;
    r = fma(r, f, 1.4676387238435006e-07);
    r = fma(r, f, 1.3550807778387664e-05);
    r = fma(r, f, 0.0009383847926296646);
    r = fma(r, f, 0.04332169878499658);
    *near = fma(r, f, 1.0);
    const double t = roots[n & 15];
    *root = __hiloint2double(__double2hiint(t) + static_cast<int>(static_cast<uint32_t>((n >> 4) + more) << 20), __double2loint(t));
  }
  __device__ __forceinline__ double real(float z) const {
    double a, b;
    parts(z, 0, &a, &b);
    return any(z) ? a * b : 0.0;
  }
  // A weight of at most 1 as an integer: adding 2^52 leaves it in the low bits of the sum.
  __device__ __forceinline__ u64 whole_if_any(float z) const {
    double a, b;
    parts(z, q, &a, &b);
    return __double_as_longlong(fma(a, b, 4503599627370496.0)) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ u64 whole(float z) const {
    const u64 x = whole_if_any(z);
    return any(z) ? x : 0ull;
  }
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

template <typename T>
__device__ __forceinline__ float largest(const Vec<T>& v) {
  const uint32_t m = max_word<T>(max_word<T>(v.raw.x, v.raw.y), max_word<T>(v.raw.z, v.raw.w));
  if constexpr (sizeof(T) == 4) return __uint_as_float(m);
  else return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}

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
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(SampleParams p, int slice) {
  constexpr int kVec = Vec<T>::kLen, kTile = kThreads * kVec;
  extern __shared__ __align__(16) unsigned char dyn[];
  T* const held = reinterpret_cast<T*>(dyn);
  const int tiles = slice / kTile;
  u64* const part = reinterpret_cast<u64*>(dyn + (RESIDENT ? static_cast<size_t>(slice) * sizeof(T) : 0));      // [tiles][warps]
  uint32_t* const ties = reinterpret_cast<uint32_t*>(part + tiles * kWarps);                                      // [tiles][warps]
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
  const float temperature = p.temperature ? p.temperature[b] : 1.f, top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;
  const int k = p.top_k ? p.top_k[b] : 0;
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
  // `body(i, vector)` for each tile in which some lane's `may(its largest value)`: what looks for large values passes over most tiles at a vote each.
  auto for_tiles = [&](auto may, auto body) {
    for (int i = 0; i < tiles; ++i) {
      const Vec<T> v = fetch((i * kThreads + tid) * kVec);
      if (__any_sync(0xffffffffu, may(largest<T>(v)))) body(i, v);
    }
  };

  // `done(z, true)` for the elements of a vector in a mask, where it is expensive: one after the other of each lane where few are in it (`done(z, false)`: none).
  auto for_mask = [&](const Vec<T>& v, int i, unsigned mask, auto done) {
    const int steps = __reduce_max_sync(0xffffffffu, __popc(mask));
    if (2 * steps > kVec) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) done(v.at(e), (mask >> e & 1u) != 0);
    } else {
      const int pos = (i * kThreads + tid) * kVec;
      for (int j = 0; j < steps; ++j) {
        float z = 0.f;
        if (mask) {
          const int at = pos + __ffs(mask) - 1;
          if constexpr (RESIDENT) z = static_cast<float>(held[at]);
          else z = clean(static_cast<float>(src[first + at]));
        }
        done(z, mask != 0);
        mask &= mask - 1;
      }
    }
  };

  // ---- the largest value
  float most = -INFINITY;                                 // this thread's
#pragma unroll 8
  for (int i = 0; i < tiles; ++i) {
    const int pos = (i * kThreads + tid) * kVec;
    const Vec<T> v = load(pos);
    if constexpr (RESIDENT) *reinterpret_cast<uint4*>(held + pos) = v.raw;
    most = fmaxf(most, largest<T>(v));
  }
  // ... and a lower bound of the sum of the weights: what the threads' largest values weigh, in fp32 (each CTA's against its own largest value)
  const bool greedy = !(temperature > 0.f);
  const float rate32 = greedy ? 0.f : 1.4426950f / temperature;
  float at_least = 0.f;
  uint32_t top_key = __reduce_max_sync(0xffffffffu, key_of(most));
  if (lane == 0) s.warp_sum[warp] = top_key;
  __syncthreads();
  top_key = __reduce_max_sync(0xffffffffu, lane < kWarps ? static_cast<uint32_t>(s.warp_sum[lane]) : 0u);
  {
    float x = exp2f((most - value_of_key(top_key)) * rate32);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) s.warp_low[warp] = x;
  }
  __syncthreads();
  if (warp == 0) {
    at_least = lane < kWarps ? s.warp_low[lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) at_least += __shfl_xor_sync(0xffffffffu, at_least, o);
  }
  cluster.barrier_wait(std::move(started));
  {
    const u64(*got)[2] = exchange(top_key, __float_as_uint(at_least));
    for (int c = 0; c < C; ++c) top_key = max(top_key, static_cast<uint32_t>(got[c][0]));
    at_least = 0.f;
    for (int c = 0; c < C; ++c)
      at_least += __uint_as_float(static_cast<uint32_t>(got[c][1])) * exp2f((value_of_key(static_cast<uint32_t>(got[c][0])) - value_of_key(top_key)) * rate32);
    at_least = at_least * 0.999f > 1.f && at_least < INFINITY ? at_least * 0.999f : 1.f;      // (1: the largest value's; NaN beside infinities)
  }
  Weigher w;
  w.top = value_of_key(top_key);
  const bool nothing = w.top == -INFINITY;
  if (nothing && rank == 0 && tid == 0) {
    report_status(p.status, EAGLE_ERR_ROW);
    if (p.tokens) p.tokens[row] = -1;
  }
  const double least = static_cast<double>(fminf(fmaxf(min_p, 0.f), 1.f));      // (NaN: 0)
  w.rate = 16.0 * 1.4426950408889634 / (greedy ? 1.0 : static_cast<double>(temperature));
  w.top_d = fminf(w.top, 3.4028234663852886e38f);
  w.floor = w.top == INFINITY ? w.top : fmaxf(__double2float_ru(static_cast<double>(w.top) - 15680.0 / w.rate), -3.4028234663852886e38f);      // (2^-980)
  w.roots = s.roots;
  w.q = min(46, 63 - (32 - __clz(p.V - 1)));
  const double half_unit = __hiloint2double((1022 - w.q) << 20, 0);
  // min-p: only next to the border a weight is needed to tell
  float sure_in = -INFINITY, sure_out = -3.4028234663852886e38f;      // (-infinity has no weight)
  if (least > 0.0) {
    const double border = static_cast<double>(w.top) + log2(least) * 16.0 / w.rate, room = 1e-6 * (fabs(static_cast<double>(w.top)) + fabs(border));
    const bool known_border = room < 1e300;               // (no infinity, no NaN)
    sure_in = known_border ? static_cast<float>(border + room) : INFINITY;
    if (known_border) sure_out = fmaxf(sure_out, static_cast<float>(border - room));
  }
  auto left = [&](float z) { return least == 0.0 || z > sure_in || (z >= sure_out && !(w.real(z) < least)); };

  // ---- the cut: tokens with a greater value stay, and the first `take` of those that equal it (`some`: these are not all of them).  `mass`: of
  // all that stay, where a search for the cut has found it.
  float cut = -INFINITY;
  uint32_t take = 0xffffffffu;
  bool some = false, known = false;
  u64 mass = 0;

  // A vector of the row's probabilities.
  auto store = [&](float* dst, int pos, auto value) {
    const int id = first + pos;
    const bool wide = ((reinterpret_cast<uintptr_t>(dst) - 4 * static_cast<uintptr_t>(off)) & 15) == 0;
    if (wide && id >= 0 && id + kVec <= p.V) {
#pragma unroll
      for (int x = 0; x < kVec; x += 4) *reinterpret_cast<float4*>(dst + id + x) = make_float4(value(x), value(x + 1), value(x + 2), value(x + 3));
    } else {
#pragma unroll
      for (int x = 0; x < kVec; ++x)
        if (id + x >= 0 && id + x < p.V) dst[id + x] = value(x);
    }
  };
  // What a row's prefix has to pass.
  auto drawn = [&](long long of_row, u64 of_all) {
    const double total = static_cast<double>(of_all), t = static_cast<double>(p.uniforms[of_row]) * total;
    return t < total ? fmax(t, 0.0) : total * 0.9999999999999999;      // (u outside of [0, 1))
  };

  // Merged histogram -> the bin in which the prefix, on top of `base`, reaches the target (that of the histogram's total), with what lies
  // before it.  CTAs send one another the sums of 32 bins each; only the 32 bins that matter are then read from all of them (all bins, of four CTAs: 5 us).
  // Every CTA finds the same.  Returns the total.
  // (A histogram is cleared, and sums are sent again, only behind a further exchange, so that nobody reads them any more.)
  auto find_bin = [&](auto is_mass, u64 base, auto target_of) {
    constexpr bool MASS = decltype(is_mass)::value;
    constexpr int kSegments = (MASS ? kMassBins : kCountBins) / 32;
    auto bin_in = [&](const Shared& of, int bin) -> u64 {
      if constexpr (MASS) return of.hist.mass[0][bin] + (static_cast<u64>(of.hist.mass[1][bin]) << 32);
      else return of.hist.count[bin];
    };
    __syncthreads();                                      // this CTA's histogram is complete
#pragma unroll
    for (int i = 0; i < kSegments / kWarps; ++i) {
      const int segment = i * kWarps + warp;
      const u64 sum = warp_sum64(bin_in(s, segment * 32 + lane));
      if (lane < C) cluster.map_shared_rank(&s.coarse[rank][segment], lane)[0] = sum;
    }
    cluster.sync();
    if (warp == 0) {
      u64 v[kSegments / 32], sum = 0;
#pragma unroll
      for (int i = 0; i < kSegments / 32; ++i) {
        v[i] = 0;
        for (int c = 0; c < C; ++c) v[i] += s.coarse[c][lane * (kSegments / 32) + i];
        sum += v[i];
      }
      const u64 inc = warp_scan64(sum, lane), total = __shfl_sync(0xffffffffu, inc, 31);
      const double target = target_of(total);
      auto reached = [&](u64 before, u64 after) { return static_cast<double>(before) < target && !(static_cast<double>(after) < target); };
      u64 before = base + inc - sum, at = 0;
      int segment = -1;
#pragma unroll
      for (int i = 0; i < kSegments / 32; ++i) {
        if (reached(before, before + v[i])) {
          segment = lane * (kSegments / 32) + i;
          at = before;
        }
        before += v[i];
      }
      const unsigned hit = __ballot_sync(0xffffffffu, segment >= 0);
      if (hit) {
        const int bin = __shfl_sync(0xffffffffu, segment, __ffs(hit) - 1) * 32 + lane;
        at = __shfl_sync(0xffffffffu, at, __ffs(hit) - 1);
        u64 x = 0;
        for (int c = 0; c < C; ++c) x += bin_in(*cluster.map_shared_rank(&s, c), bin);
        const u64 upto = at + warp_scan64(x, lane);
        if (reached(upto - x, upto)) {
          s.bin = bin;
          s.base = upto - x;
        }
      }
      if (lane == 0) s.total = total;
    }
    __syncthreads();
    return s.total;
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
  // Values of a bin are ranked against one another; a bin with too many of them is cut finer first, by their keys.  `member(z)`: lies in the bin, which
  // lies within [low, high] (about: with room at both ends); MASS: base (what lies above the bin) and target are masses, else counts.
  // The one for top-k also lists what lies in its bin and above, for those that follow: they go over this list if there is room for it.
  int kept = -1;                                          // values listed here (-1: none)
  auto rank_in_bin = [&](float low, float high, auto member, auto is_mass, u64 base, double target) {
    constexpr bool MASS = decltype(is_mass)::value;
    bool keep = !MASS;
    uint32_t lo = 0, hi = 0xffffffffu;
    if (!(low <= high)) {                                 // (NaN)
      low = -INFINITY;
      high = INFINITY;
    }
    auto for_members = [&](auto done) {
      auto one = [&](float z) {
        if (z >= low && z <= high && member(z)) {
          const uint32_t key = key_of(z);
          if (key >= lo && key <= hi) done(z, key);
        }
      };
      if (MASS && kept >= 0) {
        for (int j = tid; j < kept; j += kThreads) one(s.kept[j]);
        return;
      }
      for_tiles([&](float z) { return z >= low; }, [&](int, const Vec<T>& v) {
        if (keep) {
          unsigned mask = 0;
#pragma unroll
          for (int e = 0; e < kVec; ++e) mask |= (v.at(e) >= low ? 1u : 0u) << e;
          const int n = __popc(mask);
          int upto = n;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
          }
          uint32_t at = 0;
          if (lane == 31) at = atomicAdd(&s.n_kept, static_cast<uint32_t>(upto));
          at = __shfl_sync(0xffffffffu, at, 31) + upto - n;
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (mask >> e & 1u) {
              if (at < kKept) s.kept[at] = v.at(e);
              ++at;
            }
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) one(v.at(e));
      });
      keep = false;
    };
    for (;;) {
      if (tid == 0) { s.n = 0; s.lo = 0xffffffffu; s.hi = 0; }
      __syncthreads();
      uint32_t least = 0xffffffffu, most = 0;
      for_members([&](float, uint32_t key) {
        least = min(least, key);
        most = max(most, key);
        const uint32_t at = atomicAdd(&s.n, 1u);
        if (at < kRanked) s.list[at] = key;
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
          const u64 one = MASS ? w.whole(value_of_key(lo)) : 1;
          const double x = ceil((target - static_cast<double>(base)) / static_cast<double>(one));
          if (x < static_cast<double>(n)) need = x > 1.0 ? static_cast<u64>(x) : 1;
          s.cut_key = lo;
          s.cut_take = static_cast<uint32_t>(need);
          s.cut_base = base;
          s.cut_ties = n;
        }
        break;
      }
      if (n <= kRanked) {
        for (int c = 0; c < C; ++c) {
          const int m = static_cast<int>(got[c][0]);
          if (tid < m) s.all[mine_at + tid] = cluster.map_shared_rank(s.list, c)[tid];
          mine_at += m;
        }
        __syncthreads();
        if constexpr (MASS) {
          if (tid < n) s.weight[tid] = w.whole(value_of_key(s.all[tid]));
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
      for_members([&](float z, uint32_t key) { add_mass((top - key) >> shift, MASS ? w.whole(z) : 1ull); });
      find_bin(std::true_type{}, base, [&](u64) { return target; });
      base = s.base;
      hi = top - (s.bin << shift);
      lo = max(lo, hi - ((1u << shift) - 1u));
    }
    __syncthreads();
    cut = value_of_key(s.cut_key);
    take = s.cut_take;
    some = take < s.cut_ties;
    mass = s.cut_base + take * (MASS ? w.whole(cut) : 1);
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
    mass = w.whole(w.top);
  }
  // Bins of 1/64 from the top down, the last for all below, by a rounding that never turns an order around (which is all that is asked of it):
  // 64 (top - z) is rounded to a whole number in the low bits of its sum with 2^23.
  constexpr float kWhole = 8388608.f;
  const float shift_k = fmaxf(fminf(w.top * 64.f + kWhole, 3.0e38f), -3.0e38f);
  auto place_of = [&](float z) { return fmaf(z, -64.f, shift_k); };
  auto bin_of_k = [&](float z) { return static_cast<int>(__float_as_uint(fminf(fmaxf(place_of(z), kWhole), kWhole + (kCountBins - 1.f))) & 0x7fffffu); };
  auto last_of = [&](int bin) { return bin == kCountBins - 1 ? INFINITY : kWhole + bin; };      // places up to it lie in the bin or above

  // ---- top-k with a small k: the k-th largest of the threads' largest values is no larger than the row's, so what is above it holds the first k
  // tokens, and (values being spread over the threads) few others.  These go to every CTA with their ids, which then decides by itself.
  bool decided = false;
  if (by_k && !some && k <= kCandidates / 2) {
    clear(s.hist.count, kCountBins);
    atomicAdd(&s.hist.count[bin_of_k(most)], 1u);
    if (tid == 0) s.n = 0;
    find_bin(std::false_type{}, 0, [&](u64) { return static_cast<double>(k); });
    const float last = last_of(static_cast<int>(s.bin));
    for_tiles([&](float z) { return place_of(z) <= last; }, [&](int i, const Vec<T>& v) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = v.at(e);
        if (place_of(z) <= last && z > -INFINITY) {
          const uint32_t at = atomicAdd(&s.n, 1u);
          if (at < kCandidates) {
            s.list[at] = key_of(z);
            s.list_id[at] = first + (i * kThreads + tid) * kVec + e;
          }
        }
      }
    });
    __syncthreads();
    const u64(*got)[2] = exchange(s.n, 0);
    int n = 0;
    for (int c = 0; c < C; ++c) n += static_cast<int>(got[c][0]);
    if (n <= kCandidates) {
      decided = true;
      // values with their ids in one number that descends as the order does; the histogram's room is free now
      u64* const order = reinterpret_cast<u64*>(&s.hist), *const by_place = order + kCandidates, *const by_id = s.weight;
      for (int c = 0, at = 0; c < C; ++c) {
        const int m = static_cast<int>(got[c][0]);
        if (tid < m) order[at + tid] = static_cast<u64>(cluster.map_shared_rank(s.list, c)[tid]) << 32 | ~static_cast<uint32_t>(cluster.map_shared_rank(s.list_id, c)[tid]);
        at += m;
      }
      __syncthreads();
      const u64 mine = tid < n ? order[tid] : 0;
      const float z = value_of_key(static_cast<uint32_t>(mine >> 32));
      const int id = static_cast<int>(~static_cast<uint32_t>(mine));
      int place = 0, place_by_id = 0;
      if (tid < n) {
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
          const u64 other = order[j];
          place += other > mine;
          place_by_id += static_cast<uint32_t>(other) > static_cast<uint32_t>(mine);
        }
      }
      // prefix sums (exclusive ones, in place) over the candidates; returns the total
      auto prefix = [&](u64* of) {
        __syncthreads();
        const u64 x = tid < n ? of[tid] : 0, inc = warp_scan64(x, lane);
        if (lane == 31) s.warp_sum[warp] = inc;
        __syncthreads();
        const u64 of_warp = lane < kWarps ? s.warp_sum[lane] : 0;
        const u64 before = inc - x + warp_sum64(lane < warp ? of_warp : 0);
        if (tid < n) of[tid] = before;
        __syncthreads();
        return warp_sum64(of_warp);
      };
      bool stays = tid < n && place < k;
      const u64 weight = stays ? w.whole(z) : 0;
      if (top_p < 1.f) {
        if (tid < n) by_place[place] = weight;
        const u64 sum = prefix(by_place);
        stays = stays && static_cast<double>(by_place[place]) < static_cast<double>(top_p) * static_cast<double>(sum);
      }
      stays = stays && left(z);
      if (tid < n) by_id[place_by_id] = stays ? weight : 0;
      const u64 all = prefix(by_id);
      if (stays && p.tokens && rank == 0) {
        const double t = drawn(row, all);
        const u64 before = by_id[place_by_id];
        if (!(static_cast<double>(before) > t) && static_cast<double>(before + weight) > t) p.tokens[row] = id;
      }
      if (p.probs) {
        float* const dst = p.probs + row * p.V;
        for (int i = 0; i < tiles; ++i) store(dst, (i * kThreads + tid) * kVec, [](int) { return 0.f; });
        __syncthreads();
        const int at = id - first;
        if (stays && at >= 0 && at < slice) dst[id] = static_cast<float>(w.real(z) * (1.0 / (static_cast<double>(all) * (2.0 * half_unit))));
      }
    }
  }
  if (by_k && !some && !decided) {
    // positions outside of the row are counted as -infinity: they stand behind every token, and have no mass
    __syncthreads();
    if (tid == 0) s.n_kept = 0;
    clear(s.hist.count, kCountBins);
    for (int i = 0; i < tiles; ++i) {
      const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
      for (int e = 0; e < kVec; ++e) atomicAdd(&s.hist.count[bin_of_k(v.at(e))], 1u);
    }
    find_bin(std::false_type{}, 0, [&](u64) { return static_cast<double>(k); });
    const int bin = static_cast<int>(s.bin);
    const float room = fabsf(w.top) < 1e30f ? fabsf(w.top) * 1e-6f + 0.03125f : INFINITY;      // (a bin is 1/64, while the shift is exact enough)
    rank_in_bin(bin == kCountBins - 1 ? -INFINITY : w.top - bin * 0.015625f - room, w.top - bin * 0.015625f + room, [&](float z) { return bin_of_k(z) == bin; },
                std::false_type{}, s.base, static_cast<double>(k));
    if (s.n_kept <= kKept) kept = static_cast<int>(s.n_kept);
  }
  if (!nothing && !decided && top_p < 1.f && !(cut == w.top && take == 1)) {
    // masses of what is above the cut: bins from the top down to where nothing can be the cut any more (see above; the sums are of rounded weights,
    // which are up to half a unit larger, and below half a unit 0).  What lies below counts with the last bin.
    const double n = by_k ? k : p.V;
    const double tail = fmax((1.0 - static_cast<double>(top_p)) * (by_k ? 1.0 : static_cast<double>(at_least)) / n - half_unit, half_unit);
    const float depth = static_cast<float>((1e-3 - log2(tail)) * 16.0 / w.rate);
    // (of temperatures below 1e-35 or so it would overflow in the end: the bins are wider there)
    const float scale = fminf((kMassBins - 1.f) / depth, 1e37f);
    const float floor = cut;
    const float half_top = 0.5f * static_cast<float>(w.top_d), twice = 2.f * scale;      // (differences of halves do not overflow)
    auto bin_of = [&](float z) { return fmaf(fminf(z, 3.4028234663852886e38f), -0.5f, half_top) * twice; };
    __syncthreads();
    clear(reinterpret_cast<uint32_t*>(&s.hist), sizeof(s.hist) / 4);
    u64 rest = 0;
    auto count = [&](float z, bool in) {
      const float x = bin_of(z);
      const u64 weight = w.whole_if_any(z);
      if (in && w.any(z)) {
        if (x < kMassBins) add_mass(static_cast<int>(x), weight);
        else rest += weight;
      }
    };
    if (floor == -INFINITY) {
      for (int i = 0; i < tiles; ++i) {
        const Vec<T> v = fetch((i * kThreads + tid) * kVec);
#pragma unroll
        for (int e = 0; e < kVec; ++e) count(v.at(e), true);
      }
    } else if (kept >= 0) {
      for (int j = tid; j < kept; j += kThreads) count(s.kept[j], s.kept[j] > floor);
    } else {
      for_tiles([&](float z) { return z > floor; }, [&](int i, const Vec<T>& v) {
        unsigned mask = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) mask |= (v.at(e) > floor ? 1u : 0u) << e;
        for_mask(v, i, mask, count);
      });
    }
    rest = warp_sum64(rest);
    if (lane == 0) add_mass(kMassBins - 1, rest);
    const u64 one = floor == -INFINITY ? 0 : w.whole(cut);
    auto target_of = [&](u64 above) { return static_cast<double>(top_p) * static_cast<double>(one == 0 ? above : above + take * one); };
    const u64 above = find_bin(std::true_type{}, 0, target_of);
    const double target = target_of(above);
    if (one > 0 && static_cast<double>(above) < target) {      // among the last ones that top-k left
      const double x = ceil((target - static_cast<double>(above)) / static_cast<double>(one));
      if (x < static_cast<double>(take)) {
        take = x > 1.0 ? static_cast<uint32_t>(x) : 1u;
        some = true;
      }
      mass = above + take * one;
    } else {
      const float bin = static_cast<float>(s.bin);
      const float room = fabsf(w.top) * 1e-6f + (1.f + 1e-3f * bin) / scale;
      const bool last = bin == kMassBins - 1.f;             // (all that lies below belongs to it, so that a bin with a mass has members)
      rank_in_bin(last ? -INFINITY : w.top - (bin + 1.f) / scale - room, w.top - bin / scale + room, [&](float z) {
        const float x = bin_of(z);
        return x >= bin && (last || x < bin + 1.f) && z > floor;
      }, std::true_type{}, s.base, target);
    }
    known = true;
  }

  // ---- the mass of what stays and, where only the first of equal values do, how many of these there are: in all, before this CTA, and (for the draw
  // and the ranks) in each warp's part of each tile.  In order of the ids, `take` of the equal ones stay.
  u64 before = 0, here = 0, all = mass;
  uint32_t ties_before = 0;
  const bool sums = p.tokens || !known || least > 0.0;
  const u64 one = some && left(cut) ? w.whole(cut) : 0;
  if (!decided && (sums || some)) {
    u64 sum = 0, equal = 0;
    if (lane == 0)
      for (int i = 0; i < tiles; ++i) part[i * kWarps + warp] = ties[i * kWarps + warp] = 0;
    __syncwarp();
    for_tiles([&](float z) { return z >= cut; }, [&](int i, const Vec<T>& v) {
      u64 t = 0;
      uint32_t n = 0;
      unsigned mask = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = v.at(e);
        n += some && z == cut;
        mask |= (sums && (some ? z > cut : z >= cut) && z >= sure_out ? 1u : 0u) << e;
      }
      for_mask(v, i, mask, [&](float z, bool in) {
        const u64 weight = w.whole(z);
        if (in && left(z)) t += weight;
      });
      n = __reduce_add_sync(0xffffffffu, n);
      if (p.tokens) {
        t = warp_sum64(t);
        if (lane == 0) part[i * kWarps + warp] = t;
        t = lane == 0 ? t : 0;
      }
      if (lane == 0) ties[i * kWarps + warp] = n;
      sum += t;
      equal += lane == 0 ? n : 0;
    });
    sum = block_sum(sum);
    equal = some ? block_sum(equal) : 0;
    const u64(*got)[2] = exchange(sum, equal);
    if (sums) all = 0;
    uint32_t seen = 0;
    for (int c = 0; c < C; ++c) {
      const uint32_t n = static_cast<uint32_t>(got[c][1]), in = seen < take ? min(n, take - seen) : 0u;
      const u64 m = got[c][0] + in * one;
      if (c == rank) {
        before = all;
        here = m;
        ties_before = seen;
      }
      if (sums) all += m;
      seen += n;
    }
  }
  auto leaving = cluster.barrier_arrive();                // (of what is in the other CTAs nothing is read or written from here on)
  // ---- the draw: the CTA, the warp's part of a tile, the lane and the element in which the prefix passes u times the sum
  double t = 0.0;
  bool draw = false;
  if (p.tokens && !nothing && !decided) {
    t = drawn(row, all);
    draw = here > 0 && !(static_cast<double>(before) > t) && static_cast<double>(before + here) > t;
  }
  if (some && (p.probs || draw)) {
    if (warp == 0) {                                      // exclusive prefix sums in place; parts with what stays of the equal ones
      uint32_t carry = ties_before;
      for (int at = lane; at - lane < tiles * kWarps; at += 32) {
        const uint32_t n = at < tiles * kWarps ? ties[at] : 0;
        uint32_t inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += x;
        }
        const uint32_t seen = carry + inc - n;
        if (at < tiles * kWarps) {
          ties[at] = seen;
          part[at] += (seen < take ? min(n, take - seen) : 0u) * one;
        }
        carry += __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    __syncthreads();
  }
  // Which elements of a vector of this warp's part of a tile stay (min-p aside).
  auto which = [&](const Vec<T>& v, int group) {
    unsigned stay = 0, equal = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      stay |= (v.at(e) > cut ? 1u : 0u) << e;
      equal |= (v.at(e) == cut ? 1u : 0u) << e;
    }
    if (!some) return take > 0 ? stay | equal : stay;
    if (!__any_sync(0xffffffffu, equal != 0)) return stay;
    uint32_t inc = __popc(equal);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    uint32_t seen = ties[group] + inc - __popc(equal);
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (equal >> e & 1u) stay |= (seen++ < take ? 1u : 0u) << e;
    return stay;
  };
  if (draw && warp == 0) {
    u64 carry = before;
    int group = 0;
    for (int at = 0; at < tiles * kWarps; at += 32) {
      const u64 n = at + lane < tiles * kWarps ? part[at + lane] : 0;
      const u64 inc = warp_scan64(n, lane);
      const unsigned hit = __ballot_sync(0xffffffffu, static_cast<double>(carry + inc) > t);
      if (hit) {                                          // (it comes: the CTA's sum passes t)
        const int l = __ffs(hit) - 1;
        group = at + l;
        carry += __shfl_sync(0xffffffffu, inc - n, l);
        break;
      }
      carry += __shfl_sync(0xffffffffu, inc, 31);
    }
    const int pos = ((group / kWarps) * kThreads + (group % kWarps) * 32 + lane) * kVec;
    const Vec<T> v = fetch(pos);
    const unsigned stay = which(v, group);
    u64 e[kVec], mine = 0;
#pragma unroll
    for (int x = 0; x < kVec; ++x) {
      e[x] = (stay >> x & 1u) && left(v.at(x)) ? w.whole(v.at(x)) : 0;
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

  // ---- the distribution
  if (p.probs && !decided) {
    float* const dst = p.probs + row * p.V;
    const double inv = nothing ? 0.0 : 1.0 / (static_cast<double>(all) * (2.0 * half_unit));
    for (int i = 0; i < tiles; ++i) {
      const int pos = (i * kThreads + tid) * kVec;
      const Vec<T> v = fetch(pos);
      float out[kVec];
#pragma unroll
      for (int x = 0; x < kVec; ++x) out[x] = 0.f;
      if (__any_sync(0xffffffffu, largest<T>(v) >= cut)) {
        const unsigned stay = which(v, i * kWarps + warp);
#pragma unroll
        for (int x = 0; x < kVec; ++x) {
          const double weight = w.real(v.at(x));
          out[x] = (stay >> x & 1u) && !(weight < least) ? static_cast<float>(weight * inv) : 0.f;
        }
      }
      store(dst, pos, [&](int x) { return out[x]; });
    }
  }
  cluster.barrier_wait(std::move(leaving));               // nobody leaves while another may still read or write here
}

template <typename T>
cudaError_t launch(const SampleParams& p, int sm_count, cudaStream_t stream) {
  constexpr int kTile = kThreads * Vec<T>::kLen;
  const long long rows = static_cast<long long>(p.B) * p.R, positions = static_cast<long long>(p.V) + Vec<T>::kLen;
  // Enough CTAs to a row to hold it in the shared memory of CTAs that are two to an SM (figures for fewer and more: at the top), and more while all of them
  // find a place at once and each has more than a tile of the vocabulary (top-p alone, a row of 129537 bf16 logits 30 us, else 43; eight of 32000 19 us, else 41).
  int C = 1;
  auto slice_of = [&](int c) { return static_cast<int>(((positions + c - 1) / c + kTile - 1) / kTile * kTile); };
  while (C < kMaxCluster && (slice_of(C) * sizeof(T) > kPairBytes || (rows * C <= sm_count && slice_of(C) > kTile))) C *= 2;
  const int slice = slice_of(C);
  const bool resident = slice * sizeof(T) <= kSliceBytes;
  const size_t bytes = (resident ? slice * sizeof(T) : 0) + static_cast<size_t>(slice / kTile) * kWarps * 12;
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
