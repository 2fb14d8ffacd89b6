// Sampling from logits with temperature, top-k, top-p and min-p from random numbers the caller gives (sdlm_sample).
// sdlm_lmhead_confidence decodes greedily; this is the decoding of a request that samples.  Its probability and entropy
// are the confidences that sdlm_accept_commit takes.
//
// For a row of logits l, in the order (l descending, index ascending):
//   z = (l - max l) / T,  w = e^z
//   top-k keeps the first k;  top-p of those the shortest prefix whose weight reaches p of theirs;  min-p of those the
//   tokens with w >= min_p (the largest w is 1);  W = sum of the kept w
//   token = the lowest index whose cumulative kept weight, taken by index, exceeds u W;  prob = w_token / W;
//   entropy = -sum (w/W) ln (w/W)
// Every filter keeps a prefix of the order, so the kept tokens are those above one key and the first few that equal
// it, and nothing has to be sorted.
//
// What bounds it is reading the logits once and, where many tokens are kept, forming their weights.  A cluster of up to
// eight thread blocks takes a row, a slice each, which stays in shared memory; the passes after the first run on chip
// and meet through the cluster's shared memory:
//   1. the slice is loaded, its maximum taken;
//   2. (top-k, top-p) tokens are counted by distance from the maximum in bins of T/102: top-k's threshold lies in one bin,
//      and since a bin's weights are known to 1 %, top-p's in a window of a few;
//   3. (top-p) one pass forms the weights and adds them up above, in and below that window;
//   4. thresholds are narrowed down to one value among the few tokens of the bin or window, which were listed on the way
//      (all tokens that a small top-k can keep are, and then only the list is looked at: top-k of 50 and top-p 88 -> 76 us);
//   5. without top-p one pass forms the kept weights; every thread block then knows the weight of all slices, and the one
//      that holds u W finds its token.
// Rows of 151936 bf16 logits, 1 / 128 / 256 of them, in a graph over three sets of them: greedy 9 / 36 / 60 us (128: 1.1 TB/s),
// all tokens kept 13 / 65 / 112, top-k of 50 17 / 69 / 118, that and top-p of 0.9 29 / 86 / 155, top-p alone, which keeps
// tens of thousands of tokens, 39 / 154 / 275; on one set, which stays in L2, 4 to 8 us less.  A pass over all weights (14
// 64-bit operations a token, 61 a clock and SM) is some 30 of those 65; top-p takes one to two of them, and the thread blocks
// of a row wait for each other five to eight times.
// -inf and NaN fail every comparison below, so they need no mask of their own.
//
// The answer is a comparison of sums of up to 2^18 weights with u W or p times their total, and a token changes when a
// border moves by a millionth, so weights are formed in 64 bits and summed as whole multiples of 2^-45 (W < 2^18 then
// stays below 2^63): such sums are exact, so the order of the additions, atomics among them, changes nothing.
#include "sdlm_internal.h"
#include "sdlm_ptx.cuh"

#include <math.h>

#include <type_traits>

namespace sdlm {

constexpr int kSampleThreads = 256;               // two thread blocks an SM at 128 registers; 512 threads have 64 and spill
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 2048;                 // of distance from the maximum: T/102 each, the last one open
constexpr int kSampleGroups = kSampleBins / 32;   // sums over 32 bins: what thread blocks tell each other first
constexpr int kSampleSub = 128;                   // parts a key range is cut into
// Tokens of a bin or window that a thread block lists.  Twice as many for bf16: top-p of 128 rows of 151936 goes from 192
// to 146 us, as windows need no second look; fp32 gains nothing there and loses an eighth of its greedy rate to the
// smaller L1 (87 -> 97 us for 256 rows).
template <bool F32>
constexpr int kSampleList = F32 ? 2048 : 4096;
constexpr int kSampleMaxVocab = 1 << 18;
constexpr uint32_t kSampleCluster = 8;            // thread blocks of a row, at most (the portable cluster size)

struct SampleParams {
  const void* logits;
  long long ld;
  const float* u;
  const float* temperature;  // each of the four or null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  float* prob;
  float* entropy;
  int32_t* kept;
  int V, per, vec;           // vocabulary, slice of a thread block, 16-byte loads
};

// Keys that order like the values, 32 or 16 bits wide as the logits are (0 and -0 have one).
template <bool F32>
__device__ __forceinline__ uint32_t sample_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  const uint32_t k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return F32 ? k : k >> 16;
}
template <bool F32>
__device__ __forceinline__ float sample_value(uint32_t key) {
  if (F32) return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
  return __uint_as_float((key & 0x8000u ? key ^ 0x8000u : ~key & 0xffffu) << 16);
}

// Weight of a value: t = z log2 e (0 at the maximum; -200 below v_floor, and 2^-200 adds nothing) and w45 = 2^t 2^45 with a
// relative error below 6e-12; `whole` is that as a whole number (64-bit integers add up beside the pipe of the doubles).
struct SampleWeight {
  double t, w45;
  uint64_t whole;
};
constexpr double kSampleWhole = 4503599627370496.0;  // 2^52: adding it leaves the nearest whole number in the mantissa
__device__ __forceinline__ uint64_t sample_whole(double x) {  // a number below 2^52, to the nearest whole one
  return (uint64_t)__double_as_longlong(x + kSampleWhole) & 0xfffffffffffffull;
}
__device__ __forceinline__ SampleWeight sample_weight(float v, float v_floor, double vmax, double scale) {
  SampleWeight r;
  r.t = v >= v_floor ? ((double)v - vmax) * scale : -200.0;  // (a NaN is not)
  const double m = r.t + 1.5 * kSampleWhole;       // round(t) in the low bits
  const double f = r.t - (m - 1.5 * kSampleWhole); // |f| <= 1/2
  // 2^f = sum (f ln 2)^i / i! up to i = 7; what the series leaves out is below (ln 2 / 2)^8 / 8! = 5.2e-12
  double q = 1.5252733804059840e-05;
  q = fma(q, f, 1.5403530393381609e-04);
  q = fma(q, f, 1.3333558146428443e-03);
  q = fma(q, f, 9.6181291076284772e-03);
  q = fma(q, f, 5.5504108664821580e-02);
  q = fma(q, f, 2.4022650695910071e-01);
  q = fma(q, f, 6.9314718055994531e-01);
  q = fma(q, f, 1.0);
  r.w45 = __hiloint2double(__double2hiint(q) + ((__double2loint(m) + 45) << 20), __double2loint(q));  // at most 2^45
  r.whole = sample_whole(r.w45);
  return r;
}
// -w t as a multiple of 2^-43 (w |t| <= 0.54), for sums whose order is not fixed.
__device__ __forceinline__ uint64_t sample_entropy(const SampleWeight& w) { return sample_whole(w.w45 * w.t * -0.25); }

// Tokens above `value` are kept, and the first `take` by index of those that equal it.
struct SampleCut {
  float value;
  uint32_t take;
};

// Sums over kept tokens.
struct SampleSums {
  uint64_t mass;
  double ent;  // sum of -w t, multiples of 2^-45
  uint32_t count, ties;
};

struct alignas(16) SampleShared {  // the values behind it are read and written 16 bytes at a time
  uint32_t count[kSampleBins + 4];                // the last for tokens that cannot be taken
  uint32_t group_n[kSampleGroups];                // tokens of 32 bins, and bounds of their weight
  uint64_t group_lo[kSampleGroups], group_hi[kSampleGroups];
  uint32_t lo[2][kSampleSub], hi[2][kSampleSub];  // by parity of the level: one barrier per level then suffices
  SampleSums mine, extra[2];                      // what a thread block tells the others of its cluster
  uint64_t window[2], looked[2];
  SampleSums warp[kSampleWarps];
  uint64_t scan[kSampleWarps], scan2[kSampleWarps];
  uint32_t scan32[kSampleWarps];
  uint64_t found_before;
  uint32_t max_bits;
  int found, n_list;
  // what the first warp finds in the counts
  int b_k, b0, b1;
  uint64_t before_k;
  uint32_t sum_n[kSampleGroups], fine_k[32], n_window;  // the cluster's counts by group, of the bins of b_k's group what top-k keeps
  uint64_t sum_lo[kSampleGroups], sum_hi[kSampleGroups];
};
static_assert(sizeof(SampleShared) % 16 == 0, "the values start on a 16-byte boundary");

// Exclusive prefix of v over the thread block in thread order, and the total; all threads call it.
__device__ __forceinline__ uint64_t sample_scan(uint64_t v, uint64_t* warp_sums, uint64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kSampleWarps; ++i) {
    if (i < warp) before += warp_sums[i];
    total += warp_sums[i];
  }
  __syncthreads();  // warp_sums may be written again
  return before + incl - v;
}
template <typename N>
__device__ __forceinline__ N sample_warp_sum(N v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What the C thread blocks of a cluster have at the same place, loads in flight together (a loop over C waits for each).
template <typename N>
__device__ __forceinline__ void sample_gather(const N* at, uint32_t C, N (&v)[kSampleCluster]) {
  static_assert(sizeof(N) == 4 || sizeof(N) == 8, "");
  const uint32_t a = ptx::smem_u32(at);
#pragma unroll
  for (uint32_t r = 0; r < kSampleCluster; ++r) {
    v[r] = 0;
    if (r < C) {
      if constexpr (sizeof(N) == 4) v[r] = (N)ptx::ld_cluster_u32(ptx::mapa_u32(a, r));
      else if constexpr (std::is_same<N, double>::value) v[r] = __longlong_as_double((long long)ptx::ld_cluster_u64(ptx::mapa_u32(a, r)));
      else v[r] = (N)ptx::ld_cluster_u64(ptx::mapa_u32(a, r));
    }
  }
}
template <typename N>
__device__ __forceinline__ N sample_cluster_sum(const N* at, uint32_t C) {
  N v[kSampleCluster];
  sample_gather(at, C, v);
#pragma unroll
  for (uint32_t r = 1; r < kSampleCluster; ++r) v[0] += v[r];
  return v[0];
}

template <bool F32>
struct SampleRow {
  static constexpr int kVec = F32 ? 4 : 8;  // values in 16 bytes
  const uint4* vals;                         // the slice, -inf behind its end; n_vec is a multiple of 32, so that a warp's lanes stay together
  SampleShared* sh;
  uint32_t* list;                            // values (bits) of the tokens in question
  int n_vec, C, rank;
  double scale;                              // log2 e / T
  float vmax, v_floor, bin_scale;
  int level;                                 // key levels so far (buffer parity)

  static __device__ __forceinline__ void unpack(const uint4& q, float (&v)[kVec]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (F32) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  // Bin b holds the values about (b - 1/2 .. b + 1/2) / bin_scale below the maximum: the distance, rounded by adding 2^23.
  __device__ __forceinline__ int bin_of(float v) const {
    return __float_as_int(fminf((vmax - v) * bin_scale, (float)(kSampleBins - 1)) + 8388608.0f) - 0x4b000000;
  }
  __device__ __forceinline__ SampleWeight weight(float v) const { return sample_weight(v, v_floor, (double)vmax, scale); }

  // Bounds of the weight of n tokens of bin b, as multiples of 2^-40 rounded outwards.  The factors 1 -+ 2e-5 cover four
  // roundings: of the distance (two of 2^-24 of at most 2047 bins, a bin being 0.0098: 2.4e-6), of the exponent here (2^-24
  // of at most 28.9: 1.2e-6), of exp2f and the product (3e-7), and of each weight to 2^-45 (half of it against e^-20: 6.9e-6).
  __device__ __forceinline__ void bounds(int b, uint32_t n, uint64_t& lo, uint64_t& hi) const {
    const double kappa = scale / (double)bin_scale;  // log2 units a bin
    const float near = b == 0 ? 1.0f : exp2f((float)(-((double)b - 0.5) * kappa)) * 1.00002f;
    const float far = b == kSampleBins - 1 ? 0.0f : exp2f((float)(-((double)b + 0.5) * kappa)) * 0.99998f;
    lo = (uint64_t)((double)n * (double)far * 1099511627776.0);
    hi = n ? (uint64_t)((double)n * (double)near * 1099511627776.0) + 1u : 0u;
  }
  // Tokens of bin 32 g + lane in the whole cluster; whole warps.
  __device__ __forceinline__ uint32_t cluster_bin(int g) const {
    return sample_cluster_sum(&sh->count[32 * g + (threadIdx.x & 31)], C);
  }
  template <typename N>
  static __device__ __forceinline__ N warp_prefix(N v) {  // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const N w = __shfl_up_sync(0xffffffffu, v, o);
      if ((threadIdx.x & 31) >= o) v += w;
    }
    return v;
  }
  // Counts the tokens by bin, and finds top-k's bin (b_k, with before_k tokens before it).  The histograms stay where they
  // are: the thread blocks exchange sums over 32 bins and then only the bins in question (all of them from all of the others
  // cost more than everything else together).
  __device__ __forceinline__ void find_bins(bool by_k, int k, bool by_p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kSampleBins / 4; i += kSampleThreads) reinterpret_cast<uint4*>(sh->count)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int i = threadIdx.x; i < n_vec; i += kSampleThreads) {
      float v[kVec];
      unpack(vals[i], v);
#pragma unroll
      for (int e = 0; e < kVec; ++e) atomicAdd(&sh->count[v[e] > -INFINITY ? bin_of(v[e]) : kSampleBins], 1u);
    }
    __syncthreads();
    for (int g = warp; g < kSampleGroups; g += kSampleWarps) {
      const uint32_t n = sh->count[32 * g + lane], all = __reduce_add_sync(0xffffffffu, n);
      uint64_t lo = 0, hi = 0;
      if (by_p && all) {
        bounds(32 * g + lane, n, lo, hi);
        lo = sample_warp_sum(lo);
        hi = sample_warp_sum(hi);
      }
      if (lane == 0) {
        sh->group_n[g] = all;
        sh->group_lo[g] = lo;
        sh->group_hi[g] = hi;
      }
    }
    ptx::cluster_sync_all();
    if (warp == 0) {
      static_assert(kSampleGroups == 64, "two groups a lane");
      uint32_t n[2] = {0, 0};
      uint64_t lo[2] = {0, 0}, hi[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        n[i] = sample_cluster_sum(&sh->group_n[2 * lane + i], C);
        if (by_p) {
          lo[i] = sample_cluster_sum(&sh->group_lo[2 * lane + i], C);
          hi[i] = sample_cluster_sum(&sh->group_hi[2 * lane + i], C);
        }
      }
      int b_k = kSampleBins;
      const uint32_t incl = warp_prefix(n[0] + n[1]), tokens = __shfl_sync(0xffffffffu, incl, 31);
      if (by_k && (uint32_t)k < tokens) {
        const int src = __ffs(__ballot_sync(0xffffffffu, incl >= (uint32_t)k)) - 1;
        const uint32_t before = __shfl_sync(0xffffffffu, incl - n[0] - n[1], src), n_0 = __shfl_sync(0xffffffffu, n[0], src);
        const int g = 2 * src + (before + n_0 >= (uint32_t)k ? 0 : 1);
        uint32_t fine = cluster_bin(g);
        const uint32_t f_incl = before + (g & 1 ? n_0 : 0u) + warp_prefix(fine);
        const int at = __ffs(__ballot_sync(0xffffffffu, f_incl >= (uint32_t)k)) - 1;
        const uint32_t before_k = __shfl_sync(0xffffffffu, f_incl - fine, at);
        b_k = 32 * g + at;
        fine = lane < at ? fine : lane == at ? (uint32_t)k - before_k : 0u;
        sh->fine_k[lane] = fine;
        if (lane == 0) sh->before_k = before_k;
        // what top-k leaves of the groups
        uint64_t l, h;
        bounds(32 * g + lane, fine, l, h);
        l = sample_warp_sum(l);
        h = sample_warp_sum(h);
        const uint32_t m = __reduce_add_sync(0xffffffffu, fine);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (2 * lane + i > g) { n[i] = 0; lo[i] = hi[i] = 0; }
          if (2 * lane + i == g) { n[i] = m; lo[i] = l; hi[i] = h; }
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sh->sum_n[2 * lane + i] = n[i];
        sh->sum_lo[2 * lane + i] = lo[i];
        sh->sum_hi[2 * lane + i] = hi[i];
      }
      if (lane == 0) sh->b_k = b_k;
    }
    __syncthreads();
  }

  // The window [b0, b1] of bins that can hold top-p's threshold: the first bin whose weight from above, with all before, can
  // reach the goal, to the first whose weight from below must.  At first the goal is p of a total that is known between
  // bounds as well; once the weight before group g0 and of groups [g0, g1] is known (`before`, `mass`, multiples of 2^-45),
  // it is `want`, and the bounds hold from both ends.  For the first warp; n_window: the tokens of the window.
  __device__ __forceinline__ void find_window(bool known, int g0, int g1, double before, double mass, double want, double p64) {
    const int lane = threadIdx.x & 31, g_k = sh->b_k >> 5;
    uint64_t lo[2], hi[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool in = 2 * lane + i >= g0 && 2 * lane + i <= g1;
      lo[i] = in ? sh->sum_lo[2 * lane + i] : 0;
      hi[i] = in ? sh->sum_hi[2 * lane + i] : 0;
    }
    const uint64_t l_incl = warp_prefix(lo[0] + lo[1]), h_incl = warp_prefix(hi[0] + hi[1]);
    const double l_all = (double)__shfl_sync(0xffffffffu, l_incl, 31), h_all = (double)__shfl_sync(0xffffffffu, h_incl, 31);
    const double unit = 1.0 / 32.0, base = known ? before * unit : 0.0, end = base + mass * unit;  // in multiples of 2^-40
    // weight up to a place with bounds l, h of what lies between the first group and it, from above and from below
    auto at_most = [&](double l, double h) { return (known ? fmin(base + h, end - (l_all - l)) : h) * (1.0 + 1e-13) + 1.0; };
    auto at_least = [&](double l, double h) { return (known ? fmax(base + l, end - (h_all - h)) : l) * (1.0 - 1e-13) - 1.0; };
    auto locate = [&](bool upper) {
      const double goal = known ? want * unit : upper ? p64 * l_all * (1.0 - 1e-13) : p64 * h_all * (1.0 + 1e-13);
      const double l1 = (double)l_incl, h1 = (double)h_incl, l0 = (double)(l_incl - lo[1]), h0 = (double)(h_incl - hi[1]);
      const bool ok0 = (upper ? at_most(l0, h0) : at_least(l0, h0)) >= goal && 2 * lane >= g0;
      const bool ok1 = (upper ? at_most(l1, h1) : at_least(l1, h1)) >= goal && 2 * lane + 1 >= g0;
      const uint32_t m0 = __ballot_sync(0xffffffffu, ok0), m1 = __ballot_sync(0xffffffffu, ok1);
      const int a = m0 ? 2 * (__ffs(m0) - 1) : kSampleGroups, b = m1 ? 2 * (__ffs(m1) - 1) + 1 : kSampleGroups;
      const int g = min(min(a, b), g1);
      const uint64_t l_b = __shfl_sync(0xffffffffu, g & 1 ? l_incl - lo[1] : l_incl - lo[0] - lo[1], g >> 1);
      const uint64_t h_b = __shfl_sync(0xffffffffu, g & 1 ? h_incl - hi[1] : h_incl - hi[0] - hi[1], g >> 1);
      uint64_t l, h;
      bounds(32 * g + lane, g == g_k ? sh->fine_k[lane] : cluster_bin(g), l, h);
      const double lx = (double)(l_b + warp_prefix(l)), hx = (double)(h_b + warp_prefix(h));
      const uint32_t at = __ballot_sync(0xffffffffu, (upper ? at_most(lx, hx) : at_least(lx, hx)) >= goal);
      return 32 * g + (at ? __ffs(at) - 1 : 31);
    };
    const int b0 = locate(true), b1 = min(max(b0, locate(false)), sh->b_k);
    // tokens of the window's groups (an upper bound that is near enough)
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) n += 2 * lane + i >= b0 >> 5 && 2 * lane + i <= b1 >> 5 ? sh->sum_n[2 * lane + i] : 0u;
    if (b0 >> 5 == b1 >> 5 || (b0 >> 5) + 1 == b1 >> 5) {  // few groups: count the bins
      const int ga = b0 >> 5, gb = b1 >> 5;
      const uint32_t x = ga == g_k ? sh->fine_k[lane] : cluster_bin(ga), y = gb == ga ? 0u : gb == g_k ? sh->fine_k[lane] : cluster_bin(gb);
      n = (32 * ga + lane >= b0 && 32 * ga + lane <= b1 ? x : 0u) + (32 * gb + lane <= b1 ? y : 0u);
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      sh->b0 = b0;
      sh->b1 = b1;
      sh->n_window = n;
    }
  }

  // Lists the tokens of bins [b0, b1] that `floor` keeps whole; n_list is beyond the list's length when they do not fit.
  // For whole warps: the lane's values i * kVec + e, e in the bits of `which`.  (A lane that went on by itself would take
  // the weights of its next values alone.)
  __device__ __forceinline__ void put_on_list(uint32_t which, int i) {
    if (!__any_sync(0xffffffffu, which)) return;
    const int mine = __popc(which), incl = warp_prefix(mine), lane = threadIdx.x & 31;
    int to = 0;
    if (lane == 31) to = atomicAdd(&sh->n_list, incl);
    to = __shfl_sync(0xffffffffu, to, 31) + incl - mine;
    for (; which; which &= which - 1, ++to)
      if (to < kSampleList<F32>) list[to] = __float_as_uint(at(i * kVec + __ffs(which) - 1));
    __syncwarp();
  }
  __device__ __forceinline__ void list_bins(int b0, int b1, const SampleCut& floor) {
    if (threadIdx.x == 0) sh->n_list = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n_vec; i += kSampleThreads) {
      float v[kVec];
      unpack(vals[i], v);
      uint32_t in = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const int b = bin_of(v[e]);
        in |= v[e] > floor.value && b >= b0 && b <= b1 ? 1u << e : 0u;
      }
      put_on_list(in, i);
    }
    __syncthreads();
  }
  // The slice's value at a place known only at run time (indexing the registers it was unpacked to would put them in memory).
  __device__ __forceinline__ float at(int i) const {
    if (F32) return reinterpret_cast<const float*>(vals)[i];
    return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(vals)[i] << 16);
  }
  // f(value) for the tokens listed (of bins [b0, b1] above the floor), from the slice when the list was too short.
  template <typename F>
  __device__ __forceinline__ void each_listed(int b0, int b1, const SampleCut& floor, F f) {
    if (sh->n_list <= kSampleList<F32>) {
      for (int i = threadIdx.x; i < sh->n_list; i += kSampleThreads) {
        const float v = __uint_as_float(list[i]);
        const int b = bin_of(v);
        if (v > floor.value && b >= b0 && b <= b1) f(v);
      }
    } else {
      for (int i = threadIdx.x; i < n_vec; i += kSampleThreads) {
        float v[kVec];
        unpack(vals[i], v);
        uint32_t in = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const int b = bin_of(v[e]);
          in |= v[e] > floor.value && b >= b0 && b <= b1 ? 1u << e : 0u;
        }
        for (; in; in &= in - 1) f(at(i * kVec + __ffs(in) - 1));
        __syncwarp();
      }
    }
  }
  // A key no smaller (up) or no larger than that of any value on the inner side of v.
  __device__ __forceinline__ uint32_t key_near(float v, bool up) const {
    if (isinf(v)) return sample_key<F32>(up ? vmax : F32 ? -3.402823466e38f : -3.3895314e38f);
    const uint32_t k = sample_key<true>(v);
    return F32 ? k : up ? (k >> 16) + 1u : k >> 16;
  }

  // The value at which the tokens listed, taken from the largest down behind `before`, reach `want` (tokens, or weight when
  // MASS), and how many of the tokens that equal it are needed.  The first floor.take tokens that equal floor.value belong
  // to the list when with_floor.
  template <bool MASS>
  __device__ SampleCut narrow(int b0, int b1, const SampleCut floor, bool with_floor, uint64_t before, uint64_t want) {
    const float near = ((float)b0 - 0.5f) / bin_scale, far = ((float)b1 + 0.5f) / bin_scale;
    const float slack = 1e-6f * (fabsf(vmax) + far) + 1e-37f;  // what rounding may have moved over a bin's border
    const uint32_t k_max = sample_key<F32>(vmax);
    uint32_t r_hi = b0 > 0 ? min(k_max, key_near(vmax - near + slack, true)) : k_max;
    uint32_t r_lo = b1 < kSampleBins - 1 ? max(1u, key_near(vmax - far - slack, false)) : 1u;
    for (int lev = 0; lev < 8; ++lev) {  // a level leaves a 128th of at most 2^32 keys: five are enough
      const int buf = level++ & 1;
      uint32_t* lo = sh->lo[buf];
      uint32_t* hi = sh->hi[buf];
      if (threadIdx.x < kSampleSub) lo[threadIdx.x] = hi[threadIdx.x] = 0;
      int part = 0;
      while (((r_hi - r_lo) >> part) >= (uint32_t)kSampleSub) ++part;
      if (threadIdx.x == 0) sh->found = 0;
      __syncthreads();
      auto add = [&](float v, uint32_t n) {
        const uint32_t key = sample_key<F32>(v);
        if (key < r_lo || key > r_hi) return;
        const uint32_t i = (r_hi - key) >> part;
        if (MASS) {
          const uint64_t w = weight(v).whole * n;
          // 64 bits in two halves; the carry goes with whoever brought the lower half over
          const uint32_t w_lo = (uint32_t)w, old = atomicAdd(&lo[i], w_lo);
          const uint32_t up = (uint32_t)(w >> 32) + (old + w_lo < old ? 1u : 0u);
          if (up) atomicAdd(&hi[i], up);
        } else {
          atomicAdd(&lo[i], n);
        }
      };
      each_listed(b0, b1, floor, [&](float v) { add(v, 1); });
      if (with_floor && rank == 0 && threadIdx.x == 0) add(floor.value, floor.take);
      ptx::cluster_sync_all();
      uint64_t v = 0;
      if (threadIdx.x < kSampleSub) {
        uint32_t a[kSampleCluster], b[kSampleCluster] = {};
        sample_gather(&lo[threadIdx.x], C, a);
        if (MASS) sample_gather(&hi[threadIdx.x], C, b);
#pragma unroll
        for (uint32_t r = 0; r < kSampleCluster; ++r) v += (uint64_t)a[r] + ((uint64_t)b[r] << 32);
      }
      uint64_t total;
      const uint64_t e = before + sample_scan(v, sh->scan, total);
      if (e < want && want <= e + v) {
        sh->found = threadIdx.x;
        sh->found_before = e;
      }
      __syncthreads();
      r_hi -= (uint32_t)sh->found << part;
      before = sh->found_before;
      const uint32_t w = (1u << part) - 1u;
      r_lo = r_hi - r_lo > w ? r_hi - w : r_lo;
      __syncthreads();  // found may be written again
      if (r_hi == r_lo) break;
    }
    const float value = sample_value<F32>(r_hi);
    const uint64_t each = MASS ? max((uint64_t)1, weight(value).whole) : 1;
    return SampleCut{value, (uint32_t)((want - before + each - 1) / each)};
  }

  // Sums over the slice's tokens above the cut (with t >= min_t), by warp: warp w has a contiguous part of the slice.
  __device__ __forceinline__ int warp_vecs() const { return (n_vec / 32 + kSampleWarps - 1) / kSampleWarps * 32; }
  __device__ void kept_sums(const SampleCut& cut, double min_t, float reject) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = warp * warp_vecs(), last = min(n_vec, first + warp_vecs());
    SampleSums s{0, 0.0, 0, 0};
    for (int i = first + lane; i < last; i += 32) {
      float v[kVec];
      unpack(vals[i], v);
      float mx = v[0];
#pragma unroll
      for (int e = 1; e < kVec; ++e) mx = fmaxf(mx, v[e]);
      if (!__any_sync(0xffffffffu, mx >= reject)) continue;
      // (no branch on a single token: eight chains of 64-bit operations at a time keep their pipe fed, one does not)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const SampleWeight w = weight(v[e]);
        const bool in = v[e] > cut.value && v[e] >= reject && w.t >= min_t;
        s.mass += in ? w.whole : 0;
        s.ent = fma(in ? w.w45 : 0.0, -w.t, s.ent);
        s.count += in ? 1u : 0u;
        s.ties += v[e] == cut.value && v[e] > -INFINITY ? 1u : 0u;
      }
    }
    s.mass = sample_warp_sum(s.mass);
    s.ent = sample_warp_sum(s.ent);
    s.count = __reduce_add_sync(0xffffffffu, s.count);
    s.ties = __reduce_add_sync(0xffffffffu, s.ties);
    __syncthreads();  // the sums that were there have been read
    if (lane == 0) sh->warp[warp] = s;
    __syncthreads();
  }
  // The same over the tokens listed (of bins [b0, b1] above the floor); returns the thread block's.  In whole numbers, as the
  // list has no fixed order.
  __device__ SampleSums listed_sums(int b0, int b1, const SampleCut& floor, const SampleCut& cut, double min_t, float reject) {
    uint64_t mass = 0, ent = 0;
    uint32_t count = 0, ties = 0;
    each_listed(b0, b1, floor, [&](float v) {
      const SampleWeight w = weight(v);
      if (v > cut.value && v >= reject && w.t >= min_t) {
        mass += w.whole;
        ent += sample_entropy(w);
        ++count;
      } else if (v == cut.value) {
        ++ties;
      }
    });
    mass = sample_warp_sum(mass);
    ent = sample_warp_sum(ent);
    count = __reduce_add_sync(0xffffffffu, count);
    ties = __reduce_add_sync(0xffffffffu, ties);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh->warp[threadIdx.x >> 5] = SampleSums{mass, 4.0 * (double)ent, count, ties};
    __syncthreads();
    SampleSums all{0, 0.0, 0, 0};
#pragma unroll 1
    for (int i = 0; i < kSampleWarps; ++i) {
      all.mass += sh->warp[i].mass;
      all.ent += sh->warp[i].ent;
      all.count += sh->warp[i].count;
      all.ties += sh->warp[i].ties;
    }
    return all;
  }
};

template <bool F32>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(const SampleParams p) {
  using Row = SampleRow<F32>;
  constexpr int kVec = Row::kVec;
  extern __shared__ __align__(16) uint8_t sample_smem[];
  SampleShared* sh = reinterpret_cast<SampleShared*>(sample_smem);
  uint32_t* list = reinterpret_cast<uint32_t*>(sample_smem + sizeof(SampleShared));
  uint4* vals = reinterpret_cast<uint4*>(list + kSampleList<F32>);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t C;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
  const uint32_t rank = ptx::cluster_ctarank();
  const int row = blockIdx.x / C;
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  // the row's parameters, asked for before anything else
  const float T = p.temperature ? p.temperature[row] : 1.0f;
  const int k = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.0f;
  const float mp = p.min_p ? p.min_p[row] : 0.0f;
  const float u = p.u[row];

  // ---- the slice into shared memory, its largest value
  const int first = (int)rank * p.per, n = max(0, min(p.per, p.V - first)), n_vec = (n + 32 * kVec - 1) / (32 * kVec) * 32;
  float mx = -INFINITY;
  {
    const int whole = p.vec ? n / kVec : 0;
    if (F32) {
      const uint32_t* src = static_cast<const uint32_t*>(p.logits) + (long long)row * p.ld + first;
#pragma unroll 8
      for (int i = tid; i < whole; i += kSampleThreads) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(src) + i);
        vals[i] = q;
        mx = fmaxf(fmaxf(fmaxf(mx, __uint_as_float(q.x)), fmaxf(__uint_as_float(q.y), __uint_as_float(q.z))), __uint_as_float(q.w));
      }
      uint32_t* dst = reinterpret_cast<uint32_t*>(vals);
      for (int i = whole * kVec + tid; i < n_vec * kVec; i += kSampleThreads) {
        const uint32_t b = i < n ? src[i] : 0xff800000u;
        dst[i] = b;
        mx = fmaxf(mx, __uint_as_float(b));
      }
    } else {
      const uint16_t* src = static_cast<const uint16_t*>(p.logits) + (long long)row * p.ld + first;
      __nv_bfloat162 m2 = __floats2bfloat162_rn(-INFINITY, -INFINITY);
#pragma unroll 8
      for (int i = tid; i < whole; i += kSampleThreads) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(src) + i);
        vals[i] = q;
        const __nv_bfloat162* b = reinterpret_cast<const __nv_bfloat162*>(&q);
        m2 = __hmax2(m2, __hmax2(__hmax2(b[0], b[1]), __hmax2(b[2], b[3])));
      }
      mx = fmaxf(__low2float(m2), __high2float(m2));
      uint16_t* dst = reinterpret_cast<uint16_t*>(vals);
      for (int i = whole * kVec + tid; i < n_vec * kVec; i += kSampleThreads) {
        const uint16_t b = i < n ? src[i] : (uint16_t)0xff80u;
        dst[i] = b;
        mx = fmaxf(mx, __uint_as_float((uint32_t)b << 16));
      }
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));  // a NaN loses against any number
  if (lane == 0) sh->scan32[warp] = __float_as_uint(mx);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSampleWarps; ++i) mx = fmaxf(mx, __uint_as_float(sh->scan32[i]));
  if (tid == 0) sh->max_bits = __float_as_uint(mx);
  ptx::cluster_sync_all();
  {
    uint32_t all[kSampleCluster];
    sample_gather(&sh->max_bits, C, all);
#pragma unroll
    for (uint32_t r = 0; r < kSampleCluster; ++r) mx = r < C ? fmaxf(mx, __uint_as_float(all[r])) : mx;
  }
  if (!(mx > -INFINITY)) {  // no token can be taken
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      p.prob[row] = 0.f;
      p.entropy[row] = 0.f;
      if (p.kept) p.kept[row] = 0;
    }
    ptx::cluster_sync_all();  // the others may still read this thread block's maximum
    return;
  }
  if (mx == INFINITY) {  // +inf counts as the largest finite value
    mx = F32 ? __uint_as_float(0x7f7fffffu) : __uint_as_float(0x7f7f0000u);
    for (int i = tid; i < n_vec * kVec; i += kSampleThreads) {
      if (F32) {
        uint32_t* x = reinterpret_cast<uint32_t*>(vals) + i;
        if (*x == 0x7f800000u) *x = 0x7f7fffffu;
      } else {
        uint16_t* x = reinterpret_cast<uint16_t*>(vals) + i;
        if (*x == 0x7f80u) *x = 0x7f7fu;
      }
    }
    __syncthreads();
  }

  // ---- thresholds
  const bool greedy = !(T > 0.0f);
  Row s;
  s.vals = vals; s.sh = sh; s.list = list; s.n_vec = n_vec; s.C = (int)C; s.rank = (int)rank; s.level = 0;
  s.vmax = mx;
  s.v_floor = fmaxf(mx - 138.0f * (greedy ? 1.0f : T), -3.402823466e38f);  // 200 ln 2 T below, and no -inf
  s.scale = 1.4426950408889634074 / (double)(greedy ? 1.0f : T);
  s.bin_scale = (float)kSampleBins / (20.0f * fminf(fmaxf(greedy ? 1.0f : T, 1e-30f), 1e30f));
  SampleCut cut{-INFINITY, 0u};
  const bool by_k = k > 1 && k < p.V, by_p = top_p < 1.0f;
  SampleSums own{0, 0.0, 0, 0};  // this thread block's kept tokens, once known
  bool summed = false, few = false;
  if (greedy || k == 1) {  // the first token alone
    cut = SampleCut{mx, 1u};
  } else if (by_k || by_p) {
    const double p64 = fmax((double)top_p, 0.0);
    s.find_bins(by_k, k, by_p);
    const int b_k = sh->b_k;
    // with few tokens kept by top-k, all that can be are listed, and nothing below looks at the slice again
    few = b_k < kSampleBins && k <= kSampleList<F32> / 2;
    if (b_k < kSampleBins) {
      s.list_bins(few ? 0 : b_k, b_k, cut);
      cut = s.template narrow<false>(b_k, b_k, cut, false, sh->before_k, (uint64_t)k);
    }
    if (by_p) {
      const SampleCut top = cut;
      const bool tied_k = b_k < kSampleBins;  // top-k kept some of the tokens that equal its threshold (they are not listed)
      const uint64_t tied = tied_k ? s.weight(top.value).whole * top.take : 0;
      int b0, b1, from = 0, upto = kSampleBins - 1;
      uint64_t all_above = 0, want = 0, in_window = 0;
      own = SampleSums{0, 0.0, 0, 0};
      for (int pass = 0; pass < 2; ++pass) {
        if (warp == 0) s.find_window(pass > 0, from >> 5, upto >> 5, (double)all_above, (double)in_window, (double)want, p64);
        if (tid == 0 && !few) sh->n_list = 0;
        __syncthreads();
        b0 = sh->b0;
        b1 = sh->b1;
        // many tokens (a wide window in a thin tail): no list yet, but whole groups, and a second look with the sums known
        const bool wide = !few && pass == 0 && sh->n_window > (uint32_t)(kSampleList<F32> / 2) * C;
        if (wide) {
          b0 &= ~31;
          b1 |= 31;
        }
        // one pass over the weights of bins [from, upto]: above the window, in it (listed), below it
        uint64_t above = 0, inside = 0, all_mine = 0;
        double ent = 0.0;
        uint32_t count = 0;
        if (pass == 0 && !tied_k) {  // every token counts: eight chains of 64-bit operations at a time keep their pipe fed
          for (int i = tid; i < n_vec; i += kSampleThreads) {
            float v[kVec];
            Row::unpack(vals[i], v);
            uint32_t listed = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const SampleWeight w = s.weight(v[e]);  // (0 for -inf and NaN)
              const int b = s.bin_of(v[e]);
              const bool up = b < b0, mid = !up && b <= b1;
              all_mine += w.whole;
              above += up ? w.whole : 0;
              inside += mid ? w.whole : 0;
              ent = fma(up ? w.w45 : 0.0, -w.t, ent);
              count += up && v[e] > -INFINITY ? 1u : 0u;
              listed |= mid && v[e] > -INFINITY ? 1u << e : 0u;
            }
            if (!wide) s.put_on_list(listed, i);
          }
        } else if (few) {
          uint64_t whole_ent = 0;
          s.each_listed(0, b_k, top, [&](float v) {
            const SampleWeight w = s.weight(v);
            const int b = s.bin_of(v);
            all_mine += w.whole;
            if (b < b0) {
              above += w.whole;
              whole_ent += sample_entropy(w);
              ++count;
            } else if (b <= b1) {
              inside += w.whole;
            }
          });
          ent = 4.0 * (double)whole_ent;
        } else {
          for (int i = tid; i < n_vec; i += kSampleThreads) {
            float v[kVec];
            Row::unpack(vals[i], v);
            uint32_t some = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const int b = s.bin_of(v[e]);
              some |= v[e] > top.value && b >= from && b <= upto ? 1u << e : 0u;
            }
            if (!__any_sync(0xffffffffu, some)) continue;  // (a weight at a time instead: bf16 6 % faster, fp32 2 % slower)
            uint32_t listed = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const SampleWeight w = s.weight(v[e]);
              const int b = s.bin_of(v[e]);
              const bool in = some >> e & 1u, up = in && b < b0, mid = in && !up && b <= b1;
              all_mine += in ? w.whole : 0;
              above += up ? w.whole : 0;
              inside += mid ? w.whole : 0;
              ent = fma(up ? w.w45 : 0.0, -w.t, ent);
              count += up ? 1u : 0u;
              listed |= mid ? 1u << e : 0u;
            }
            if (!wide) s.put_on_list(listed, i);
          }
        }
        above = sample_warp_sum(above);
        ent = sample_warp_sum(ent);
        inside = sample_warp_sum(inside);
        all_mine = sample_warp_sum(all_mine);
        count = __reduce_add_sync(0xffffffffu, count);
        if (lane == 0) {
          sh->warp[warp] = SampleSums{above, ent, count, 0u};
          sh->scan[warp] = inside;
          sh->scan2[warp] = all_mine;
        }
        __syncthreads();
        if (tid == 0) {
          SampleSums a{0, 0.0, 0, 0};
          uint64_t w_in = 0, w_all = 0;
          for (int i = 0; i < kSampleWarps; ++i) {
            a.mass += sh->warp[i].mass;
            a.ent += sh->warp[i].ent;
            a.count += sh->warp[i].count;
            w_in += sh->scan[i];
            w_all += sh->scan2[i];
          }
          sh->extra[pass] = a;
          sh->window[pass] = w_in;
          sh->looked[pass] = w_all;
        }
        ptx::cluster_sync_all();
        all_above += sample_cluster_sum(&sh->extra[pass].mass, C);
        in_window = sample_cluster_sum(&sh->window[pass], C);
        
        own.mass += sh->extra[pass].mass;
        own.ent += sh->extra[pass].ent;
        own.count += sh->extra[pass].count;
        if (pass == 0) {
          const uint64_t all = sample_cluster_sum(&sh->looked[pass], C) + tied;
          const double goal = ceil(p64 * (double)all);
          want = goal >= (double)all ? all : goal < 1.0 ? 1 : (uint64_t)goal;
          if (tied_k && b_k <= b1) in_window += tied;  // (b_k is in the window then, as the window ends there at the latest)
        }
        if (!wide) break;
        from = b0;
        upto = b1;
      }
      cut = s.template narrow<true>(b0, b1, top, tied_k && b_k <= b1, all_above, want);
      if (tied_k && cut.value == top.value) cut.take = min(cut.take, top.take);
      // this thread block's kept tokens: those above the window and the listed ones above the cut
      const SampleSums in = s.listed_sums(b0, b1, top, cut, -INFINITY, -INFINITY);
      own.mass += in.mass;
      own.ent += in.ent;
      own.count += in.count;
      own.ties += in.ties;
      if (tied_k && cut.value == top.value) {  // (these were left out)
        uint32_t t = 0;
        if (few) {
          s.each_listed(b_k, b_k, SampleCut{-INFINITY, 0u}, [&](float v) { t += v == cut.value ? 1u : 0u; });
        } else {
          for (int i = tid; i < n_vec; i += kSampleThreads) {
            float v[kVec];
            Row::unpack(vals[i], v);
#pragma unroll
            for (int e = 0; e < kVec; ++e) t += v[e] == cut.value ? 1u : 0u;
          }
        }
        t = __reduce_add_sync(0xffffffffu, t);
        if (lane == 0) sh->scan32[warp] = t;
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < kSampleWarps; ++i) own.ties += sh->scan32[i];
      }
      summed = true;
    }
  }
  // w >= min_p as t >= log2 min_p; `reject`: a value that no kept token is below
  double min_t = -INFINITY;
  float reject = cut.value;
  if (mp > 0.0f) {
    min_t = log2(fmin((double)mp, 1.0));
    if (cut.value > -INFINITY && s.weight(cut.value).t >= min_t) {
      min_t = -INFINITY;  // the cut already stands above it
    } else {
      summed = false;
      const double down = min_t / s.scale;
      reject = fmaxf(reject, (float)((double)mx + down - 1e-6 * (fabs((double)mx) - down)));
    }
  }

  // ---- what is kept in each slice
  bool warps_known = false;
  if (!summed && few) {
    own = s.listed_sums(0, sh->b_k, SampleCut{-INFINITY, 0u}, cut, min_t, reject);
  } else if (!summed) {
    s.kept_sums(cut, min_t, reject);
    warps_known = true;
    own = SampleSums{0, 0.0, 0, 0};
#pragma unroll 1
    for (int i = 0; i < kSampleWarps; ++i) {
      own.mass += sh->warp[i].mass;
      own.ent += sh->warp[i].ent;
      own.count += sh->warp[i].count;
      own.ties += sh->warp[i].ties;
    }
  }
  if (tid == 0) sh->mine = own;
  ptx::cluster_sync_all();
  const bool has_cut = cut.value > -INFINITY;
  const SampleWeight tie = s.weight(has_cut ? cut.value : mx);
  const uint64_t tie_fix = has_cut ? tie.whole : 0;
  uint32_t take = has_cut && tie.t >= min_t ? cut.take : 0u;
  uint64_t W = 0, my_first = 0, my_mass = 0;
  double sum_ent = 0.0;
  uint32_t my_take = 0, kept = 0;
  uint64_t masses[kSampleCluster];
  double ents[kSampleCluster];
  uint32_t counts[kSampleCluster], tied[kSampleCluster];
  sample_gather(&sh->mine.mass, C, masses);
  sample_gather(&sh->mine.ent, C, ents);
  sample_gather(&sh->mine.count, C, counts);
  sample_gather(&sh->mine.ties, C, tied);
#pragma unroll
  for (uint32_t r = 0; r < kSampleCluster; ++r) {  // (zeros from C on)
    const uint32_t t = min(take, tied[r]);
    const uint64_t all = masses[r] + (uint64_t)t * tie_fix;
    if (r == rank) {
      my_first = W;
      my_mass = all;
      my_take = t;
    }
    W += all;
    take -= t;
    kept += counts[r] + t;
    sum_ent += ents[r];
    if (has_cut) sum_ent = fma((double)t, -tie.w45 * tie.t, sum_ent);
  }
  ptx::cluster_sync_all();  // nothing of another thread block is read after this

  // ---- the token
  const double at = floor((u > 0.0f ? (double)u : 0.0) * (double)W);
  const uint64_t target = at >= (double)(W - 1) ? W - 1 : (uint64_t)at;
  if (rank == 0 && tid == 0) {
    const double total = (double)W * (1.0 / 35184372088832.0);  // 2^45
    p.entropy[row] = fmaxf(0.0f, (float)(log(total) + 0.69314718055994530942 * sum_ent * (1.0 / 35184372088832.0) / total));
    if (p.kept) p.kept[row] = (int32_t)kept;
  }
  if (target < my_first || target >= my_first + my_mass) return;
  uint64_t rest = target - my_first;
  if (!warps_known) s.kept_sums(cut, min_t, reject);
  // the warp whose part holds it
  uint32_t t_left = my_take;
  int w = 0;
  for (; w < kSampleWarps - 1; ++w) {
    const uint32_t t = min(t_left, sh->warp[w].ties);
    const uint64_t m = sh->warp[w].mass + (uint64_t)t * tie_fix;
    if (rest < m) break;
    rest -= m;
    t_left -= t;
  }
  if (w != warp) return;
  const int v_first = warp * s.warp_vecs(), v_last = min(n_vec, v_first + s.warp_vecs());
  for (int i0 = v_first; i0 < v_last; i0 += 32) {
    float v[kVec];
    uint64_t m[kVec], mass = 0;
    uint32_t ties = 0;
    if (i0 + lane < v_last) {
      Row::unpack(vals[i0 + lane], v);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const SampleWeight x = s.weight(v[e]);
      m[e] = v[e] > cut.value && x.t >= min_t ? x.whole : 0;
      ties += v[e] == cut.value && has_cut ? 1u : 0u;
      mass += m[e];
    }
    uint32_t t_incl = ties;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, t_incl, o);
      if (lane >= o) t_incl += x;
    }
    uint32_t t_mine = t_left > t_incl - ties ? min(ties, t_left - (t_incl - ties)) : 0u;  // of this lane's, the first so many
    uint64_t incl = mass + (uint64_t)t_mine * tie_fix;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, incl > rest);
    if (past) {
      const int src = __ffs(past) - 1;
      const uint64_t before = __shfl_sync(0xffffffffu, incl, src > 0 ? src - 1 : 0);
      if (lane == src) {
        uint64_t left = rest - (src > 0 ? before : 0);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          uint64_t x = m[e];
          if (v[e] == cut.value && has_cut && t_mine) {
            x = tie_fix;
            --t_mine;
          }
          if (left < x) {
            p.token[row] = first + (i0 + lane) * kVec + e;
            p.prob[row] = (float)((double)x / (double)W);
            break;
          }
          left -= x;
        }
      }
      return;
    }
    rest -= __shfl_sync(0xffffffffu, incl, 31);
    t_left -= min(t_left, __shfl_sync(0xffffffffu, t_incl, 31));
  }
}

cudaError_t setup_sample(sdlm_ctx*) {
  const int most = (int)sizeof(SampleShared) + kSampleList<true> * 4 + (kSampleMaxVocab / 8 + 8) * 4 + 512;  // (bf16: half the slice)
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  return e;
}

}  // namespace sdlm

using namespace sdlm;

extern "C" sdlm_status sdlm_sample(sdlm_ctx* ctx, int32_t rows, int32_t vocab, sdlm_logit_type type, const void* logits,
                                   int64_t row_stride, const float* u, const float* temperature, const int32_t* top_k,
                                   const float* top_p, const float* min_p, int32_t* token, float* prob, float* entropy,
                                   int32_t* n_kept, void* stream) {
  if (!ctx || !logits || !u || !token || !prob || !entropy || rows < 1 || vocab < 1) return SDLM_ERR_INVALID_ARG;
  if (type != SDLM_LOGITS_BF16 && type != SDLM_LOGITS_F32) return SDLM_ERR_INVALID_ARG;
  if (row_stride < vocab || row_stride > (1ll << 40)) return SDLM_ERR_INVALID_ARG;
  const bool f32 = type == SDLM_LOGITS_F32;
  const uintptr_t at = reinterpret_cast<uintptr_t>(logits);
  if (at % (f32 ? 4 : 2)) return SDLM_ERR_INVALID_ARG;
  if (vocab > kSampleMaxVocab) return SDLM_ERR_UNSUPPORTED;  // sums of weights in 64 bits; a slice in shared memory
  if (rows > (1 << 27)) return SDLM_ERR_SHAPE;
  if (!same_device(ctx)) return SDLM_ERR_INVALID_ARG;
  // Outputs must not lie over logits or each other; over the rows' parameters only row for row (a row's thread blocks have
  // all read theirs when its results are written, other rows' have not).
  const size_t per_row = (size_t)rows * 4, logits_b = ((size_t)(rows - 1) * row_stride + vocab) * (f32 ? 4 : 2);
  const void* const outs[] = {token, prob, entropy, n_kept};
  const void* const ins[] = {u, temperature, top_k, top_p, min_p};
  for (int i = 0; i < 4; ++i) {
    if (!outs[i]) continue;
    if (ranges_overlap(outs[i], per_row, logits, logits_b)) return SDLM_ERR_INVALID_ARG;
    for (int o = 0; o < i; ++o)
      if (ranges_overlap(outs[i], per_row, outs[o], per_row)) return SDLM_ERR_INVALID_ARG;
    for (const void* in : ins)
      if (in && in != outs[i] && ranges_overlap(outs[i], per_row, in, per_row)) return SDLM_ERR_INVALID_ARG;
  }
  SampleParams p;
  p.logits = logits; p.ld = row_stride; p.u = u; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.token = token; p.prob = prob; p.entropy = entropy; p.kept = n_kept;
  p.V = vocab;
  // Thread blocks of a row, in powers of two up to eight (the portable cluster size): a slice of at most 80 KB, so that two
  // fit an SM, and eight where all rows then run at once.  More of them have less to do each but meet as often: 128 rows of
  // 151936 bf16 logits, top-k 51 us with four and 77 with eight; one row, top-p: 63 and 49 (before later steps).
  const int esz = f32 ? 4 : 2;
  unsigned c = 1;
  const int most = rows * 8 <= ctx->sm_count ? 16384 : 81920;
  while (c < 8 && (long long)vocab * esz > (long long)most * c) c *= 2;
  p.per = (int)(((vocab + c - 1) / c + 7) / 8 * 8);
  p.vec = at % 16 == 0 && (row_stride * esz) % 16 == 0;
  const size_t list = (size_t)(f32 ? kSampleList<true> : kSampleList<false>) * 4;
  const size_t smem = sizeof(SampleShared) + list + ((size_t)p.per * esz + 511) / 512 * 512;  // (whole warps of 16 bytes a lane)
  const dim3 grid((unsigned)rows * c);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = f32 ? launch_overlapped_cluster(sample_kernel<true>, grid, dim3(kSampleThreads), smem, st, c, p)
                            : launch_overlapped_cluster(sample_kernel<false>, grid, dim3(kSampleThreads), smem, st, c, p);
  ctx->launches++;
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? SDLM_OK : SDLM_ERR_CUDA;
}
