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
// What bounds it is reading the logits once.  A cluster of up to eight thread blocks takes a row, a slice each, which
// stays in shared memory as order-preserving integer keys; all passes after the first run on chip and meet through
// the cluster's shared memory.  A threshold is found by histograms: first over bins of T/32 below the maximum, where
// few neighbours collide, then over the keys of the bin that the threshold falls in, until a bin holds one key.
//
// The answer is a comparison of sums of up to 2^18 weights with u W or p times their total, and a token changes when a
// border moves by a millionth, so weights are formed in 64 bits and summed as whole multiples of 2^-45 (W < 2^18 then
// stays below 2^63): such sums are exact, so the order of the additions, atomics among them, changes nothing.
#include "sdlm_internal.h"
#include "sdlm_ptx.cuh"

#include <math.h>

namespace sdlm {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 1024;
constexpr int kSampleMaxVocab = 1 << 18;

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
  int V, per, seg, vec;      // vocabulary, slice of a thread block, slice of a thread, 16-byte loads
};

// A row's slice in shared memory as keys that order like the values: key 0 for a token that cannot be taken (-inf or
// NaN); +inf counts as the largest finite value, -0 as 0.
template <bool F32>
struct SampleKey;
template <>
struct SampleKey<true> {
  using type = uint32_t;
  static __device__ __forceinline__ uint32_t of(uint32_t bits) {
    if ((bits & 0x7fffffffu) > 0x7f800000u || bits == 0xff800000u) return 0u;
    if (bits == 0x7f800000u) bits = 0x7f7fffffu;
    if (bits == 0x80000000u) bits = 0u;
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
  }
};
template <>
struct SampleKey<false> {
  using type = uint16_t;
  static __device__ __forceinline__ uint32_t of(uint32_t bits) {
    if ((bits & 0x7fffu) > 0x7f80u || bits == 0xff80u) return 0u;
    if (bits == 0x7f80u) bits = 0x7f7fu;
    if (bits == 0x8000u) bits = 0u;
    return bits & 0x8000u ? ~bits & 0xffffu : bits | 0x8000u;
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    return __uint_as_float((key & 0x8000u ? key ^ 0x8000u : ~key & 0xffffu) << 16);
  }
};

// Weight of a value: t = z log2 e, w = 2^t with a relative error below 1e-11, and w as a multiple of 2^-45.
struct SampleWeight {
  double t, w;
  uint64_t fix;
};
__device__ __forceinline__ SampleWeight sample_weight(float v, double vmax, double scale) {
  SampleWeight r;
  r.t = fmax(((double)v - vmax) * scale, -300.0);  // 2^-300 is below every positive min_p and adds nothing
  const double kMagic = 6755399441055744.0;        // 1.5 * 2^52: adding it leaves round(t) in the low bits
  const double m = r.t + kMagic;
  const double f = r.t - (m - kMagic);             // |f| <= 1/2
  // 2^f = sum (f ln 2)^i / i! up to i = 9; what the series leaves out is below (ln 2 / 2)^10 / 10! = 7e-12
  const double x = f * 0.69314718055994530942;
  double q = 1.0 / 362880.0;
  q = fma(q, x, 1.0 / 40320.0);
  q = fma(q, x, 1.0 / 5040.0);
  q = fma(q, x, 1.0 / 720.0);
  q = fma(q, x, 1.0 / 120.0);
  q = fma(q, x, 1.0 / 24.0);
  q = fma(q, x, 1.0 / 6.0);
  q = fma(q, x, 0.5);
  q = fma(q, x, 1.0);
  q = fma(q, x, 1.0);
  r.w = __hiloint2double(__double2hiint(q) + (__double2loint(m) << 20), __double2loint(q));
  // w 2^45 rounded to a whole number: it is at most 2^45, so adding 2^52 leaves it in the mantissa
  r.fix = (uint64_t)__double_as_longlong(fma(r.w, 35184372088832.0, 4503599627370496.0)) & 0xfffffffffffffull;
  return r;
}

// What a thread block tells the others of its cluster.
struct SampleExchange {
  uint64_t mass;
  double wt;       // sum of w t over the kept tokens above the threshold key
  uint32_t count, ties, max_key, pad;
};

struct alignas(16) SampleShared {  // the keys behind it are read and written 16 bytes at a time
  uint32_t count[2][kSampleBins];             // by parity of the level: one barrier per level then suffices
  uint32_t lo[2][kSampleBins], hi[2][kSampleBins];
  SampleExchange mine;
  uint64_t scan[kSampleWarps];
  uint32_t scan32[kSampleWarps];
  double scan_d[kSampleWarps];
  uint64_t found_before, total;
  int found_bin;
};

struct SampleCut {
  uint32_t key, take;  // tokens above `key` are kept, and the first `take` of those that equal it
};

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

template <bool F32>
struct SampleRow {
  using Key = typename SampleKey<F32>::type;
  const Key* keys;
  SampleShared* sh;
  int n_pad, C, rank;
  double vmax, scale;       // largest value; log2 e / T
  float vmaxf, bin_scale;
  uint32_t kmax;
  int level;                // histogram levels so far (buffer parity)

  __device__ __forceinline__ int bin_of(float v) const { return min(kSampleBins - 1, __float2int_rz((vmaxf - v) * bin_scale)); }

  // Finds the cut that leaves the first k tokens (MASS false; want = k) or the shortest prefix with `frac` of the weight
  // (MASS true), among the tokens above floor.key and the first floor.take that equal it.  Returns false when
  // nothing is cut off.
  template <bool MASS>
  __device__ bool cut(uint64_t want, double frac, const SampleCut floor, SampleCut& out) {
    uint32_t r_lo = 1, r_hi = kmax;
    int in_bin = -1, shift = 0;
    uint64_t before = 0;
    for (int lev = 0; lev < 8; ++lev) {  // a level leaves a 1024th of at most 2^32 keys: five are enough
      const int buf = level & 1;
      uint32_t* cnt = sh->count[buf];
      uint32_t* lo = sh->lo[buf];
      uint32_t* hi = sh->hi[buf];
      for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) {
        if (MASS) lo[i] = hi[i] = 0; else cnt[i] = 0;
      }
      if (threadIdx.x == 0) sh->found_bin = 0;
      __syncthreads();
      auto add = [&](uint32_t key, uint32_t n) {
        const float v = SampleKey<F32>::value(key);
        int i;
        if (lev == 0) {
          i = bin_of(v);
        } else {
          if (key < r_lo || key > r_hi || bin_of(v) != in_bin) return;
          i = (int)((r_hi - key) >> shift);
        }
        if (MASS) {
          const uint64_t w = sample_weight(v, vmax, scale).fix * n;
          if (w == 0) return;
          // 64 bits in two halves; the carry goes with whoever brought the lower half over
          const uint32_t w_lo = (uint32_t)w, old = atomicAdd(&lo[i], w_lo);
          const uint32_t up = (uint32_t)(w >> 32) + (old + w_lo < old ? 1u : 0u);
          if (up) atomicAdd(&hi[i], up);
        } else {
          atomicAdd(&cnt[i], n);
        }
      };
      for (int i = threadIdx.x; i < n_pad; i += kSampleThreads) {
        const uint32_t key = keys[i];
        if (key > floor.key) add(key, 1);
      }
      if (floor.take && rank == 0 && threadIdx.x == 0) add(floor.key, floor.take);
      ++level;
      ptx::cluster_sync_all();
      // two neighbouring bins a thread, summed over the cluster
      uint64_t v0 = 0, v1 = 0;
      for (int r = 0; r < C; ++r) {
        if (MASS) {
          const uint2 l = ptx::ld_cluster_v2(ptx::mapa_u32(ptx::smem_u32(&lo[2 * threadIdx.x]), r));
          const uint2 h = ptx::ld_cluster_v2(ptx::mapa_u32(ptx::smem_u32(&hi[2 * threadIdx.x]), r));
          v0 += ((uint64_t)h.x << 32) + l.x;
          v1 += ((uint64_t)h.y << 32) + l.y;
        } else {
          const uint2 c = ptx::ld_cluster_v2(ptx::mapa_u32(ptx::smem_u32(&cnt[2 * threadIdx.x]), r));
          v0 += c.x;
          v1 += c.y;
        }
      }
      uint64_t total;
      const uint64_t e0 = before + sample_scan(v0 + v1, sh->scan, total), e1 = e0 + v0;
      if (lev == 0) {
        if (MASS) {
          const double t = ceil(frac * (double)total);
          want = t >= (double)total ? total : t < 1.0 ? 1 : (uint64_t)t;
        } else if (want >= total) {
          return false;
        }
      }
      if (e0 < want && want <= e1) { sh->found_bin = 2 * threadIdx.x; sh->found_before = e0; }
      if (e1 < want && want <= e1 + v1) { sh->found_bin = 2 * threadIdx.x + 1; sh->found_before = e1; }
      __syncthreads();
      const int bin = sh->found_bin;
      before = sh->found_before;
      __syncthreads();
      if (lev == 0) {
        // keys of the bin: values between vmax - (bin + 1) / s and vmax - bin / s, widened by what rounding may move
        in_bin = bin;
        const float near = (float)bin / bin_scale, far = (float)(bin + 1) / bin_scale;
        const float slack = 1e-6f * (fabsf(vmaxf) + far) + 1e-37f;
        r_hi = kmax;
        r_lo = 1;
        if (bin > 0) r_hi = min(kmax, key_near(vmaxf - near + slack, true));
        if (bin < kSampleBins - 1) r_lo = max(1u, key_near(vmaxf - far - slack, false));
      } else {
        r_hi -= (uint32_t)bin << shift;
        const uint32_t w = (1u << shift) - 1u;
        r_lo = r_hi - r_lo > w ? r_hi - w : r_lo;
        if (shift == 0) break;
      }
      shift = 0;
      while (((r_hi - r_lo) >> shift) >= (uint32_t)kSampleBins) ++shift;
    }
    out.key = r_hi;
    const uint64_t each = MASS ? max((uint64_t)1, sample_weight(SampleKey<F32>::value(r_hi), vmax, scale).fix) : 1;
    out.take = (uint32_t)((want - before + each - 1) / each);
    return true;
  }

  // A key no smaller (up) or no larger than that of any value on the inner side of v.
  __device__ __forceinline__ uint32_t key_near(float v, bool up) const {
    if (isinf(v)) return up ? kmax : 1u;
    const uint32_t k = SampleKey<true>::of(__float_as_uint(v));
    return F32 ? k : up ? (k >> 16) + 1u : k >> 16;
  }
};

template <bool F32>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const SampleParams p) {
  using Key = typename SampleKey<F32>::type;
  extern __shared__ __align__(16) uint8_t sample_smem[];
  SampleShared* sh = reinterpret_cast<SampleShared*>(sample_smem);
  Key* keys = reinterpret_cast<Key*>(sample_smem + sizeof(SampleShared));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t C, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
  rank = ptx::cluster_ctarank();
  const int row = blockIdx.x / C;
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();

  // ---- the slice into shared memory, its largest key
  const int first = (int)rank * p.per, n = max(0, min(p.per, p.V - first)), n_pad = kSampleThreads * p.seg;
  uint32_t kmax = 0;
  if (F32) {
    const uint32_t* src = static_cast<const uint32_t*>(p.logits) + (long long)row * p.ld + first;
    const int whole = p.vec ? n / 4 : 0;
#pragma unroll 4
    for (int i = tid; i < whole; i += kSampleThreads) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(src) + i);
      const uint4 k = make_uint4(SampleKey<true>::of(v.x), SampleKey<true>::of(v.y), SampleKey<true>::of(v.z), SampleKey<true>::of(v.w));
      reinterpret_cast<uint4*>(keys)[i] = k;
      kmax = max(max(kmax, max(k.x, k.y)), max(k.z, k.w));
    }
    for (int i = whole * 4 + tid; i < n_pad; i += kSampleThreads) {
      const uint32_t k = i < n ? SampleKey<true>::of(src[i]) : 0u;
      keys[i] = (Key)k;
      kmax = max(kmax, k);
    }
  } else {
    const uint16_t* src = static_cast<const uint16_t*>(p.logits) + (long long)row * p.ld + first;
    const int whole = p.vec ? n / 8 : 0;
#pragma unroll 4
    for (int i = tid; i < whole; i += kSampleThreads) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(src) + i);
      const uint32_t in[4] = {v.x, v.y, v.z, v.w};
      uint32_t out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t a = SampleKey<false>::of(in[e] & 0xffffu), b = SampleKey<false>::of(in[e] >> 16);
        out[e] = a | b << 16;
        kmax = max(kmax, max(a, b));
      }
      reinterpret_cast<uint4*>(keys)[i] = make_uint4(out[0], out[1], out[2], out[3]);
    }
    for (int i = whole * 8 + tid; i < n_pad; i += kSampleThreads) {
      const uint32_t k = i < n ? SampleKey<false>::of(src[i]) : 0u;
      keys[i] = (Key)k;
      kmax = max(kmax, k);
    }
  }
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) sh->scan32[warp] = kmax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSampleWarps; ++i) kmax = max(kmax, sh->scan32[i]);
  if (tid == 0) sh->mine.max_key = kmax;
  ptx::cluster_sync_all();
  for (uint32_t r = 0; r < C; ++r) kmax = max(kmax, ptx::ld_cluster_u32(ptx::mapa_u32(ptx::smem_u32(&sh->mine.max_key), r)));
  if (kmax == 0) {  // no token can be taken
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      p.prob[row] = 0.f;
      p.entropy[row] = 0.f;
      if (p.kept) p.kept[row] = 0;
    }
    ptx::cluster_sync_all();  // the others may still read this thread block's maximum
    return;
  }

  // ---- thresholds
  const float T = p.temperature ? p.temperature[row] : 1.0f;
  const bool greedy = !(T > 0.0f);
  SampleRow<F32> s;
  s.keys = keys; s.sh = sh; s.n_pad = n_pad; s.C = (int)C; s.rank = (int)rank;
  s.kmax = kmax; s.level = 0;
  s.vmaxf = SampleKey<F32>::value(kmax);
  s.vmax = (double)s.vmaxf;
  s.scale = 1.4426950408889634074 / (double)(greedy ? 1.0f : T);
  s.bin_scale = (float)kSampleBins / (32.0f * fminf(fmaxf(greedy ? 1.0f : T, 1e-30f), 1e30f));
  SampleCut cut{0u, 0u};
  const int k = p.top_k ? p.top_k[row] : 0;
  if (greedy || k == 1) {
    cut = SampleCut{kmax, 1u};
  } else {
    SampleCut c;
    if (k > 0 && k < p.V && s.template cut<false>((uint64_t)k, 0.0, cut, c)) cut = c;
    const float top_p = p.top_p ? p.top_p[row] : 1.0f;
    if (top_p < 1.0f && s.template cut<true>(0, fmax((double)top_p, 0.0), cut, c)) cut = c;
  }
  const float mp = p.min_p ? p.min_p[row] : 0.0f;
  const double min_w = mp > 0.0f ? fmin((double)mp, 1.0) : -1.0;

  // ---- what is kept, by contiguous slices of the threads
  uint64_t mass = 0;
  double wt = 0.0;
  uint32_t count = 0, ties = 0;
  const Key* seg = keys + tid * p.seg;
  for (int i = 0; i < p.seg; ++i) {
    const uint32_t key = seg[i];
    if (key > cut.key) {
      const SampleWeight w = sample_weight(SampleKey<F32>::value(key), s.vmax, s.scale);
      if (w.w >= min_w) {
        mass += w.fix;
        wt = fma(w.w, w.t, wt);
        ++count;
      }
    } else if (key == cut.key && key != 0) {
      ++ties;
    }
  }
  uint64_t cta_mass, cta_ties;
  const uint64_t mass_before = sample_scan(mass, sh->scan, cta_mass);
  const uint64_t ties_before = sample_scan(ties, sh->scan, cta_ties);
#pragma unroll
  for (int o = 16; o; o >>= 1) wt += __shfl_xor_sync(0xffffffffu, wt, o);
  count = __reduce_add_sync(0xffffffffu, count);
  if (lane == 0) {
    sh->scan_d[warp] = wt;
    sh->scan32[warp] = count;
  }
  __syncthreads();
  if (tid == 0) {
    SampleExchange x{cta_mass, 0.0, 0u, (uint32_t)cta_ties, kmax, 0u};
    for (int i = 0; i < kSampleWarps; ++i) {
      x.wt += sh->scan_d[i];
      x.count += sh->scan32[i];
    }
    sh->mine = x;  // (whoever still reads max_key gets the cluster's maximum, which does as well)
  }
  ptx::cluster_sync_all();
  const SampleWeight tie = sample_weight(SampleKey<F32>::value(cut.key), s.vmax, s.scale);
  const uint64_t tie_fix = cut.key ? tie.fix : 0;
  uint32_t take = cut.key && tie.w >= min_w ? cut.take : 0u;
  uint64_t W = 0, my_first = 0, my_mass = 0;
  uint32_t my_take = 0, kept = 0;
  double sum_wt = 0.0;
  for (uint32_t r = 0; r < C; ++r) {
    const uint32_t a = ptx::mapa_u32(ptx::smem_u32(&sh->mine), r);
    const uint64_t m = ptx::ld_cluster_u64(a + offsetof(SampleExchange, mass));
    const uint32_t t = min(take, ptx::ld_cluster_u32(a + offsetof(SampleExchange, ties)));
    const uint64_t all = m + (uint64_t)t * tie_fix;
    if (r == rank) {
      my_first = W;
      my_mass = all;
      my_take = t;
    }
    W += all;
    take -= t;
    kept += ptx::ld_cluster_u32(a + offsetof(SampleExchange, count)) + t;
    sum_wt += __longlong_as_double((long long)ptx::ld_cluster_u64(a + offsetof(SampleExchange, wt))) + (double)t * (cut.key ? tie.w * tie.t : 0.0);
  }
  ptx::cluster_sync_all();  // nothing of another thread block is read after this

  // ---- the token
  const float u = p.u[row];
  const double at = floor((u > 0.0f ? (double)u : 0.0) * (double)W);
  const uint64_t target = at >= (double)(W - 1) ? W - 1 : (uint64_t)at;
  if (rank == 0 && tid == 0) {
    const double total = (double)W * (1.0 / 35184372088832.0);
    p.entropy[row] = fmaxf(0.0f, (float)(log(total) - 0.69314718055994530942 * sum_wt / total));
    if (p.kept) p.kept[row] = (int32_t)kept;
  }
  if (target < my_first || target >= my_first + my_mass) return;
  const uint64_t rest = target - my_first;
  const uint32_t t_before = (uint32_t)min((uint64_t)my_take, ties_before);
  const uint64_t start = mass_before + (uint64_t)t_before * tie_fix;
  const uint64_t own = mass + (uint64_t)min(my_take - t_before, ties) * tie_fix;
  const uint32_t who = __ballot_sync(0xffffffffu, rest >= start && rest < start + own);
  if (!who) return;
  // the warp goes through that thread's slice together, 32 tokens at a time
  const int src = __ffs(who) - 1;
  uint64_t left = rest - __shfl_sync(0xffffffffu, start, src);
  uint32_t t_left = my_take - __shfl_sync(0xffffffffu, t_before, src);
  const int base = (warp * 32 + src) * p.seg;
  for (int i0 = 0; i0 < p.seg; i0 += 32) {
    const uint32_t key = i0 + lane < p.seg ? keys[base + i0 + lane] : 0u;
    const uint32_t eq = __ballot_sync(0xffffffffu, key == cut.key && key != 0);
    uint64_t w = 0;
    if (key > cut.key) {
      const SampleWeight x = sample_weight(SampleKey<F32>::value(key), s.vmax, s.scale);
      if (x.w >= min_w) w = x.fix;
    } else if ((eq >> lane & 1u) && __popc(eq & ((1u << lane) - 1u)) < t_left) {
      w = tie_fix;
    }
    uint64_t incl = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, incl > left);
    if (past) {
      if (lane == __ffs(past) - 1) {
        p.token[row] = first + base + i0 + lane;
        p.prob[row] = (float)((double)w / (double)W);
      }
      return;
    }
    left -= __shfl_sync(0xffffffffu, incl, 31);
    t_left -= min(t_left, (uint32_t)__popc(eq));
  }
}

static_assert(sizeof(SampleShared) % 16 == 0, "the keys start on a 16-byte boundary");

cudaError_t setup_sample(sdlm_ctx*) {
  const int most = (int)sizeof(SampleShared) + (kSampleMaxVocab / 8 + 2 * kSampleThreads) * 4;
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
  SampleParams p;
  p.logits = logits; p.ld = row_stride; p.u = u; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.token = token; p.prob = prob; p.entropy = entropy; p.kept = n_kept;
  p.V = vocab;
  // one thread block for every 8192 tokens or so, in powers of two up to eight (the portable cluster size)
  unsigned c = 1;
  while (c < 8 && vocab > 8192 * (int)c) c *= 2;
  p.per = (int)(((vocab + c - 1) / c + 7) / 8 * 8);
  // a thread's slice is an odd number of 32-bit words, so that the threads of a warp start in different banks
  const int words = f32 ? (p.per + kSampleThreads - 1) / kSampleThreads : (p.per + 2 * kSampleThreads - 1) / (2 * kSampleThreads);
  p.seg = (words | 1) * (f32 ? 1 : 2);
  const int esz = f32 ? 4 : 2;
  p.vec = at % 16 == 0 && (row_stride * esz) % 16 == 0;
  const size_t smem = sizeof(SampleShared) + (size_t)kSampleThreads * p.seg * esz;
  const dim3 grid((unsigned)rows * c);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = f32 ? launch_overlapped_cluster(sample_kernel<true>, grid, dim3(kSampleThreads), smem, st, c, p)
                            : launch_overlapped_cluster(sample_kernel<false>, grid, dim3(kSampleThreads), smem, st, c, p);
  ctx->launches++;
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? SDLM_OK : SDLM_ERR_CUDA;
}
