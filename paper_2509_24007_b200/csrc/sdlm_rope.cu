// Rotary positions of query and key rows at positions the caller gives, with the per-head RMS norm of both in the
// same pass (sdlm_qk_norm_rope).  sdlm_rope_block rotates the rows right behind the cached history, whole heads, in
// the rotate-half convention; the nodes of a drafted tree (two siblings share a position), prompts, the layout of
// neighbouring pairs, partly rotated heads and contexts beyond the trained length need this one.
//
//   y = x / sqrt(mean_d(x^2) + eps) * w          (left out without weights)
//   out[a_i] = y[a_i] m cos(t_i) - y[b_i] m sin(t_i),   out[b_i] = y[b_i] m cos(t_i) + y[a_i] m sin(t_i),  i < rot/2
//   t_i = position * f_i;  (a_i, b_i) = (i, i + rot/2) or (2i, 2i + 1);  out = y beyond rot
//
// Bound by memory: every element is read and written once.  d/16 lanes take a head, each of them 16 elements that
// hold eight whole pairs in either layout, so that a pair never leaves its thread and the mean takes log2(d/16)
// shuffles.  A warp keeps to one row and goes through its heads, so that the row's angles are worked out once per
// warp.  The angle is formed in turns: position * (f_i / 2 pi) in 64 bits, its fraction in 32 (a position of a
// million times a frequency near 1 keeps no fraction worth having in 32 bits); the frequencies are worked out on the
// host in 64 bits and travel as kernel arguments.  Everything else is fp32 with one rounding to bf16 at the end.
//
// 16381 rows of 40 + 8 heads of 128 (403 MB): 73 us, 5.5 TB/s; 672 rows of 16 + 2 heads: 4.3 us; one row: 2.8 us, which
// is a launch.
#include "sdlm_internal.h"
#include "sdlm_ptx.cuh"

#include <math.h>
#include <string.h>

namespace sdlm {

constexpr int kRopeThreads = 128;

struct RopeParams {
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  __nv_bfloat16* q_out;
  __nv_bfloat16* k_out;
  const __nv_bfloat16* q_weight;  // or null: no norm
  const __nv_bfloat16* k_weight;
  const int32_t* positions;  // [rows], or null: the row's number within its sequence
  const int32_t* seq_len;    // null: positions stand for themselves; else they count from the slot's length
  const int32_t* seq_ids;
  DevHeader* hdr;
  long long q_stride, k_stride;  // elements from one row to the next
  long long rows;
  int D, max_batch, n_heads, n_heads2, rot, interleaved;
  int parts;                     // warps that share a row's heads
  float eps, mscale;
  double freq[64];               // turns per position of pair i
};

// cos and sin of 2 pi * turns for the eight pairs of a lane, times the attention factor of the scaling
__device__ __forceinline__ void rope_angles(const RopeParams& p, double pos, int first_pair, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double t = pos * p.freq[first_pair + e];
    const float f = (float)(t - rint(t));
    sincospif(2.0f * f, &sn[e], &cs[e]);
    cs[e] *= p.mscale;
    sn[e] *= p.mscale;
  }
}

template <int HD>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int TPH = HD / 16;     // lanes of one head
  constexpr int HPW = 32 / TPH;    // heads a warp works on at a time
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  const long long unit = (long long)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  const long long row = unit / p.parts;
  if (row >= p.rows) return;
  const int part = (int)(unit % p.parts), lane = threadIdx.x & 31, l = lane % TPH;
  const int heads = p.n_heads + p.n_heads2, groups = (heads + HPW - 1) / HPW;

  const bool rotated = l < p.rot / 16;
  // the lane's two chunks of eight elements: the halves of eight pairs, or sixteen neighbours
  const bool halves = rotated && !p.interleaved;
  const int c0 = halves ? l : 2 * l, c1 = halves ? l + p.rot / 16 : 2 * l + 1;

  uint4 x0, x1;
  auto fetch = [&](int g) {
    const int h = g * HPW + lane / TPH;
    x0 = x1 = make_uint4(0, 0, 0, 0);
    if (g < groups && h < heads) {
      const uint4* src = reinterpret_cast<const uint4*>(h < p.n_heads ? p.q + row * p.q_stride + (long long)h * HD
                                                                      : p.k + row * p.k_stride + (long long)(h - p.n_heads) * HD);
      x0 = src[c0];
      x1 = src[c1];
    }
  };
  fetch(part);

  const long long b = row / p.D;
  const int j = (int)(row % p.D);
  long long pos = p.positions ? p.positions[row] : j;
  if (p.seq_len) {
    const int slot = p.seq_ids ? p.seq_ids[b] : (int)b;
    if (slot < 0 || slot >= p.max_batch) {  // never follow a bad slot number out of the tables: the row is left alone
      if (lane == 0 && part == 0 && atomicCAS(&p.hdr->status[0], 0, (int)SDLM_ERR_DEVICE_CHECK) == 0) p.hdr->status[1] = slot;
      return;
    }
    pos += p.seq_len[slot];
  }
  float cs[8], sn[8];
  if (rotated) rope_angles(p, (double)pos, 8 * l, cs, sn);

  for (int g = part; g < groups; g += p.parts) {
    const uint4 a0 = x0, a1 = x1;
    fetch(g + p.parts);
    const int h = g * HPW + lane / TPH;
    const bool is_q = h < p.n_heads;
    float v[16];
    const __nv_bfloat162* e0 = reinterpret_cast<const __nv_bfloat162*>(&a0);
    const __nv_bfloat162* e1 = reinterpret_cast<const __nv_bfloat162*>(&a1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f0 = __bfloat1622float2(e0[i]), f1 = __bfloat1622float2(e1[i]);
      v[2 * i] = f0.x; v[2 * i + 1] = f0.y;
      v[8 + 2 * i] = f1.x; v[8 + 2 * i + 1] = f1.y;
    }
    const __nv_bfloat16* w = is_q ? p.q_weight : p.k_weight;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
    for (int o = TPH / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (w && h < heads) {
      const float inv = rsqrtf(ss / (float)HD + p.eps);
      const uint4 w0 = reinterpret_cast<const uint4*>(w)[c0], w1 = reinterpret_cast<const uint4*>(w)[c1];
      const __nv_bfloat162* g0 = reinterpret_cast<const __nv_bfloat162*>(&w0);
      const __nv_bfloat162* g1 = reinterpret_cast<const __nv_bfloat162*>(&w1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f0 = __bfloat1622float2(g0[i]), f1 = __bfloat1622float2(g1[i]);
        v[2 * i] *= inv * f0.x; v[2 * i + 1] *= inv * f0.y;
        v[8 + 2 * i] *= inv * f1.x; v[8 + 2 * i + 1] *= inv * f1.y;
      }
    }
    if (rotated) {
      if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = v[2 * e], c = v[2 * e + 1];
          v[2 * e] = a * cs[e] - c * sn[e];
          v[2 * e + 1] = c * cs[e] + a * sn[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = v[e], c = v[8 + e];
          v[e] = a * cs[e] - c * sn[e];
          v[8 + e] = c * cs[e] + a * sn[e];
        }
      }
    }
    if (h < heads) {
      uint4 o0, o1;
      uint32_t* u0 = reinterpret_cast<uint32_t*>(&o0);
      uint32_t* u1 = reinterpret_cast<uint32_t*>(&o1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u0[i] = ptx::pack_bf16(v[2 * i], v[2 * i + 1]);
        u1[i] = ptx::pack_bf16(v[8 + 2 * i], v[8 + 2 * i + 1]);
      }
      uint4* dst = reinterpret_cast<uint4*>(is_q ? p.q_out + (row * p.n_heads + h) * HD
                                                 : p.k_out + (row * p.n_heads2 + (h - p.n_heads)) * HD);
      dst[c0] = o0;
      dst[c1] = o1;
    }
  }
}

// Turns per position of every rotated pair, and the factor on cosine and sine, in 64 bits.
static bool rope_frequencies(const sdlm_rope& r, int rot, double* freq, float* mscale) {
  const double two_pi = 6.283185307179586476925286766559;
  double theta = r.theta, m = 1.0;
  const double s = r.factor;
  if (r.scaling == SDLM_ROPE_NTK) theta *= pow(s, rot / (rot - 2.0));
  double lo = 0.0, hi = 0.0;
  if (r.scaling == SDLM_ROPE_YARN) {
    // pairs that turn more than beta_fast times within the trained length keep their frequency, pairs that turn less
    // than beta_slow times have it divided by the factor, those in between are mixed linearly
    lo = floor(rot * log(r.trained_len / (r.beta_fast * two_pi)) / (2.0 * log((double)r.theta)));
    hi = ceil(rot * log(r.trained_len / (r.beta_slow * two_pi)) / (2.0 * log((double)r.theta)));
    lo = lo < 0.0 ? 0.0 : lo;
    hi = hi > rot - 1.0 ? rot - 1.0 : hi;
    if (s > 1.0) m = 0.1 * log(s) + 1.0;
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(theta, -2.0 * i / rot);
    if (r.scaling == SDLM_ROPE_LINEAR) f /= s;
    if (r.scaling == SDLM_ROPE_YARN) {
      double ramp = (i - lo) / (hi > lo ? hi - lo : 0.001);
      ramp = ramp < 0.0 ? 0.0 : ramp > 1.0 ? 1.0 : ramp;
      f = f / s * ramp + f * (1.0 - ramp);
    }
    freq[i] = f / two_pi;
    if (!isfinite(freq[i])) return false;
  }
  *mscale = r.attn_factor > 0.f ? r.attn_factor : (float)m;
  return true;
}

}  // namespace sdlm

using namespace sdlm;

extern "C" sdlm_status sdlm_qk_norm_rope(sdlm_ctx* ctx, int32_t batch, int32_t D, const int32_t* seq_ids,
                                         const int32_t* positions, int32_t relative, const sdlm_rope* rope, float eps,
                                         int32_t n_heads, const void* q, int64_t q_stride, const void* q_weight,
                                         void* q_out, int32_t n_heads2, const void* k, int64_t k_stride,
                                         const void* k_weight, void* k_out, void* stream) {
  if (!ctx || !rope || !q || !q_out || batch < 1 || D < 1 || n_heads < 1 || n_heads2 < 0 || (n_heads2 > 0 && (!k || !k_out)))
    return SDLM_ERR_INVALID_ARG;
  if (n_heads > 65536 || n_heads2 > 65536) return SDLM_ERR_SHAPE;
  const int d = ctx->cfg.head_dim;
  const long long rows = (long long)batch * D;
  if (n_heads2 == 0) {
    k = nullptr; k_out = nullptr; k_weight = nullptr; k_stride = 0;
  }
  if (!aligned16(q) || !aligned16(q_out) || (q_weight && !aligned16(q_weight))) return SDLM_ERR_INVALID_ARG;
  if (k && (!aligned16(k) || !aligned16(k_out) || (k_weight && !aligned16(k_weight)))) return SDLM_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps)) return SDLM_ERR_INVALID_ARG;
  const long long qw = (long long)n_heads * d, kw = (long long)n_heads2 * d;
  // (a stride of 2^40 elements is beyond any memory; the bound keeps the products below in 64 bits)
  if (q_stride < qw || q_stride % 8 || q_stride > (1ll << 40) || (k && (k_stride < kw || k_stride % 8 || k_stride > (1ll << 40))))
    return SDLM_ERR_INVALID_ARG;
  if (!(rope->theta > 1.f) || isinf(rope->theta)) return SDLM_ERR_INVALID_ARG;
  const int rot = rope->rot_dim == 0 ? d : rope->rot_dim;
  if (rot < 2 || rot > d) return SDLM_ERR_INVALID_ARG;
  if (rot % 16) return SDLM_ERR_UNSUPPORTED;  // a lane holds eight whole pairs
  if (rope->interleaved != 0 && rope->interleaved != 1) return SDLM_ERR_INVALID_ARG;
  if (rope->scaling < SDLM_ROPE_PLAIN || rope->scaling > SDLM_ROPE_YARN) return SDLM_ERR_INVALID_ARG;
  if (rope->scaling != SDLM_ROPE_PLAIN && (!(rope->factor > 0.f) || isinf(rope->factor))) return SDLM_ERR_INVALID_ARG;
  if (rope->scaling == SDLM_ROPE_YARN &&
      (rope->trained_len < 1 || !(rope->beta_fast > 0.f) || !(rope->beta_slow > 0.f) || isinf(rope->beta_fast) || isinf(rope->beta_slow)))
    return SDLM_ERR_INVALID_ARG;
  if (!(rope->attn_factor >= 0.f) || isinf(rope->attn_factor)) return SDLM_ERR_INVALID_ARG;
  const bool counted = relative != 0 || !positions;
  if (counted && batch > ctx->cfg.max_batch) return SDLM_ERR_SHAPE;
  if (!same_device(ctx)) return SDLM_ERR_INVALID_ARG;
  // Rows may be rotated in place (out is x, dense rows); any other overlap would have rows read after they are written.
  const size_t qn = ((size_t)(rows - 1) * q_stride + qw) * 2, kn = k ? ((size_t)(rows - 1) * k_stride + kw) * 2 : 0;
  const size_t qo = (size_t)rows * qw * 2, ko = (size_t)rows * kw * 2;
  if (q_out == q ? q_stride != qw : ranges_overlap(q, qn, q_out, qo)) return SDLM_ERR_INVALID_ARG;
  if (k && (k_out == k ? k_stride != kw : ranges_overlap(k, kn, k_out, ko))) return SDLM_ERR_INVALID_ARG;
  if (k && (ranges_overlap(q, qn, k_out, ko) || ranges_overlap(k, kn, q_out, qo) || ranges_overlap(q_out, qo, k_out, ko)))
    return SDLM_ERR_INVALID_ARG;
  const struct { const void* p; size_t bytes; } others[] = {{positions, (size_t)rows * 4}, {counted ? seq_ids : nullptr, (size_t)batch * 4},
                                                           {q_weight, (size_t)d * 2}, {k_weight, (size_t)d * 2}};
  for (const auto& in : others)
    if (in.p && (ranges_overlap(q_out, qo, in.p, in.bytes) || (k && ranges_overlap(k_out, ko, in.p, in.bytes)))) return SDLM_ERR_INVALID_ARG;
  RopeParams p;
  p.q = static_cast<const __nv_bfloat16*>(q); p.k = static_cast<const __nv_bfloat16*>(k);
  p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_out);
  p.q_weight = static_cast<const __nv_bfloat16*>(q_weight); p.k_weight = static_cast<const __nv_bfloat16*>(k_weight);
  p.positions = positions; p.seq_len = counted ? ctx->seq_len : nullptr; p.seq_ids = seq_ids; p.hdr = ctx->hdr;
  p.q_stride = q_stride; p.k_stride = k_stride; p.rows = rows;
  p.D = D; p.max_batch = ctx->cfg.max_batch; p.n_heads = n_heads; p.n_heads2 = n_heads2;
  p.rot = rot; p.interleaved = rope->interleaved; p.eps = eps;
  if (ctx->rope_rot != rot || memcmp(&ctx->rope_of, rope, sizeof(*rope)) != 0) {
    ctx->rope_rot = 0;
    for (double& f : ctx->rope_freq) f = 0.0;
    if (!rope_frequencies(*rope, rot, ctx->rope_freq, &ctx->rope_mscale)) return SDLM_ERR_INVALID_ARG;
    ctx->rope_of = *rope;
    ctx->rope_rot = rot;
  }
  memcpy(p.freq, ctx->rope_freq, sizeof(p.freq));
  p.mscale = ctx->rope_mscale;
  const int hpw = 32 / (d / 16), groups = (n_heads + n_heads2 + hpw - 1) / hpw;
  // few rows: one warp for every group of heads; many: fewer warps a row, which then form the angles less often
  const long long want = (long long)ctx->sm_count * 32;
  long long parts = (want + rows - 1) / rows;
  p.parts = (int)(parts < 1 ? 1 : parts > groups ? groups : parts);
  const long long blocks = (rows * p.parts + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  if (blocks > 0x7fffffffll) return SDLM_ERR_SHAPE;
  const cudaError_t e = d == 128 ? launch_overlapped(qk_norm_rope_kernel<128>, dim3((unsigned)blocks), dim3(kRopeThreads), 0,
                                                     static_cast<cudaStream_t>(stream), p)
                                 : launch_overlapped(qk_norm_rope_kernel<64>, dim3((unsigned)blocks), dim3(kRopeThreads), 0,
                                                     static_cast<cudaStream_t>(stream), p);
  ctx->launches++;
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? SDLM_OK : SDLM_ERR_CUDA;
}
