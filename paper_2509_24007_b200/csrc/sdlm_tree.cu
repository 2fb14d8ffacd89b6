// Attention of a tree of drafted tokens over the paged cache (sdlm_tree_attn): the verification pass of Sec. 3.4 for
// several drafted continuations at once.  Node j of sequence b (a drafted token hanging from node parent[j] < j, or
// from the cached history) attends to the whole history, to the nodes on its path and to itself:
//   out[b,j,h,:] = softmax_t( q[b,j,h,:] . K_t * scale ) V_t,   t over the cached tokens of b, the ancestors of j, j.
//
// The G = Hq/Hkv query heads of a KV head and the tree's nodes are stacked: row node * G + g of (sequence, KV head).
// A task is 256 stacked rows of one (sequence, KV head), two tiles of 128; its keys are the cached tiles (64 tokens
// each) and one tile of the tree's own keys:
//     S = Q K^T      M = 128 rows, N = 64 keys, K = d       A and B from shared memory
//     O += P V       M = 128 rows, N = d,       K = 64      A = P from tensor memory, B = V^T from shared memory
// Few rows are bound by the cache's bytes, many by the products.  Two groups of softmax warps take turns on the tensor
// core, each with an S, two P buffers and an O of its own, so that the next scores are there when a group has written
// its weights: with more than 128 rows they have a tile each and share every key tile, with fewer both have the same
// rows, one takes the even and one the odd key tiles, and they add up at the end.  The key tiles of all tasks form one sequence that is
// cut into equal contiguous ranges, one per thread block (one per SM); the part of a task in one range is a piece.  A
// piece that is not its whole task leaves its sums unnormalised with their reference, and a second kernel joins them
// in the order of their thread blocks, so that results do not depend on timing.
//
// Roles: warps 0 and 3 bring K and V^T tiles into a ring each (they run ahead over piece boundaries; the tree's own tile
// they write themselves, V transposed), warps 1 and 2 issue the MMAs of the first and of the second softmax group,
// warps 4..7 / 8..11 are the first / second group of softmax warps: a thread has one row and its 64 scores in
// registers (no exchange between threads), stages queries and writes rows out.  Only key tiles that are not seen whole
// look at the row's 64-bit visibility word.
//
// Measured in a graph over three sets of inputs at 1965 MHz (16 query and 2 KV heads of 128 where not said otherwise): one
// sequence of 1024, one node: 12.9 us; 32 sequences of 512..4096, 13 nodes (80 MB): 34 us, 2.3 TB/s (30 on one set, which
// stays in L2); 8 of 32768, 32 nodes: 89 us, 3.0 TB/s and 0.77 PFLOP/s; 64 of 512..4096, 64 nodes, 40 and 8 heads: 270 to 284
// us, 2.5 TB/s and 0.55 PFLOP/s.  Called for seconds the last two take 102 and 305 us, at the 1.67 to 1.8 GHz the power cap
// leaves.  Heads of 64 (4 over 2): 32 of 512..4096, 13 nodes 24 us, 64 of 4096, 64 nodes 57 us.  What bounds it is the round of a key tile
// between an issuer and its softmax group (S ready, scores read, weights written, P V issued): about half of the time
// goes into its waits and barriers, with all arithmetic taken out the third case still takes 44 us.
#include "sdlm_internal.h"
#include "sdlm_ptx.cuh"

#include <float.h>
#include <math.h>

namespace sdlm {

constexpr int kTreeThreads = 384;
constexpr int kTreeRows = 256;        // stacked rows of a task
constexpr float kTreeRebase = 8.0f;   // log2 units a score may exceed its row's reference by
// Key tiles' worth of work the schedule charges for a task's queries and output.  2, 4, 8, 12, 24: 32.0, 32.0, 29.7, 29.8,
// 31.8 us for 32 sequences of 512..4096, and 293, 280, 269, 274, 293 us for 64 with 64 nodes.
constexpr int kTreeItemCost = 8;
constexpr int kTreeSmemLimit = 232448;

struct TreeParams {
  const __nv_bfloat16* pool;
  const int32_t* page_table;
  const int32_t* seq_len;
  const int32_t* seq_ids;
  const int32_t* n_nodes;   // or null: n for every sequence
  const int32_t* parent;
  const __nv_bfloat16* q;
  const __nv_bfloat16* k_tree;
  const __nv_bfloat16* v_tree;
  __nv_bfloat16* out;
  DevHeader* hdr;
  float* part_o;            // [2 * thread blocks][256][d] unnormalised sums
  float2* part_ml;          // [2 * thread blocks][256] reference (log2 units), sum
  TreeCut* cuts;            // [thread blocks] the task that a thread block's range begins in
  float scale_log2;
  uint32_t inv_G;           // 2^32 / G rounded up: R / G = R * inv_G >> 32 for the R < 64 G there are; 0 for G = 1
  int batch, n, Hq, Hkv, G, mpps, num_pages, max_batch, n_k, n_v, q_tiles;
};

// Node of stacked row R (see inv_G).
__device__ __forceinline__ int tree_node(const TreeParams& p, int R) { return p.inv_G ? (int)__umulhi((uint32_t)R, p.inv_G) : R; }

// Largest of a thread's 64 scores (four chains), NaN left out; with EDGE only over the keys whose bit is set.
template <bool EDGE>
__device__ __forceinline__ float tree_row_max(const uint32_t (&x)[64], uint32_t lo, uint32_t hi) {
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 64; i += 2) {
    float a = __uint_as_float(x[i]), b = __uint_as_float(x[i + 1]);
    if (EDGE) {
      const uint32_t bits = i < 32 ? lo : hi;
      if (!(bits >> (i & 31) & 1u)) a = -INFINITY;
      if (!(bits >> ((i + 1) & 31) & 1u)) b = -INFINITY;
    }
    mx[(i >> 1) & 3] = ptx::max3(mx[(i >> 1) & 3], a, b);
  }
  return fmaxf(ptx::max3(mx[0], mx[1], mx[2]), mx[3]);
}
// A thread's 64 weights 2^(x * scale + neg_ref) as bf16 pairs into 32 tensor-memory columns at taddr; returns their sum
// before rounding.  Rounding the weights to bf16 is what the matrix product takes: 2^-8 of each weight at most, of either
// sign.  (Summing the rounded ones instead costs two instructions more a weight on the pipe that is busiest here, and
// moves the result's error by less than its own rounding.)  Two pairs of every eight take the power of two from the
// cubic, the others from the special-function unit.
template <bool EDGE>
__device__ __forceinline__ float tree_weights(const uint32_t (&x)[64], uint32_t taddr, float scale, float neg_ref, uint32_t lo, uint32_t hi) {
  const float2 scale2 = make_float2(scale, scale), neg_ref2 = make_float2(neg_ref, neg_ref);
  float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t packed[16];
    const uint32_t bits = c ? hi : lo;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float2 t = ptx::fma2_f2(make_float2(__uint_as_float(x[c * 32 + i]), __uint_as_float(x[c * 32 + i + 1])), scale2, neg_ref2);
      float2 w;
      if (((i >> 1) & 3) == 1) {
        w = ptx::exp2_poly2<true>(t);
      } else {
        w.x = ptx::ex2(t.x);
        w.y = ptx::ex2(t.y);
      }
      if (EDGE) {
        if (!(bits >> i & 1u)) w.x = 0.f;
        if (!(bits >> (i + 1) & 1u)) w.y = 0.f;
      }
      sum[(i >> 1) & 1] = ptx::add2_f2(sum[(i >> 1) & 1], w);
      packed[i >> 1] = ptx::pack_bf16(w.x, w.y);
    }
    ptx::tmem_st16(taddr + c * 16, packed);
  }
  const float2 s = ptx::add2_f2(sum[0], sum[1]);
  return s.x + s.y;
}

__device__ __forceinline__ void tree_status(const TreeParams& p, int code, int slot, int detail) {
  if (atomicCAS(&p.hdr->status[0], 0, code) == 0) {
    p.hdr->status[1] = slot;
    p.hdr->status[2] = detail;
  }
}

// Values of the tree's nodes that are not finite: a weight of zero times one is NaN in the product, which covers all nodes
// for all rows.  They are zero in the tile, and are added to the rows that see their node once those are written (a weight
// above zero times an infinity or NaN is one).
__device__ __forceinline__ uint32_t tree_largest(uint32_t most, const uint4& v) {  // of |bf16| pairs, NaN above all
  __nv_bfloat162 m = *reinterpret_cast<__nv_bfloat162*>(&most);
  const __nv_bfloat162* b = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __hmax2_nan(m, __habs2(b[i]));
  return *reinterpret_cast<uint32_t*>(&m);
}
__device__ __forceinline__ bool tree_spoiled(uint32_t pair) {  // one of two bf16 is not finite
  return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}
// Puts zero in their place in the V^T tile that a warp has written (whole warps); the nodes that have any.
template <int HD>
__device__ __noinline__ uint64_t tree_clean(uint8_t* tile, const __nv_bfloat16* v, size_t stride, int nodes) {
  const int lane = threadIdx.x & 31;
  uint32_t lo = 0, hi = 0;
  __syncwarp();
  for (int i = lane; i < nodes * HD; i += 32) {
    const int key = i / HD, col = i % HD;
    if (isfinite(__bfloat162float(v[key * stride + col]))) continue;
    *reinterpret_cast<uint16_t*>(tile + col * 128 + (((key >> 3) ^ (col & 7)) << 4) + (key & 7) * 2) = 0;
    if (key < 32) lo |= 1u << key; else hi |= 1u << (key - 32);
  }
  __syncwarp();
  lo = __reduce_or_sync(0xffffffffu, lo);
  hi = __reduce_or_sync(0xffffffffu, hi);
  return (uint64_t)hi << 32 | lo;
}
template <typename T>  // columns [first, last) of a row written by this thread; v: the sequence's values of its KV head
__device__ __noinline__ void tree_add_spoiled(T* row, int first, int last, const __nv_bfloat16* v, size_t stride, const int32_t* parent,
                                              int node, uint64_t spoiled) {
  for (int i = node; i >= 0;) {
    if (spoiled >> i & 1u)
      for (int c = first; c < last; ++c) {
        const float x = __bfloat162float(v[i * stride + c]);
        if (!isfinite(x)) row[c] = (T)((float)row[c] + x);
      }
    const int up = parent[i];
    i = up < i ? up : -1;
  }
}

// ---- the schedule -----------------------------------------------------------------------------------------
// Sequence b has Hkv * ceil(G * nodes / 256) tasks of (item cost + key tiles) positions each; a slot number outside the
// tables, or a sequence without nodes, has none.  Thread block c has the positions [c * span, (c + 1) * span).
struct TreeSeq {
  int slot, len, nodes, rts, tiles;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b) {
  TreeSeq s;
  s.slot = p.seq_ids ? p.seq_ids[b] : b;
  s.nodes = p.n_nodes ? min(max(p.n_nodes[b], 0), p.n) : p.n;
  if (s.slot < 0 || s.slot >= p.max_batch) s.nodes = 0;
  s.len = s.nodes > 0 ? max(0, min(p.seq_len[s.slot], p.mpps * kPageSize)) : 0;
  s.rts = (p.G * s.nodes + kTreeRows - 1) / kTreeRows;
  s.tiles = (s.len + kPageSize - 1) / kPageSize + 1;  // cached tiles and the tree's
  return s;
}
__device__ __forceinline__ int tree_positions(const TreeParams& p, const TreeSeq& s) {
  return p.Hkv * s.rts * (kTreeItemCost + s.tiles);
}
struct TreePiece {
  TreeSeq s;
  int b, hk, rt, t0, t1;  // key tiles [t0, t1) of 256 rows of a KV head
  int slot_i;  // 0: the piece of the task that holds the range's first position, 1: a later one
};
// Walks the pieces of a thread block's positions, counted from its first one; every role keeps a walk of its own.
struct TreeWalk {
  int cur, b, base;  // base: first position of sequence b (negative where it lies in an earlier range)
};
__device__ __forceinline__ bool tree_next(const TreeParams& p, TreeWalk& w, int n_pos, TreePiece& t) {
  while (w.cur < n_pos) {
    t.s = tree_seq(p, w.b);
    const int per = kTreeItemCost + t.s.tiles, tasks = p.Hkv * t.s.rts;
    if (w.cur >= w.base + per * tasks) {  // positions are left, so a later sequence has them
      w.base += per * tasks;
      ++w.b;
      continue;
    }
    const int ti = (w.cur - w.base) / per, start = w.base + ti * per;
    const int in0 = w.cur - start, in1 = min(n_pos - start, per);
    w.cur = start + in1;
    t.t0 = max(0, in0 - kTreeItemCost);
    t.t1 = max(0, in1 - kTreeItemCost);
    if (t.t1 <= t.t0) continue;  // only positions that stand for a task's start
    t.b = w.b;
    t.hk = ti / t.s.rts;
    t.rt = ti - t.hk * t.s.rts;
    t.slot_i = start <= 0 ? 0 : 1;
    return true;
  }
  return false;
}

// What a thread block's roles start from: its first piece, the walk behind it, its number of positions.
struct TreeStart {
  TreePiece t;
  TreeWalk w;
  int n_pos, have;
};
template <int HD>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_attn_kernel(const TreeParams p) {
  constexpr int KH = HD / 64;                    // 64-wide panels of K and of Q
  constexpr int CH = HD / 8;                     // 16-byte chunks of a row
  constexpr int K_PANEL_B = kPageSize * 128;     // 64 keys x 64 dims
  constexpr int TILE_B = HD * 128;               // K (d/64 panels) or V^T (d rows of 64 keys) of a key tile
  constexpr int Q_PANEL_B = 128 * 128;           // 128 rows x 64 dims
  constexpr int Q_B = KH * Q_PANEL_B;            // one tile's queries
  // tensor memory: S of softmax group X at columns X*128 .. + 63, its P buffers (two bf16 a column) at X*128 + 64 + 32b, O at
  // 256 + X*128
  constexpr uint32_t O_COL = 256, TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_s = smem;                 // [q_tiles][Q_B]
  uint8_t* k_ring = q_s + (size_t)p.q_tiles * Q_B;
  const int NK = p.n_k, NV = p.n_v;
  uint8_t* v_ring = k_ring + (size_t)NK * TILE_B;
  uint64_t* full_k = reinterpret_cast<uint64_t*>(v_ring + (size_t)NV * TILE_B);
  uint64_t* k_free = full_k + NK;
  uint64_t* full_v = k_free + NK;
  uint64_t* v_free = full_v + NV;
  uint64_t* s_full = v_free + NV;      // [X]
  uint64_t* s_free = s_full + 2;       // [X]: scores in registers
  uint64_t* p_full = s_free + 2;       // [X][buffer]: weights written
  uint64_t* pv_done = p_full + 4;      // [X][buffer]: O += P V of its item, and of those before, complete
  uint64_t* q_full = pv_done + 4;      // queries staged, the piece before read out of tensor memory, both issuers there
  uint64_t* l_bar = q_full + 1;        // both groups have left their rows' references and sums in tensor memory
  uint64_t* drain = l_bar + 1;
  uint64_t* spoiled = drain + 2;       // [16] by piece: nodes with values that are not finite
  TreeStart* start = reinterpret_cast<TreeStart*>(spoiled + 16);
  int* warp_sum = reinterpret_cast<int*>(start + 1);  // [12]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(warp_sum + 12);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 32) {
    for (int s = 0; s < NK; ++s) {
      ptx::mbar_init(&full_k[s], 1);  // the copying warp
      ptx::mbar_init(&k_free[s], 2);  // both issuers
    }
    for (int s = 0; s < NV; ++s) {
      ptx::mbar_init(&full_v[s], 1);
      ptx::mbar_init(&v_free[s], 2);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(&s_full[s], 1);
      ptx::mbar_init(&s_free[s], 4);
    }
    for (int s = 0; s < 4; ++s) {
      ptx::mbar_init(&p_full[s], 4);  // one arrival per softmax warp of the group
      ptx::mbar_init(&pv_done[s], 1);
    }
    ptx::mbar_init(q_full, 10);  // softmax warps and issuers
    ptx::mbar_init(l_bar, 8);
    ptx::mbar_init(&drain[0], 1);
    ptx::mbar_init(&drain[1], 1);
    *abort = 0;
    ptx::fence_barrier_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, TMEM_COLS);
    ptx::tmem_relinquish();
  }
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();  // queries, tree and cache may come from the kernels before this one

  // ---- this thread block's range of positions
  const int per_thread = (p.batch + kTreeThreads - 1) / kTreeThreads;
  int mine = 0;
  for (int i = 0; i < per_thread; ++i) {
    const int b = tid * per_thread + i;
    if (b >= p.batch) break;
    const TreeSeq s = tree_seq(p, b);
    if (blockIdx.x == 0 && (s.slot < 0 || s.slot >= p.max_batch)) tree_status(p, SDLM_ERR_DEVICE_CHECK, s.slot, b);
    mine += tree_positions(p, s);
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) warp_sum[warp] = upto;
  ptx::tc_fence_before();
  __syncthreads();  // barriers initialised, tensor memory allocated, sums of the warps written
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  int total = 0;
  upto -= mine;
#pragma unroll
  for (int i = 0; i < kTreeThreads / 32; ++i) {
    if (i < warp) upto += warp_sum[i];
    total += warp_sum[i];
  }
  const int span = total > 0 ? (int)(((uint32_t)total + gridDim.x - 1) / gridDim.x) : 1;
  const long long lo64 = (long long)blockIdx.x * span;
  const int lo = lo64 < total ? (int)lo64 : total;
  if (mine > 0 && upto <= lo && lo < upto + mine) {  // the thread whose sequences hold the first position
    for (int b = tid * per_thread;; ++b) {
      const TreeSeq s = tree_seq(p, b);
      const int n = tree_positions(p, s);
      if (lo < upto + n) {
        const int per = kTreeItemCost + s.tiles, ti = (lo - upto) / per, hk = ti / s.rts;
        p.cuts[blockIdx.x] = TreeCut{upto + ti * per, span, total, b, hk, ti - hk * s.rts, s.tiles, s.nodes};
        TreeStart st;
        st.n_pos = min(total - lo, span);
        st.w = TreeWalk{0, b, upto - lo};
        st.have = tree_next(p, st.w, st.n_pos, st.t) ? 1 : 0;
        *start = st;
        break;
      }
      upto += n;
    }
  }
  if (tid == 0 && lo >= total) {
    p.cuts[blockIdx.x].span = 0;
    start->have = 0;
  }
  __syncthreads();
  const int n_pos = start->n_pos;  // (not looked at without a first piece)
  TreeWalk walk = start->w;
  TreePiece t = start->t;
  bool have = start->have != 0;

  if (warp < 4) {
    if (warp == 0 || warp == 3) {
      // ---------------------------------------------------------------- key tiles: K (warp 0), V^T (warp 3)
      // Cached tiles by bulk copies, NK (NV) tiles ahead of the issuers and over piece boundaries; the tree's own tile by the
      // warp itself.  (Asking for tiles further ahead into L2 as well made long contexts 14 % slower.)
      const bool v_part = warp == 3;
      const int ring = v_part ? NV : NK;
      uint8_t* dst = v_part ? v_ring : k_ring;
      uint64_t* full = v_part ? full_v : full_k;
      uint64_t* freed = v_part ? v_free : k_free;
      bool ok = true;
      int slot = 0, used = 0;
      uint32_t ph = 1, n_piece = 0;  // phase of the slot's use before
      if (have) asm volatile("bar.sync 1, 320;" ::: "memory");  // the softmax warps have asked for their first queries
      for (; ok && have; have = tree_next(p, walk, n_pos, t), ++n_piece) {
        const int cached = t.s.tiles - 1, end = min(t.t1, cached);
        const int32_t* pages = p.page_table + (size_t)t.s.slot * p.mpps;
        const size_t head_off = (size_t)t.hk * 2 * kv_tile_elems(HD);
        int page_w = 0, page_next = t.t0 + lane < end ? pages[t.t0 + lane] : 0;  // page numbers, 32 tiles at a time, and the next 32
        for (int tl = t.t0; tl < t.t1; ++tl) {
          if (used >= ring) ok = ptx::mbar_wait_warp(&freed[slot], ph, abort);
          if (!ok) break;
          uint8_t* tile = dst + (size_t)slot * TILE_B;
          const int at = (tl - t.t0) & 31;
          if (at == 0) {
            page_w = page_next;
            page_next = tl + 32 + lane < end ? pages[tl + 32 + lane] : 0;
          }
          if (tl < cached) {
            int page = __shfl_sync(0xffffffffu, page_w, at);
            if (ptx::elect_one()) {
              if (page < 0 || page >= p.num_pages) {  // never follow a bad table entry out of the pool
                tree_status(p, SDLM_ERR_DEVICE_CHECK, t.s.slot, page);
                page = 0;
              }
              const size_t page_elems = (size_t)p.Hkv * 2 * kv_tile_elems(HD);
              ptx::mbar_arrive_expect_tx(&full[slot], TILE_B);
              ptx::bulk_g2s(tile, p.pool + page * page_elems + head_off + (v_part ? kv_tile_elems(HD) : 0), TILE_B, &full[slot]);
            }
          } else {
            const __nv_bfloat16* src = (v_part ? p.v_tree : p.k_tree) + ((size_t)t.b * p.n * p.Hkv + t.hk) * HD;
            const size_t stride = (size_t)p.Hkv * HD;
            if (!v_part) {  // keys: row by row, swizzled; rows behind the last node are zero
#pragma unroll 4
              for (int i = 0; i < 2 * CH; ++i) {
                const int idx = lane + i * 32, key = idx / CH, c = idx % CH;
                ptx::cp_async16(ptx::smem_u32(tile + (c >> 3) * K_PANEL_B + key * 128 + (((c & 7) ^ (key & 7)) << 4)),
                                src + min(key, t.s.nodes - 1) * stride + c * 8, key < t.s.nodes ? 16u : 0u);
              }
              ptx::cp_async_commit();
              ptx::cp_async_wait<0>();
            } else {  // values: blocks of eight keys by eight columns, transposed in registers
              uint32_t most = 0;
#pragma unroll 2
              for (int i = 0; i < CH / 4; ++i) {
                const int blk = lane + i * 32, kb = blk / CH, c = blk % CH;
                uint4 v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  v[e] = make_uint4(0, 0, 0, 0);
                  if (kb * 8 + e < t.s.nodes) v[e] = *(reinterpret_cast<const uint4*>(src + (kb * 8 + e) * stride) + c);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) most = tree_largest(most, v[e]);
#pragma unroll
                for (int col = 0; col < 8; ++col) {
                  uint32_t o[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const uint32_t a = reinterpret_cast<const uint32_t*>(&v[2 * e])[col >> 1];
                    const uint32_t c2 = reinterpret_cast<const uint32_t*>(&v[2 * e + 1])[col >> 1];
                    o[e] = __byte_perm(a, c2, col & 1 ? 0x7632 : 0x5410);
                  }
                  *reinterpret_cast<uint4*>(tile + (c * 8 + col) * 128 + ((kb ^ col) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                }
              }
              // Read once the products of this tile are complete.  The ring lets this warp run at most 8 pieces ahead of the
              // issuers, which stay in a piece until all its rows are written.
              uint64_t bad = 0;
              if (__any_sync(0xffffffffu, tree_spoiled(most))) bad = tree_clean<HD>(tile, src, stride, t.s.nodes);
              if (lane == 0) spoiled[n_piece & 15u] = bad;
            }
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&full[slot]);
          }
          __syncwarp();
          ++used;
          if (++slot == ring) { slot = 0; ph ^= 1u; }
        }
      }
      if (lane == 0 && (!ok || *abort)) {  // winding down: let the copies already issued land
        tree_status(p, SDLM_ERR_TIMEOUT, -2, v_part ? 14 : 11);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------- MMA issuer of softmax group X
      // Items of a group are the key tiles it takes; in order of issue: S of the first, then S of item i + 1, as soon as the
      // group has the scores of item i in registers, and O += P V of item i.  Each group has an issuer of its own: an MMA
      // occupies its issuer for about as long as it runs, and with one issuer for both each group's waits are the other's
      // too.  An issuer also passes over the tiles that only the other group takes, so that every ring slot is given back
      // by both.  The whole warp runs the loop and the waits, one elected lane issues (see ptx::elect_one); ring slots and
      // phases are counted up, not divided out.
      const int X = warp - 1;
      const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((64u >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(HD >> 3) << 17) | ((128u >> 4) << 24);
      const uint64_t d_q = ptx::umma_smem_desc(ptx::smem_u32(q_s)), d_kr = ptx::umma_smem_desc(ptx::smem_u32(k_ring)),
                     d_vr = ptx::umma_smem_desc(ptx::smem_u32(v_ring));
      const uint32_t d_s = tmem_base + X * 128, d_o = tmem_base + O_COL + X * 128;
      bool ok = true;
      int slot_k = 0, slot_v = 0;
      uint32_t ph_k = 0, ph_v = 0, pc = 0, n_s = 0, n_pv = 0;  // ring phases, pieces, items so far
      for (; ok && have; have = tree_next(p, walk, n_pos, t)) {
        const bool two = p.G * t.s.nodes - t.rt * kTreeRows > 128;
        const int n_tiles = t.t1 - t.t0, step = two ? 1 : 2, first = two ? 0 : X;
        const uint64_t d_a = d_q + (uint64_t)((two && X ? Q_B : 0) >> 4);
        // (an issuer arrives too: where its group has no key tile the piece ends without it, and q_full must not be a phase
        // further when it comes to look)
        if (lane == 0) ptx::mbar_arrive(q_full);
        ok = ptx::mbar_wait_warp(q_full, pc & 1u, abort);
        ++pc;
        int at_k = 0, at_v = 0;  // tiles of the piece passed so far
        // passes over tiles up to `upto`; false when a wait ran out
        auto skip = [&](int& at, int upto, int& slot, uint32_t& ph, int ring, uint64_t* full, uint64_t* freed) {
          for (; at < upto; ++at) {
            if (!ptx::mbar_wait_warp(&full[slot], ph, abort)) return false;
            if (lane == 0) ptx::mbar_arrive(&freed[slot]);
            if (++slot == ring) { slot = 0; ph ^= 1u; }
          }
          return true;
        };
        auto issue_s = [&](int tile) {
          if (!skip(at_k, tile, slot_k, ph_k, NK, full_k, k_free)) return false;
          if (!ptx::mbar_wait2_warp(&full_k[slot_k], ph_k, n_s ? &s_free[X] : nullptr, (n_s - 1) & 1u, abort)) return false;
          ptx::tc_fence_after();
          const uint64_t d_k = d_kr + (uint64_t)((slot_k * TILE_B) >> 4);
          if (ptx::elect_one()) {
#pragma unroll
            for (int kh = 0; kh < KH; ++kh)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                ptx::umma_bf16_ss(d_s, d_a + (uint64_t)((kh * Q_PANEL_B + k * 32) >> 4), d_k + (uint64_t)((kh * K_PANEL_B + k * 32) >> 4),
                                  idesc_s, (kh | k) ? 1u : 0u);
            ptx::umma_commit(&s_full[X]);
            ptx::umma_commit(&k_free[slot_k]);
          }
          __syncwarp();
          ++n_s;
          ++at_k;
          if (++slot_k == NK) { slot_k = 0; ph_k ^= 1u; }
          return true;
        };
        if (first < n_tiles) ok = ok && issue_s(first);
        for (int tile = first; tile < n_tiles && ok; tile += step) {
          if (tile + step < n_tiles && !issue_s(tile + step)) { ok = false; break; }
          if (!skip(at_v, tile, slot_v, ph_v, NV, full_v, v_free)) { ok = false; break; }
          const uint32_t buf = n_pv & 1u;
          if (!ptx::mbar_wait2_warp(&full_v[slot_v], ph_v, &p_full[X * 2 + buf], (n_pv >> 1) & 1u, abort)) { ok = false; break; }
          ptx::tc_fence_after();
          const uint64_t d_v = d_vr + (uint64_t)((slot_v * TILE_B) >> 4);
          const uint32_t d_p = d_s + 64 + buf * 32;
          if (ptx::elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              ptx::umma_bf16_ts(d_o, d_p + k * 8, d_v + (uint64_t)((k * 32) >> 4), idesc_o, (tile > first || k) ? 1u : 0u);
            ptx::umma_commit(&pv_done[X * 2 + buf]);
            ptx::umma_commit(&v_free[slot_v]);
          }
          __syncwarp();
          ++n_pv;
          ++at_v;
          if (++slot_v == NV) { slot_v = 0; ph_v ^= 1u; }
        }
        ok = ok && skip(at_k, n_tiles, slot_k, ph_k, NK, full_k, k_free) && skip(at_v, n_tiles, slot_v, ph_v, NV, full_v, v_free);
      }
      if (!ok && lane == 0) {  // winding down: the MMAs already issued must finish before TMEM and smem are released
        tree_status(p, SDLM_ERR_TIMEOUT, -2, 12);
        ptx::umma_commit(&drain[X]);
        ptx::mbar_wait_brief(&drain[X], 0);
      }
      __syncwarp();
    }
  } else {
    // ---------------------------------------------------------------- queries, softmax and output
    // Thread = row of its group's tile: all keys of a group, all columns of O (half of them where both groups have
    // the same rows).
    const int X = (warp - 4) >> 2, qd = warp & 3, row = qd * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(qd * 32) << 16);
    const uint32_t s_addr = lane_addr + (uint32_t)X * 128, o_addr = lane_addr + O_COL + (uint32_t)X * 128;
    uint32_t cnt = 0, pc = 0, n_piece = 0;  // items of the group so far, pieces of one tile so far, pieces
    bool ok = true, opening = true, two = false;
    for (; ok && have; have = tree_next(p, walk, n_pos, t), ++n_piece) {
      const int rows_all = min(kTreeRows, p.G * t.s.nodes - t.rt * kTreeRows);
      const bool was_two = two;
      two = rows_all > 128;
      const int row0 = t.rt * kTreeRows + (two ? X * 128 : 0), rows = min(128, p.G * t.s.nodes - row0);
      {
        // Queries into shared memory, swizzled as an MMA operand; rows beyond the end are zero.  Each group stages its
        // tile, or half of the only one.  Behind a piece with two tiles the first group stages all of the only one: nothing
        // has joined the groups there, and products of the first, which it has waited for itself, may still read tile 0 when
        // the second is done.  (A piece with one tile joins them below.)
        const bool halves = !two && !was_two;
        const int st = tid - 128 - X * 128, q_first = halves ? X * (128 * CH / 2) : 0, q_n = halves ? CH / 2 : two || X == 0 ? CH : 0;
        const uint32_t qd_s = ptx::smem_u32(q_s + (two ? X * Q_B : 0));
#pragma unroll 2
        for (int i = 0; i < q_n; ++i) {
          const int idx = q_first + st + i * 128, r = idx / CH, c = idx % CH;
          const int R = row0 + min(r, rows - 1), node = tree_node(p, R), g = R - node * p.G;
          ptx::cp_async16(qd_s + (c >> 3) * Q_PANEL_B + r * 128 + (((c & 7) ^ (r & 7)) << 4),
                          p.q + (((size_t)t.b * p.n + node) * p.Hq + (size_t)t.hk * p.G + g) * HD + c * 8, r < rows ? 16u : 0u);
        }
        ptx::cp_async_commit();
        if (opening) {  // the cached tiles are asked for behind the queries, which would else wait for a whole ring of them
          asm volatile("bar.arrive 1, 320;" ::: "memory");
          opening = false;
        }
        ptx::cp_async_wait<0>();
        ptx::fence_proxy_async();
        ptx::tc_fence_before();  // this thread's reads of the piece before are done
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(q_full);
      }
      const int my_node = tree_node(p, row0 + row);
      uint32_t vis_lo = 0, vis_hi = 0;  // the nodes this row sees, where the piece has the tree's keys
      if (t.t1 == t.s.tiles && row < rows) {
        for (int i = my_node; i >= 0;) {
          if (i < 32) vis_lo |= 1u << i; else vis_hi |= 1u << (i - 32);
          const int up = p.parent[(size_t)t.b * p.n + i];
          i = up < i ? up : -1;  // a parent that is not an earlier node: the node hangs from the history
        }
      }
      const int cached = t.s.tiles - 1, whole = t.s.len / kPageSize;
      const int step = two ? 1 : 2, first = t.t0 + (two ? 0 : X), end = t.t1;
      float m_ref = -INFINITY, l = 0.f;
      for (int tl = first; tl < end; tl += step) {
        const uint32_t buf = cnt & 1u;
        // the scores, and the P buffer of the item before the last one (whose weights the product has long read)
        if (!ptx::mbar_wait2_warp(&s_full[X], cnt & 1u, cnt >= 2 ? &pv_done[X * 2 + buf] : nullptr, ((cnt >> 1) - 1) & 1u, abort)) { ok = false; break; }
        if (qd * 32 >= rows) {  // a warp of rows beyond the end: its lanes of P and O are nobody's
          if (lane == 0) {
            ptx::mbar_arrive(&s_free[X]);
            ptx::mbar_arrive(&p_full[X * 2 + buf]);
          }
          ++cnt;
          continue;
        }
        ptx::tc_fence_after();
        uint32_t x[64];
        ptx::tmem_ld64(s_addr, x);
        ptx::tmem_ld_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&s_free[X]);
        const bool edge = tl >= whole;  // some key of this tile is not seen by every row
        uint32_t lo = vis_lo, hi = vis_hi;
        if (edge && tl < cached) {  // the history ends inside this tile
          const int in_last = t.s.len - whole * kPageSize;
          lo = in_last >= 32 ? 0xffffffffu : (1u << in_last) - 1u;
          hi = in_last > 32 ? (1u << (in_last - 32)) - 1u : 0u;
        }
        const float mx = (edge ? tree_row_max<true>(x, lo, hi) : tree_row_max<false>(x, 0, 0)) * p.scale_log2;  // the scale is positive
        const bool move = mx > m_ref + kTreeRebase || (m_ref == -INFINITY && mx > -INFINITY);
        if (__any_sync(0xffffffffu, move)) {
          float alpha = 1.0f;
          if (move) {
            alpha = m_ref == -INFINITY ? 0.f : ptx::ex2(m_ref - mx);
            m_ref = mx;
            l *= alpha;
          }
          if (tl > first) {  // O holds sums relative to the old references: they follow once the item before is in them
            if (!ptx::mbar_wait_warp(&pv_done[X * 2 + (buf ^ 1)], ((cnt - 1) >> 1) & 1u, abort)) { ok = false; break; }
            ptx::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < HD / 16; ++c) {
              uint32_t o[16];
              ptx::tmem_ld16(o_addr + c * 16, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              ptx::tmem_st16(o_addr + c * 16, o);
            }
          }
        }
        // weights 2^(s * scale - reference), rounded to bf16, two per column, into this item's buffer.
        // A key the row does not see gets weight zero.
        const float neg_ref = m_ref == -INFINITY ? 0.f : -m_ref;
        const uint32_t p_addr = s_addr + 64 + buf * 32;
        l += edge ? tree_weights<true>(x, p_addr, p.scale_log2, neg_ref, lo, hi) : tree_weights<false>(x, p_addr, p.scale_log2, neg_ref, 0, 0);
        if (mx == INFINITY) l = NAN;  // (the cubic would give the quotient of two infinities a weight)
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[X * 2 + buf]);
        ++cnt;
      }
      // (the second group has nothing where a piece of one tile is a single key tile)
      if (ok && first < end) ok = ptx::mbar_wait_warp(&pv_done[X * 2 + ((cnt - 1) & 1u)], ((cnt - 1) >> 1) & 1u, abort);
      float a_mine = 1.0f, a_other = 0.f;
      if (ok && !two) {
        // the row's two results meet: references and sums through the S columns, which are free now
        ptx::tc_fence_after();
        ptx::tmem_st1(s_addr, __float_as_uint(m_ref));
        ptx::tmem_st1(s_addr + 1, __float_as_uint(l));
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(l_bar);
        if (!ptx::mbar_wait_warp(l_bar, pc & 1u, abort)) ok = false;
        ++pc;
        if (ok) {
          ptx::tc_fence_after();
          uint32_t om, ol;
          ptx::tmem_ld1(lane_addr + (uint32_t)(X ^ 1) * 128, om);
          ptx::tmem_ld1(lane_addr + (uint32_t)(X ^ 1) * 128 + 1, ol);
          ptx::tmem_ld_wait();
          const float m2 = __uint_as_float(om), m_all = fmaxf(m_ref, m2);
          a_mine = m_ref == -INFINITY ? 0.f : ptx::ex2(m_ref - m_all);
          a_other = m2 == -INFINITY ? 0.f : ptx::ex2(m2 - m_all);
          l = l * a_mine + __uint_as_float(ol) * a_other;
          m_ref = m_all;
        }
      }
      if (ok && qd * 32 < rows) {
        ptx::tc_fence_after();
        const bool all = t.t0 == 0 && t.t1 == t.s.tiles;
        const float inv = all ? 1.0f / l : 1.0f;
        a_mine *= inv;
        a_other *= inv;
        const int c_first = two ? 0 : X * (HD / 32), c_last = two ? HD / 16 : c_first + HD / 32;
        const bool have_1 = end > t.t0 + 1;  // the second group has had a key tile
        const float a_0 = X == 0 || two ? a_mine : a_other, a_1 = X == 0 ? a_other : a_mine;
        const uint32_t o_0 = two ? o_addr : lane_addr + O_COL;
        const int g = row0 + row - my_node * p.G;
        __nv_bfloat16* out_row = p.out + (((size_t)t.b * p.n + my_node) * p.Hq + (size_t)t.hk * p.G + g) * HD;
        const size_t part_row = (size_t)(2 * blockIdx.x + t.slot_i) * kTreeRows + (two ? X * 128 : 0) + row;
        float4* part = reinterpret_cast<float4*>(p.part_o + part_row * HD);
        if (!all && row < rows && (two || X == 0)) p.part_ml[part_row] = make_float2(m_ref, l);
#pragma unroll 2
        for (int c = c_first; c < c_last; ++c) {
          uint32_t o[16], o2[16];
          ptx::tmem_ld16(o_0 + c * 16, o);
          if (!two && have_1) ptx::tmem_ld16(lane_addr + O_COL + 128 + c * 16, o2);
          ptx::tmem_ld_wait();
          float f[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            f[i] = __uint_as_float(o[i]) * a_0;
            if (!two && have_1) f[i] = fmaf(__uint_as_float(o2[i]), a_1, f[i]);
          }
          if (row < rows) {
            if (all) {
              uint32_t w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) w[i] = ptx::pack_bf16(f[2 * i], f[2 * i + 1]);
              reinterpret_cast<uint4*>(out_row + c * 16)[0] = make_uint4(w[0], w[1], w[2], w[3]);
              reinterpret_cast<uint4*>(out_row + c * 16)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) part[c * 4 + i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
          }
        }
        if (t.t1 == t.s.tiles && row < rows && spoiled[n_piece & 15u]) {
          const size_t stride = (size_t)p.Hkv * HD;
          const __nv_bfloat16* v = p.v_tree + ((size_t)t.b * p.n * p.Hkv + t.hk) * HD;
          const int32_t* parent = p.parent + (size_t)t.b * p.n;
          if (all) tree_add_spoiled(out_row, c_first * 16, c_last * 16, v, stride, parent, my_node, spoiled[n_piece & 15u]);
          else tree_add_spoiled(reinterpret_cast<float*>(part), c_first * 16, c_last * 16, v, stride, parent, my_node, spoiled[n_piece & 15u]);
        }
      }
    }
    if (!ok && lane == 0) tree_status(p, SDLM_ERR_TIMEOUT, -2, 13);
    ptx::tc_fence_before();
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

// Joins the pieces of every task that range boundaries cut.  Boundary c = blockIdx.x + 1 is where the range of thread
// block c begins; the boundaries inside a task share its rows, and blockIdx.y and the warps share a boundary's, a warp
// a row at a time:  O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i, M the largest m_i, in the order of the pieces.
// It adds 4 to 9 us to a call, most of which is its launch behind the last thread block and three dependent reads
// (cut, references, rows); 4, 8 and 16 thread blocks a boundary measured within 2 %.
constexpr int kTreeMergeY = 8, kTreeMergeThreads = 256;
template <int HD>
__global__ void __launch_bounds__(kTreeMergeThreads) tree_merge_kernel(const TreeParams p) {
  constexpr int V = HD / 32;                           // values of a row per lane
  constexpr int KL = (kAttnMaxCtas + 31) / 32;         // pieces of a row per lane, at most
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  const int c = blockIdx.x + 1;
  const TreeCut cut = p.cuts[c];
  if (cut.span == 0 || cut.start >= c * (long long)cut.span) return;  // the task begins here: not cut
  const int per = kTreeItemCost + cut.tiles, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = cut.start / cut.span, last = (cut.start + per - 1) / cut.span;  // thread blocks with parts of the task
  const int rows = min(kTreeRows, p.G * cut.nodes - cut.rt * kTreeRows), cuts = last - first, at = c - first - 1;
  const int r_lo = rows * at / cuts, r_hi = rows * (at + 1) / cuts;
  // lane's pieces: row index in the partial results, or -1 (a range that holds only positions that stand for a start)
  int slot[KL];
  bool whole = false;
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    const int k = first + lane + 32 * i;
    slot[i] = -1;
    if (k <= last) {
      const long long k_lo = (long long)k * cut.span, k_hi = min(k_lo + cut.span, (long long)cut.total);
      const int g0 = (int)max(0ll, max(0ll, k_lo - cut.start) - kTreeItemCost);
      const int g1 = (int)max(0ll, min((long long)per, k_hi - cut.start) - kTreeItemCost);
      if (g1 > g0) slot[i] = (2 * k + (cut.start <= k_lo ? 0 : 1)) * kTreeRows;
      whole |= g0 == 0 && g1 == cut.tiles;
    }
  }
  if (__any_sync(0xffffffffu, whole)) return;  // one thread block had all key tiles and wrote the output
  for (int r = r_lo + (int)blockIdx.y * (kTreeMergeThreads / 32) + warp; r < r_hi; r += kTreeMergeY * (kTreeMergeThreads / 32)) {
    float w[KL], M = -INFINITY, L = 0.f;
    float2 ml[KL];
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      if (slot[i] >= 0) ml[i] = p.part_ml[slot[i] + r];
      M = fmaxf(M, ml[i].x);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      w[i] = exp2f(ml[i].x - M);
      if (w[i] < FLT_MIN) w[i] = FLT_MIN;     // nothing beside the others, but an infinity stays one
      if (ml[i].x == -INFINITY) w[i] = 0.f;   // a piece in which the row saw nothing adds nothing
      L = fmaf(w[i], ml[i].y, L);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    float acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.f;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int n = min(32, last - first + 1 - 32 * i);
      for (int j = 0; j < n; j += 8) {  // eight rows in flight; a row of weight zero is read from a place that has one, and left out
        float o[8][V], wk[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          wk[e] = __shfl_sync(0xffffffffu, w[i], (j + e) & 31);
          const int sk = __shfl_sync(0xffffffffu, slot[i], (j + e) & 31);
          if (j + e >= n) wk[e] = 0.f;
          const float* src = p.part_o + (size_t)(wk[e] > 0.f ? sk + r : r) * HD + lane * V;
#pragma unroll
          for (int v = 0; v < V; v += 2) {
            const float2 x = *reinterpret_cast<const float2*>(src + v);
            o[e][v] = x.x;
            o[e][v + 1] = x.y;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int v = 0; v < V; ++v) acc[v] = wk[e] > 0.f ? fmaf(o[e][v], wk[e], acc[v]) : acc[v];
      }
    }
    const int R = cut.rt * kTreeRows + r, node = tree_node(p, R), g = R - node * p.G;
    const float inv = 1.0f / L;
    __nv_bfloat16* dst = p.out + (((size_t)cut.b * p.n + node) * p.Hq + (size_t)cut.hk * p.G + g) * HD + lane * V;
#pragma unroll
    for (int v = 0; v < V; v += 2) *reinterpret_cast<uint32_t*>(dst + v) = ptx::pack_bf16(acc[v] * inv, acc[v + 1] * inv);
  }
}

// ---------------------------------------------------------------------------------------------
template <int HD>
static cudaError_t tree_launch(sdlm_ctx* ctx, TreeParams& p, cudaStream_t st) {
  const int tile_b = HD * 128;
  // alignment slack, the tiles' queries, 17 barriers, 16 sets of nodes, the schedule, flags; two barriers per ring slot
  const int fixed = 1024 + p.q_tiles * (HD / 64) * 128 * 128 + (17 + 16) * 8 + (int)sizeof(TreeStart) + 12 * 4 + 16;
  const int slots = (kTreeSmemLimit - fixed) / (tile_b + 16);
  if (slots < 4) return cudaErrorLaunchOutOfResources;
  p.n_k = p.n_v = slots / 2 > 8 ? 8 : slots / 2;
  const size_t smem = (size_t)fixed + (size_t)(p.n_k + p.n_v) * (tile_b + 16);
  const int ctas = ctx->sm_count < kAttnMaxCtas ? ctx->sm_count : kAttnMaxCtas;
  cudaError_t e = launch_overlapped(tree_attn_kernel<HD>, dim3(ctas), dim3(kTreeThreads), smem, st, p);
  ctx->launches++;
  if (e != cudaSuccess) return e;
  e = launch_overlapped(tree_merge_kernel<HD>, dim3(ctas - 1, kTreeMergeY), dim3(kTreeMergeThreads), 0, st, p);
  ctx->launches++;
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t setup_tree(sdlm_ctx* ctx) {
  if (ctx->cfg.head_dim == 128)
    return cudaFuncSetAttribute(tree_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTreeSmemLimit);
  return cudaFuncSetAttribute(tree_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTreeSmemLimit);
}

}  // namespace sdlm

using namespace sdlm;

extern "C" sdlm_status sdlm_tree_attn(sdlm_ctx* ctx, int32_t batch, int32_t n, const int32_t* seq_ids, const int32_t* n_nodes,
                                      const int32_t* parent, const void* q, const void* k_tree, const void* v_tree,
                                      void* out, void* stream) {
  if (!ctx || !parent || !q || !k_tree || !v_tree || !out || batch < 1 || n < 1) return SDLM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(out)) return SDLM_ERR_INVALID_ARG;
  if (batch > ctx->cfg.max_batch || n > kMaxTreeNodes) return SDLM_ERR_SHAPE;
  if (!(ctx->scale > 0.0f)) return SDLM_ERR_UNSUPPORTED;
  if (!same_device(ctx)) return SDLM_ERR_INVALID_ARG;
  const sdlm_config& c = ctx->cfg;
  // rows are read by thread blocks that others, which have their outputs already, do not wait for
  const size_t row_b = (size_t)batch * n * c.head_dim * 2, q_b = row_b * c.n_q_heads, kv_b = row_b * c.n_kv_heads;
  const size_t seqs_b = (size_t)batch * 4;  // (every role walks the schedule by itself and reads these as it goes)
  if (ranges_overlap(out, q_b, q, q_b) || ranges_overlap(out, q_b, k_tree, kv_b) || ranges_overlap(out, q_b, v_tree, kv_b) ||
      ranges_overlap(out, q_b, parent, seqs_b * n) || (n_nodes && ranges_overlap(out, q_b, n_nodes, seqs_b)) ||
      (seq_ids && ranges_overlap(out, q_b, seq_ids, seqs_b)))
    return SDLM_ERR_INVALID_ARG;
  const long long rts = ((long long)ctx->group * n + kTreeRows - 1) / kTreeRows;
  const long long positions = (long long)batch * c.n_kv_heads * rts * (kTreeItemCost + (long long)c.max_pages_per_seq + 1);
  if (positions >= (1ll << 30)) return SDLM_ERR_SHAPE;  // they are counted in 32 bits
  TreeParams p;
  p.pool = reinterpret_cast<const __nv_bfloat16*>(ctx->pool);
  p.page_table = ctx->page_table; p.seq_len = ctx->seq_len; p.seq_ids = seq_ids; p.n_nodes = n_nodes; p.parent = parent;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k_tree = static_cast<const __nv_bfloat16*>(k_tree); p.v_tree = static_cast<const __nv_bfloat16*>(v_tree);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.hdr = ctx->hdr;
  p.part_o = reinterpret_cast<float*>(ctx->ws + ctx->lay.tree_o);
  p.part_ml = reinterpret_cast<float2*>(ctx->ws + ctx->lay.tree_ml);
  p.cuts = reinterpret_cast<TreeCut*>(ctx->ws + ctx->lay.tree_cuts);
  p.scale_log2 = ctx->scale * 1.4426950408889634f;
  p.batch = batch; p.n = n; p.Hq = c.n_q_heads; p.Hkv = c.n_kv_heads; p.G = ctx->group;
  p.mpps = c.max_pages_per_seq; p.num_pages = c.num_pages; p.max_batch = c.max_batch;
  p.n_k = p.n_v = 0;
  p.q_tiles = ctx->group * n > 128 ? 2 : 1;
  p.inv_G = ctx->group == 1 ? 0u : (uint32_t)((1ull << 32) / (unsigned)ctx->group + 1);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (c.head_dim == 128 ? tree_launch<128>(ctx, p, st) : tree_launch<64>(ctx, p, st)) == cudaSuccess ? SDLM_OK : SDLM_ERR_CUDA;
}
