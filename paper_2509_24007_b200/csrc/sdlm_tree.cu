// Attention of a tree of drafted tokens over the paged cache (sdlm_tree_attn): the verification pass of Sec. 3.4 for
// several drafted continuations at once.  Node j of sequence b (a drafted token hanging from node parent[j] < j, or
// from the cached history) attends to the whole history, to the nodes on its path and to itself:
//   out[b,j,h,:] = softmax_t( q[b,j,h,:] . K_t * scale ) V_t,   t over the cached tokens of b, the ancestors of j, j.
//
// The G = Hq/Hkv query heads of a KV head and the tree's nodes are stacked: row node * G + g of (sequence, KV head).
// A task is 256 stacked rows of one (sequence, KV head), two tiles of 128 that share every cached tile and take turns
// on the tensor cores; its keys are the cached tiles (64 tokens each) and one tile of the tree's own keys, taken two
// at a time (a group):
//     S = Q K^T      M = 128 rows, N = 128 keys, K = d      A and B from shared memory
//     O += P V       M = 128 rows, N = d,        K = 128    A = P from tensor memory, B = V^T from shared memory
// Few rows are bound by the cache's bytes, many by the products.  The groups of all tasks form one sequence that is
// cut into equal contiguous ranges, one per thread block (one per SM); the part of a task in one range is a piece.  A
// piece that is not its whole task leaves its sums unnormalised with their reference, and a second kernel joins them
// in the order of their thread blocks, so that results do not depend on timing.
//
// Roles: warp 0 copies cached tiles (K and V^T have rings of their own and run ahead over piece boundaries), warp 1
// issues all MMAs, warps 2 and 3 put the tree's keys and values into the ring slot of the last group (V transposed),
// warps 4..11 / 12..19 are the softmax of the first / second tile (two threads a row, one for each key tile of the
// group, that agree on the row's reference through shared memory) and also stage the tile's queries and write its
// rows out.  Only groups with a partly visible tile look at the row's 64-bit visibility word.
#include "sdlm_internal.h"
#include "sdlm_ptx.cuh"

namespace sdlm {

constexpr int kTreeThreads = 640;
constexpr int kTreeRows = 256;        // stacked rows of a task
constexpr float kTreeRebase = 8.0f;   // log2 units a score may exceed its row's reference by
constexpr int kTreeItemCost = 2;      // groups' worth of work the schedule charges for a task's queries and output
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
  int batch, n, Hq, Hkv, G, mpps, num_pages, max_batch, n_k, n_v, q_tiles, merge_rows;
};

__device__ __forceinline__ uint64_t tree_smem_desc(uint32_t saddr) {
  // K-major operand, 128-byte swizzle, 8-row groups 1024 bytes apart; descriptor version 1 (sm_100)
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// D (tensor memory) = or += A (tensor memory: 128 lanes, two bf16 of consecutive k per 32-bit column) * B (shared memory)
__device__ __forceinline__ void tree_umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Largest of a thread's 64 scores; with EDGE only over the keys whose bit is set.
template <bool EDGE>
__device__ __forceinline__ float tree_row_max(const uint32_t (&x)[64], uint32_t lo, uint32_t hi) {
  float mx = -INFINITY;
  if (EDGE) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (lo >> i & 1u) mx = fmaxf(mx, __uint_as_float(x[i]));
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (hi >> i & 1u) mx = fmaxf(mx, __uint_as_float(x[32 + i]));
  } else {
#pragma unroll
    for (int i = 0; i < 64; i += 2) mx = ptx::max3(mx, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
  }
  return mx;
}
// A thread's 64 weights 2^(x * scale + neg_ref) as bf16 pairs into 32 tensor-memory columns at taddr; returns the sum
// of the rounded weights, the ones O is formed from (a row that one key dominates then comes out as that key's V row
// exactly).  Rounding the weights to bf16 is what the matrix product takes: 2^-9 of each weight at most, of either
// sign.  Three pairs of every eight take the power of two from the cubic, the others from the special-function unit.
template <bool EDGE>
__device__ __forceinline__ float tree_weights(const uint32_t (&x)[64], uint32_t taddr, float scale, float neg_ref, uint32_t lo, uint32_t hi) {
  const float2 scale2 = make_float2(scale, scale), neg_ref2 = make_float2(neg_ref, neg_ref);
  float2 l2 = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t packed[16];
    const uint32_t bits = c ? hi : lo;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float2 t = ptx::fma2_f2(make_float2(__uint_as_float(x[c * 32 + i]), __uint_as_float(x[c * 32 + i + 1])), scale2, neg_ref2);
      float2 wf;
      if (((i >> 1) & 7) < 3) {
        wf = ptx::exp2_poly2(t);
      } else {
        wf.x = ptx::ex2(t.x);
        wf.y = ptx::ex2(t.y);
      }
      if (EDGE) {
        if (!(bits >> i & 1u)) wf.x = 0.f;
        if (!(bits >> (i + 1) & 1u)) wf.y = 0.f;
      }
      const __nv_bfloat162 w = __floats2bfloat162_rn(wf.x, wf.y);
      const uint32_t wb = *reinterpret_cast<const uint32_t*>(&w);
      l2 = ptx::add2_f2(l2, make_float2(__uint_as_float(wb << 16), __uint_as_float(wb & 0xffff0000u)));
      packed[i >> 1] = wb;
    }
    ptx::tmem_st16(taddr + c * 16, packed);
  }
  return l2.x + l2.y;
}

__device__ __forceinline__ void tree_status(const TreeParams& p, int code, int slot, int detail) {
  if (atomicCAS(&p.hdr->status[0], 0, code) == 0) {
    p.hdr->status[1] = slot;
    p.hdr->status[2] = detail;
  }
}

// ---- the schedule -----------------------------------------------------------------------------------------
// Sequence b has Hkv * ceil(G * nodes / 256) tasks of (item cost + groups) positions each; a slot number outside the
// tables, or a sequence without nodes, has none.  Thread block c has the positions [c * span, (c + 1) * span).
struct TreeSeq {
  int slot, len, nodes, rts, groups;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b) {
  TreeSeq s;
  s.slot = p.seq_ids ? p.seq_ids[b] : b;
  s.nodes = p.n_nodes ? min(max(p.n_nodes[b], 0), p.n) : p.n;
  if (s.slot < 0 || s.slot >= p.max_batch) s.nodes = 0;
  s.len = s.nodes > 0 ? max(0, min(p.seq_len[s.slot], p.mpps * kPageSize)) : 0;
  s.rts = (p.G * s.nodes + kTreeRows - 1) / kTreeRows;
  s.groups = ((s.len + kPageSize - 1) / kPageSize + 2) / 2;  // cached tiles and the tree's, two at a time
  return s;
}
__device__ __forceinline__ long long tree_positions(const TreeParams& p, const TreeSeq& s) {
  return (long long)p.Hkv * s.rts * (kTreeItemCost + s.groups);
}
struct TreePiece {
  TreeSeq s;
  int b, hk, rt, g0, g1;
  int slot_i;  // 0: the piece of the task that holds the range's first position, 1: a later one
};
// Walks the pieces of a thread block's positions, counted from its first one; every role keeps a walk of its own.
struct TreeWalk {
  int cur, b, base;  // base: first position of sequence b (negative where it lies in an earlier range)
};
__device__ __forceinline__ bool tree_next(const TreeParams& p, TreeWalk& w, int n_pos, TreePiece& t) {
  while (w.cur < n_pos) {
    t.s = tree_seq(p, w.b);
    const int per = kTreeItemCost + t.s.groups, tasks = p.Hkv * t.s.rts;
    if (w.cur >= w.base + (long long)per * tasks) {  // positions are left, so a later sequence has them
      w.base += per * tasks;
      ++w.b;
      continue;
    }
    const int ti = (w.cur - w.base) / per, start = w.base + ti * per;
    const int in0 = w.cur - start, in1 = min(n_pos - start, per);
    w.cur = start + in1;
    t.g0 = max(0, in0 - kTreeItemCost);
    t.g1 = max(0, in1 - kTreeItemCost);
    if (t.g1 <= t.g0) continue;  // only positions that stand for a task's start
    t.b = w.b;
    t.hk = ti / t.s.rts;
    t.rt = ti - t.hk * t.s.rts;
    t.slot_i = start <= 0 ? 0 : 1;
    return true;
  }
  return false;
}

template <int HD>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_attn_kernel(const TreeParams p) {
  constexpr int KH = HD / 64;                    // 64-wide panels of K and of Q
  constexpr int CH = HD / 8;                     // 16-byte chunks of a row
  constexpr int K_PANEL_B = kPageSize * 128;     // one key tile's panel: 64 keys x 128 bytes
  constexpr int K_PART_B = 2 * KH * K_PANEL_B;   // K of a group: [panel][tile of the group][64 keys x 128 bytes]
  constexpr int VT_B = HD * 128;                 // one key tile's V^T: d rows x 128 bytes
  constexpr int V_PART_B = 2 * VT_B;             // V^T of a group: [tile of the group][d x 128 bytes]
  constexpr int Q_PANEL_B = 128 * 128;           // 128 rows x 64 dims
  constexpr int Q_B = KH * Q_PANEL_B;            // one tile's queries
  // tensor memory: S of tile X at columns X*128 (P of key tile j over columns X*128 + 64j .. + 31); O of tile X at
  // 256 + X*128
  constexpr uint32_t O_COL = 256, TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_s = smem;                 // [q_tiles][Q_B]
  uint8_t* k_ring = q_s + (size_t)p.q_tiles * Q_B;
  const int NK = p.n_k, NV = p.n_v;
  uint8_t* v_ring = k_ring + (size_t)NK * K_PART_B;
  uint64_t* full_k = reinterpret_cast<uint64_t*>(v_ring + (size_t)NV * V_PART_B);
  uint64_t* k_free = full_k + NK;
  uint64_t* full_v = k_free + NK;
  uint64_t* v_free = full_v + NV;
  uint64_t* s_full = v_free + NV;      // [tile]
  uint64_t* p_full = s_full + 2;       // [tile]
  uint64_t* m_bar = p_full + 2;        // [tile]: both halves of a row have written their maximum
  uint64_t* l_bar = m_bar + 2;         // [tile]: ... their sum
  uint64_t* o_done = l_bar + 2;        // [tile]
  uint64_t* q_full = o_done + 2;       // [tile]: queries staged, the piece before read out of tensor memory
  uint64_t* drain = q_full + 2;
  long long* sched = reinterpret_cast<long long*>(drain + 1);  // [total, first position, its sequence, that one's base]
  long long* warp_sum = sched + 4;                             // [20]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(warp_sum + 20);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* tree_k = abort + 1;    // tree tiles whose ring slot is free to be written
  volatile int* tree_v = abort + 2;
  __nv_bfloat16* m_s = reinterpret_cast<__nv_bfloat16*>(tmem_slot + 4);  // [tile][half][128 rows]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 32) {
    for (int s = 0; s < NK; ++s) {
      ptx::mbar_init(&full_k[s], 3);  // the copies, and the two warps that write the tree's tile (or the copying thread for them)
      ptx::mbar_init(&k_free[s], 1);
    }
    for (int s = 0; s < NV; ++s) {
      ptx::mbar_init(&full_v[s], 3);
      ptx::mbar_init(&v_free[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(&s_full[s], 1);
      ptx::mbar_init(&p_full[s], 8);  // one arrival per softmax warp of the tile
      ptx::mbar_init(&m_bar[s], 8);
      ptx::mbar_init(&l_bar[s], 8);
      ptx::mbar_init(&o_done[s], 1);
      ptx::mbar_init(&q_full[s], 8);
    }
    ptx::mbar_init(drain, 1);
    *abort = 0;
    *tree_k = 0;
    *tree_v = 0;
    sched[1] = -1;
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
  long long mine = 0;
  for (int i = 0; i < per_thread; ++i) {
    const int b = tid * per_thread + i;
    if (b >= p.batch) break;
    const TreeSeq s = tree_seq(p, b);
    if (blockIdx.x == 0 && (s.slot < 0 || s.slot >= p.max_batch)) tree_status(p, SDLM_ERR_DEVICE_CHECK, s.slot, b);
    mine += tree_positions(p, s);
  }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) warp_sum[warp] = upto;
  ptx::tc_fence_before();
  __syncthreads();  // barriers initialised, tensor memory allocated, sums of the warps written
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  long long total = 0;
  upto -= mine;
#pragma unroll
  for (int i = 0; i < kTreeThreads / 32; ++i) {
    if (i < warp) upto += warp_sum[i];
    total += warp_sum[i];
  }
  const long long span = total > 0 ? (total + gridDim.x - 1) / gridDim.x : 1;
  const long long lo = (long long)blockIdx.x * span;
  if (mine > 0 && upto <= lo && lo < upto + mine) {  // the thread whose sequences hold the first position
    for (int b = tid * per_thread;; ++b) {
      const TreeSeq s = tree_seq(p, b);
      const long long n = tree_positions(p, s);
      if (lo < upto + n) {
        sched[1] = lo;
        sched[2] = b;
        sched[3] = upto;
        const int per = kTreeItemCost + s.groups, ti = (int)((lo - upto) / per), hk = ti / s.rts;
        p.cuts[blockIdx.x] = TreeCut{upto + (long long)ti * per, span, total, b, hk, ti - hk * s.rts, s.groups, s.nodes};
        break;
      }
      upto += n;
    }
  }
  if (tid == 0 && lo >= total) p.cuts[blockIdx.x].span = 0;
  __syncthreads();
  const int n_pos = lo < total ? (int)(total - lo < span ? total - lo : span) : 0;
  TreeWalk walk{0, (int)sched[2], (int)(sched[3] - lo)};
  TreePiece t;

  // Registers move between warp groups inside the thread block's own allocation (640 threads x 96 at launch):
  // 128 x 56 + 512 x 104 stays below it, so the raise below never waits for registers that nobody gives back.
  static_assert(128 * 56 + 512 * 104 <= kTreeThreads * 96, "register budget of the warp groups");
  if (warp < 4) {
    ptx::reg_dealloc<56>();
    if (warp == 0) {
      // ---------------------------------------------------------------- cached tiles: bulk copies
      // K runs NK groups ahead of the issuer and V^T NV groups, over piece boundaries: two walks, one for each.
      bool ok = true;
      TreeWalk wv = walk;
      TreePiece tv;
      int gk = 0, gv = 0, g_k = 0, g_v = 0, tk_n = 0, tv_n = 0;
      bool more_k = tree_next(p, walk, n_pos, t), more_v = tree_next(p, wv, n_pos, tv);
      if (more_k) g_k = t.g0;
      if (more_v) g_v = tv.g0;
      int win_base[2] = {-1, -1}, win_b[2] = {-1, -1}, win_page[2] = {0, 0};
      auto copy_part = [&](const TreePiece& tp, int g, int gi, bool v_part) {  // warp-wide; lane 0 issues
        const int ring = v_part ? NV : NK, slot_i = gi % ring;
        const uint32_t use = (uint32_t)(gi / ring);
        const int w = v_part ? 1 : 0, base = (2 * g) & ~31;
        const int cached = (tp.s.len + kPageSize - 1) / kPageSize, tiles = max(0, min(2, cached - 2 * g));
        const bool with_tree = g == tp.s.groups - 1;
        if (win_base[w] != base || win_b[w] != tp.b) {
          win_base[w] = base;
          win_b[w] = tp.b;
          win_page[w] = base + lane < cached ? p.page_table[(size_t)tp.s.slot * p.mpps + base + lane] : 0;
        }
        const int page0 = __shfl_sync(0xffffffffu, win_page[w], (2 * g) & 31);
        const int page1 = __shfl_sync(0xffffffffu, win_page[w], (2 * g + 1) & 31);
        if (lane == 0) {
          uint64_t* freed = v_part ? &v_free[slot_i] : &k_free[slot_i];
          uint64_t* full = v_part ? &full_v[slot_i] : &full_k[slot_i];
          if (use > 0 && !ptx::mbar_wait_paced(freed, (use - 1) & 1u, abort)) ok = false;
          if (ok) {
            if (with_tree) {  // warps 2 and 3 write the tree's tile and arrive for it
              __threadfence_block();
              if (v_part) *tree_v = tv_n + 1; else *tree_k = tk_n + 1;
            } else {
              ptx::mbar_arrive(full);
              ptx::mbar_arrive(full);
            }
            ptx::mbar_arrive_expect_tx(full, (uint32_t)(tiles * (v_part ? VT_B : KH * K_PANEL_B)));
            for (int j = 0; j < tiles; ++j) {
              int page = j ? page1 : page0;
              if (page < 0 || page >= p.num_pages) {  // never follow a bad table entry out of the pool
                tree_status(p, SDLM_ERR_DEVICE_CHECK, tp.s.slot, page);
                page = 0;
              }
              const uint8_t* src = reinterpret_cast<const uint8_t*>(p.pool + kv_tile_offset(page, tp.hk, 0, p.Hkv, HD));
              if (v_part) {
                ptx::bulk_g2s(v_ring + (size_t)slot_i * V_PART_B + j * VT_B, src + KH * K_PANEL_B, VT_B, full);
              } else {
#pragma unroll
                for (int kh = 0; kh < KH; ++kh)
                  ptx::bulk_g2s(k_ring + (size_t)slot_i * K_PART_B + (kh * 2 + j) * K_PANEL_B, src + kh * K_PANEL_B, K_PANEL_B, full);
              }
            }
          }
        }
        if (with_tree) { if (v_part) ++tv_n; else ++tk_n; }
        ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
      };
      // Order of the copies: K of the first NK groups, then for every group its V^T and the K of the group NK further
      // on, which is the order in which the issuer gives the buffers back.
      while (more_v && ok) {
        while (more_k && ok && gk < gv + NK) {
          copy_part(t, g_k, gk++, false);
          if (++g_k == t.g1) {
            more_k = tree_next(p, walk, n_pos, t);
            if (more_k) g_k = t.g0;
          }
        }
        if (!ok) break;
        copy_part(tv, g_v, gv++, true);
        if (++g_v == tv.g1) {
          more_v = tree_next(p, wv, n_pos, tv);
          if (more_v) g_v = tv.g0;
        }
      }
      if (lane == 0 && (!ok || *abort)) {  // winding down: let the copies already issued land
        tree_status(p, SDLM_ERR_TIMEOUT, -2, 11);
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer
      // Per group and tile: O_x += P_x(before) V(before), then S_x = Q_x K^T over the columns that P_x was read from.
      // The whole warp runs the loop and the waits; one elected lane issues (see ptx::elect_one).
      const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(HD >> 3) << 17) | ((128u >> 4) << 24);
      const uint64_t d_q = tree_smem_desc(ptx::smem_u32(q_s));
      const uint64_t d_kr = tree_smem_desc(ptx::smem_u32(k_ring)), d_vr = tree_smem_desc(ptx::smem_u32(v_ring));
      bool ok = true;
      int gk = 0, gp[2] = {0, 0}, pc[2] = {0, 0};  // groups so far, groups and pieces of each tile so far
      while (ok && tree_next(p, walk, n_pos, t)) {
        const int n_x = p.G * t.s.nodes - t.rt * kTreeRows > 128 ? 2 : 1;
        const int n_groups = t.g1 - t.g0, n_tiles = (t.s.len + kPageSize - 1) / kPageSize + 1;
        for (int x = 0; x < n_x && ok; ++x)
          ok = __all_sync(0xffffffffu, ptx::mbar_wait_parked(&q_full[x], (uint32_t)pc[x] & 1u, abort));
        for (int g = 0; g <= n_groups && ok; ++g) {
          for (int x = 0; x < n_x && ok; ++x) {
            if (g > 0) {  // O_x += P_x(g-1) V(g-1)
              const int gi = gk + g - 1, vs = gi % NV, tiles = min(2, n_tiles - 2 * (t.g0 + g - 1));
              if (x == 0 && !__all_sync(0xffffffffu, ptx::mbar_wait_parked(&full_v[vs], (uint32_t)(gi / NV) & 1u, abort))) { ok = false; break; }
              if (!__all_sync(0xffffffffu, ptx::mbar_wait_parked(&p_full[x], (uint32_t)(gp[x] + g - 1) & 1u, abort))) { ok = false; break; }
              ptx::tc_fence_after();
              const uint64_t d_v = d_vr + (uint64_t)((vs * V_PART_B) >> 4);
              if (ptx::elect_one()) {
                for (int j = 0; j < tiles; ++j)
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    tree_umma_ts(tmem_base + O_COL + x * 128, tmem_base + x * 128 + j * 64 + k * 8,
                                 d_v + (uint64_t)((j * VT_B + k * 32) >> 4), idesc_o, (g - 1 | j | k) ? 1u : 0u);
                if (x == n_x - 1) ptx::umma_commit(&v_free[vs]);
                if (g == n_groups) ptx::umma_commit(&o_done[x]);
              }
              __syncwarp();
            }
            if (g < n_groups) {  // S_x(g) = Q_x K(g)^T
              const int gi = gk + g, ks = gi % NK;
              if (x == 0 && !__all_sync(0xffffffffu, ptx::mbar_wait_parked(&full_k[ks], (uint32_t)(gi / NK) & 1u, abort))) { ok = false; break; }
              ptx::tc_fence_after();
              const uint64_t d_k = d_kr + (uint64_t)((ks * K_PART_B) >> 4);
              if (ptx::elect_one()) {
#pragma unroll
                for (int kh = 0; kh < KH; ++kh)
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    ptx::umma_bf16_ss(tmem_base + x * 128, d_q + (uint64_t)((x * Q_B + kh * Q_PANEL_B + k * 32) >> 4),
                                      d_k + (uint64_t)((kh * 2 * K_PANEL_B + k * 32) >> 4), idesc_s, (kh | k) ? 1u : 0u);
                ptx::umma_commit(&s_full[x]);
                if (x == n_x - 1) ptx::umma_commit(&k_free[ks]);  // the K part of this group may be replaced
              }
              __syncwarp();
            }
          }
        }
        gk += n_groups;
        for (int x = 0; x < n_x; ++x) {
          gp[x] += n_groups;
          ++pc[x];
        }
      }
      if (!ok && lane == 0) {  // winding down: the MMAs already issued must finish before TMEM and smem are released
        tree_status(p, SDLM_ERR_TIMEOUT, -2, 12);
        ptx::umma_commit(drain);
        ptx::mbar_wait_brief(drain, 0);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------- the tree's own keys and values
      const int st = tid - 64;  // 64 threads
      bool ok = true;
      int gk = 0, n_done = 0;
      while (ok && tree_next(p, walk, n_pos, t)) {
        const int gi = gk + (t.g1 - t.g0) - 1;
        gk += t.g1 - t.g0;
        if (t.g1 != t.s.groups) continue;
        const int jt = ((t.s.len + kPageSize - 1) / kPageSize) & 1;  // the tile's place in the group
        const size_t stride = (size_t)p.Hkv * HD;
        const size_t first = ((size_t)t.b * p.n * p.Hkv + t.hk) * HD;
        // keys: row by row, 16 bytes at a time; rows behind the last node are zero
        if (!ptx::counter_wait(tree_k, n_done, abort)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        uint8_t* kd = k_ring + (size_t)(gi % NK) * K_PART_B + jt * K_PANEL_B;
#pragma unroll 4
        for (int i = 0; i < CH; ++i) {
          const int idx = st + i * 64, key = idx / CH, c = idx % CH;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (key < t.s.nodes) v = *(reinterpret_cast<const uint4*>(p.k_tree + first + key * stride) + c);
          *reinterpret_cast<uint4*>(kd + (c >> 3) * (2 * K_PANEL_B) + key * 128 + (((c & 7) ^ (key & 7)) << 4)) = v;
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full_k[gi % NK]);
        // values: blocks of eight keys by eight columns, transposed in registers
        if (!ptx::counter_wait(tree_v, n_done, abort)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++n_done;
        uint8_t* vd = v_ring + (size_t)(gi % NV) * V_PART_B + jt * VT_B;
        for (int i = 0; i < CH / 8; ++i) {
          const int blk = st + i * 64, kb = blk / CH, c = blk % CH;
          uint4 v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = make_uint4(0, 0, 0, 0);
            if (kb * 8 + e < t.s.nodes) v[e] = *(reinterpret_cast<const uint4*>(p.v_tree + first + (kb * 8 + e) * stride) + c);
          }
#pragma unroll
          for (int col = 0; col < 8; ++col) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t a = reinterpret_cast<const uint32_t*>(&v[2 * e])[col >> 1];
              const uint32_t c2 = reinterpret_cast<const uint32_t*>(&v[2 * e + 1])[col >> 1];
              o[e] = __byte_perm(a, c2, col & 1 ? 0x7632 : 0x5410);
            }
            *reinterpret_cast<uint4*>(vd + (c * 8 + col) * 128 + ((kb ^ col) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full_v[gi % NV]);
      }
      if (!ok && lane == 0) tree_status(p, SDLM_ERR_TIMEOUT, -2, 14);
      __syncwarp();
    }
  } else {
    ptx::reg_alloc<104>();
    // ---------------------------------------------------------------- queries, softmax and output
    // Thread = (row of tile X, half h): the keys of the group's key tile h, the columns h*d/2 .. of O.
    const int X = (warp - 4) >> 3, h = ((warp - 4) >> 2) & 1, qd = warp & 3, row = qd * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(qd * 32) << 16);
    const uint32_t s_col = (uint32_t)X * 128 + (uint32_t)h * 64, o_col = O_COL + (uint32_t)X * 128 + (uint32_t)h * (HD / 2);
    __nv_bfloat16* m_mine = m_s + (X * 2 + h) * 128 + row;
    const __nv_bfloat16* m_other = m_s + (X * 2 + (h ^ 1)) * 128 + row;
    int gi = 0, pc = 0;
    bool ok = true;
    while (ok && tree_next(p, walk, n_pos, t)) {
      const int row0 = t.rt * kTreeRows + X * 128, rows = min(128, p.G * t.s.nodes - row0);
      if (rows <= 0) continue;  // the task has no second tile
      {
        // Queries into shared memory, swizzled as an MMA operand; rows beyond the end are zero.
        uint4 v[CH / 2];
        const int st = tid - 128 - X * 256;
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) {
          const int idx = st + i * 256, r = idx / CH, c = idx % CH;
          v[i] = make_uint4(0, 0, 0, 0);
          if (r < rows) {
            const int node = (row0 + r) / p.G, g = row0 + r - node * p.G;
            v[i] = *(reinterpret_cast<const uint4*>(p.q + (((size_t)t.b * p.n + node) * p.Hq + (size_t)t.hk * p.G + g) * HD) + c);
          }
        }
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) {
          const int idx = st + i * 256, r = idx / CH, c = idx % CH;
          *reinterpret_cast<uint4*>(q_s + X * Q_B + (c >> 3) * Q_PANEL_B + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
        }
        ptx::fence_proxy_async();
        ptx::tc_fence_before();  // this thread's reads of the piece before are done
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&q_full[X]);
      }
      const int my_node = (row0 + row) / p.G;
      uint32_t vis_lo = 0, vis_hi = 0;  // the nodes this row sees, where the piece has the tree's keys
      if (t.g1 == t.s.groups && row < rows) {
        for (int i = my_node; i >= 0;) {
          if (i < 32) vis_lo |= 1u << i; else vis_hi |= 1u << (i - 32);
          const int up = p.parent[(size_t)t.b * p.n + i];
          i = up < i ? up : -1;  // a parent that is not an earlier node: the node hangs from the history
        }
      }
      const int cached = (t.s.len + kPageSize - 1) / kPageSize, whole = t.s.len / kPageSize;
      float m_ref = -INFINITY, l = 0.f;
      for (int g = t.g0; g < t.g1; ++g) {
        // S(g) complete; so is O += P(g-1) V(g-1), which was issued before it
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_parked(&s_full[X], (uint32_t)gi & 1u, abort))) { ok = false; break; }
        ptx::tc_fence_after();
        const bool edge = 2 * g + 2 > whole;  // some key of this group is not seen by every row
        uint32_t lo = 0xffffffffu, hi = 0xffffffffu;
        if (edge) {
          const int tl = 2 * g + h, in_last = t.s.len - whole * kPageSize;
          if (tl == cached) { lo = vis_lo; hi = vis_hi; }
          else if (tl > cached) lo = hi = 0;
          else if (tl == whole) {  // the history ends inside this tile
            lo = in_last >= 32 ? 0xffffffffu : (1u << in_last) - 1u;
            hi = in_last > 32 ? (1u << (in_last - 32)) - 1u : 0u;
          }
        }
        uint32_t x[64];
        ptx::tmem_ld64(lane_addr + s_col, x);
        ptx::tmem_ld_wait();
        float mx = edge ? tree_row_max<true>(x, lo, hi) : tree_row_max<false>(x, lo, hi);
        // The row's two threads must use one reference: each leaves its maximum, rounded to bf16, in shared
        // memory and takes the larger of the two rounded values (any common value near the maximum serves).
        const __nv_bfloat16 mine_m = __float2bfloat16_rn(mx * p.scale_log2);  // the scale is positive
        *m_mine = mine_m;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&m_bar[X]);
        if (!__all_sync(0xffffffffu, ptx::mbar_wait_parked(&m_bar[X], (uint32_t)gi & 1u, abort))) { ok = false; break; }
        mx = fmaxf(__bfloat162float(mine_m), __bfloat162float(*m_other));
        const bool move = mx > m_ref + kTreeRebase || (m_ref == -INFINITY && mx > -INFINITY);
        if (__any_sync(0xffffffffu, move)) {
          float alpha = 1.0f;
          if (move) {
            alpha = m_ref == -INFINITY ? 0.f : ptx::ex2(m_ref - mx);
            m_ref = mx;
            l *= alpha;
          }
          if (g > t.g0) {  // O holds sums relative to the old references (nothing before the first group)
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) {
              uint32_t o[16];
              ptx::tmem_ld16(lane_addr + o_col + c * 16, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              ptx::tmem_st16(lane_addr + o_col + c * 16, o);
            }
          }
        }
        // weights 2^(s * scale - reference), rounded to bf16, two per column over the first half of this
        // thread's S columns.  A key the row does not see gets weight zero.
        const float neg_ref = m_ref == -INFINITY ? 0.f : -m_ref;
        l += edge ? tree_weights<true>(x, lane_addr + s_col, p.scale_log2, neg_ref, lo, hi)
                  : tree_weights<false>(x, lane_addr + s_col, p.scale_log2, neg_ref, lo, hi);
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[X]);
        ++gi;
      }
      if (ok && !__all_sync(0xffffffffu, ptx::mbar_wait(&o_done[X], (uint32_t)pc & 1u, abort))) ok = false;
      if (ok) {
        // every MMA of the tile is complete: the row's two sums meet in its S columns
        ptx::tc_fence_after();
        ptx::tmem_st1(lane_addr + s_col, __float_as_uint(l));
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&l_bar[X]);
        if (!__all_sync(0xffffffffu, ptx::mbar_wait(&l_bar[X], (uint32_t)pc & 1u, abort))) ok = false;
      }
      if (ok) {
        ptx::tc_fence_after();
        uint32_t other;
        ptx::tmem_ld1(lane_addr + ((uint32_t)X * 128 + (uint32_t)(h ^ 1) * 64), other);
        ptx::tmem_ld_wait();
        l += __uint_as_float(other);
        const bool all = t.g0 == 0 && t.g1 == t.s.groups;
        const float inv = all ? 1.0f / l : 1.0f;
        const int g = row0 + row - my_node * p.G;
        __nv_bfloat16* out_row = p.out + (((size_t)t.b * p.n + my_node) * p.Hq + (size_t)t.hk * p.G + g) * HD + h * (HD / 2);
        const size_t part_row = (size_t)(2 * blockIdx.x + t.slot_i) * kTreeRows + X * 128 + row;
        float4* part = reinterpret_cast<float4*>(p.part_o + part_row * HD + h * (HD / 2));
        if (!all && h == 0 && row < rows) p.part_ml[part_row] = make_float2(m_ref, l);
#pragma unroll
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[16];
          ptx::tmem_ld16(lane_addr + o_col + c * 16, o);
          ptx::tmem_ld_wait();
          if (row < rows) {
            if (all) {
              uint32_t w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) w[i] = ptx::pack_bf16(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
              reinterpret_cast<uint4*>(out_row + c * 16)[0] = make_uint4(w[0], w[1], w[2], w[3]);
              reinterpret_cast<uint4*>(out_row + c * 16)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                part[c * 4 + i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                              __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
            }
          }
        }
        ++pc;
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

// Joins the pieces of every task that a range boundary cuts: boundary blockIdx.x belongs to the thread block whose
// range begins there; the first boundary inside a task does the task's rows, merge_rows of them per thread block, a
// warp a row:  O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i, M the largest m_i, in the order of the thread blocks.
template <int HD>
__global__ void __launch_bounds__(128) tree_merge_kernel(const TreeParams p) {
  constexpr int V = HD / 32;  // values of a row per lane
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  const int c = blockIdx.x + 1;
  const TreeCut cut = p.cuts[c];
  if (cut.span == 0) return;
  const long long lo = (long long)c * cut.span;
  if (cut.start >= lo || cut.start < lo - cut.span) return;  // not cut here, or an earlier boundary does it
  const int per = kTreeItemCost + cut.groups, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = min(kTreeRows, p.G * cut.nodes - cut.rt * kTreeRows);
  const int last = (int)((cut.start + per - 1) / cut.span);  // thread block that has the task's last position
  for (int r = blockIdx.y * p.merge_rows + warp; r < min(rows, (int)(blockIdx.y + 1) * p.merge_rows); r += 4) {
    float M = -INFINITY, L = 0.f, acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    bool done = false;
    for (int k = c - 1; k <= last; ++k) {
      const long long k_lo = (long long)k * cut.span, k_hi = min(k_lo + cut.span, cut.total);
      const int g0 = (int)max(0ll, max(0ll, k_lo - cut.start) - kTreeItemCost);
      const int g1 = (int)max(0ll, min((long long)per, k_hi - cut.start) - kTreeItemCost);
      if (g1 <= g0) continue;
      if (g0 == 0 && g1 == cut.groups) { done = true; break; }  // one thread block had all of it and wrote the output
      const size_t part_row = (size_t)(2 * k + (cut.start <= k_lo ? 0 : 1)) * kTreeRows + r;
      const float2 ml = p.part_ml[part_row];
      if (ml.x == -INFINITY) continue;  // the row saw none of the piece's keys
      const float m_new = fmaxf(M, ml.x), a = M == -INFINITY ? 0.f : exp2f(M - m_new), w = exp2f(ml.x - m_new);
      M = m_new;
      L = L * a + ml.y * w;
      const float* o = p.part_o + part_row * HD + lane * V;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = acc[i] * a + o[i] * w;
    }
    if (done) return;
    const int R = cut.rt * kTreeRows + r, node = R / p.G, g = R - node * p.G;
    const float inv = 1.0f / L;
    __nv_bfloat16* dst = p.out + (((size_t)cut.b * p.n + node) * p.Hq + (size_t)cut.hk * p.G + g) * HD + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = ptx::pack_bf16(acc[i] * inv, acc[i + 1] * inv);
  }
}

// ---------------------------------------------------------------------------------------------
template <int HD>
static cudaError_t tree_launch(sdlm_ctx* ctx, TreeParams& p, cudaStream_t st) {
  const int part_b = 2 * kPageSize * HD * 2;  // K (or V^T) of one group of two tiles
  // alignment slack, the tiles' queries, 13 barriers, the schedule, flags, the row maxima; two barriers per ring slot
  const int fixed = 1024 + p.q_tiles * (HD / 64) * 128 * 128 + 13 * 8 + 24 * 8 + 16 + 2 * 2 * 128 * 2;
  const int slots = (kTreeSmemLimit - fixed) / (part_b + 16);
  if (slots < 4) return cudaErrorLaunchOutOfResources;
  p.n_v = slots / 2 > 6 ? 6 : slots / 2;  // K is asked for a product earlier than V^T: the odd slot goes to its ring
  p.n_k = slots - p.n_v > 6 ? 6 : slots - p.n_v;
  const size_t smem = (size_t)fixed + (size_t)(p.n_k + p.n_v) * (part_b + 16);
  const int ctas = ctx->sm_count < kAttnMaxCtas ? ctx->sm_count : kAttnMaxCtas;
  // a merging thread block takes four rows (one a warp) where few tasks share the GPU, up to 32 where many do
  const long long tasks = (long long)p.batch * p.Hkv * ((p.G * p.n + kTreeRows - 1) / kTreeRows);
  p.merge_rows = tasks * 16 >= ctas ? 32 : 4;
  cudaError_t e = launch_overlapped(tree_attn_kernel<HD>, dim3(ctas), dim3(kTreeThreads), smem, st, p);
  ctx->launches++;
  if (e != cudaSuccess) return e;
  const int blocks = (p.G * p.n < kTreeRows ? p.G * p.n : kTreeRows) + p.merge_rows - 1;
  e = launch_overlapped(tree_merge_kernel<HD>, dim3(ctas - 1, blocks / p.merge_rows), dim3(128), 0, st, p);
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

static inline bool tree_a16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

extern "C" sdlm_status sdlm_tree_attn(sdlm_ctx* ctx, int32_t batch, int32_t n, const int32_t* seq_ids, const int32_t* n_nodes,
                                      const int32_t* parent, const void* q, const void* k_tree, const void* v_tree,
                                      void* out, void* stream) {
  if (!ctx || !parent || !q || !k_tree || !v_tree || !out || batch < 1 || n < 1) return SDLM_ERR_INVALID_ARG;
  if (!tree_a16(q) || !tree_a16(k_tree) || !tree_a16(v_tree) || !tree_a16(out)) return SDLM_ERR_INVALID_ARG;
  if (batch > ctx->cfg.max_batch || n > kMaxTreeNodes) return SDLM_ERR_SHAPE;
  if (!(ctx->scale > 0.0f)) return SDLM_ERR_UNSUPPORTED;
  if (!same_device(ctx)) return SDLM_ERR_INVALID_ARG;
  const sdlm_config& c = ctx->cfg;
  const long long rts = ((long long)ctx->group * n + kTreeRows - 1) / kTreeRows;
  const long long positions = (long long)batch * c.n_kv_heads * rts * (kTreeItemCost + ((long long)c.max_pages_per_seq + 2) / 2);
  // a thread block counts positions from its first one in 32 bits, a sequence's own among them
  if (positions / batch >= (1ll << 30) || positions / ctx->sm_count >= (1ll << 30)) return SDLM_ERR_SHAPE;
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
  p.n_k = p.n_v = p.merge_rows = 0;
  p.q_tiles = ctx->group * n > 128 ? 2 : 1;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (c.head_dim == 128 ? tree_launch<128>(ctx, p, st) : tree_launch<64>(ctx, p, st)) == cudaSuccess ? SDLM_OK : SDLM_ERR_CUDA;
}
