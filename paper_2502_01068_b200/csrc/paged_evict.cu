// Eviction from the paged cache by accumulated attention weight, in place.
//
// A sequence of more than `limit` entries keeps, for each KV head, its last `window` entries and, of the n = len - window before them,
// the m = keep - window of largest weight (ties to the lower slot).  Slots 0 .. m - 1 are a set without order, the window is in order:
//   a kept candidate in a slot below m stays where it is; the r-th free slot below m takes the r-th kept candidate from slot m on;
//   window entry len - window + i moves to slot m + i.
// So an eviction moves no more rows than it has to: those that leave the slots given up, and the window.
//
// Two launches.  evict_plan_kernel ranks: one cluster per (sequence, KV head) finds the m-th largest weight by a most-significant-digit
// radix search on the order-preserving integer image of the weights and writes, in slot order, which slots are free and which
// candidates move.  evict_move_kernel moves: one cluster per (sequence, KV head) and pool.  Everything that moves comes from slots
// >= m, so pages that lie below m altogether take their entries first, in any order; the pages from m on are read from and written
// to, and go through shared memory in ascending order, a barrier of the cluster between reading a round and writing it: what a later
// round reads lies behind everything an earlier one wrote, because the window moves down.
// Weights and ids go to buffers of their own, so that the call may be given again, and a reader may still hold the old ones.
//
// 8-bit pages: a page's entries share a scale; a page that receives entries takes the largest scale of the pages that its entries
// come from (those that stay among them), and codes from smaller scales are encoded again, code * old / new, rounded to nearest even:
// powers of two, so only codes that fall below 2^-6 lose bits.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace fastkv {

namespace {

constexpr int kBins = 256;

// Monotone map fp32 -> uint32 (larger float <=> larger integer); -0 counts as +0, NaN of either sign below everything else.
__device__ __forceinline__ uint32_t rank_key(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (u == 0x80000000u) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// The length that a call goes by: 0 and `ok` false where it does not fit (such a sequence is left alone and reported).
__device__ __forceinline__ int evict_len(const EvictParams& p, int b, bool& ok) {
  const int len = p.lens[b];
  const long long room = static_cast<long long>(p.c.max_pages) << p.c.page_log2;
  ok = len >= 0 && len <= room && len <= p.stride && len <= p.max_len;
  return ok ? len : 0;
}

struct PlanView {
  int* kept_below;                 // kept candidates in slots below m
  int* hole;                       // [m]: -1, or the slot's number among the free ones
  int* from;                       // [m]: slot of the kept candidate of rank r, written for those in slots >= m
};
__device__ __forceinline__ PlanView plan_of(const EvictParams& p, int b, int g) {
  const int m = p.keep - p.window;
  int* base = p.plan + (static_cast<long long>(b) * p.c.n_kv_heads + g) * ((2ll * m + 4) / 4 * 4);
  return {base, base + 1, base + 1 + m};
}

template <int THREADS>
struct alignas(16) PlanShared {
  int hist[kBins * 32];            // lane-private digit counters: hist[bin * 32 + lane]
  int total_hist[2][kBins];        // the cluster's histogram of a pass (every CTA adds into it), double-buffered by pass parity
  int warp_tot[2][THREADS / 32];
  alignas(8) int counts[8][2];     // per CTA of the cluster: (#above threshold, #equal to it)
  int digit, k_rem;
};

}  // namespace

// Every thread owns consecutive candidates of its CTA's chunk, so slot order is thread order.  ITEMS > 0: the candidates stay in
// registers for all passes; ITEMS == 0: any number, read again for every pass.
template <int CLUSTER, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) evict_plan_kernel(const EvictParams p) {
  constexpr int kWarps = THREADS / 32, kPerBin = THREADS / kBins;
  static_assert(THREADS % kBins == 0 && kPerBin >= 1 && kPerBin <= 4, "256, 512 or 1024 threads");
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ PlanShared<THREADS> sh;
  constexpr bool CACHED = ITEMS > 0;
  constexpr int R = CACHED ? ITEMS : 1;
  const int rank = static_cast<int>(cluster.block_rank());
  const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  for (int i = tid; i < 2 * kBins; i += THREADS) (&sh.total_hist[0][0])[i] = 0;
  for (int i = tid; i < kBins * 32; i += THREADS) sh.hist[i] = 0;
  cluster.sync();                  // nobody adds into a histogram that is not cleared yet
  pdl_launch_dependents();
  pdl_wait();
  bool ok;
  const int len = evict_len(p, b, ok);
  if (!ok && rank == 0 && g == 0 && tid == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_EVICT_LEN);
  const bool over = len > p.limit;                   // (uniform over the cluster)
  if (rank == 0 && g == 0 && tid == 0 && p.new_lens != nullptr) p.new_lens[b] = over ? p.keep : p.lens[b];
  if (!over) return;
  const int n = len - p.window, m = p.keep - p.window;         // candidates, and how many of them stay
  const float* S = p.weights + (static_cast<long long>(b) * p.c.n_kv_heads + g) * p.stride;
  const PlanView plan = plan_of(p, b, g);

  const int chunk = ((n + CLUSTER - 1) / CLUSTER + 3) & ~3;
  const int c_begin = min(n, rank * chunk), c_end = min(n, c_begin + chunk);
  const int per = CACHED ? ITEMS : (chunk + THREADS - 1) / THREADS;
  const int t_begin = min(c_end, c_begin + tid * per), t_end = min(c_end, t_begin + per);
  const int n_mine = t_end - t_begin;

  uint32_t key[R];
  uint32_t live = 0;               // bit r: candidate r exists and still matches the threshold's prefix
  if (CACHED) {
    const float* mine = S + t_begin;
    if (n_mine == R && R % 4 == 0 && (reinterpret_cast<uintptr_t>(mine) & 15u) == 0) {
#pragma unroll
      for (int r = 0; r < R; r += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(mine + r));
        key[r] = rank_key(v.x); key[r + 1] = rank_key(v.y); key[r + 2] = rank_key(v.z); key[r + 3] = rank_key(v.w);
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) key[r] = r < n_mine ? rank_key(__ldg(mine + r)) : 0u;
    }
    live = n_mine >= 32 ? 0xffffffffu : ((1u << n_mine) - 1u);
  }

  uint32_t tau = 0;
  int k_rem = m;
  if (m > 0) {
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      if (CACHED) {
        if (live != 0) {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if ((live >> r) & 1u) atomicAdd(&sh.hist[((key[r] >> shift) & 0xFFu) * 32 + lane], 1);
        }
      } else {
        for (int i = t_begin; i < t_end; ++i) {
          const uint32_t u = rank_key(__ldg(S + i));
          if (pass == 0 || ((u ^ tau) >> (shift + 8)) == 0) atomicAdd(&sh.hist[((u >> shift) & 0xFFu) * 32 + lane], 1);
        }
      }
      __syncthreads();
      {
        // kPerBin threads per bin, each sums (and clears for the next pass) its share of the 32 lane counters
        const int bin = tid / kPerBin, part = tid % kPerBin;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < 32 / kPerBin; ++i) {
          int* c = &sh.hist[bin * 32 + ((part * (32 / kPerBin) + i + bin) & 31)];
          sum += *c;
          *c = 0;
        }
        if (kPerBin >= 2) sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        if (kPerBin >= 4) sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (part == 0 && sum != 0) {
#pragma unroll
          for (int r = 0; r < CLUSTER; ++r) atomicAdd(cluster.map_shared_rank(&sh.total_hist[pass & 1][bin], r), sum);
        }
      }
      cluster.sync();
      if (warp == 0) {
        // 8 bins per lane, highest bins first: lane 0 owns bins 255..248
        int cnt[8], tot = 0;
        const int4 lo = *reinterpret_cast<const int4*>(&sh.total_hist[pass & 1][248 - lane * 8]);
        const int4 hi = *reinterpret_cast<const int4*>(&sh.total_hist[pass & 1][252 - lane * 8]);
        cnt[0] = hi.w; cnt[1] = hi.z; cnt[2] = hi.y; cnt[3] = hi.x;
        cnt[4] = lo.w; cnt[5] = lo.z; cnt[6] = lo.y; cnt[7] = lo.x;
#pragma unroll
        for (int i = 0; i < 8; ++i) tot += cnt[i];
        int incl = tot;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += v;
        }
        int above = incl - tot;
        if (above < k_rem && k_rem <= incl) {          // exactly one lane holds the k_rem-th largest
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (above < k_rem && k_rem <= above + cnt[i]) {
              sh.digit = 255 - (lane * 8 + i);
              sh.k_rem = k_rem - above;
            }
            above += cnt[i];
          }
        }
      }
      __syncthreads();
      if (tid < kBins) sh.total_hist[pass & 1][tid] = 0;   // for the pass after next; nobody adds into it before the next barrier
      const uint32_t digit = static_cast<uint32_t>(sh.digit);
      tau |= digit << shift;
      k_rem = sh.k_rem;
      if (CACHED && live != 0) {
        uint32_t still = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) still |= (((key[r] >> shift) & 0xFFu) == digit ? 1u : 0u) << r;
        live &= still;
      }
    }
  }
  // tau: image of the smallest weight that stays; need_eq: how many candidates equal to it do
  const int need_eq = m > 0 ? k_rem : 0;
  int n_gt = 0, n_eq = 0;
  if (m > 0) {
    if (CACHED) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        n_gt += (r < n_mine && key[r] > tau) ? 1 : 0;
        n_eq += (r < n_mine && key[r] == tau) ? 1 : 0;
      }
    } else {
      for (int i = t_begin; i < t_end; ++i) {
        const uint32_t u = rank_key(__ldg(S + i));
        n_gt += (u > tau) ? 1 : 0;
        n_eq += (u == tau) ? 1 : 0;
      }
    }
  }
  // exclusive scans in thread order: within the warp, over the warps, over the cluster's CTAs
  int gt_incl = n_gt, eq_incl = n_eq;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int va = __shfl_up_sync(0xffffffffu, gt_incl, o), ve = __shfl_up_sync(0xffffffffu, eq_incl, o);
    if (lane >= o) { gt_incl += va; eq_incl += ve; }
  }
  if (lane == 31) { sh.warp_tot[0][warp] = gt_incl; sh.warp_tot[1][warp] = eq_incl; }
  __syncthreads();
  if (warp == 0) {
    int a = lane < kWarps ? sh.warp_tot[0][lane] : 0, e = lane < kWarps ? sh.warp_tot[1][lane] : 0;
    const int a0 = a, e0 = e;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int va = __shfl_up_sync(0xffffffffu, a, o), ve = __shfl_up_sync(0xffffffffu, e, o);
      if (lane >= o) { a += va; e += ve; }
    }
    if (lane < kWarps) { sh.warp_tot[0][lane] = a - a0; sh.warp_tot[1][lane] = e - e0; }
    const int a_tot = __shfl_sync(0xffffffffu, a, 31), e_tot = __shfl_sync(0xffffffffu, e, 31);
    if (lane < CLUSTER) *reinterpret_cast<int2*>(cluster.map_shared_rank(&sh.counts[rank][0], lane)) = make_int2(a_tot, e_tot);
  }
  __syncthreads();
  const int gt_excl = sh.warp_tot[0][warp] + gt_incl - n_gt, eq_excl = sh.warp_tot[1][warp] + eq_incl - n_eq;
  cluster.sync();
  int eq_before = 0, kept_before = 0;
#pragma unroll
  for (int r = 0; r < CLUSTER; ++r) {
    if (r < rank) {
      kept_before += sh.counts[r][0] + max(0, min(sh.counts[r][1], need_eq - eq_before));
      eq_before += sh.counts[r][1];
    }
  }
  int eq_rank = eq_before + eq_excl;                       // rank of this thread's first candidate equal to tau
  int pos = kept_before + gt_excl + min(eq_rank, need_eq) - min(eq_before, need_eq);    // kept candidates before it
  auto place = [&](int i, uint32_t u) {
    const bool is_eq = u == tau && m > 0;
    const bool kept = m > 0 && (u > tau || (is_eq && eq_rank < need_eq));
    if (i == m) *plan.kept_below = pos;
    if (i < m) plan.hole[i] = kept ? -1 : i - pos;
    else if (kept) plan.from[pos] = i;
    pos += kept ? 1 : 0;
    eq_rank += is_eq ? 1 : 0;
  };
  if (CACHED) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < n_mine) place(t_begin + r, key[r]);
  } else {
    for (int i = t_begin; i < t_end; ++i) place(i, rank_key(__ldg(S + i)));
  }
  // (limit >= keep, so there are more candidates than m, and slot m is one of them)
}

namespace {

constexpr int kMoveThreads = 512, kMoveWarps = kMoveThreads / 32;
constexpr int kRoundRows = 128;            // rows of a round that a CTA holds in shared memory: one page at most, or several

__device__ __forceinline__ uint32_t recode2(uint32_t w, float f) {        // two codes times f <= 1, rounded to nearest even
  uint32_t h;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(w));
  float lo, hi;
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi * f), "f"(lo * f));
  return r;
}
__device__ __forceinline__ uint4 recode16(uint4 v, float f) {
  if (f == 1.0f) return v;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = recode2(w[i] & 0xffffu, f) | (recode2(w[i] >> 16, f) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace

// blockIdx.y: K, V, or weights and ids; blockIdx.z: (sequence, KV head); blockIdx.x: CTA of the cluster.
template <bool kE4M3, int kRowBytes>
__global__ void __launch_bounds__(kMoveThreads, 1) evict_move_kernel(const EvictParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  constexpr int kLanesPerRow = kRowBytes / 16, kRowsPerWarp = 32 / kLanesPerRow;
  __shared__ __align__(16) uint8_t stage[kRoundRows * kRowBytes];
  __shared__ float scale_from[kRoundRows], page_scale[kRoundRows / 16];
  const int CL = gridDim.x, rank = blockIdx.x, kind = blockIdx.y;
  const int b = blockIdx.z / p.c.n_kv_heads, g = blockIdx.z - b * p.c.n_kv_heads;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  pdl_wait();
  bool ok;
  const int len = evict_len(p, b, ok);
  const bool over = len > p.limit;
  const int m = p.keep - p.window, shift = len - p.keep;
  const PlanView plan = plan_of(p, b, g);
  const int kept_below = over ? *plan.kept_below : 0;
  // the slot whose entry slot j of the result takes
  auto origin = [&](int j) -> int {
    if (j >= m) return j + shift;
    const int h = plan.hole[j];
    return h < 0 ? j : plan.from[kept_below + h];
  };
  if (kind == 2) {
    const long long row = (static_cast<long long>(b) * p.c.n_kv_heads + g) * p.stride;
    const int n = over ? p.keep : len;
    for (int j = rank * kMoveThreads + tid; j < n; j += CL * kMoveThreads) {
      const int o = over ? origin(j) : j;
      p.new_weights[row + j] = p.weights[row + o];
      if (p.ids != nullptr) p.new_ids[row + j] = p.ids[row + o];
    }
    return;
  }
  if (!over) return;                                 // (uniform over the cluster)
  uint8_t* const pool = kind == 0 ? p.c.k_pages : p.c.v_pages;
  float* const scales = kind == 0 ? p.c.k_scales : p.c.v_scales;
  const int P = 1 << p.c.page_log2, mask = P - 1;
  const int* const table = p.c.block_table + static_cast<size_t>(b) * p.c.max_pages;
  // block (page, KV head) that holds a slot; -1 and a report for a page that does not exist
  auto block_at = [&](int slot) -> int {
    const long long blk = pool_block(table[slot >> p.c.page_log2], p.c.n_pages, p.c.n_kv_heads, g);
    if (blk < 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_EVICT_PAGE);
    return static_cast<int>(blk);
  };
  auto row_at = [&](int blk, int slot) -> uint8_t* {
    return pool + ((static_cast<long long>(blk) << p.c.page_log2) + (slot & mask)) * kRowBytes;
  };
  const int piece = lane % kLanesPerRow, sub = lane / kLanesPerRow;

  // ---- pages that lie below m: free slots take their entries ----
  const int m0 = m & ~mask;
  const int span = P < 32 ? P : 32;                  // slots of a warp's step; 8-bit pages go by whole pages
  const int gw = rank * kMoveWarps + warp, n_warps = CL * kMoveWarps;
  const int unit = kE4M3 ? P : span;                 // slots a warp takes at a time
  for (int u0 = gw * unit; u0 < m0; u0 += n_warps * unit) {
    const int to_blk = block_at(u0);
    if (to_blk < 0) continue;
    float own = 1.0f, now = 1.0f;                    // 8-bit pages: the page's scale, before and after
    bool again = false;                              // what stays has to be encoded again
    if (kE4M3) {
      own = scales[to_blk];
      float most = 0.0f;
      bool stays = false, comes = false;
      for (int s0 = 0; s0 < P; s0 += 32) {
        if (s0 + lane < P) {
          const int j = u0 + s0 + lane, o = origin(j);
          if (o == j) {
            stays = true;
          } else {
            const int blk = block_at(o);
            if (blk >= 0) { most = fmaxf(most, scales[blk]); comes = true; }
          }
        }
      }
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      stays = __any_sync(0xffffffffu, stays);
      comes = __any_sync(0xffffffffu, comes);
      if (!comes) continue;
      now = stays ? fmaxf(own, most) : most;
      again = stays && now != own;
    }
    for (int s0 = 0; s0 < unit; s0 += 32) {
      // this lane's slot: where its row comes from
      const int j = u0 + s0 + lane;
      int o = -1, blk = -1;
      float f = 1.0f;
      if (s0 + lane < unit) {
        o = origin(j);
        if (o == j && !again) o = -1;
        if (o >= 0) {
          blk = block_at(o);
          if (kE4M3 && blk >= 0) f = scales[blk] / now;
        }
      }
      unsigned todo = __ballot_sync(0xffffffffu, blk >= 0);
      constexpr int kAhead = 4;                      // loads of a lane in flight
      while (todo != 0) {
        uint4 v[kAhead];
        int to[kAhead];
        float by[kAhead];
#pragma unroll
        for (int x = 0; x < kAhead; ++x) {
          // the next rows of the step, one for each group of lanes
          int who = -1;
#pragma unroll
          for (int y = 0; y < kRowsPerWarp; ++y) {
            const int first = __ffs(todo) - 1;
            if (y == sub) who = first;
            if (first >= 0) todo &= todo - 1;
          }
          const int from = __shfl_sync(0xffffffffu, o, max(who, 0)), fb = __shfl_sync(0xffffffffu, blk, max(who, 0));
          by[x] = __shfl_sync(0xffffffffu, f, max(who, 0));
          to[x] = who;
          if (who >= 0) v[x] = *reinterpret_cast<const uint4*>(row_at(fb, from) + piece * 16);
        }
#pragma unroll
        for (int x = 0; x < kAhead; ++x)
          if (to[x] >= 0)
            *reinterpret_cast<uint4*>(row_at(to_blk, u0 + s0 + to[x]) + piece * 16) = kE4M3 ? recode16(v[x], by[x]) : v[x];
      }
    }
    if (kE4M3) {
      __syncwarp();
      if (lane == 0 && now != own) scales[to_blk] = now;
    }
  }

  // ---- the pages from m on, in rounds of kRoundRows slots a CTA ----
  for (int r0 = m0; r0 < p.keep; r0 += CL * kRoundRows) {
    const int j0 = r0 + rank * kRoundRows, rows = max(0, min(kRoundRows, p.keep - j0));
    constexpr int kGroups = kMoveThreads / kLanesPerRow;
    const int grp = tid / kLanesPerRow;
    for (int i = grp; i < rows; i += kGroups) {
      const int o = origin(j0 + i), blk = block_at(o);
      if (blk >= 0) *reinterpret_cast<uint4*>(stage + i * kRowBytes + piece * 16) = *reinterpret_cast<const uint4*>(row_at(blk, o) + piece * 16);
      if (piece == 0) scale_from[i] = blk < 0 ? -1.0f : kE4M3 ? scales[blk] : 1.0f;      // -1: a row that is not to be had
    }
    __syncthreads();
    if (kE4M3) {
      for (int q = tid; q * P < rows; q += kMoveThreads) {
        float most = 0.0f;
        for (int i = q * P; i < min(rows, (q + 1) * P); ++i) most = fmaxf(most, scale_from[i]);
        page_scale[q] = most;
      }
    }
    cluster.sync();                                  // everybody has read the round
    for (int i = grp; i < rows; i += kGroups) {
      const int j = j0 + i;
      if (scale_from[i] < 0.0f) continue;
      const int blk = block_at(j);
      if (blk < 0) continue;
      uint4 v = *reinterpret_cast<const uint4*>(stage + i * kRowBytes + piece * 16);
      if (kE4M3) v = recode16(v, scale_from[i] / page_scale[i >> p.c.page_log2]);
      *reinterpret_cast<uint4*>(row_at(blk, j) + piece * 16) = v;
    }
    if (kE4M3) {
      for (int q = tid; q * P < rows; q += kMoveThreads) {
        const int blk = block_at(j0 + q * P);
        if (blk >= 0 && page_scale[q] > 0.0f) scales[blk] = page_scale[q];
      }
    }
    __syncthreads();                                 // the stage is free again
  }
}

namespace {

template <int CLUSTER, int ITEMS, int THREADS>
cudaError_t launch_plan_t(const EvictParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(CLUSTER, p.c.n_kv_heads, p.c.batch);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CLUSTER;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  fill_pdl_attribute(&attr[1]);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, evict_plan_kernel<CLUSTER, ITEMS, THREADS>, p);
}

}  // namespace

cudaError_t launch_evict_plan(const EvictParams& p, cudaStream_t stream) {
  const int n = p.max_len - p.window;                // the most candidates
  if (n <= 4 * 256) return launch_plan_t<1, 4, 256>(p, stream);
  if (n <= 16 * 256) return launch_plan_t<1, 16, 256>(p, stream);
  if (n <= 2 * 16 * 256) return launch_plan_t<2, 16, 256>(p, stream);
  if (n <= 4 * 16 * 256) return launch_plan_t<4, 16, 256>(p, stream);
  if (n <= 8 * 4 * 1024) return launch_plan_t<8, 4, 1024>(p, stream);
  if (n <= 8 * 16 * 1024) return launch_plan_t<8, 16, 1024>(p, stream);
  return launch_plan_t<8, 0, 1024>(p, stream);
}

namespace {

template <bool kE4M3, int kRowBytes>
cudaError_t launch_move_t(const EvictParams& p, cudaStream_t stream) {
  // CTAs of a cluster: as many as keep all SMs busy with few pairs
  const long long pairs = static_cast<long long>(p.c.batch) * p.c.n_kv_heads;
  int cl = 8;
  while (cl > 1 && (pairs * 2 * cl > 4 * 148 || cl * kRoundRows >= 4 * p.keep)) cl /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cl, 3, static_cast<unsigned>(pairs));
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  fill_pdl_attribute(&attr[1]);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, evict_move_kernel<kE4M3, kRowBytes>, p);
}

}  // namespace

cudaError_t launch_evict_move(const EvictParams& p, bool e4m3, cudaStream_t stream) {
  if (p.row_bytes == 256) return launch_move_t<false, 256>(p, stream);
  if (p.row_bytes == 128) return e4m3 ? launch_move_t<true, 128>(p, stream) : launch_move_t<false, 128>(p, stream);
  if (p.row_bytes == 64) return launch_move_t<true, 64>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
