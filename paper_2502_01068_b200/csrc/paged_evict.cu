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
// What bounds it: latency.  The bytes of a cut (2304 entries to 2048: 256 rows of K and V per KV head and the weights) are few, and each row
// is found by loads that wait for one another: slot, source, page, (scale,) row.  One B200, 8 KV heads of 128: one sequence of 2304 15 us
// (ranking 5, an empty launch 2 each), 131072 to 13107 51 us (ranking 20: 64 CTAs, 4 us until the weights are there, 2 a digit; moving
// 25 for 102 MB, 62 % of a copy).  In 8 bits 64 of 2304 take 84 us and 4 of 26214 to 13107 102 on pages as appends leave them, where entries that
// stay in a page whose scale grows are read and encoded again; on pages whose scales are equal already 40 and 65 (moving 28 and 40), which is
// what calls in a row on the same pages measure.  More warps on an SM (48 or 40 registers a thread) gained nothing in 8 bits: 42 and 41 us, 68 and
// 74 on equal scales (39 and 69 at the time).
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
  int* free_slot;                  // [m]: the free slots in ascending order
  int* page_first;                 // [pages below m, + 1]: free slots before the page
};
__device__ __forceinline__ PlanView plan_of(const EvictParams& p, int b, int g) {
  const int m = p.keep - p.window;
  int* base = p.plan + (static_cast<long long>(b) * p.c.n_kv_heads + g) * p.plan_words;
  return {base, base + 1, base + 1 + m, base + 1 + 2ll * m, base + 1 + 3ll * m};
}

// Copies of the digit histogram, so that the lanes of a warp seldom meet on one counter: all 32 in blocks of 1024 threads, which sum them
// quickly; 8 in blocks of 256, where summing (and clearing) 32 cost more than the meetings (2304 candidates: 12.8 us and 7).
template <int THREADS> constexpr int kCopies = THREADS >= 1024 ? 32 : 8;

template <int THREADS>
struct alignas(16) PlanShared {
  int hist[kBins * kCopies<THREADS>];      // hist[bin * copies + lane % copies]
  int total_hist[2][kBins];        // the cluster's histogram of a pass (every CTA adds into it), double-buffered by pass parity
  int warp_tot[2][THREADS / 32];
  alignas(8) int counts[8][2];     // per CTA of the cluster: (#above threshold, #equal to it)
  int digit, k_rem, whole;
};

}  // namespace

// A warp owns consecutive candidates of its CTA's chunk, 32 a row, a lane each: slot order is warp, row, lane, and what comes before a
// candidate in its row is a ballot's.  ITEMS > 0: up to so many rows stay in registers for all passes; ITEMS == 0: any number, read again for
// every pass.
template <int CLUSTER, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_plan_kernel(const EvictParams p) {
  constexpr int kWarps = THREADS / 32, kPerBin = THREADS / kBins, kCopy = kCopies<THREADS>;
  static_assert(THREADS % kBins == 0 && kPerBin >= 1 && kPerBin <= 4, "256, 512 or 1024 threads");
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ PlanShared<THREADS> sh;
  constexpr bool CACHED = ITEMS > 0;
  constexpr int R = CACHED ? ITEMS : 1;
  const int rank = static_cast<int>(cluster.block_rank());
  const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  auto everybody = [&]() {         // a barrier of the cluster
    if constexpr (CLUSTER == 1) __syncthreads(); else cluster.sync();
  };
  if (CLUSTER > 1)
    for (int i = tid; i < 2 * kBins; i += THREADS) (&sh.total_hist[0][0])[i] = 0;
  for (int i = tid; i < kBins * kCopy; i += THREADS) sh.hist[i] = 0;
  everybody();                     // nobody adds into a histogram that is not cleared yet
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
  const int n_rows = (c_end - c_begin + THREADS - 1) / THREADS;             // of a warp; at most ITEMS
  const int first = c_begin + warp * n_rows * 32 + lane;                    // this lane's candidate of the warp's first row
  const int end = c_begin + min(c_end - c_begin, (warp + 1) * n_rows * 32);

  uint32_t key[R];
  uint32_t live = 0;               // bit r: candidate r exists and still matches the threshold's prefix
  if (CACHED) {
    float w[R];                    // (all loads first, whatever the row: in a branch each would wait for the one before)
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = __ldg(S + max(min(first + r * 32, end - 1), 0));
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool there = r < n_rows && first + r * 32 < end;
      key[r] = there ? rank_key(w[r]) : 0u;
      live |= (there ? 1u : 0u) << r;
    }
  }
  // every row of the warp: f(candidate, whether this lane has one, its key)
  auto rows = [&](auto&& f) {
    if constexpr (CACHED) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (r < n_rows) f(first + r * 32, first + r * 32 < end, key[r]);
    } else {
      for (int r = 0; r < n_rows; ++r) {
        const int i = first + r * 32;
        f(i, i < end, i < end ? rank_key(__ldg(S + i)) : 0u);
      }
    }
  };

  uint32_t tau = 0;
  int k_rem = m;
  if (m > 0) {
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      if (CACHED) {
        if (live != 0) {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if ((live >> r) & 1u) atomicAdd(&sh.hist[((key[r] >> shift) & 0xFFu) * kCopy + lane % kCopy], 1);
        }
      } else {
        rows([&](int, bool there, uint32_t u) {
          if (there && (pass == 0 || ((u ^ tau) >> (shift + 8)) == 0)) atomicAdd(&sh.hist[((u >> shift) & 0xFFu) * kCopy + lane % kCopy], 1);
        });
      }
      __syncthreads();
      {
        // kPerBin threads per bin, each sums (and clears for the next pass) its share of the copies
        const int bin = tid / kPerBin, part = tid % kPerBin;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kCopy / kPerBin; i += 4) {        // (the start is rotated by bin: neighbours use different banks)
          int4* c = reinterpret_cast<int4*>(&sh.hist[bin * kCopy + ((part * (kCopy / kPerBin) + i + 4 * bin) & (kCopy - 1))]);
          const int4 v = *c;
          sum += (v.x + v.y) + (v.z + v.w);
          *c = make_int4(0, 0, 0, 0);
        }
        if (kPerBin >= 2) sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        if (kPerBin >= 4) sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (CLUSTER == 1) {
          if (part == 0) sh.total_hist[pass & 1][bin] = sum;
        } else if (part == 0 && sum != 0) {
#pragma unroll
          for (int r = 0; r < CLUSTER; ++r) atomicAdd(cluster.map_shared_rank(&sh.total_hist[pass & 1][bin], r), sum);
        }
      }
      everybody();
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
              sh.whole = cnt[i] == k_rem - above;
            }
            above += cnt[i];
          }
        }
      }
      __syncthreads();
      if (CLUSTER > 1 && tid < kBins) sh.total_hist[pass & 1][tid] = 0;   // for the pass after next; nobody adds into it before the next barrier
      const uint32_t digit = static_cast<uint32_t>(sh.digit);
      tau |= digit << shift;
      k_rem = sh.k_rem;
      // All that match the prefix stay: no more digits (with zeros for them the threshold is at or below each, and those equal to it are no
      // more than k_rem).
      if (sh.whole) break;
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
  int n_gt = 0, n_eq = 0;          // of the warp
  if (m > 0) {
    rows([&](int, bool there, uint32_t u) {
      n_gt += __popc(__ballot_sync(0xffffffffu, there && u > tau));
      n_eq += __popc(__ballot_sync(0xffffffffu, there && u == tau));
    });
  }
  // before this warp's: scans over the CTA's warps and over the cluster's CTAs
  if (lane == 0) { sh.warp_tot[0][warp] = n_gt; sh.warp_tot[1][warp] = n_eq; }
  __syncthreads();
  int gt_before = 0, eq_before = 0, gt_cta = 0, eq_cta = 0;
  {
    const int a0 = lane < kWarps ? sh.warp_tot[0][lane] : 0, e0 = lane < kWarps ? sh.warp_tot[1][lane] : 0;
    gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? a0 : 0);
    eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? e0 : 0);
    gt_cta = __reduce_add_sync(0xffffffffu, a0);
    eq_cta = __reduce_add_sync(0xffffffffu, e0);
  }
  int kept_ctas = 0, eq_ctas = 0;  // kept candidates, and candidates equal to tau, of the CTAs before
  if constexpr (CLUSTER > 1) {
    if (warp == 0 && lane < CLUSTER) *reinterpret_cast<int2*>(cluster.map_shared_rank(&sh.counts[rank][0], lane)) = make_int2(gt_cta, eq_cta);
    cluster.sync();
#pragma unroll
    for (int r = 0; r < CLUSTER; ++r) {
      if (r < rank) {
        kept_ctas += sh.counts[r][0] + max(0, min(sh.counts[r][1], need_eq - eq_ctas));
        eq_ctas += sh.counts[r][1];
      }
    }
  }
  int eq_rank = eq_ctas + eq_before;                       // of the warp's next candidate equal to tau
  int pos = kept_ctas + gt_before + min(eq_rank, need_eq) - min(eq_ctas, need_eq);      // kept candidates before the warp's next row
  const uint32_t below = (1u << lane) - 1u;
  rows([&](int i, bool there, uint32_t u) {
    const bool eq = there && u == tau && m > 0;
    const uint32_t all_eq = __ballot_sync(0xffffffffu, eq);
    const bool kept = there && m > 0 && (u > tau || (eq && eq_rank + __popc(all_eq & below) < need_eq));
    const uint32_t all_kept = __ballot_sync(0xffffffffu, kept);
    const int at = pos + __popc(all_kept & below);         // kept candidates before this one
    if (there) {
      if (i <= m && (i & ((1 << p.c.page_log2) - 1)) == 0) plan.page_first[i >> p.c.page_log2] = i - at;
      if (i == m) *plan.kept_below = at;
      if (i < m) {
        plan.hole[i] = kept ? -1 : i - at;
        if (!kept) plan.free_slot[i - at] = i;
      } else if (kept) {
        plan.from[at] = i;
      }
    }
    pos += __popc(all_kept);
    eq_rank += __popc(all_eq);
  });
  // (limit >= keep, so there are more candidates than m, and slot m is one of them)
}

namespace {

// Rows of a round that a CTA holds in shared memory are a multiple of kRowsUnit, so that pages are whole: as many as a window of the call
// needs for one round, up to kStageMost bytes (one CTA an SM, or three).  A round waits for reads, a barrier of the cluster and writes,
// whatever its size: 25647 entries cut to their last 17173, in 8 bits, took 111 us in 17 rounds of 128 rows a CTA, in two rounds 46.
constexpr int kRowsUnit = 128;
template <int THREADS> constexpr int kStageMost = THREADS >= 1024 ? 160 << 10 : 64 << 10;
constexpr int kHeld = 3;                    // 8-bit pages: free slots that a lane holds at a time (2: 75 us for four of 26214, 3: 72)
constexpr int kOwnPages = 16;              // 8-bit pages that a warp takes at a time, at most

__device__ __forceinline__ uint32_t recode2(uint32_t w, float f) {        // two codes times f <= 1, rounded to nearest even
  uint32_t h;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(w));
  float lo, hi;
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi * f), "f"(lo * f));
  return r;
}
// Sixteen codes times f <= 1, a power of two.  Conversions are slow (an SM does 16 a cycle, and two codes take two of them), so four codes
// that are all normal numbers before and after, and not NaN, have their exponents lowered in one subtraction.
__device__ __forceinline__ uint4 recode16(uint4 v, float f) {
  if (f == 1.0f) return v;
  const uint32_t bits = __float_as_uint(f);
  const int down = 127 - static_cast<int>(bits >> 23);                    // f = 2^-down
  const bool plain = (bits & 0x7fffffu) == 0u && down > 0 && down < 14;
  const uint32_t by = static_cast<uint32_t>(plain ? down : 0) * 0x08080808u;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // every byte: the exponent is above `down` (the sum stays at 0x80 or above), and the code is not all ones
    const uint32_t above = ((w[i] & 0x78787878u) | 0x80808080u) - by - 0x08080808u, nan = (w[i] & 0x7f7f7f7fu) + 0x01010101u;
    if (plain && (above & ~nan & 0x80808080u) == 0x80808080u) w[i] -= by;
    else w[i] = recode2(w[i] & 0xffffu, f) | (recode2(w[i] >> 16, f) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16 bytes from memory to shared memory, on their way until copies_wait().
__device__ __forceinline__ void copy16_async(uint8_t* to, const uint8_t* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

}  // namespace

// blockIdx.y: K, V, or weights and ids; blockIdx.z: (sequence, KV head); blockIdx.x: CTA of the cluster.
template <bool kE4M3, int kRowBytes, int kMoveThreads>
__global__ void __launch_bounds__(kMoveThreads, 1024 / kMoveThreads) evict_move_kernel(const EvictParams p) {
  constexpr int kMoveWarps = kMoveThreads / 32;
  cg::cluster_group cluster = cg::this_cluster();
  constexpr int kLanesPerRow = kRowBytes / 16, kRowsPerWarp = 32 / kLanesPerRow;
  // rows of a round (before the rounds, the warps' lists of moves); their scales, or -1; the new scales of their pages
  extern __shared__ __align__(16) uint8_t stage[];
  float* const scale_from = reinterpret_cast<float*>(stage + p.stage_bytes);
  float* const page_scale = scale_from + p.round_rows;
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
  const int gw = warp * CL + rank, n_warps = CL * kMoveWarps;
  // Rows that the lanes name (from `from`, null: none, to `to`, in 8 bits times f) move, several at a time: the warp's list of them lies in
  // shared memory, and a group of lanes takes every kRowsPerWarp-th.
  struct Move { const uint8_t* from; uint8_t* to; };
  static_assert(sizeof(Move) == 16, "what the lists have room for");
  Move* const moves = reinterpret_cast<Move*>(stage) + warp * 32;
  __shared__ float move_scale[kMoveWarps][kE4M3 ? 32 : 1];
  auto move_rows = [&](const uint8_t* from, uint8_t* to, float f) {
    const unsigned have = __ballot_sync(0xffffffffu, from != nullptr);
    if (from != nullptr) {
      const int at = __popc(have & ((1u << lane) - 1u));
      moves[at] = {from, to};
      if (kE4M3) move_scale[warp][at] = f;
    }
    __syncwarp();
    const int n = __popc(have);
    constexpr int kAhead = 4;                        // loads of a lane in flight: more cost the warps that hide the rest (8: 74 -> 97 us, four of 26214)
    for (int i0 = sub; i0 < n; i0 += kAhead * kRowsPerWarp) {
      uint4 v[kAhead];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int i = i0 + x * kRowsPerWarp;
        if (i < n) v[x] = *reinterpret_cast<const uint4*>(moves[i].from + piece * 16);
      }
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int i = i0 + x * kRowsPerWarp;
        if (i < n) *reinterpret_cast<uint4*>(moves[i].to + piece * 16) = kE4M3 ? recode16(v[x], move_scale[warp][i]) : v[x];
      }
    }
    __syncwarp();
  };
  if constexpr (!kE4M3) {
    // Free slots in any order, an even share of them a warp, 64 at a time: a move is found by three loads that wait for one another, so several of them at once.
    const int n_free = plan.page_first[m0 >> p.c.page_log2];
    const int share = (n_free + n_warps - 1) / n_warps, end = min(n_free, (gw + 1) * share);
    for (int h0 = gw * share; h0 < end; h0 += 64) {
      int dst[2], src[2];
      const uint8_t* from[2];
      uint8_t* to[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int h = min(h0 + z * 32 + lane, end - 1);
        dst[z] = plan.free_slot[h];
        src[z] = plan.from[kept_below + h];
      }
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int dst_blk = block_at(dst[z]), src_blk = block_at(src[z]);
        const bool there = h0 + z * 32 + lane < end && dst_blk >= 0 && src_blk >= 0;
        from[z] = there ? row_at(src_blk, src[z]) : nullptr;
        to[z] = there ? row_at(dst_blk, dst[z]) : nullptr;
      }
#pragma unroll
      for (int z = 0; z < 2; ++z) move_rows(from[z], to[z], 1.0f);
    }
  } else {
    // A warp takes several pages whole: first every page's new scale, and which of its slots are free, then the rows.
    __shared__ unsigned most_of[kMoveWarps][kOwnPages], free_of[kMoveWarps][kOwnPages][4];
    __shared__ uint8_t again_of[kMoveWarps][kOwnPages];
    const int n_pages = m0 >> p.c.page_log2;
    // an even share, in as many parts as it takes for one to have no more than some 96 free slots: those stay in the lanes' registers
    const int most_pages = min(kOwnPages, max(1, n_pages == 0 ? 1 : static_cast<int>(32ll * kHeld * n_pages / max(plan.page_first[n_pages], 1))));
    const int parts = max(1, (n_pages + n_warps * most_pages - 1) / (n_warps * most_pages));
    const int per = max(1, (n_pages + n_warps * parts - 1) / (n_warps * parts));
    for (int pa = gw * per; pa < n_pages; pa += n_warps * per) {
      const int pb = min(pa + per, n_pages);
      const int first = plan.page_first[pa + min(lane, pb - pa)];            // of page pa + lane, and behind the last
      const int ha = __shfl_sync(0xffffffffu, first, 0), hb = __shfl_sync(0xffffffffu, first, pb - pa);
      if (ha == hb) continue;
      const int n_own = __shfl_down_sync(0xffffffffu, first, 1) - first;     // free slots of page pa + lane
      if (lane < kOwnPages) {
        most_of[warp][lane] = 0u;
        for (int z = 0; z < 4; ++z) free_of[warp][lane][z] = 0u;
      }
      int own_blk = -1;
      float own = 1.0f;
      if (pa + lane < pb && n_own > 0) {
        own_blk = block_at((pa + lane) << p.c.page_log2);
        if (own_blk >= 0) own = scales[own_blk];
      }
      __syncwarp();
      // kHeld free slots of the warp's pages a lane, from h0 on: three loads that wait for one another, so several of them at once
      int src[kHeld], dst[kHeld], src_blk[kHeld];
      float was[kHeld];
      auto take = [&](int h0) {
#pragma unroll
        for (int z = 0; z < kHeld; ++z) {
          const int h = min(h0 + z * 32 + lane, hb - 1);
          dst[z] = plan.free_slot[h];
          src[z] = plan.from[kept_below + h];
        }
#pragma unroll
        for (int z = 0; z < kHeld; ++z) src_blk[z] = block_at(src[z]);
#pragma unroll
        for (int z = 0; z < kHeld; ++z) was[z] = scales[max(src_blk[z], 0)];
      };
      for (int h0 = ha; h0 < hb; h0 += 32 * kHeld) {
        take(h0);
#pragma unroll
        for (int z = 0; z < kHeld; ++z) {
          if (h0 + z * 32 + lane < hb) {
            const int pg = (dst[z] >> p.c.page_log2) - pa, slot = dst[z] & mask;
            atomicOr(&free_of[warp][pg][slot >> 5], 1u << (slot & 31));
            if (src_blk[z] >= 0) atomicMax(&most_of[warp][pg], __float_as_uint(was[z]));     // (positive: their bits compare alike)
          }
        }
      }
      __syncwarp();
      // lane = page: the new scale, and what becomes of the entries that stay
      float now = own;
      bool again = false;
      if (own_blk >= 0) {
        const float most = __uint_as_float(most_of[warp][lane]);
        const bool stays = n_own < P;
        now = stays ? fmaxf(own, most) : most > 0.0f ? most : own;
        again = stays && now != own;
      }
      const unsigned pages_again = __ballot_sync(0xffffffffu, again);
      if (again) again_of[warp][__popc(pages_again & ((1u << lane) - 1u))] = static_cast<uint8_t>(lane);
      __syncwarp();
      for (int r0 = 0, rows = __popc(pages_again) << p.c.page_log2; r0 < rows; r0 += 32) {
        const int pg = r0 + lane < rows ? again_of[warp][(r0 + lane) >> p.c.page_log2] : 0, r = (r0 + lane) & mask;
        const int blk = __shfl_sync(0xffffffffu, own_blk, pg);
        const float f = __shfl_sync(0xffffffffu, own, pg) / __shfl_sync(0xffffffffu, now, pg);
        const bool mine = r0 + lane < rows && ((free_of[warp][pg][r >> 5] >> (r & 31)) & 1u) == 0;
        uint8_t* const at = mine ? row_at(blk, r) : nullptr;
        move_rows(at, at, f);
      }
      for (int h0 = ha; h0 < hb; h0 += 32 * kHeld) {
        if (hb - ha > 32 * kHeld) take(h0);          // (otherwise the lanes still hold them)
#pragma unroll
        for (int z = 0; z < kHeld; ++z) {
          if (h0 + z * 32 >= hb) break;              // (uniform)
          const bool there = h0 + z * 32 + lane < hb;
          const int pg = there ? (dst[z] >> p.c.page_log2) - pa : 0;
          const int dst_blk = __shfl_sync(0xffffffffu, own_blk, pg);
          const float to = __shfl_sync(0xffffffffu, now, pg);
          const bool moves_on = there && dst_blk >= 0 && src_blk[z] >= 0;
          move_rows(moves_on ? row_at(src_blk[z], src[z]) : nullptr, moves_on ? row_at(dst_blk, dst[z]) : nullptr, was[z] / to);
        }
      }
      if (own_blk >= 0 && now != own) scales[own_blk] = now;
      __syncwarp();                                  // the masks are free again
    }
  }

  // ---- the pages from m on, in rounds of some slots a CTA: a lane looks a row up, the warp copies it ----
  __syncthreads();                                   // the lists have been read
  const int R = p.round_rows;
  for (int r0 = m0; r0 < p.keep; r0 += CL * R) {
    const int j0 = r0 + rank * R, rows = max(0, min(R, p.keep - j0));
    for (int i0 = warp * 32; i0 < rows; i0 += kMoveThreads) {
      const int i = i0 + lane;
      const uint8_t* from = nullptr;
      if (i < rows) {
        const int o = origin(j0 + i), blk = block_at(o);
        if (blk >= 0) from = row_at(blk, o);
        scale_from[i] = blk < 0 ? -1.0f : kE4M3 ? scales[blk] : 1.0f;        // -1: a row that is not to be had
      }
#pragma unroll
      for (int r = 0; r < 32; r += kRowsPerWarp) {
        const unsigned long long src = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(from), r + sub);
        if (src != 0) copy16_async(stage + (i0 + r + sub) * kRowBytes + piece * 16, reinterpret_cast<const uint8_t*>(src) + piece * 16);
      }
    }
    copies_wait();
    __syncthreads();
    if (kE4M3) {
      // the largest scale of each page's rows (positive: their bits compare alike)
      for (int q = tid; q * 16 < rows; q += kMoveThreads) page_scale[q] = 0.0f;
      __syncthreads();
      for (int i = tid; i < rows; i += kMoveThreads) {
        const float most = scale_from[i];
        if (most > 0.0f) atomicMax(reinterpret_cast<unsigned*>(&page_scale[i >> p.c.page_log2]), __float_as_uint(most));
      }
    }
    cluster.sync();                                  // everybody has read the round
    for (int i0 = warp * 32; i0 < rows; i0 += kMoveThreads) {
      const int i = i0 + lane;
      uint8_t* to = nullptr;
      float f = 1.0f;
      if (i < rows && scale_from[i] >= 0.0f) {
        const int blk = block_at(j0 + i);
        if (blk >= 0) to = row_at(blk, j0 + i);
        if (kE4M3) f = scale_from[i] / page_scale[i >> p.c.page_log2];
      }
#pragma unroll
      for (int r = 0; r < 32; r += kRowsPerWarp) {
        const unsigned long long dst = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), r + sub);
        const float by = kE4M3 ? __shfl_sync(0xffffffffu, f, r + sub) : 1.0f;
        if (dst != 0) {
          const uint4 v = *reinterpret_cast<const uint4*>(stage + (i0 + r + sub) * kRowBytes + piece * 16);
          *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(dst) + piece * 16) = kE4M3 ? recode16(v, by) : v;
        }
      }
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
  // short sequences: a CTA each, of 512 threads as long as all of them run at once, else of 256
  if (n <= 16 * 256) {
    if (static_cast<long long>(p.c.batch) * p.c.n_kv_heads <= 2 * 148) return n <= 2 * 512 ? launch_plan_t<1, 2, 512>(p, stream) : launch_plan_t<1, 8, 512>(p, stream);
    return n <= 4 * 256 ? launch_plan_t<1, 4, 256>(p, stream) : launch_plan_t<1, 16, 256>(p, stream);
  }
  // longer ones: clusters of CTAs of 512 threads and up to 16 candidates a thread, as small as the length allows when there are many
  const long long pairs = static_cast<long long>(p.c.batch) * p.c.n_kv_heads;
  if (n <= 2 * 16 * 512) return pairs * 4 <= 148 ? launch_plan_t<4, 8, 512>(p, stream) : launch_plan_t<2, 16, 512>(p, stream);
  if (n <= 4 * 16 * 512) return pairs * 8 <= 148 ? launch_plan_t<8, 8, 512>(p, stream) : launch_plan_t<4, 16, 512>(p, stream);
  if (n <= 8 * 16 * 512) return launch_plan_t<8, 16, 512>(p, stream);
  if (n <= 8 * 16 * 1024) return launch_plan_t<8, 16, 1024>(p, stream);
  return launch_plan_t<8, 0, 1024>(p, stream);
}

namespace {

template <bool kE4M3, int kRowBytes, int kThreads>
cudaError_t launch_move_t(EvictParams p, int cl, cudaStream_t stream) {
  // the window and what of m's page lies below it
  const long long rows = p.window + ((p.keep - p.window) & ((1 << p.c.page_log2) - 1)), unit = kRowsUnit;
  const long long each = (rows + cl * unit - 1) / (cl * unit) * unit, most = kStageMost<kThreads> / kRowBytes / unit * unit;
  p.round_rows = static_cast<int>(max(unit, min(each, most)));
  p.stage_bytes = max(p.round_rows * kRowBytes, kThreads * 16);
  constexpr int kMost = kStageMost<kThreads> + kStageMost<kThreads> / kRowBytes * 5;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(evict_move_kernel<kE4M3, kRowBytes, kThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    configured.set(dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cl, 3, static_cast<unsigned>(p.c.batch * p.c.n_kv_heads));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = p.stage_bytes + p.round_rows * 5;         // (a scale a row, and one for 16 of them)
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  fill_pdl_attribute(&attr[1]);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, evict_move_kernel<kE4M3, kRowBytes, kThreads>, p);
}

template <bool kE4M3, int kRowBytes>
cudaError_t launch_move_r(const EvictParams& p, cudaStream_t stream) {
  // CTAs of a cluster: as many as keep all SMs busy with few pairs; where even eight leave SMs with one CTA or none, large ones
  const long long pairs = static_cast<long long>(p.c.batch) * p.c.n_kv_heads;
  int cl = 8;
  while (cl > 1 && (pairs * 2 * cl > 4 * 148 || cl * kRowsUnit >= 4 * p.keep)) cl /= 2;
  if (cl == 8 && pairs * 2 * cl <= 148) return launch_move_t<kE4M3, kRowBytes, 1024>(p, cl, stream);
  return launch_move_t<kE4M3, kRowBytes, 256>(p, cl, stream);
}

}  // namespace

cudaError_t launch_evict_move(const EvictParams& p, bool e4m3, cudaStream_t stream) {
  if (p.row_bytes == 256) return launch_move_r<false, 256>(p, stream);
  if (p.row_bytes == 128) return e4m3 ? launch_move_r<true, 128>(p, stream) : launch_move_r<false, 128>(p, stream);
  if (p.row_bytes == 64) return launch_move_r<true, 64>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
