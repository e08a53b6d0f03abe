// Attention of a few new query tokens per sequence over the paged cache, in bf16 or in 8-bit codes with a power-of-two scale
// for each (page, KV head).
//
//   out[b, i, h] = sum_t softmax_t(scale <q[b, i, h], K[t, h / G]>) V[t, h / G],   t < len_b - (q_len - 1 - i)
//
// Memory-bound: every cached K and V row is read once (2 d bytes per entry and KV head in 8 bits, 4 d in bf16) for the G * q_len
// query rows that share it.  The products run as warp-level m16n8k16 tensor-core products, whose only job is to keep the
// instruction count per entry low; a tcgen05 tile has 128 rows and these have 8 or 16.
//
// Split-KV: a CTA takes a split of the entries of one (sequence, KV head, tile of query rows), or an even share of all of them;
// inside it four warps compute, each with a ring of shared-memory stages that a warp of its own fills with tiled TMA copies (32
// entries of K and V a stage in 8 bits, 16 in bf16) and its own online softmax.
//   S [rows x 16 entries] = Q K^T: A = the query rows, B = K rows as stored;
//   O^T [d x rows] += V^T P^T:     A = V through the transposing matrix load, B = P in the layout S comes out in.
// Pages hold 16 rows or more, so that a step of 16 entries never straddles two pages.
//
// 8-bit pages: a code is exact in fp16, so K and V are widened in registers and the products are fp16 x fp16 -> fp32 (warp-level
// products of 8-bit operands are no native instruction here: a step of theirs took 30 cycles against 8).  The queries (bf16) go
// into fp16 after a power-of-two shift per row that brings the row's largest element to [2^14, 2^15): exact down to 2^-28 of it,
// and what is smaller is off by at most 2^-39 of the largest.  K's scale multiplies the logits.  V's scale stays out of the weights,
// whose range in fp16 is short: the codes of a step (16 or 32 entries of one page) are summed with weights 2^(l - m) that count from the
// step's own largest logit m, and the sum joins the running outputs in fp32, times V's scale and 2^(m - M).  So neither the
// scales of other pages nor the weights of other steps cost a step's entries any of their bits.  Pages of 16 join twice as often (32
// sequences of up to 1638 entries, four query tokens: 28.9 us, with pages of 128 26.9).
// P goes in as 16-bit terms (value and rounding remainders).  Three in bf16: 24 bits, whatever the weight.  Two in fp16: 22 bits, or
// (both terms rounded to a multiple of 2^-24, the weights 2^15 times too large) off by at most 2^-39 of the step's largest weight: all
// in all 2^-22 of sum p |v| and, step by step, 2^-39 of the largest weight times the sum of the |v|.
//
// Measured, in us (and the share of a plain copy's bandwidth over the bytes the entries take): one sequence of 131072 entries,
// 8 bits, 46.6 (88 %); eight of 4K to 64K, 107 (91 %); 64 of 1638 to 2048, bf16, 75 (98 %); 32 of 819 to 1638 with four query
// tokens, 8 bits, 27 (48 %: two row tiles double the products and the softmax, so that the instructions bound it); 257 entries 5.1:
// launch, table -> page -> copy, one pass, merge.
#include <type_traits>

#include "paged.cuh"

namespace fastkv {

namespace {

constexpr int kSub = 16;            // entries of one step of the second product; a page holds a whole number of them
// 8-bit pages: the weights of the second product are 2^15 times too large, so that the remainder term of the largest of them is far
// from fp16's subnormals, and the running outputs 2^16 times too small, between fp32's two ends: 2^15 entries of the largest value,
// 448 * 2^120, and all weights together stay finite, and a weight times V's scale keeps its bits down to 2^-95.
constexpr float kWeightGain = 32768.0f, kOutGain = 65536.0f;
constexpr float kScaleGain = 1.0f / (kWeightGain * kOutGain);   // what V's scale, 2^-64 or more, is multiplied by at the join

__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// D[16x8] += A[16x16] B[16x8], fp32 accumulators; `first`: D = A B.
template <bool kHalf>
__device__ __forceinline__ void mma16(float (&c)[4], bool first, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  const float z0 = first ? 0.0f : c[0], z1 = first ? 0.0f : c[1], z2 = first ? 0.0f : c[2], z3 = first ? 0.0f : c[3];
  if constexpr (kHalf)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
}
// Two floats to a pair of 16-bit values (`lo` in the low half), and what the rounding left over.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if constexpr (kHalf) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool kHalf>
__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi) {
  if constexpr (kHalf) {
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(w));
  } else {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
  }
}
// The two low, or the two high, codes of a word as fp16 values.
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, b;\n\t}" : "=r"(r) : "r"(w));
  return r;
}

// All ones in the elements of a word that are NaN or infinite.
template <bool kE4M3>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return kE4M3 ? __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) : __vcmpeq2(w & 0x7f807f80u, 0x7f807f80u);
}

// A CTA is four warps that compute and four that bring the data, one for each of them; two CTAs per SM.  The chain from a chunk's
// logits to its outputs is long and every warp walks it alone, so what counts is how much independent work the compiler can
// weave into it, and that takes registers: the launch's 128 a thread are split 216 to 40.  Starting a chunk's copies (page, box,
// barrier) held a computing warp up for ~600 cycles, a third of its pass; a warp of its own does it in the meantime and runs
// ahead into the CTA's next segment.
constexpr int kWarps = 4, kComputing = 32 * kWarps, kThreads = 2 * kComputing;
constexpr int kLaunchRegs = 128, kComputeRegs = 216, kBringRegs = 40;
static_assert(kComputeRegs + kBringRegs == 2 * kLaunchRegs, "the warpgroups' shares add up to what the CTA was launched with");
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// kOwnPage: 8-bit pages of 16 entries, where the two halves of a chunk lie in different pages.
template <int D, bool kE4M3, int RT, bool kOwnPage>
struct PagedCfg {
  static constexpr int kItem = kE4M3 ? 1 : 2;
  // 8-bit rows go through in chunks of 32 entries: two independent halves, and the work that does not depend on the chunk's size
  // (waits, shuffles, rescaling) is paid half as often.
  static constexpr int kSubs = kE4M3 ? 2 : 1;
  static constexpr int kChunk = kSub * kSubs;                              // entries per stage
  static constexpr int kBoxSubs = kOwnPage ? 1 : kSubs;                    // 16-entry steps that one TMA box brings
  static constexpr int kParts = kOwnPage ? kSubs : 1;                      // parts of a chunk whose sums join apart
  static constexpr int kRowBytes = D * kItem;
  static constexpr int kBoxes = kRowBytes > 128 ? kRowBytes / 128 : 1;     // 128-byte column blocks of a row (or one of 64)
  static constexpr int kBoxRow = kRowBytes / kBoxes;
  static constexpr int kBoxBytes = kChunk * kBoxRow;
  static constexpr int kStageBytes = 2 * kBoxes * kBoxBytes;               // by column block: K's rows, V's rows (see the copies)
  // Per computing warp, of 8 KB each for head_dim 128.  A third stage of 8-bit rows makes long caches slower (131072 entries: 52
  // against 49.5 us): what is in flight is enough, and fewer streams leave memory pages open longer.
  static constexpr int kStages = kE4M3 ? 2 : 3;
  static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
  static constexpr int kRows = 8 * RT;
  static constexpr int kMergeCols = RT == 1 ? 64 : 32;                     // the warps' outputs meet so many columns at a time
  static constexpr int kMergeLd = kMergeCols + 4;
  static constexpr int kMergeBytes = kWarps * kRows * (kMergeLd * 4 + 8);
  static constexpr int kSmem = kRingBytes + kMergeBytes + 1024;
};

// Sum over the block of one value per thread; every thread gets it.  `scratch`: one word per warp.
template <int kBlock>
__device__ __forceinline__ long long block_sum(long long x, long long* scratch) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
  __syncthreads();
  long long s = 0;
#pragma unroll
  for (int w = 0; w < kBlock / 32; ++w) s += scratch[w];
  return s;
}

__device__ __forceinline__ int chunks_of(const PagedAttnParams& p, int b, int chunk_log2) {
  return chunk_count(usable_len(p.lens[b], p.c.max_pages, p.c.page_log2), chunk_log2);
}

// CTAs that get a share: no more than there are units, so that every CTA between a pair's first and last holds a piece of it.
__device__ __forceinline__ int sharing_ctas(const PagedAttnParams& p, long long total) {
  return static_cast<int>(min(static_cast<long long>(p.ctas), total));
}
// First unit of CTA c when `total` units are dealt evenly to n CTAs.
__device__ __forceinline__ long long share_begin(long long total, int c, int n) { return total * c / n; }

}  // namespace

// p.balanced == 0: one segment per CTA, (split of the entries, KV head, row tile, sequence).  p.balanced == 1: the chunks of all
// (sequence, row tile, KV head) triples in a row are dealt evenly to the grid's CTAs, so that sequences of very different
// lengths load every SM alike; a CTA walks the segments its share touches.
template <int D, bool kE4M3, int RT, bool kOwnPage>
__global__ void __launch_bounds__(kThreads, 2)
paged_attn_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const PagedAttnParams p) {
  using Cfg = PagedCfg<D, kE4M3, RT, kOwnPage>;
  constexpr int KS = D / 16, MT = D / 16, kRows = Cfg::kRows, kStages = Cfg::kStages, NSUB = Cfg::kSubs, kParts = Cfg::kParts;
  constexpr int kChunk = Cfg::kChunk, kChunkLog2 = kE4M3 ? 5 : 4;
  constexpr int kTerms = kE4M3 ? 2 : 3;         // 16-bit terms of a weight: 11 + 11 bits of fp16, 8 + 8 + 8 of bf16
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint64_t full[kWarps][kStages], empty[kWarps][kStages];
  __shared__ float2 scale_of[kWarps][kStages][NSUB];       // 8-bit pages, by 16 entries of a stage: K's scale, V's times kScaleGain
  __shared__ float weight_of[kWarps][kRows];               // what a warp's outputs count for in the merge
  __shared__ long long at_of[kRows];                       // where a row's result goes, in units of D floats
  __shared__ int abort_flag;
  __shared__ long long scratch[kThreads / 32];
  __shared__ int s_first;
  __shared__ long long s_base;

  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len;

  if (t == 0) {
    tma_prefetch_desc(&tmap_k);
    if (!p.joint) tma_prefetch_desc(&tmap_v);
    abort_flag = 0;
    s_first = -1;
  }
  if (lane == 0 && warp < kWarps) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&full[warp][i], kE4M3 ? 2 : 1); mbar_init(&empty[warp][i], 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // ---- this CTA's share: units [u, u_end) of a row of (sequence, row tile x KV head, chunk) ----
  const int HT = Hkv * p.row_tiles;
  int b = 0, ht = 0, split = 0, c0, c1, n_chunks;
  long long u = 0, u_end = 0, u_begin = 0;
  if (!p.balanced) {
    unsigned rest = blockIdx.x;                   // row tiles fastest: they read the same entries
    const int tile = rest % p.row_tiles; rest /= p.row_tiles;
    split = rest % p.splits; rest /= p.splits;
    ht = tile * Hkv + rest % Hkv;
    b = rest / Hkv;
  }
  __syncthreads();
  pdl_wait();
  if (p.balanced) {
    const int per = (p.c.batch + kThreads - 1) / kThreads, b0 = min(t * per, p.c.batch), b1 = min(b0 + per, p.c.batch);
    long long mine = 0;
    for (int x = b0; x < b1; ++x) mine += chunks_of(p, x, kChunkLog2);
    const long long total = block_sum<kThreads>(mine, scratch) * HT;
    // chunks of the sequences before this thread's
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += y;
    }
    before -= mine;
    for (int w = 0; w < warp; ++w) before += scratch[w];
    const int ctas = sharing_ctas(p, total);
    if (static_cast<int>(blockIdx.x) < ctas) {
      u_begin = u = share_begin(total, blockIdx.x, ctas);
      u_end = share_begin(total, blockIdx.x + 1, ctas);
    }
    if (u < u_end && before * HT <= u && u < (before + mine) * HT) {
      long long base = before;
      for (int x = b0; x < b1; ++x) {
        const int n = chunks_of(p, x, kChunkLog2);
        if (u < (base + n) * HT) { s_first = x; s_base = base * HT; break; }
        base += n;
      }
    }
    __syncthreads();
    b = s_first;
    if (b < 0) return;                          // nothing for this CTA
    n_chunks = chunks_of(p, b, kChunkLog2);
    ht = static_cast<int>((u - s_base) / n_chunks);
    c0 = static_cast<int>((u - s_base) - static_cast<long long>(ht) * n_chunks);
    c1 = static_cast<int>(min(static_cast<long long>(n_chunks), c0 + (u_end - u)));
  } else {
    n_chunks = chunks_of(p, b, kChunkLog2);
    const int per = (n_chunks + p.splits - 1) / p.splits;
    c0 = min(split * per, n_chunks);
    c1 = min(n_chunks, c0 + per);
  }

  // Moves on to the next segment of the share; false when there is none.
  auto advance = [&]() -> bool {
    if (!p.balanced) return false;
    u += c1 - c0;
    if (u >= u_end) return false;
    if (++ht == HT) {
      ht = 0;
      do { n_chunks = chunks_of(p, ++b, kChunkLog2); } while (n_chunks == 0);       // u < u_end: there is one
    }
    c0 = 0;
    c1 = static_cast<int>(min(static_cast<long long>(n_chunks), u_end - u));
    return true;
  };
  const int pair = warp & (kWarps - 1);                    // the computing warp, and the one that brings its data
  uint8_t* const ring_ptr = smem + pair * kStages * Cfg::kStageBytes;
  // inside a column block of a stage: K and V alternate by box (of a chunk's 32 rows, or of 16)
  constexpr uint32_t box_bytes = Cfg::kBoxSubs * kSub * Cfg::kBoxRow, sub_stride = (kOwnPage ? 2 : 1) * kSub * Cfg::kBoxRow;
  const uint32_t k_off = p.v_first ? box_bytes : 0, v_off = p.v_first ? 0 : box_bytes;
  int stage = 0;                                           // position in the ring, carried from segment to segment
  uint32_t phase = 0;
  auto step = [&]() { if (++stage == kStages) { stage = 0; phase ^= 1; } };
  bool ok = true;                                          // false: a wait gave up; nothing more is copied or computed

  if (warp >= kWarps) {
    // ================= a warp that brings data =================
    give_registers<kBringRegs>();
    const uint64_t policy = p.row_tiles == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
    const int page_subs_log2 = p.c.page_log2 - 4;          // steps of 16 entries in a page
    int issued = 0;                                        // chunks whose copies were started, up to kStages
    do {
      const int g = ht % Hkv;
      const int len = usable_len(p.lens[b], p.c.max_pages, p.c.page_log2);
      const int my_chunks = c1 - c0 > pair ? (c1 - c0 - pair + kWarps - 1) / kWarps : 0;
      const int* const table = p.c.block_table + static_cast<size_t>(b) * p.c.max_pages;
      const int n_subs = (len + kSub - 1) / kSub;
      // Page and scales of the 16-entry step x for lane x % 32, fetched for 32 steps at a time, a batch ahead: table -> scale is
      // a chain of two trips to memory.
      auto block_of = [&](int x) -> int {                  // block (page * Hkv + g) of this lane's step, -1 behind the end
        const int i = x / NSUB, sub = (c0 + pair + i * kWarps) * NSUB + x % NSUB;
        if (i >= my_chunks || sub >= n_subs) return -1;
        const long long blk = pool_block(table[sub >> page_subs_log2], p.c.n_pages, Hkv, g);
        if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PAGED_PAGE); return g; }   // page 0 instead
        return static_cast<int>(blk);
      };
      auto scales_at = [&](int blk) -> float2 {
        if (!kE4M3 || blk < 0) return make_float2(1.0f, 0.0f);
        return make_float2(p.c.k_scales[blk], p.c.v_scales[blk] * kScaleGain);
      };
      int blk_cur = block_of(lane), blk_next = block_of(32 + lane);
      float2 sc_cur = scales_at(blk_cur), sc_next = scales_at(blk_next);
      for (int i = 0; i < my_chunks; ++i) {
        if ((i * NSUB & 31) == 0 && i > 0) {               // the next batch of 32 steps becomes the current one
          blk_cur = blk_next;
          sc_cur = sc_next;
          blk_next = block_of(i * NSUB + 32 + lane);
          sc_next = scales_at(blk_next);
        }
        if (issued == kStages) {                           // the stage has to be empty again
          ok = mbar_wait_nap(&empty[pair][stage], phase ^ 1, &abort_flag, p.hdr, SITE_PAGED_EMPTY, p.wait_limit);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        } else {
          ++issued;
        }
        int blk[NSUB];
#pragma unroll
        for (int y = 0; y < NSUB; ++y) blk[y] = max(__shfl_sync(0xffffffffu, blk_cur, (i * NSUB + y) & 31), 0);
        const bool withheld = pair == 0 && i == p.skip_copy;     // test hook
        if (lane == 0 && !withheld) {
          // One copy brings a box of K and the same box of V (the pools are two planes of one tensor map); where the pools lie
          // too far apart for that, two copies fill the same places.  A step behind the sequence's end brings page 0.
          uint64_t* bar = &full[pair][stage];
          mbar_arrive_expect_tx(bar, Cfg::kStageBytes);
#pragma unroll
          for (int y = 0; y < NSUB; ++y) {
            if (y >= kParts) break;
            const int sub = (c0 + pair + i * kWarps) * NSUB + y;
            const int row = (sub & ((1 << page_subs_log2) - 1)) * kSub;
            uint8_t* dst = ring_ptr + stage * Cfg::kStageBytes + y * sub_stride;
#pragma unroll
            for (int x = 0; x < Cfg::kBoxes; ++x) {
              if (p.joint) {
                tma_load_4d(dst + x * 2 * Cfg::kBoxBytes, &tmap_k, bar, x * 64, row, blk[y], 0, policy);
              } else {
                tma_load_3d(dst + x * 2 * Cfg::kBoxBytes + k_off, &tmap_k, bar, x * 64, row, blk[y], policy);
                tma_load_3d(dst + x * 2 * Cfg::kBoxBytes + v_off, &tmap_v, bar, x * 64, row, blk[y], policy);
              }
            }
          }
        }
        if constexpr (kE4M3) {
          // The scales follow: the first ones are a trip to memory behind the table, which the copies need not wait for.
          const int here = lane - (i * NSUB & 31);         // this lane's step of the chunk, if it has one
          if (here >= 0 && here < NSUB) scale_of[pair][stage][here] = sc_cur;
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[pair][stage]);
        }
        __syncwarp();
        step();
      }
    } while (ok && advance());
    if (lane == 0) {                                       // no copy is in flight when the warp leaves, whatever the others do
      for (int j = 0; j < issued; ++j) {
        if (stage == 0) { stage = kStages; phase ^= 1; }
        --stage;
        if (pair != 0 || p.skip_copy < 0) mbar_wait_drain(&full[pair][stage], phase, p.hdr, SITE_PAGED_WAIT);
        else mbar_wait_drain(&full[pair][stage], phase, nullptr, SITE_PAGED_WAIT, p.wait_limit);   // the withheld one never arrives
      }
    }
    return;
  }

  // ================= the warps that compute =================
  take_registers<kComputeRegs>();
  const int quad = lane >> 2, c = lane & 3;                // fragment coordinates
  const uint32_t ring = smem_u32(ring_ptr);
  const uint32_t row7 = lane & 7;
  const uint32_t swz = Cfg::kBoxRow == 128 ? row7 : (row7 >> 1);      // 16-byte piece p of row r sits at p ^ swz
  float* const mo = reinterpret_cast<float*>(smem + Cfg::kRingBytes);                          // [warps][rows][columns]
  float2* const mml = reinterpret_cast<float2*>(mo + kWarps * kRows * Cfg::kMergeLd);        // [warps][rows]: max, sum
  auto meet = []() { asm volatile("bar.sync 1, %0;" ::"n"(kComputing) : "memory"); };

  do {
    const int g = ht % Hkv, tile = ht / Hkv, row_base = tile * kRows;
    const int asked = p.lens[b];
    const int len = usable_len(asked, p.c.max_pages, p.c.page_log2);
    if (t == 0 && c0 == 0 && ht == 0 && asked != len) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PAGED_LEN);
    const int my_chunks = ok && c1 - c0 > warp ? (c1 - c0 - warp + kWarps - 1) / kWarps : 0;

    // ---- query fragments: rows quad and (RT == 2) quad + 8 of the tile, absent rows zero ----
    uint32_t qa[KS][2 * RT];
    float q_scale[RT];                            // logit per accumulated unit (log2)
    int sees[RT];                                 // entries the row sees
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int r = row_base + rt * 8 + quad;
      const bool there = r < p.rows;
      const int i = there ? r / G : 0, h = g * G + (there ? r - i * G : 0);
      sees[rt] = len - (T - 1 - i);
      const uint16_t* qp = p.q + ((static_cast<size_t>(b) * T + i) * p.n_q_heads + h) * D;
      q_scale[rt] = p.scale_log2;
      if constexpr (kE4M3) {
        // element order of the 8-bit K rows: k index 2c, 2c + 1, 2c + 8, 2c + 9 of a step is element 4c .. 4c + 3
        uint2 w[KS];
        float m = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          w[ks] = there ? *reinterpret_cast<const uint2*>(qp + ks * 16 + c * 4) : make_uint2(0u, 0u);
          float a, d;
          unpack16<false>(w[ks].x, a, d);
          m = fmaxf(m, fmaxf(fabsf(a), fabsf(d)));
          unpack16<false>(w[ks].y, a, d);
          m = fmaxf(m, fmaxf(fabsf(a), fabsf(d)));
        }
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        int up = m > 0.0f ? 14 - scale_log2(__float_as_uint(m)) : 0;
        up = up > 120 ? 120 : up;                 // of a subnormal row; otherwise within [-113, 120] as it stands
        const float f = __uint_as_float(pow2_bits(up));
        q_scale[rt] *= __uint_as_float(pow2_bits(-up));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          float a, d;
          unpack16<false>(w[ks].x, a, d);
          qa[ks][rt] = pack16<true>(a * f, d * f);
          unpack16<false>(w[ks].y, a, d);
          qa[ks][RT + rt] = pack16<true>(a * f, d * f);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qa[ks][rt] = there ? *reinterpret_cast<const uint32_t*>(qp + ks * 16 + c * 2) : 0u;
          qa[ks][RT + rt] = there ? *reinterpret_cast<const uint32_t*>(qp + ks * 16 + c * 2 + 8) : 0u;
        }
      }
    }
    // O^T per row tile: [0] (d0, row 2c), [1] (d0, row 2c + 1), [2] (d1, row 2c), [3] (d1, row 2c + 1); (d0, d1) is
    // (quad, quad + 8) of the 16-wide step mt for bf16 and (2 quad, 2 quad + 1) for 8-bit rows
    float o[RT][MT][4];
    float m_run[RT], l_part[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m_run[rt] = -INFINITY;
      l_part[rt] = 0.0f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[rt][mt][e] = 0.0f;
    }

    bool spoilt = false;                          // elements of V were cleared because not every row sees them

    // One pass over the chunk in stage st.  kTail: some row does not see all of it (the sequence's end, and what follows a query's
    // own token).  Products that follow one another are independent (a dependent one waits 21 cycles, the tensor cores take one
    // every 8), and the matrix loads are asked for a phase ahead of their use: K's together, V's before the softmax step whose
    // latency they hide in.
    auto pass = [&](auto tail_, int i, int st) {
      constexpr bool kTail = decltype(tail_)::value;
      const int key0 = (c0 + warp + i * kWarps) * kChunk;
      const uint32_t ks_addr = ring + st * Cfg::kStageBytes + k_off, vs_addr = ring + st * Cfg::kStageBytes + v_off;
      // What a row does not see must not reach it: its logit is masked, but a zero weight does not silence a NaN or an infinity in
      // V.  Between the query tokens' own entries, which only some rows see, such elements are cleared, and handed to the rows
      // that do see them when the segment is through.
      if (kTail && T > 1) {
        const int own0 = max(0, len - (T - 1) - key0), own1 = min(kChunk, len - key0);
        uint8_t* vs = ring_ptr + st * Cfg::kStageBytes + v_off;
        constexpr int kPieces = Cfg::kBoxRow / 16;
        const int n = max(own1 - own0, 0) * kPieces;
        bool found = false;
        for (int j = lane; j < Cfg::kBoxes * n; j += 32) {
          const int x = j / n, rem = j - x * n, r = own0 + rem / kPieces;
          uint4* const at = reinterpret_cast<uint4*>(vs + x * 2 * Cfg::kBoxBytes + r / kSub * sub_stride + r % kSub * Cfg::kBoxRow + rem % kPieces * 16);
          uint4 w = *at;
          const uint32_t bad = not_finite<kE4M3>(w.x) | not_finite<kE4M3>(w.y) | not_finite<kE4M3>(w.z) | not_finite<kE4M3>(w.w);
          if (bad != 0) {
            w.x &= ~not_finite<kE4M3>(w.x); w.y &= ~not_finite<kE4M3>(w.y); w.z &= ~not_finite<kE4M3>(w.z); w.w &= ~not_finite<kE4M3>(w.w);
            *at = w;
            found = true;
          }
        }
        if (__any_sync(0xffffffffu, found)) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");                 // before the stage's next copies
          spoilt = true;
        }
        __syncwarp();
      }
      if (kTail && len - key0 < kChunk) {
        // what lies behind the sequence's end in the page is not its own
        const int rows = len - key0;
        uint8_t* vs = ring_ptr + st * Cfg::kStageBytes + v_off;
        constexpr int kPieces = Cfg::kBoxRow / 16;
        const int n = (kChunk - rows) * kPieces;
        for (int j = lane; j < Cfg::kBoxes * n; j += 32) {
          const int x = j / n, rem = j - x * n, r = rows + rem / kPieces;
          *reinterpret_cast<uint4*>(vs + x * 2 * Cfg::kBoxBytes + r / kSub * sub_stride + r % kSub * Cfg::kBoxRow + rem % kPieces * 16) =
              make_uint4(0u, 0u, 0u, 0u);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before the stage's next copies
        __syncwarp();
      }
      // ---- S = Q K^T, 8 entries a tile: lane holds (row quad, entries nt * 8 + 2c, + 1) in [0], [1], row quad + 8 in [2], [3] ----
      float s[2 * NSUB][4];
      {
        const uint32_t at = ks_addr + row7 * Cfg::kBoxRow + (((lane >> 3) ^ swz) << 4);
        constexpr int kLoads = Cfg::kRowBytes / 64;             // matrix loads of eight K rows: 64 bytes of each
        uint32_t kb[kLoads][2 * NSUB][4];
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
#pragma unroll
          for (int nt = 0; nt < 2 * NSUB; ++nt)
            ldsm_x4(kb[l][nt], (at ^ ((l & 1) << 6)) + (l >> 1) * 2 * Cfg::kBoxBytes + (nt >> 1) * sub_stride + (nt & 1) * 8 * Cfg::kBoxRow);
        constexpr int kEach = kE4M3 ? 4 : 2;                    // 16-element steps that a load brings
        float d[4][4];                                          // four sums at a time: the tiles, or halves of two tiles
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
#pragma unroll
          for (int y = 0; y < kEach; ++y)
#pragma unroll
            for (int nt = 0; nt < 2 * NSUB; ++nt) {
              const int ks = l * kEach + y;
              const uint32_t q0 = qa[ks][0], q1 = RT == 2 ? qa[ks][RT - 1] : 0u, q2 = qa[ks][RT], q3 = RT == 2 ? qa[ks][2 * RT - 1] : 0u;
              if constexpr (kE4M3) mma16<true>(d[nt], ks == 0, q0, q1, q2, q3, widen_lo(kb[l][nt][y]), widen_hi(kb[l][nt][y]));
              else mma16<false>(d[(y & 1) * 2 + nt], ks < 2, q0, q1, q2, q3, kb[l][nt][2 * y], kb[l][nt][2 * y + 1]);
            }
#pragma unroll
        for (int nt = 0; nt < 2 * NSUB; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][e] = kE4M3 ? d[nt][e] : d[nt][e] + d[2 + nt][e];
      }
      // V's fragments, as loaded.  8-bit rows: entries 0..7 and 8..15 of step y, pieces 2l and 2l + 1; bf16: 16 elements x 16 entries
      constexpr int kVLoads = Cfg::kRowBytes / 32;
      uint32_t vb[kVLoads][NSUB][4];
      {
        const uint32_t at = kE4M3 ? vs_addr + (((lane >> 3) & 1) * 8 + row7) * Cfg::kBoxRow + (((lane >> 4) ^ swz) << 4)
                                  : vs_addr + ((lane >> 4) * 8 + row7) * Cfg::kBoxRow + ((((lane >> 3) & 1) ^ swz) << 4);
#pragma unroll
        for (int l = 0; l < kVLoads; ++l)
#pragma unroll
          for (int y = 0; y < NSUB; ++y)
            ldsm_x4_trans(vb[l][y], (at ^ ((l & 3) << 5)) + (l >> 2) * 2 * Cfg::kBoxBytes + y * sub_stride);
      }
      float2 sc[NSUB];                              // the pages' scales
#pragma unroll
      for (int y = 0; y < NSUB; ++y) sc[y] = kE4M3 ? scale_of[warp][st][y] : make_float2(1.0f, 1.0f);
      uint32_t pt[RT][kTerms][NSUB][2];             // the weights as B fragments, term by term
      float a0[RT], a1[RT];                         // what the outputs of rows 2c and 2c + 1 are scaled by
      float g0[RT][kParts], g1[RT][kParts];         // 8-bit pages: and what their new sums are
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        // ---- online softmax of row quad (+ 8 rt): its logits sit in the four lanes of the quad ----
        if constexpr (kTail) {
#pragma unroll
          for (int nt = 0; nt < 2 * NSUB; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (key0 + nt * 8 + c * 2 + e >= sees[rt]) s[nt][rt * 2 + e] = -INFINITY;
        }
        float f[NSUB], most[NSUB], top[NSUB];       // most: the largest unit; top: what it is as a logit (log2)
#pragma unroll
        for (int y = 0; y < NSUB; ++y) {
          f[y] = fmaxf(q_scale[rt] * sc[y].x, 1.17549435e-38f);          // positive, so that a masked logit stays -inf
          most[y] = fmaxf(fmaxf(s[2 * y][2 * rt], s[2 * y][2 * rt + 1]), fmaxf(s[2 * y + 1][2 * rt], s[2 * y + 1][2 * rt + 1]));
          most[y] = fmaxf(most[y], __shfl_xor_sync(0xffffffffu, most[y], 1));
          most[y] = fmaxf(most[y], __shfl_xor_sync(0xffffffffu, most[y], 2));
          top[y] = most[y] * f[y];
        }
        float m_new = m_run[rt];
#pragma unroll
        for (int y = 0; y < NSUB; ++y) m_new = fmaxf(m_new, top[y]);
        const float ref = m_new == -INFINITY ? 0.0f : m_new;             // nothing seen yet: everything stays at zero
        const float alpha = ex2(m_run[rt] - ref);
        float pr[NSUB][4];
        if constexpr (kE4M3) {
          float from[kParts], gain[kParts], sum[kParts];                 // from: the unit that a part's weights count from
#pragma unroll
          for (int z = 0; z < kParts; ++z) {
            from[z] = kOwnPage ? most[z] : fmaxf(most[0], most[NSUB - 1]);
            gain[z] = ex2((kOwnPage ? top[z] : fmaxf(top[0], top[NSUB - 1])) - ref);
            if (from[z] == -INFINITY) from[z] = 0.0f;
            sum[z] = 0.0f;
          }
#pragma unroll
          for (int y = 0; y < NSUB; ++y) {
            const int z = kOwnPage ? y : 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[y][e] = ex2((s[2 * y + (e >> 1)][2 * rt + (e & 1)] - from[z]) * f[y]);      // at most 1
            sum[z] += (pr[y][0] + pr[y][1]) + (pr[y][2] + pr[y][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[y][e] *= kWeightGain;
          }
#pragma unroll
          for (int z = 0; z < kParts; ++z) {
            l_part[rt] = fmaf(sum[z], gain[z], z == 0 ? l_part[rt] * alpha : l_part[rt]);
            gain[z] *= sc[z].y;
            g0[rt][z] = __shfl_sync(0xffffffffu, gain[z], 8 * c);
            g1[rt][z] = __shfl_sync(0xffffffffu, gain[z], 8 * c + 4);
          }
        } else {
          float sum = 0.0f;
#pragma unroll
          for (int y = 0; y < NSUB; ++y) {
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[y][e] = ex2(fmaf(s[2 * y + (e >> 1)][2 * rt + (e & 1)], f[y], -ref));
            sum += (pr[y][0] + pr[y][1]) + (pr[y][2] + pr[y][3]);
          }
          l_part[rt] = fmaf(l_part[rt], alpha, sum);
        }
        m_run[rt] = m_new;
        a0[rt] = __shfl_sync(0xffffffffu, alpha, 8 * c);
        a1[rt] = __shfl_sync(0xffffffffu, alpha, 8 * c + 4);
        // the weights as 16-bit terms: the leading bits cut off, then what is left (the last term rounded)
        constexpr uint32_t kKeep = kE4M3 ? 0xffffe000u : 0xffff0000u;
#pragma unroll
        for (int y = 0; y < NSUB; ++y) {
#pragma unroll
          for (int w = 0; w < kTerms; ++w) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float lo = pr[y][2 * x], hi = pr[y][2 * x + 1];
              if (w + 1 < kTerms) {
                lo = __uint_as_float(__float_as_uint(lo) & kKeep);
                hi = __uint_as_float(__float_as_uint(hi) & kKeep);
                pr[y][2 * x] -= lo;
                pr[y][2 * x + 1] -= hi;
              }
              if (!kE4M3 && w + 1 < kTerms) pt[rt][w][y][x] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
              else pt[rt][w][y][x] = pack16<kE4M3>(lo, hi);
            }
          }
        }
      }
      // ---- O^T = O^T alpha + V^T P^T.  The products of a chunk (of each page's part) start from zero and join the running outputs with
      // one rounding to nearest: the tensor cores cut their sums off, and over thousands of chunks that bias shows. ----
      auto join = [&](float (&acc)[4], const float (&x)[4], int rt, int z) {
        if constexpr (kE4M3) {
          const float b0 = z == 0 ? a0[rt] : 1.0f, b1 = z == 0 ? a1[rt] : 1.0f;
          acc[0] = fmaf(x[0], g0[rt][z], acc[0] * b0); acc[1] = fmaf(x[1], g1[rt][z], acc[1] * b1);
          acc[2] = fmaf(x[2], g0[rt][z], acc[2] * b0); acc[3] = fmaf(x[3], g1[rt][z], acc[3] * b1);
        } else {
          acc[0] = fmaf(acc[0], a0[rt], x[0]); acc[1] = fmaf(acc[1], a1[rt], x[1]);
          acc[2] = fmaf(acc[2], a0[rt], x[2]); acc[3] = fmaf(acc[3], a1[rt], x[3]);
        }
      };
      constexpr int kTogether = 4 / RT / kParts;    // 16-element tiles of the head dimension whose sums run side by side
#pragma unroll
      for (int m0 = 0; m0 < MT; m0 += kTogether) {
        float x[kParts][kTogether][RT][4];
        uint32_t v[NSUB][kTogether][4];
#pragma unroll
        for (int y = 0; y < NSUB; ++y)
#pragma unroll
          for (int z = 0; z < kTogether; ++z) {
            const int m = m0 + z;
            if constexpr (kE4M3) {
              // a word holds elements (2 quad, 2 quad + 1) of entry 2c, then of entry 2c + 1: bring equal elements together
              const uint32_t w0 = __byte_perm(vb[m / 2][y][2 * (m & 1)], 0, 0x3120), w1 = __byte_perm(vb[m / 2][y][2 * (m & 1) + 1], 0, 0x3120);
              v[y][z][0] = widen_lo(w0); v[y][z][1] = widen_hi(w0); v[y][z][2] = widen_lo(w1); v[y][z][3] = widen_hi(w1);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) v[y][z][e] = vb[m][0][e];
            }
          }
#pragma unroll
        for (int n = 0; n < NSUB * kTerms; ++n) {     // by half, then by term; halves that join apart take turns
          const int y = kOwnPage ? n % NSUB : n / kTerms, w = kOwnPage ? n / NSUB : n % kTerms, part = kOwnPage ? y : 0;
#pragma unroll
          for (int z = 0; z < kTogether; ++z)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              mma16<kE4M3>(x[part][z][rt], n < kParts, v[y][z][0], v[y][z][1], v[y][z][2], v[y][z][3], pt[rt][w][y][0], pt[rt][w][y][1]);
        }
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int z = 0; z < kTogether; ++z)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) join(o[rt][m0 + z], x[part][z][rt], rt, part);
      }
    };
    const int all_see = chunks_all_see(len, T, kChunkLog2);
    for (int i = 0; i < my_chunks; ++i) {
      ok = mbar_wait_bounded(&full[warp][stage], phase, &abort_flag, p.hdr, SITE_PAGED_WAIT, p.wait_limit);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (c0 + warp + i * kWarps < all_see) pass(std::false_type{}, i, stage);
      else pass(std::true_type{}, i, stage);
      __syncwarp();                                // every lane is done with the stage
      if (lane == 0) mbar_arrive(&empty[warp][stage]);
      step();
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      l_part[rt] += __shfl_xor_sync(0xffffffffu, l_part[rt], 1);
      l_part[rt] += __shfl_xor_sync(0xffffffffu, l_part[rt], 2);
    }
    pdl_launch_dependents();
    if (spoilt) {                                  // rare: the elements that were cleared, from the pool
#pragma unroll 1
      for (int key = max(len - (T - 1), 0); key < len; ++key) {
        const int x = key / kChunk - c0 - warp;
        if (x < 0 || x % kWarps != 0 || x / kWarps >= my_chunks) continue;     // another warp's chunk
        long long blk = pool_block(p.c.block_table[static_cast<size_t>(b) * p.c.max_pages + (key >> p.c.page_log2)], p.c.n_pages, Hkv, g);
        if (blk < 0) blk = g;                      // as the copies take it
        const uint8_t* const row = p.c.v_pages + ((blk << p.c.page_log2) + (key & ((1 << p.c.page_log2) - 1))) * Cfg::kRowBytes;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float v;
            if constexpr (kE4M3) v = (row[m * 16 + 2 * quad + z] & 0x7f) == 0x7f ? NAN : 0.0f;
            else v = __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[m * 16 + quad + 8 * z]) << 16);
            if (isfinite(v)) continue;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (key < len - (T - 1 - (row_base + rt * 8 + 2 * c + e) / G)) o[rt][m][2 * z + e] += v;
          }
      }
    }
    // ---- the warps merge through shared memory: a thread per row weighs the warps, then the outputs join, columns by columns ----
    const int n_rows = min(kRows, p.rows - row_base);
    const bool whole = p.balanced ? c0 == 0 && c1 == n_chunks : p.splits == 1;
    meet();                                        // the last segment's merge has been read
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
      if (c == 0) mml[warp * kRows + rt * 8 + quad] = make_float2(ok ? m_run[rt] : -INFINITY, ok ? l_part[rt] : 0.0f);
#pragma unroll
    for (int cut = 0; cut < D / Cfg::kMergeCols; ++cut) {
      if (cut > 0) meet();                         // the columns before have been read
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int m = 0; m < Cfg::kMergeCols / 16; ++m) {
          const float (&x)[4] = o[rt][cut * (Cfg::kMergeCols / 16) + m];
          float* row0 = mo + (warp * kRows + rt * 8 + 2 * c) * Cfg::kMergeLd + m * 16;
          if constexpr (kE4M3) {
            *reinterpret_cast<float2*>(row0 + 2 * quad) = make_float2(x[0], x[2]);
            *reinterpret_cast<float2*>(row0 + Cfg::kMergeLd + 2 * quad) = make_float2(x[1], x[3]);
          } else {
            row0[quad] = x[0]; row0[Cfg::kMergeLd + quad] = x[1];
            row0[quad + 8] = x[2]; row0[Cfg::kMergeLd + quad + 8] = x[3];
          }
        }
      }
      meet();
      if (cut == 0) {
        if (t < n_rows) {
          float M = -INFINITY, L = 0.0f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) M = fmaxf(M, mml[w * kRows + t].x);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float2 ml = mml[w * kRows + t];
            if (ml.y != 0.0f) L = fmaf(ml.y, ex2(ml.x - M), L);                   // warps without entries weigh nothing; NaN stays
          }
          const float last = !whole ? 1.0f : L != 0.0f ? (kE4M3 ? kOutGain : 1.0f) / L : 0.0f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float2 ml = mml[w * kRows + t];
            weight_of[w][t] = ml.y != 0.0f ? ex2(ml.x - M) * last : 0.0f;
          }
          if (whole) {
            const int r = row_base + t, i = r / G, h = g * G + r - i * G;
            const long long at = (static_cast<long long>(b) * T + i) * p.n_q_heads + h;
            at_of[t] = at;
            if (p.lse != nullptr) p.lse[at] = L != 0.0f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
          } else {
            // where a piece waits for the merge: static launches by (pair, split), balanced ones by CTA (first segment or later)
            const long long at = (p.balanced ? 2 * static_cast<long long>(blockIdx.x) + (u != u_begin) : static_cast<long long>(blockIdx.x)) * kRows + t;
            at_of[t] = at;
            p.part_ml[at] = make_float2(M, L);
          }
        }
        meet();
      }
      constexpr int kQuads = Cfg::kMergeCols / 4;
      float* const dst = whole ? p.out : p.part_o;
      for (int x = t; x < n_rows * kQuads; x += kComputing) {
        const int r = x / kQuads, col = (x - r * kQuads) * 4;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = weight_of[w][r];
          const float4 y = *reinterpret_cast<const float4*>(mo + (w * kRows + r) * Cfg::kMergeLd + col);
          sum.x = fmaf(y.x, f, sum.x); sum.y = fmaf(y.y, f, sum.y); sum.z = fmaf(y.z, f, sum.z); sum.w = fmaf(y.w, f, sum.w);
        }
        *reinterpret_cast<float4*>(dst + at_of[r] * D + cut * Cfg::kMergeCols + col) = sum;
      }
    }
  } while (advance());
}

// Merges the pieces of one query row, a block each: the warps share the pieces out, every one of them weighs all pieces for itself,
// and their sums meet once.  All of it is latency (an empty kernel here costs 1 us, this one 2.3 for 37 pieces a row): the outputs are
// asked for before their weights are known, what can be is worked out before the wait for the main kernel, and there is little
// code, because instructions that run once come from memory, too (loops unrolled for 24 loads in flight: 4 us).
constexpr int kMergeWarps = 8;
template <int D, bool kE4M3>
__global__ void __launch_bounds__(32 * kMergeWarps, 2) paged_merge_kernel(const PagedAttnParams p) {
  constexpr int kChunkLog2 = kE4M3 ? 5 : 4, V = D / 32, kAhead = 8;
  __shared__ float acc[kMergeWarps][D];
  pdl_launch_dependents();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, warps = blockDim.x >> 5, G = p.group, kRows = p.tile_rows;
  // block -> (query token of the batch, head)
  const unsigned bi = blockIdx.x / p.n_q_heads;
  const int h = blockIdx.x - bi * p.n_q_heads, b = bi / p.q_len, i = bi - b * p.q_len, g = h / G;
  const int row = i * G + h - g * G, tile = row / kRows, r = row - tile * kRows, HT = p.c.n_kv_heads * p.row_tiles;
  const int ht = tile * p.c.n_kv_heads + g;
  long long first, rest;                          // piece 0 is at `first`, piece s > 0 at rest + s * step
  int n, step;
  if (p.balanced) {
    long long before = 0, total = 0;              // every warp for itself
    for (int x = lane; x < p.c.batch; x += 32) {
      const int k = chunks_of(p, x, kChunkLog2);
      total += k;
      if (x < b) before += k;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, o);
      before += __shfl_xor_sync(0xffffffffu, before, o);
    }
    total *= HT;
    const int mine = chunks_of(p, b, kChunkLog2), ctas = sharing_ctas(p, total);
    const long long p0 = before * HT + static_cast<long long>(ht) * mine, p1 = p0 + mine;
    first = rest = 0;
    n = step = 0;
    if (mine == 0) {
      // no CTA of the main kernel came by to report a length below zero
      if (t == 0 && h == 0 && i == 0 && p.lens[b] < 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PAGED_LEN);
    } else {
      const int ca = static_cast<int>(((p0 + 1) * ctas - 1) / total), cb = static_cast<int>((p1 * ctas - 1) / total);
      if (ca == cb) {                             // one CTA had all of it and wrote the result
        pdl_wait();                               // who waits for this kernel waits for the main one
        return;
      }
      n = cb - ca + 1;
      step = 2;
      rest = 2 * static_cast<long long>(ca);
      first = rest + (share_begin(total, ca, ctas) != p0);
    }
  } else {
    n = p.splits;
    step = p.row_tiles;
    first = rest = (static_cast<long long>(b) * p.c.n_kv_heads + g) * n * step + tile;
  }
  const float* const outputs = p.part_o + (rest * kRows + r) * D + lane * V;
  const float2* const sums = p.part_ml + rest * kRows + r;
  const size_t apart = static_cast<size_t>(step) * kRows;
  const long long extra = (first - rest) * kRows;
  struct Part { float x[V]; };
  auto load = [&](int s) -> Part {
    const float* const at = outputs + (s == 0 ? extra : s * apart) * D;
    Part y;
    if constexpr (V == 4) {
      const float4 w = __ldcg(reinterpret_cast<const float4*>(at));
      y.x[0] = w.x; y.x[1] = w.y; y.x[2] = w.z; y.x[3] = w.w;
    } else {
      const float2 w = __ldcg(reinterpret_cast<const float2*>(at));
      y.x[0] = w.x; y.x[1] = w.y;
    }
    return y;
  };
  auto sums_of = [&](int s) -> float2 { return __ldcg(sums + (s == 0 ? extra : s * apart)); };
  const float2 none = make_float2(-INFINITY, 0.0f);
  pdl_wait();                                     // the lengths were there before any block of the main kernel let this one start
  const float2 ml0 = lane < n ? sums_of(lane) : none, ml1 = 32 + lane < n ? sums_of(32 + lane) : none;
  Part ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (warp + k * warps < n) ahead[k] = load(warp + k * warps);
  float M = fmaxf(ml0.x, ml1.x), L = 0.0f;
  for (int s = 64 + lane; s < n; s += 32) M = fmaxf(M, sums_of(s).x);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  // pieces without entries weigh nothing; NaN stays
  auto weight = [&](const float2& ml) -> float { return ml.y == 0.0f ? 0.0f : ex2(ml.x - M); };
  const float w0 = weight(ml0), w1 = weight(ml1);
  L = ml0.y * w0 + ml1.y * w1;
  for (int s = 64 + lane; s < n; s += 32) {
    const float2 ml = sums_of(s);
    L += ml.y * weight(ml);
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int s = warp + k * warps;
    if (s < n) {                                  // at most 64 pieces this way, kAhead * kMergeWarps
      const float f = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] = fmaf(ahead[k].x[e], f, sum[e]);
    }
  }
#pragma unroll 2
  for (int s = warp + kAhead * warps; s < n; s += warps) {
    const Part y = load(s);
    const float f = weight(sums_of(s));
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = fmaf(y.x[e], f, sum[e]);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) acc[warp][lane * V + e] = sum[e];
  __syncthreads();
  const size_t at = (static_cast<size_t>(b) * p.q_len + i) * p.n_q_heads + h;
  const float scale = L != 0.0f ? (kE4M3 ? kOutGain : 1.0f) / L : 0.0f;
  for (int x = t; x < D; x += blockDim.x) {
    float o = 0.0f;
#pragma unroll 4
    for (int w = 0; w < warps; ++w) o += acc[w][x];
    p.out[at * D + x] = o * scale;
  }
  if (p.lse != nullptr && t == 0) p.lse[at] = L != 0.0f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

PagedAttnPlan plan_paged_attn(int batch, int n_kv_heads, int rows, bool e4m3, int max_len, long long total_len) {
  PagedAttnPlan pl;
  const int chunk = e4m3 ? 2 * kSub : kSub;
  const long long chunks = chunk_count(max_len, e4m3 ? 5 : 4);
  // More than 8 query rows: 16 of them share an entry's loads, unless the call is so small that CTAs of 8 rows all run at once and
  // have some 512 entries or fewer each to go through (four query tokens, 16 and 8 rows a CTA, in us: one sequence of 250 entries,
  // 8 bits, 6.7 and 5.8, of 2000 8.9 and 8.1, of 13107 13.9 and 14.6; 16 of 380, bf16, 13.9 and 10.0; 32 of 819 to 1638, 8 bits,
  // 26.8 and 39).
  const long long pairs_of_8 = static_cast<long long>(batch) * n_kv_heads * ((rows + 7LL) / 8);
  pl.row_tiles_of_8 = rows <= 8 || (pairs_of_8 <= kPagedCtas && pairs_of_8 * max_len <= 512LL * kPagedCtas) ? 1 : 2;
  pl.row_tiles = chunk_count(rows, pl.row_tiles_of_8 == 1 ? 3 : 4);
  const long long pairs = static_cast<long long>(batch) * n_kv_heads * pl.row_tiles;
  // Splits: as many as run at once, each with a chunk for every warp.  Short sequences stay whole: the merge costs 2 to 3 us, a
  // warp's pass over a chunk 0.75 us in 8 bits and 0.55 us in bf16 (one sequence, 8 bits: 400 entries 7.2 us whole and 6.7 in
  // four splits, 320 entries 5.8 and 6.2; bf16: 400 entries 6.8 and 5.7, four sequences of 257 6.8 and 7.1).
  long long splits = kPagedCtas / pairs;
  const long long useful = chunks <= (e4m3 ? 12 : 18) ? 1 : (chunks + kWarps - 1) / kWarps;
  if (splits > useful) splits = useful;
  if (splits > kPagedCtas) splits = kPagedCtas;
  if (splits < 1) splits = 1;
  pl.splits = static_cast<int>(splits);
  pl.balanced = 0;
  pl.ctas = 0;
  // Static or dealt out evenly: entries that the busiest CTA goes through against the mean.  Static launches of several waves even
  // themselves out but for about half a sequence.  Against that stands what a balanced launch pays: CTAs start and join two
  // segments or more, and the merge looks at every row; measured, some 512 entries' time and 5 more for every pair, 7.5 where 16 rows
  // share a CTA.  Static and balanced, in us: eight sequences of 4K to 64K entries, 8 bits, 235 and 105; four of 500 to 20000 29.5 and
  // 27.8; 16 of 400 to 8000 44 and 37; 16 of 200 to 4000 26 and 27; 24 of 100 to 1638 19.5 and 26; 64 of 100 to 1000 24.5 and 38, of
  // 2K to 8K 128 and 110; four query tokens, 32 of 819 to 1638, 27 and 44, 16 of 400 to 8000 61 and 55.
  const double per = static_cast<double>((chunks + splits - 1) / splits) * chunk;
  const double even = static_cast<double>(total_len) * n_kv_heads * pl.row_tiles / kPagedCtas;
  const double busiest = pairs * splits <= kPagedCtas ? per : even + 0.5 * per;
  if (batch >= 2 && busiest - even > 512.0 + (pl.row_tiles_of_8 == 1 ? 5.0 : 7.5) * pairs) {
    pl.balanced = 1;
    pl.ctas = kPagedCtas;
    pl.splits = 1;
  }
  return pl;
}

static size_t pieces_of_plan(const PagedAttnPlan& plan, int batch, int n_kv_heads) {
  if (plan.balanced) return 2 * static_cast<size_t>(plan.ctas);
  return plan.splits == 1 ? 0 : static_cast<size_t>(batch) * n_kv_heads * plan.row_tiles * plan.splits;
}
size_t paged_attn_partials_offset(const PagedAttnPlan& plan, int batch, int n_kv_heads) {
  const size_t rows = pieces_of_plan(plan, batch, n_kv_heads) * 8 * plan.row_tiles_of_8;
  return sizeof(WorkspaceHeader) + (rows * sizeof(float2) + 255) / 256 * 256;
}
size_t paged_attn_workspace_bytes(const PagedAttnPlan& plan, int batch, int n_kv_heads, int head_dim) {
  const size_t rows = pieces_of_plan(plan, batch, n_kv_heads) * 8 * plan.row_tiles_of_8;
  return paged_attn_partials_offset(plan, batch, n_kv_heads) + rows * head_dim * sizeof(float);
}

template <int D, bool kE4M3, int RT, bool kOwnPage>
static cudaError_t launch_w(const CUtensorMap& tk, const CUtensorMap& tv, PagedAttnParams& p, cudaStream_t stream, int* launches) {
  using Cfg = PagedCfg<D, kE4M3, RT, kOwnPage>;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(paged_attn_kernel<D, kE4M3, RT, kOwnPage>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
    if (e != cudaSuccess) return e;
    // the split of the registers holds for this launch size only: a build that differs must not run
    cudaFuncAttributes fa;
    if ((e = cudaFuncGetAttributes(&fa, paged_attn_kernel<D, kE4M3, RT, kOwnPage>)) != cudaSuccess) return e;
    if (fa.numRegs != kLaunchRegs) return cudaErrorLaunchOutOfResources;
    configured.set(dev);
  }
  const long long blocks = p.balanced ? p.ctas : static_cast<long long>(p.c.batch) * p.row_tiles * p.c.n_kv_heads * p.splits;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  p.tile_rows = Cfg::kRows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, paged_attn_kernel<D, kE4M3, RT, kOwnPage>, tk, tv, static_cast<const PagedAttnParams&>(p));
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (!p.balanced && p.splits == 1) return cudaSuccess;
  cfg.gridDim = dim3(static_cast<unsigned>(p.c.batch) * p.q_len * p.n_q_heads);
  // warps of a row's block: no more than it has pieces, of balanced launches twice what it has on the average
  const long long pairs = static_cast<long long>(p.c.batch) * p.c.n_kv_heads * p.row_tiles;
  const long long pieces = p.balanced ? 1 + 2 * static_cast<long long>(p.ctas) / pairs : p.splits;
  cfg.blockDim = dim3(32 * static_cast<unsigned>(pieces < kMergeWarps ? pieces : kMergeWarps));
  cfg.dynamicSmemBytes = 0;
  e = cudaLaunchKernelEx(&cfg, paged_merge_kernel<D, kE4M3>, static_cast<const PagedAttnParams&>(p));
  if (e == cudaSuccess) *launches = 2;
  return e;
}

template <int D, bool kE4M3>
static cudaError_t launch_f(const CUtensorMap& tk, const CUtensorMap& tv, PagedAttnParams& p, const PagedAttnPlan& plan,
                            cudaStream_t stream, int* launches) {
  if constexpr (kE4M3) {
    if (p.c.page_log2 == 4)
      return plan.row_tiles_of_8 == 1 ? launch_w<D, kE4M3, 1, true>(tk, tv, p, stream, launches) : launch_w<D, kE4M3, 2, true>(tk, tv, p, stream, launches);
  }
  return plan.row_tiles_of_8 == 1 ? launch_w<D, kE4M3, 1, false>(tk, tv, p, stream, launches) : launch_w<D, kE4M3, 2, false>(tk, tv, p, stream, launches);
}

cudaError_t launch_paged_attn(const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, PagedAttnParams& p, const PagedAttnPlan& plan,
                              int head_dim, bool e4m3, cudaStream_t stream, int* launches) {
  *launches = 0;
  p.row_tiles = plan.row_tiles;
  p.splits = plan.splits;
  p.balanced = plan.balanced;
  p.ctas = plan.ctas;
  if (head_dim == 128)
    return e4m3 ? launch_f<128, true>(tmap_k, tmap_v, p, plan, stream, launches) : launch_f<128, false>(tmap_k, tmap_v, p, plan, stream, launches);
  if (head_dim == 64)
    return e4m3 ? launch_f<64, true>(tmap_k, tmap_v, p, plan, stream, launches) : launch_f<64, false>(tmap_k, tmap_v, p, plan, stream, launches);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
