// Attention of a batch's new query tokens over a prefix that several sequences share, computed once for all of them, and its merge with
// the attention over each sequence's own entries (paged_attn.cu).
//
// The query rows of all sequences that share a prefix (query tokens x heads of a KV group) are one matrix against the prefix's K and V:
// tiles of 128 rows, so that the products belong on the 5th-generation tensor cores and the prefix's pages cross HBM once instead of
// once per sequence.  The chunks (128 entries) of all (prefix, KV head, pair of row tiles) units in a row are dealt evenly to one
// persistent CTA per SM; a CTA walks the segments that its share touches and leaves each one's (reference, sum, output) as a piece:
// unit and CTA number both only grow along the walk, so unit + CTA names a piece.  prefix_merge_kernel joins a row's pieces and its own
// entries' attention.
//
// A CTA's roles:
//   loaders    one warp: K and V tiles page by page (TMA, a box per page and 64 columns) into their rings, ahead into the next
//              segment; one warp: a segment's Q, as soon as the one before is through with it;
//   widening   (8-bit pages) four warps: codes from the raw ring to bf16 tiles in the layout that TMA would write, times the
//              page's scale: a power of two, so exact;
//   issuers    one warp per row tile: per chunk O += P V of the chunk before, then S = Q K^T (tcgen05.mma 128 x 128 x d, fp32 in
//              tensor memory), in that order from one thread, so that S may overwrite the P that the contraction before has read;
//   softmax    eight warps per row tile, two threads per row: online softmax in log2 units with a lazily raised reference; P goes
//              back, in bf16, into the first half of the thread's own S columns.
// With more than 128 rows the two tiles hold different rows and take every chunk, their contractions alternating.  With 128 or fewer
// both work on the same rows and take every other chunk: one's softmax runs under the other's contractions.
// Tensor memory (512 columns): S (and P inside it) of tile A at 0, of tile B at 128; O of A at 256, of B at 256 + d.
//
// P is rounded to bf16 (2^-9 of each weight, of either sign): that is what the output is rounded to; the row sums take it unrounded.
// Logits, exponentials, sums, outputs and their merge are fp32.
//
// Every wait is bounded; a wait that gives up raises the status word and the CTA-wide abort flag, the roles stop issuing work, copies and
// contractions in flight are waited for, tensor memory is released.
#include "paged.cuh"
#include "paged_mma.cuh"

namespace fastkv {

namespace {

constexpr int kTile = 128;                     // rows of a tile, entries of a chunk
constexpr int kCtrlWarps = 4;                  // K and V, issuer of tile A, issuer of tile B, Q
constexpr int kSoftmaxWarps = 8;               // per tile
constexpr int kWideWarps = 4;
constexpr int kHalfBytes = kTile * 128;        // 128 rows x 64 bf16: one swizzled column block of a tile
constexpr float kSlackLog2 = 8.0f;

template <int D, bool kE4M3>
struct PrefixCfg {
  static constexpr int KH = D / 64;
  static constexpr int kTileBytes = KH * kHalfBytes;
  static constexpr int kStages = kE4M3 && D == 128 ? 1 : 2;               // bf16 tiles of K, and of V
  static constexpr int kRawBytes = kTile * D;                              // codes of a chunk's K or V
  static constexpr int kRaw = kE4M3 ? (D == 128 ? 5 : 8) : 1;              // (one unused in bf16)
  static constexpr int kWarps = kCtrlWarps + 2 * kSoftmaxWarps + (kE4M3 ? kWideWarps : 0);
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kXchBytes = 2 * 2 * 2 * kTile * 4;                  // what the two halves of a row exchange
  static constexpr int kSmem = (2 + 2 * kStages) * kTileBytes + (kE4M3 ? kRaw * kRawBytes : 0) + kXchBytes + 1024;
};

// Chunks are numbered along a CTA's share.  Chunk n's K and V are in tile n % kStages, and their barriers are those of n's parity, also
// where there is one tile: then a row tile that takes every other chunk waits on barriers of its own, in order (one that waited for a
// phase two ahead would be answered by the phase before), and the two issuers start every segment together.
template <int NR>
struct PrefixBarriers {
  uint64_t q_full, q_empty, v_tail;
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t raw_full[NR], raw_empty[NR];
  uint64_t s_full[2], p_full[2];               // per tile: S is there; every softmax warp has stored its part of P
  uint64_t o_done[2], o_free[2];               // per tile: a segment's O is complete; its softmax warps have read it
  uint64_t turn[2];                            // turn[x]: the other tile's issuer has issued the block that goes before x's next one
  uint64_t drained[2];
  uint32_t tmem_base;
  int abort_flag;
  int first_group;
  long long first_chunk;
  int first_unit;
  long long scratch[32], scratch_u[32];
};

// ---- which rows and entries belong together ----
struct Group {
  int seq0, tokens, len, chunks, pairs;        // first sequence, query tokens, entries, chunks of them, pairs of row tiles
};
__device__ __forceinline__ Group group_of(const PrefixParams& p, int i) {
  Group g;
  int lo = 0, hi = p.c.batch;
  if (p.cu_seqs != nullptr) {
    lo = min(max(__ldcg(p.cu_seqs + i), 0), p.c.batch);
    hi = min(max(__ldcg(p.cu_seqs + i + 1), lo), p.c.batch);
  }
  g.seq0 = lo;
  g.tokens = (hi - lo) * p.q_len;
  g.len = usable_len(__ldcg(p.lens + i), p.max_pages, p.c.page_log2);
  g.chunks = chunk_count(g.len, 7);
  g.pairs = g.chunks == 0 ? 0 : (g.tokens + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens);
  return g;
}
__device__ __forceinline__ int sharing_ctas(const PrefixParams& p, long long total) {
  return static_cast<int>(min(static_cast<long long>(p.ctas), total));
}

// A segment of a CTA's share: chunks [c0, c1) of one unit.
struct Segment {
  int group, g, pair, c0, c1, unit;
  Group of;
  int n0;                                      // number of its first chunk along the share
  int token0, tokens;                          // of the unit: first query token of the batch, and how many
  bool dual;                                   // two tiles of different rows
  __device__ __forceinline__ void set(const PrefixParams& p) {
    const int first = pair * 2 * p.tile_tokens;
    token0 = of.seq0 * p.q_len + first;
    tokens = min(of.tokens - first, 2 * p.tile_tokens);
    dual = tokens > p.tile_tokens;
  }
  // chunks that tile x takes, and the number of its j-th: all, or those of its parity
  __device__ __forceinline__ int skip(int x) const { return dual ? 0 : (n0 ^ x) & 1; }
  __device__ __forceinline__ int chunks_of(int x) const { return dual ? c1 - c0 : (c1 - c0 + 1 - skip(x)) >> 1; }
  __device__ __forceinline__ int chunk(int x, int j) const { return n0 + (dual ? j : skip(x) + 2 * j); }
  __device__ __forceinline__ int rows_of(const PrefixParams& p, int x) const {
    return (dual ? (x == 0 ? p.tile_tokens : tokens - p.tile_tokens) : tokens) * p.group;
  }
};

__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b, float s) {     // eight codes to bf16, times s
  uint4 r;
  float lo, hi;
  unpack16<true>(widen_lo(a), lo, hi); r.x = pack16<false>(lo * s, hi * s);
  unpack16<true>(widen_hi(a), lo, hi); r.y = pack16<false>(lo * s, hi * s);
  unpack16<true>(widen_lo(b), lo, hi); r.z = pack16<false>(lo * s, hi * s);
  unpack16<true>(widen_hi(b), lo, hi); r.w = pack16<false>(lo * s, hi * s);
  return r;
}

}  // namespace

template <int D, bool kE4M3>
__global__ void __launch_bounds__(PrefixCfg<D, kE4M3>::kThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                   const __grid_constant__ CUtensorMap tmap_v, const PrefixParams p) {
  using Cfg = PrefixCfg<D, kE4M3>;
  constexpr int NS = Cfg::kStages, NR = Cfg::kRaw, KH = Cfg::KH, kThreads = Cfg::kThreads, kWarps = Cfg::kWarps;
  extern __shared__ __align__(1024) uint8_t smem[];       // the tiles need 1024-byte alignment (128-byte swizzle atoms)
  uint8_t* const sQ = smem;                               // two row tiles
  uint8_t* const sK = sQ + 2 * Cfg::kTileBytes;
  uint8_t* const sV = sK + NS * Cfg::kTileBytes;
  uint8_t* const sRaw = sV + NS * Cfg::kTileBytes;
  float* const xch_all = reinterpret_cast<float*>(sRaw + (kE4M3 ? NR * Cfg::kRawBytes : 0));
  using Barriers = PrefixBarriers<NR>;
  static_assert(sizeof(Barriers) <= 1024, "the barriers have a kilobyte");
  Barriers* const bars = reinterpret_cast<Barriers*>(reinterpret_cast<uint8_t*>(xch_all) + Cfg::kXchBytes);

  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int Hkv = p.c.n_kv_heads, G = p.group;
  pdl_launch_dependents();
  if (smem_u32(smem) & 1023u) {                           // never seen; would garble every tile
    if (t == 0) raise_status(p.hdr, FASTKV_ERR_UNSUPPORTED, SITE_PREFIX_Q);
    pdl_wait();
    return;
  }
  // The kernel before this one is the attention over the sequences' own entries, and whoever wrote this one's inputs had finished before any
  // of its blocks let this one start: only the end of this kernel has to wait for it.

  // ---- this CTA's share ----
  long long u = 0, u_end = 0;
  Segment first;
  {
    const int n = p.n_prefixes;
    const int per = (n + kThreads - 1) / kThreads, i0 = min(t * per, n), i1 = min(i0 + per, n);
    long long mine = 0, units = 0;                        // chunks and units of this thread's prefixes
    for (int i = i0; i < i1; ++i) {
      const Group g = group_of(p, i);
      units += static_cast<long long>(g.pairs) * Hkv;
      mine += static_cast<long long>(g.pairs) * Hkv * g.chunks;
      if (blockIdx.x == 0) {
        if (g.len != __ldcg(p.lens + i)) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_LEN);
        if (p.cu_seqs != nullptr) {
          const int a = __ldcg(p.cu_seqs + i), b = __ldcg(p.cu_seqs + i + 1);
          if (a < 0 || b < a || b > p.c.batch) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_GROUP);
        }
      }
    }
    long long before = mine, before_u = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, before, o), z = __shfl_up_sync(0xffffffffu, before_u, o);
      if (lane >= o) { before += y; before_u += z; }
    }
    if (lane == 31) { bars->scratch[warp] = before; bars->scratch_u[warp] = before_u; }
    if (t == 0) bars->first_group = -1;
    __syncthreads();
    before -= mine;
    before_u -= units;
    long long total = 0, total_u = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) { before += bars->scratch[w]; before_u += bars->scratch_u[w]; }
      total += bars->scratch[w];
      total_u += bars->scratch_u[w];
    }
    if (total_u > p.max_units) {                          // groups that overlap: there is no room for their pieces
      if (blockIdx.x == 0 && t == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_GROUP);
      total = 0;
    }
    const int ctas = sharing_ctas(p, total);
    if (static_cast<int>(blockIdx.x) < ctas) {
      u = total * blockIdx.x / ctas;
      u_end = total * (blockIdx.x + 1) / ctas;
    }
    if (u < u_end && before <= u && u < before + mine) {
      long long at = before, at_u = before_u;
      for (int i = i0; i < i1; ++i) {
        const Group g = group_of(p, i);
        const long long k = static_cast<long long>(g.pairs) * Hkv * g.chunks;
        if (u < at + k) { bars->first_group = i; bars->first_chunk = at; bars->first_unit = static_cast<int>(at_u); break; }
        at += k;
        at_u += static_cast<long long>(g.pairs) * Hkv;
      }
    }
    __syncthreads();
    if (u >= u_end) {                                     // nothing for this CTA (uniform)
      pdl_wait();
      return;
    }
    first.group = bars->first_group;
    first.of = group_of(p, first.group);
    const long long in_group = u - bars->first_chunk;
    const int unit = static_cast<int>(in_group / first.of.chunks);
    first.g = unit / first.of.pairs;
    first.pair = unit - first.g * first.of.pairs;
    first.unit = bars->first_unit + unit;
    first.c0 = static_cast<int>(in_group - static_cast<long long>(unit) * first.of.chunks);
    first.c1 = static_cast<int>(min(static_cast<long long>(first.of.chunks), first.c0 + (u_end - u)));
    first.n0 = 0;
    first.set(p);
  }
  // Moves on to the next segment of the share; false when there is none.
  auto advance = [&](Segment& s, long long& at) -> bool {
    at += s.c1 - s.c0;
    s.n0 += s.c1 - s.c0;
    if (at >= u_end) return false;
    ++s.unit;
    if (++s.pair == s.of.pairs) {
      s.pair = 0;
      if (++s.g == Hkv) {
        s.g = 0;
        do { s.of = group_of(p, ++s.group); } while (s.of.pairs == 0);                 // at < u_end: there is one
      }
    }
    s.c0 = 0;
    s.c1 = static_cast<int>(min(static_cast<long long>(s.of.chunks), u_end - at));
    s.set(p);
    return true;
  };

  if (t == 0) {
    mbar_init(&bars->q_full, 1);
    mbar_init(&bars->q_empty, 2);
    mbar_init(&bars->v_tail, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->k_full[i], kE4M3 ? kWideWarps : 1); mbar_init(&bars->k_empty[i], 2);
      mbar_init(&bars->v_full[i], kE4M3 ? kWideWarps : 1); mbar_init(&bars->v_empty[i], 2);
    }
    for (int i = 0; i < NR; ++i) { mbar_init(&bars->raw_full[i], 1); mbar_init(&bars->raw_empty[i], kWideWarps); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->p_full[i], kSoftmaxWarps);
      mbar_init(&bars->o_done[i], 1);
      mbar_init(&bars->o_free[i], kSoftmaxWarps);
      mbar_init(&bars->turn[i], 1);
      mbar_init(&bars->drained[i], 1);
    }
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tma_prefetch_desc(&tmap_q);
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;
  volatile int* const abort_flag = &bars->abort_flag;
  const long long limit = p.wait_limit;
  const int P = 1 << p.c.page_log2, pages = kTile >> p.c.page_log2;      // pages of a chunk
  Segment s = first;
  long long at = u;
  // Block (page * Hkv + g) of page j of chunk c, -1 behind the prefix's end.
  auto block_of = [&](const Segment& x, int c, int j) -> int {
    const int key = c * kTile + (j << p.c.page_log2);
    if (j >= pages || key >= x.of.len) return -1;
    const long long blk = pool_block(__ldcg(p.table + static_cast<size_t>(x.group) * p.max_pages + (key >> p.c.page_log2)), p.c.n_pages, Hkv, x.g);
    if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_PAGE); return x.g; }       // page 0 instead
    return static_cast<int>(blk);
  };

  if (warp == 0) {
    // ---------------- loader of K and V ----------------
    const uint64_t pol_kv = l2_policy_evict_normal();
    constexpr int kCols = kE4M3 ? 1 : KH;                 // boxes of a page's rows
    const uint32_t box_bytes = static_cast<uint32_t>(P) * (kE4M3 ? D : 128);
    bool ok = true;
    int n = 0;                                            // chunks so far
    int k_out = 0, v_out = 0, tails = 0;                  // copies started into the rings, and cut ones of V
    auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait_parked(bar, parity, abort_flag, p.hdr, SITE_PREFIX_RING, limit));
    };
    // a chunk's boxes of K or V into dst, one lane each
    auto bring = [&](const CUtensorMap* map, uint8_t* dst, uint64_t* bar, int blk) {
      const unsigned have = __ballot_sync(0xffffffffu, lane < pages * kCols && blk >= 0);
      if (lane == 0) mbar_arrive_expect_tx(bar, __popc(have) * box_bytes);
      __syncwarp();
      if ((have >> lane) & 1u) {
        const int j = lane / kCols, col = lane % kCols;
        tma_load_3d(dst + col * kHalfBytes + j * box_bytes, map, bar, col * 64, 0, blk, pol_kv);
      }
    };
    do {
      int next = block_of(s, s.c0, lane / kCols);
      for (int c = s.c0; c < s.c1 && ok; ++c, ++n) {
        const int blk = next;
        if (c + 1 < s.c1) next = block_of(s, c + 1, lane / kCols);
        if constexpr (kE4M3) {
          for (int kv = 0; kv < 2; ++kv) {
            const int r = 2 * n + kv, slot = r % NR;
            if (r >= NR) ok = wait(&bars->raw_empty[slot], (r / NR - 1) & 1);
            if (!ok) break;
            bring(kv ? &tmap_v : &tmap_k, sRaw + slot * Cfg::kRawBytes, &bars->raw_full[slot], blk);
            k_out = r + 1;
          }
        } else {
          const int par = n & 1;
          const uint32_t freed = ((n >> 1) & 1) ^ 1;      // phase of chunk n - 2's release
          if (n >= 2) ok = wait(&bars->k_empty[par], freed);
          if (!ok) break;
          bring(&tmap_k, sK + n % NS * Cfg::kTileBytes, &bars->k_full[par], blk);
          k_out = n + 1;
          if (n >= 2) ok = wait(&bars->v_empty[par], freed);
          if (!ok) break;
          const int have = s.of.len - c * kTile;
          uint8_t* const dst = sV + n % NS * Cfg::kTileBytes;
          if (have >= kTile) {
            bring(&tmap_v, dst, &bars->v_full[par], blk);
            v_out = n + 1;
          } else {
            // the prefix's last entries: a zero weight does not silence a NaN behind them, so those rows are cleared
            bring(&tmap_v, dst, &bars->v_tail, blk);
            ok = wait(&bars->v_tail, tails & 1);
            if (!ok) { mbar_wait_drain(&bars->v_tail, tails & 1, p.hdr, SITE_PREFIX_DRAIN, limit); break; }
            ++tails;
            for (int i = lane; i < (kTile - have) * 8 * KH; i += 32) {
              const int col = i / ((kTile - have) * 8), rest = i - col * (kTile - have) * 8;
              *reinterpret_cast<uint4*>(dst + col * kHalfBytes + have * 128 + rest * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->v_full[par]);
          }
        }
      }
    } while (ok && advance(s, at));
    // nothing may still be landing in shared memory when the CTA ends
    if (!ok && lane == 0) {
      if constexpr (kE4M3) {
        for (int r = max(0, k_out - NR); r < k_out; ++r) mbar_wait_drain(&bars->raw_full[r % NR], (r / NR) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      } else {
        for (int j = max(0, k_out - 2); j < k_out; ++j) mbar_wait_drain(&bars->k_full[j & 1], (j >> 1) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
        for (int j = max(0, v_out - 2); j < v_out; ++j) mbar_wait_drain(&bars->v_full[j & 1], (j >> 1) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      }
    }
  } else if (warp == 3) {
    // ---------------- loader of Q ----------------
    const uint64_t pol_q = l2_policy_evict_first();
    const uint32_t q_bytes = static_cast<uint32_t>(KH) * 128 * G * p.tile_tokens;
    bool ok = true;
    int segs = 0;
    do {
      if (segs > 0) ok = __all_sync(0xffffffffu, mbar_wait_parked(&bars->q_empty, (segs - 1) & 1, abort_flag, p.hdr, SITE_PREFIX_Q, limit));
      if (!ok) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(&bars->q_full, (s.dual ? 2 : 1) * q_bytes);
        for (int x = 0; x < (s.dual ? 2 : 1); ++x)
          for (int c = 0; c < KH; ++c)
            tma_load_3d(sQ + x * Cfg::kTileBytes + c * kHalfBytes, &tmap_q, &bars->q_full, c * 64, s.g * G, s.token0 + x * p.tile_tokens, pol_q);
      }
      __syncwarp();
      ++segs;
    } while (advance(s, at));
    if (lane == 0) mbar_wait_drain(&bars->q_full, (segs - 1) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
  } else if (warp < kCtrlWarps) {
    // ---------------- issuer of one row tile ----------------
    const int x = warp - 1;
    constexpr uint32_t idesc_s = umma_idesc_bf16_f32(kTile, kTile);
    constexpr uint32_t idesc_o = umma_idesc_bf16_f32(kTile, D) | (1u << 16);    // B (V) is MN-major
    const uint32_t s_tmem = tmem_base + x * kTile, o_tmem = tmem_base + 256 + x * D;
    bool ok = true;
    int segs = 0, o_segs = 0;                             // segments before this one; those in which this tile had chunks
    int pn = 0, turns = 0;
    int issued = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity, int site) -> bool {
      return __all_sync(0xffffffffu, mbar_wait_nap(bar, parity, abort_flag, p.hdr, site, limit));
    };
    do {
      const int nk = s.chunks_of(x);
      const uint32_t q_addr = smem_u32(sQ + (s.dual ? x : 0) * Cfg::kTileBytes);
      auto releases = [&](uint64_t* bar) {                // a stage is free when both issuers have released it
        tc_commit(bar);
        if (!s.dual) tc_commit(bar);
      };
      ok = wait(&bars->q_full, segs & 1, SITE_PREFIX_Q);
      for (int j = 0; nk > 0 && j <= nk && ok; ++j) {
        if (s.dual) {
          if (x == 0 && turns > 0) ok = wait(&bars->turn[0], (turns - 1) & 1, SITE_PREFIX_TURN);
          if (x == 1) ok = wait(&bars->turn[1], turns & 1, SITE_PREFIX_TURN);
          ++turns;
        }
        // V's contraction does not wait for the next K: where K and V have one tile each, the next K is widened behind the V that takes
        // this one's place
        if (ok && j > 0) {
          const int n = s.chunk(x, j - 1);
          ok = wait(&bars->v_full[n & 1], (n >> 1) & 1, SITE_PREFIX_V);
          if (ok) ok = wait(&bars->p_full[x], pn & 1, SITE_PREFIX_P);
          ++pn;
          if (ok && j == 1 && o_segs > 0) ok = wait(&bars->o_free[x], (o_segs - 1) & 1, SITE_PREFIX_O);
        }
        if (!ok) break;
        tc_fence_after_sync();
        if (j > 0) {                                      // O (+)= P V
          const int n = s.chunk(x, j - 1), st = n % NS;
          const uint64_t b0 = umma_desc_mn_sw128(smem_u32(sV + st * Cfg::kTileBytes), kHalfBytes);
#pragma unroll
          for (int kk = 0; kk < kTile / 16; ++kk)         // 16 entries = 8 packed columns of P, 2048 bytes of V per step
            if (elect_one())
              tc_mma_bf16_ts(o_tmem, s_tmem + (kk >> 2) * 64 + (kk & 3) * 8, b0 + static_cast<uint64_t>(kk * (2048 >> 4)), idesc_o,
                             (j > 1 || kk > 0) ? 1u : 0u);
          if (elect_one()) releases(&bars->v_empty[n & 1]);
          issued = 1;
        }
        if (j < nk) {                                     // S = Q K^T
          const int n = s.chunk(x, j), st = n % NS;
          ok = wait(&bars->k_full[n & 1], (n >> 1) & 1, SITE_PREFIX_K);
          if (!ok) break;
          tc_fence_after_sync();
          const uint64_t a0 = umma_desc_k_sw128(q_addr), b0 = umma_desc_k_sw128(smem_u32(sK + st * Cfg::kTileBytes));
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {           // 64-element block kk / 4, 32 bytes per step inside it
            const uint64_t step = static_cast<uint64_t>(((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4);
            if (elect_one()) tc_mma_bf16(s_tmem, a0 + step, b0 + step, idesc_s, kk > 0 ? 1u : 0u);
          }
          if (elect_one()) {
            releases(&bars->k_empty[n & 1]);
            if (!(x == 0 && n == p.skip_commit)) tc_commit(&bars->s_full[x]);     // (test hook: a completion that is never signalled)
          }
          issued = 1;
        }
        if (s.dual && elect_one()) mbar_arrive(&bars->turn[x ^ 1]);
      }
      if (!ok) break;
      if (elect_one()) {
        if (nk > 0) { tc_commit(&bars->o_done[x]); tc_commit(&bars->q_empty); }
        else mbar_arrive(&bars->q_empty);
      }
      if (nk > 0) ++o_segs;
      ++segs;
    } while (advance(s, at));
    // every contraction issued has finished before tensor memory is released
    if (issued) {
      if (elect_one()) tc_commit(&bars->drained[x]);
      __syncwarp();
      mbar_wait_drain(&bars->drained[x], 0, p.hdr, SITE_PREFIX_DRAIN, limit);
    }
  } else if (warp < kCtrlWarps + 2 * kSoftmaxWarps) {
    // ---------------- softmax: eight warps per row tile, two threads per row, 64 entries of the chunk each ----------------
    const int gw = warp - kCtrlWarps;
    const int x = gw >> 3, g8 = gw & 7;                   // row tile; warp of the tile
    const int quarter = warp & 3, half = g8 >> 2;         // a tile's warps cover the four lane quarters twice
    const int r = quarter * 32 + lane;                    // row of the tile = tensor-memory lane
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + x * kTile + half * 64;         // this thread's 64 S columns; P goes into the first 32
    const uint32_t o_addr = lane_addr + 256 + x * D + half * (D / 2);  // this thread's D / 2 columns of O
    float* const xch = xch_all + x * (2 * 2 * kTile);
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + x * 4 + quarter) : "memory"); };
    constexpr int HN = kTile / 2;
    bool ok = true;
    int sn = 0, o_segs = 0;                               // this tile's chunks, and segments with chunks, so far
    do {
      const int nk = s.chunks_of(x), rows = s.rows_of(p, x);
      const bool active = quarter * 32 < rows;            // (uniform for the two warps of a lane quarter)
      const long long piece = static_cast<long long>(s.unit) + blockIdx.x;
      float2* const ml = p.part_ml + (piece * 2 + x) * p.tile_rows;
      if (!active) {
        // no rows: the warp only keeps step (nobody may run ahead of a barrier by two phases)
        for (int j = 0; j < nk; ++j, ++sn) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait_nap(&bars->s_full[x], sn & 1, abort_flag, p.hdr, SITE_PREFIX_S, limit));
          if (ok && lane == 0) mbar_arrive(&bars->p_full[x]);
        }
        if (nk > 0) {
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait_nap(&bars->o_done[x], o_segs & 1, abort_flag, p.hdr, SITE_PREFIX_O, limit));
          if (ok && lane == 0) mbar_arrive(&bars->o_free[x]);
          ++o_segs;
        }
        continue;
      }
      float m_ref = -INFINITY, l = 0.0f;                  // the reference is the same in both threads of a row; l is this half's
      // Both warps of a pair walk every chunk and meet at the pair's barrier once per chunk whatever happens: a warp whose
      // wait gave up skips the work of the chunk, never the barrier.
      for (int j = 0; j < nk; ++j, ++sn) {
        const int buf = sn & 1;
        if (ok) ok = mbar_wait_bounded(&bars->s_full[x], sn & 1, abort_flag, p.hdr, SITE_PREFIX_S, limit);
        ok = __all_sync(0xffffffffu, ok);
        const int c = s.c0 + s.chunk(x, j) - s.n0;
        const int seen = s.of.len - c * kTile - half * HN; // entries of this half
        const bool tail = seen < HN;
        float half_max = -INFINITY;
        if (ok) {
          tc_fence_after_sync();
#pragma unroll
          for (int cc = 0; cc < HN / 32; ++cc) {
            float v[32];
            tmem_ld_32x32(s_addr + cc * 32, v);
            if (tail) {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = cc * 32 + i < seen ? v[i] : -INFINITY;
            }
            float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int i = 4; i < 32; i += 4) {
              mx[0] = fmaxf(mx[0], v[i]); mx[1] = fmaxf(mx[1], v[i + 1]); mx[2] = fmaxf(mx[2], v[i + 2]); mx[3] = fmaxf(mx[3], v[i + 3]);
            }
            half_max = fmaxf(half_max, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
          }
        }
        xch[(buf * 2 + half) * kTile + r] = half_max;
        pair_sync();
        if (!ok) continue;
        const float most = fmaxf(half_max, xch[(buf * 2 + (half ^ 1)) * kTile + r]) * p.scale_log2;     // the scale is positive
        const bool move = most > m_ref + kSlackLog2;
        const float alpha = move ? ex2(m_ref - most) : 1.0f;        // 0 at a row's first logits
        if (move) { m_ref = most; l *= alpha; }
        if (j >= 1 && __any_sync(0xffffffffu, move)) {
          // O is complete up to the chunk before: the contraction that added it was issued before this chunk's S, by the same thread
#pragma unroll
          for (int cc = 0; cc < D / 64; ++cc) {
            float o[32];
            tmem_ld_32x32(o_addr + cc * 32, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= alpha;
            tmem_st_32x32(o_addr + cc * 32, o);
          }
          tmem_wait_st();
        }
        const float neg_ref = m_ref == -INFINITY ? 0.0f : -m_ref;   // nothing seen yet: every weight is 2^-inf
        float ls[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int cc = 0; cc < HN / 32; ++cc) {
          float v[32];
          tmem_ld_32x32(s_addr + cc * 32, v);
          if (tail) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = cc * 32 + i < seen ? v[i] : -INFINITY;
          }
          float packed[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float e0 = ex2(fmaf(v[i], p.scale_log2, neg_ref));
            const float e1 = ex2(fmaf(v[i + 1], p.scale_log2, neg_ref));
            ls[i & 2] += e0;
            ls[(i & 2) + 1] += e1;
            packed[i / 2] = __uint_as_float(pack16<false>(e0, e1));
          }
          tmem_st_32x16(s_addr + cc * 16, packed);
        }
        l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->p_full[x]);
      }
      if (nk == 0) {
        if (half == 0 && r < rows) ml[r] = make_float2(-INFINITY, 0.0f);
        continue;
      }
      // ---- the segment's piece: columns of O by rows, so that a warp's stores are whole lines ----
      {
        const int buf = sn & 1;                           // the exchange buffer that the last chunk did not use
        xch[(buf * 2 + half) * kTile + r] = l;
        pair_sync();
        l += xch[(buf * 2 + (half ^ 1)) * kTile + r];
        pair_sync();                                      // the next segment's first chunk uses that buffer again
        if (ok) ok = mbar_wait_bounded(&bars->o_done[x], o_segs & 1, abort_flag, p.hdr, SITE_PREFIX_O, limit);
        ok = __all_sync(0xffffffffu, ok);
        ++o_segs;
        if (!ok) continue;
        tc_fence_after_sync();
        if (half == 0 && r < rows) ml[r] = make_float2(m_ref, l);
        float* const po = p.part_o + ((piece * 2 + x) * D + half * (D / 2)) * p.tile_rows + r;
#pragma unroll
        for (int cc = 0; cc < D / 64; ++cc) {
          float o[32];
          tmem_ld_32x32(o_addr + cc * 32, o);
          if (r < rows) {
#pragma unroll
            for (int i = 0; i < 32; ++i) __stcg(po + static_cast<long long>(cc * 32 + i) * p.tile_rows, o[i]);
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->o_free[x]);
      }
    } while (advance(s, at));
  } else {
    // ---------------- widening: codes to bf16 tiles ----------------
    if constexpr (kE4M3) {
      const int w = warp - kCtrlWarps - 2 * kSoftmaxWarps;               // rows 32 w .. of every tile
      bool ok = true;
      int n = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity, int site) -> bool {
        return __all_sync(0xffffffffu, mbar_wait_nap(bar, parity, abort_flag, p.hdr, site, limit));
      };
      // scales of page `lane` of a chunk
      auto scales_of = [&](const Segment& y, int c) -> float2 {
        const int blk = block_of(y, c, lane);
        return blk < 0 ? make_float2(0.0f, 0.0f) : make_float2(__ldcg(p.c.k_scales + blk), __ldcg(p.c.v_scales + blk));
      };
      constexpr int kPieces = D / 16;                     // 16-byte pieces of a row
      constexpr int kRowsAt = 32 / kPieces;               // rows of a warp's step
      // Eight lanes (what shared memory serves at a time) take four pieces of one column block of two neighbouring rows: the
      // swizzle puts their 16-byte stores into eight different places of a line.
      const int c4 = lane & 3, block = D == 128 ? (lane >> 3) & 1 : 0;
      const int row_in = ((lane >> 2) & 1) + (D == 128 ? (lane >> 4) * 2 : (lane >> 3) * 2);
      do {
        float2 next = scales_of(s, s.c0);
        for (int c = s.c0; c < s.c1 && ok; ++c, ++n) {
          const float2 sc = next;
          if (c + 1 < s.c1) next = scales_of(s, c + 1);
          const int have = s.of.len - c * kTile;
          for (int kv = 0; kv < 2; ++kv) {
            const int raw = 2 * n + kv, slot = raw % NR;
            ok = wait(&bars->raw_full[slot], (raw / NR) & 1, SITE_PREFIX_RAW);
            const int gone = n - NS;                      // the chunk whose tile this one takes
            if (ok && gone >= 0) ok = wait(kv ? &bars->v_empty[gone & 1] : &bars->k_empty[gone & 1], (gone >> 1) & 1, SITE_PREFIX_RAW);
            if (!ok) break;
            const uint8_t* const src = sRaw + slot * Cfg::kRawBytes;
            uint8_t* const dst = (kv ? sV : sK) + n % NS * Cfg::kTileBytes + block * kHalfBytes;
#pragma unroll 4
            for (int y = 0; y < 32 / kRowsAt; ++y) {
              const int r = w * 32 + y * kRowsAt + row_in;
              const float f = __shfl_sync(0xffffffffu, kv ? sc.y : sc.x, (w * 32 + y * kRowsAt) >> p.c.page_log2);
              uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
              if (r < have) {                             // behind the prefix's end: zeros
                const uint4 v = *reinterpret_cast<const uint4*>(src + r * D + (block * 4 + c4) * 16);
                a = widen8(v.x, v.y, f);
                b = widen8(v.z, v.w, f);
              }
              *reinterpret_cast<uint4*>(dst + r * 128 + (((2 * c4) ^ (r & 7)) << 4)) = a;
              *reinterpret_cast<uint4*>(dst + r * 128 + (((2 * c4 + 1) ^ (r & 7)) << 4)) = b;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(kv ? &bars->v_full[n & 1] : &bars->k_full[n & 1]);
              mbar_arrive(&bars->raw_empty[slot]);
            }
          }
        }
      } while (ok && advance(s, at));
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
  pdl_wait();                                             // who waits for this kernel waits for the one before it, too
}

// Joins a query row's pieces and the attention over its own entries.  A warp takes 32 rows (lane = row; the pieces hold columns by rows)
// and 8 columns; blockIdx: (32 rows, KV head, 32 columns).
template <int D>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const PrefixParams p) {
  __shared__ long long chunk0[kMaxPrefixes + 1];          // chunks and units of the prefixes before
  __shared__ int unit0[kMaxPrefixes + 1];
  __shared__ long long scratch[4], scratch_u[4];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len, n = p.n_prefixes;
  pdl_launch_dependents();
  {
    const int per = (n + 127) / 128, i0 = min(t * per, n), i1 = min(i0 + per, n);
    long long mine = 0, units = 0;
    for (int i = i0; i < i1; ++i) {
      const Group g = group_of(p, i);
      units += static_cast<long long>(g.pairs) * Hkv;
      mine += static_cast<long long>(g.pairs) * Hkv * g.chunks;
    }
    long long before = mine, before_u = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, before, o), z = __shfl_up_sync(0xffffffffu, before_u, o);
      if (lane >= o) { before += y; before_u += z; }
    }
    if (lane == 31) { scratch[warp] = before; scratch_u[warp] = before_u; }
    __syncthreads();
    before -= mine;
    before_u -= units;
    for (int w = 0; w < warp; ++w) { before += scratch[w]; before_u += scratch_u[w]; }
    for (int i = i0; i < i1; ++i) {
      const Group g = group_of(p, i);
      chunk0[i] = before;
      unit0[i] = static_cast<int>(before_u);
      before += static_cast<long long>(g.pairs) * Hkv * g.chunks;
      before_u += static_cast<long long>(g.pairs) * Hkv;
      if (i == n - 1) { chunk0[n] = before; unit0[n] = static_cast<int>(min(before_u, 0x7fffffffll)); }
    }
    __syncthreads();
  }
  const long long total = unit0[n] > p.max_units ? 0 : chunk0[n];
  const int R = blockIdx.x * 32 + lane, g = blockIdx.y, col = blockIdx.z * 32 + warp * 8;
  const int token = R / G, b = token / T, h = g * G + R - token * G;
  const bool there = b < p.c.batch;
  // ---- this row's pieces: `count` of them from `piece` on, and the same rows' other half of the chunks where one tile took both ----
  int count = 0, both = 1;
  const float2* ml = p.part_ml;
  const float* po = p.part_o;
  if (there && total > 0) {
    int lo = 0, hi = n;                                   // the last prefix that starts at or before b
    if (p.cu_seqs != nullptr)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldcg(p.cu_seqs + mid) <= b) lo = mid; else hi = mid;
      }
    const Group gr = group_of(p, lo);
    const int in = token - gr.seq0 * T;
    if (in >= 0 && in < gr.tokens && gr.pairs > 0) {
      const int pair = in / (2 * p.tile_tokens), rest = in - pair * 2 * p.tile_tokens;
      const bool dual = min(gr.tokens - pair * 2 * p.tile_tokens, 2 * p.tile_tokens) > p.tile_tokens;
      const int tile = rest / p.tile_tokens, row = (rest - tile * p.tile_tokens) * G + R - token * G;
      const long long unit = static_cast<long long>(g) * gr.pairs + pair, q0 = chunk0[lo] + unit * gr.chunks, q1 = q0 + gr.chunks;
      const int ctas = sharing_ctas(p, total);
      const int ca = static_cast<int>(((q0 + 1) * ctas - 1) / total), cb = static_cast<int>((q1 * ctas - 1) / total);
      const long long piece = unit0[lo] + unit + ca;
      count = cb - ca + 1;
      both = dual ? 1 : 2;
      ml += (piece * 2 + tile) * p.tile_rows + row;
      po += ((piece * 2 + tile) * D + col) * p.tile_rows + row;
    }
  }
  pdl_wait();
  const int most = __reduce_max_sync(0xffffffffu, count * both);
  float M = -INFINITY, L = 0.0f, acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
  auto join = [&](float m, float l, const float (&o)[8]) {
    if (l == 0.0f) return;                                // nothing seen; NaN stays
    const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.0f : top;
    const float a = ex2(M - ref), w = ex2(m - ref);
    M = top;
    L = fmaf(L, a, l * w);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = fmaf(acc[i], a, o[i] * w);
  };
  const size_t step_ml = static_cast<size_t>(p.tile_rows), step_o = static_cast<size_t>(D) * p.tile_rows;
  constexpr int kAhead = 4;
  for (int s0 = 0; s0 < most; s0 += kAhead) {
    float2 v[kAhead];
    float o[kAhead][8];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = s0 + k;
      v[k] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[k][i] = 0.0f;
      if (s < count * both) {
        const size_t tile = both == 2 ? s : 2 * s;        // tiles of a piece lie side by side
        v[k] = __ldcg(ml + tile * step_ml);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[k][i] = __ldcg(po + tile * step_o + static_cast<size_t>(i) * p.tile_rows);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) join(v[k].x, v[k].y, o[k]);
  }
  if (!there) return;
  const size_t at = static_cast<size_t>(token) * p.n_q_heads + h;
  {
    const float own = __ldcg(p.own_lse + at);
    const float4 y0 = __ldcg(reinterpret_cast<const float4*>(p.own_out + at * D + col)), y1 = __ldcg(reinterpret_cast<const float4*>(p.own_out + at * D + col + 4));
    const float o[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
    join(own * 1.4426950408889634f, own == -INFINITY ? 0.0f : 1.0f, o);
  }
  const float f = L != 0.0f ? 1.0f / L : 0.0f;
  uint4 w;
  w.x = pack16<false>(acc[0] * f, acc[1] * f); w.y = pack16<false>(acc[2] * f, acc[3] * f);
  w.z = pack16<false>(acc[4] * f, acc[5] * f); w.w = pack16<false>(acc[6] * f, acc[7] * f);
  *reinterpret_cast<uint4*>(p.out + at * D + col) = w;
  if (p.lse != nullptr && col == 0) p.lse[at] = L != 0.0f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

namespace {

template <int D, bool kE4M3>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, cudaStream_t stream, int* launches) {
  using Cfg = PrefixCfg<D, kE4M3>;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(prefix_attn_kernel<D, kE4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
    if (e != cudaSuccess) return e;
    configured.set(dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.ctas);
  cfg.blockDim = dim3(Cfg::kThreads);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, prefix_attn_kernel<D, kE4M3>, tq, tk, tv, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  const long long rows = static_cast<long long>(p.c.batch) * p.q_len * p.group;
  cfg.gridDim = dim3(static_cast<unsigned>((rows + 31) / 32), p.c.n_kv_heads, D / 32);
  cfg.blockDim = dim3(128);
  cfg.dynamicSmemBytes = 0;
  e = cudaLaunchKernelEx(&cfg, prefix_merge_kernel<D>, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace

cudaError_t launch_prefix_attn(const CUtensorMap& tmap_q, const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, const PrefixParams& p,
                               int head_dim, bool e4m3, cudaStream_t stream, int* launches) {
  if (head_dim == 128) return e4m3 ? launch_t<128, true>(tmap_q, tmap_k, tmap_v, p, stream, launches) : launch_t<128, false>(tmap_q, tmap_k, tmap_v, p, stream, launches);
  if (head_dim == 64) return e4m3 ? launch_t<64, true>(tmap_q, tmap_k, tmap_v, p, stream, launches) : launch_t<64, false>(tmap_q, tmap_k, tmap_v, p, stream, launches);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
