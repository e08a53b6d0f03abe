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
//              segment, with the pages' scales; one warp: a segment's Q, as soon as the one before is through with it;
//   widening   (8-bit pages) eight warps: Q into two e4m3 terms, in place; V's codes from their ring to bf16 times the page's scale, so
//              that the scales of pages far apart cost a weight none of its bits (exact);
//   issuers    one warp per row tile: per step of 64 entries O += P V of the chunk before, then S = Q K^T into the buffer that P is read
//              from (tcgen05.mma 128 x 64 x d and 128 x d x 64, fp32 in tensor memory), in that order from one thread;
//   softmax    four warps per row tile, a thread per row, which holds a step's 64 logits in registers: online softmax in log2 units with a
//              lazily raised reference; P goes back, in bf16, into the first half of the row's S columns.
// K of 8-bit pages is multiplied as it is stored (kind::f8f6f4), its scale goes onto the logits: widened like V it would cost the same
// 1300 cycles a chunk again (8 x 131072: 115 us, as stored 95).
// With more than 128 rows the two tiles hold different rows and take every chunk, their contractions alternating.  With 128 or fewer
// both work on the same rows and take every other chunk: one's softmax runs under the other's contractions.  With 64 or fewer the second
// tile's rows are its last 64 (its descriptor of Q starts 64 rows early), so that the two tiles' softmax warps are on different schedulers.
// Tensor memory (512 columns): S (and P inside it) of tile A at 0, of tile B at 128, two buffers of 64 each; O of A at 256, of B at 256 + d.
//
// What bounds it (32 query heads over 8 KV heads of 128; the kernel inside a call, one B200).  64 sequences over 32768 bf16 entries, 256 rows a
// KV head: 41 us for 134 MB and 34 GFLOP (20.5 and 20.9 us at the rates of a copy and of a large product); a step takes 1700 cycles, of
// which each softmax warp is busy for 1400 (the tensor pipe is active for 44 % of the kernel; 128 entries a step and one buffer of S, so that
// softmax and products wait for one another, took 50 us when this took 43).  8 x 131072 in 8 bits, 32 rows: 82 us
// for 269 MB: widening a chunk of V (1300 cycles) and a step's softmax by one warp (1000, twice a chunk and tile) are as long as each other;
// four copies of the rows in a tile with a quarter of the entries each brought 6 us and cost the merge 10, a third tile of V nothing.
// Short shares: 2 us until the first copy (lengths, barriers, tensor memory), 2 us for a segment's output.
//
// P is rounded to bf16 (by at most 2^-8 of each weight, of either sign), which is what the output is rounded to.  The output is divided by the
// sum of the rounded weights, so that a row of one entry that outweighs the others has none of that error (2 x 512: 0.21 % off on the whole,
// 0.25 divided by the other sum, which takes 3 % less time); lse takes the sum of the unrounded ones.
// Logits, exponentials, sums, outputs and their merge are fp32.
//
// Every wait is bounded; a wait that gives up raises the status word and the CTA-wide abort flag, the roles stop issuing work, copies and
// contractions in flight are waited for, tensor memory is released.
#include <type_traits>

#include "paged.cuh"
#include "paged_mma.cuh"

namespace fastkv {

namespace {

constexpr int kTile = 128;                     // rows of a tile, entries of a chunk
constexpr int kStep = 64;                      // entries of a softmax step: half a chunk, so that a tile's S has two buffers
constexpr int kCtrlWarps = 4;                  // loader of K and V, issuer of tile A, issuer of tile B, loader of Q
constexpr int kSoftmaxWarps = 4;               // per tile
constexpr int kWideWarps = 8;                  // 8-bit pages: Q into its two terms, V to bf16
constexpr int kHalfBytes = kTile * 128;        // 128 rows x 64 16-bit values: one swizzled column block of a tile
// A row's reference is set kSlackLog2 + kRoomLog2 above its largest logit and moves when a logit comes nearer than kRoomLog2 (which rescales
// the row's output and keeps its warp for 2000 cycles).  So a weight is 2^-15 at most, and what is not divided by the sum of the weights yet
// stays finite for V of any finite bf16 as long as the entries weigh no more than 2^14 of the largest would, and for V up to 2^113 whatever
// the entries; V of 2^-95 and above keeps its bits.  Weights are relative to the reference, and so is whatever rounds them; further away
// than 32 their exponents would lose a bit.  (Slack of 2^8: 100 us, 2^16: 96, 2^24: 96, 8 x 131072 in 8 bits, whole call, with one sum of the
// weights.)
constexpr float kSlackLog2 = 16.0f, kRoomLog2 = 15.0f;

// kOne: every unit has at most one tile of rows (the batch has no more), so that Q needs half the space.
template <int D, bool kE4M3, bool kOne>
struct PrefixCfg {
  static constexpr int KH = D / 64;
  static constexpr int kTileBytes = KH * kHalfBytes;
  // Tiles of Q, K and V, and in 8 bits V's raw chunks.  V waits for the softmax: two tiles of V in bf16 leave a load less time than memory
  // takes.
  static constexpr int kRawBytes = kTile * D;                              // codes of a chunk's K or V
  static constexpr int kKBytes = kE4M3 ? kRawBytes : kTileBytes;
  static constexpr int kQTiles = kOne ? 1 : 2, kKTiles = kE4M3 ? (D == 128 && !kOne ? 3 : 4) : (kOne ? 3 : 2), kVTiles = kE4M3 ? 2 : 3;
  static constexpr int kRaw = kE4M3 ? (D == 128 && !kOne ? 3 : 4) : 1;     // raw chunks of V (none in bf16)
  static constexpr int kWarps = kCtrlWarps + 2 * kSoftmaxWarps + (kE4M3 ? kWideWarps : 0);
  static constexpr int kThreads = 32 * kWarps;
  // behind the tiles: the scan of the prefixes, rows' shifts, pages' scales, barriers
  static constexpr int kScanBytes = 512, kExtra = kScanBytes + 2 * kTile + 512 + 896;
  static constexpr int kSmem = (kQTiles + kVTiles) * kTileBytes + kKTiles * kKBytes + (kE4M3 ? kRaw * kRawBytes : 0) + kExtra;
  static_assert(kWarps <= 32 && kSmem <= 232448, "shared memory of a CTA");
  // 8-bit pages: the launch's 96 registers a thread go 40 to the control warps, 120 to the softmax warps and 96 to the widening ones.
  static constexpr int kLaunchRegs = 96, kCtrlRegs = 40, kSoftmaxRegs = 120, kWideRegs = 96;
  static_assert(kCtrlRegs + 2 * kSoftmaxRegs + 2 * kWideRegs <= 5 * kLaunchRegs, "the warpgroups' shares are within what the CTA was launched with");
};

// Chunks are numbered along a CTA's share.  Chunk n's K and V are in tiles n % kKTiles and n % kVTiles, their barriers are number n % 8.
// A wait for a phase that is two ahead of its barrier, or two behind, would be answered wrongly.  So a barrier serves chunks of one
// parity (a row tile that takes every other chunk has barriers of its own and waits on each in order), the two issuers start every
// segment together, when all earlier chunks have been used, and the eighth chunk behind one is not loaded before the softmax has it
// behind itself (the fourth may be).  q_full and q_wide are one barrier each: the next segment's Q waits for both issuers and for every
// softmax warp to have come to this segment (q_empty), since a tile without chunks in a segment would not hold it up, and its softmax
// warps may still be writing the output of the one before.
constexpr int kBars = 8;
// Scales of a chunk's pages, K's and behind them V's: the softmax may still read a chunk's when the fourth behind it is loaded, never when
// the eighth is.
constexpr int kScaleSlots = 8, kScales = 16;

// What the roles have to know of a segment; the loader of Q leaves it with Q.
struct Brief {
  int unit, n0, chunks;                        // number of its first chunk along the share, and how many
  int seen, tokens, dual;                      // entries from its first chunk to the prefix's end; query tokens; two tiles of different rows
  int group, g, c0, len;                       // prefix, KV head, first chunk of the prefix, entries of the prefix
  // chunks that tile x takes, and the number of its j-th along the share: all, or those of its parity
  __device__ __forceinline__ int skip(int x) const { return dual ? 0 : (n0 ^ x) & 1; }
  __device__ __forceinline__ int chunks_of(int x) const { return dual ? chunks : (chunks + 1 - skip(x)) >> 1; }
  __device__ __forceinline__ int chunk(int x, int j) const { return n0 + (dual ? j : skip(x) + 2 * j); }
  // rows of tile x that come before the unit's first
  __device__ __forceinline__ int ahead(int x, int group) const { return x == 1 && !dual && tokens * group <= 64 ? 64 : 0; }
};

template <int NR>
struct PrefixBarriers {
  uint64_t q_full, q_empty, q_wide, v_tail;
  uint64_t k_full[kBars], k_empty[kBars], v_full[kBars], v_empty[kBars];
  uint64_t raw_full[NR], raw_empty[NR];        // 8-bit pages: V's codes
  uint64_t s_full[2][2], p_full[2][2];         // per tile and buffer: S is there; every softmax warp has stored its part of P
  uint64_t o_step[2];                          // per tile: O has the next step's product
  uint64_t o_done[2], o_free[2];               // per tile: a segment's O is complete; the softmax warps have read it
  uint64_t drained[2];
  Brief brief[2];                              // of even and odd segments
  uint32_t tmem_base;
  int abort_flag, first_group, first_unit;
  long long first_chunk;
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
// a / b of what is not negative: in 32 bits, several times as fast, wherever both fit.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}
__device__ __forceinline__ int sharing_ctas(const PrefixParams& p, long long total) {
  return static_cast<int>(min(static_cast<long long>(p.ctas), total));
}

// The deal.  A CTA that goes from one unit to the next spends what three chunks take on it (the output's way out, the next queries' way in:
// 5.5 us of 1.9 a chunk), so every unit counts for its chunks and three more in front of them, which are nobody's work; with less than two
// chunks for a CTA they would only make shares uneven, and chunks alone count.  (48 x 4 tokens over 4 prefixes, 11 chunks a CTA:
// 38.6 us with chunks alone, 36.0 with units; 64 over one prefix of 32768, 14 chunks a CTA: 40.2 and 38.2; with one sum of the weights.)
__device__ __forceinline__ int unit_cost(const PrefixParams& p, long long chunks) { return chunks >= 2ll * p.ctas ? 3 : 0; }

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
};

// Two floats to a pair of e4m3 codes, to nearest even (`lo` in the low byte).
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// D[tmem] (+)= A[smem] * B[smem]^T, e4m3 x e4m3 -> fp32, 32 elements of the contraction, issued by one thread.
__device__ __forceinline__ void tc_mma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// K-major operand tile in rows of 64 bytes with the 64-byte swizzle: groups of 8 rows are 512 bytes apart.
__device__ __forceinline__ uint64_t umma_desc_k_sw64(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(1) << 16;
  d |= static_cast<uint64_t>(512 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(4) << 61;                            // layout: SWIZZLE_64B
  return d;
}
// Eight codes as fp16: one conversion for two of them, of which an SM does 16 a cycle.
__device__ __forceinline__ uint4 widen8_half(uint32_t a, uint32_t b) { return make_uint4(widen_lo(a), widen_hi(a), widen_lo(b), widen_hi(b)); }

// Codes as bf16 times a power of two, without conversions (two of them for a pair, with the rounding back to bf16, took twice as long):
// a code's bits moved to bf16's places are the code times 2^-120, subnormals included, and a bf16 product brings it back, exactly.
// Only NaN (all ones, what 480 would be) needs to be told apart: the largest of the bits stays behind in `most`.
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t widen2_bf16(uint32_t em, uint32_t sign, uint32_t up, uint32_t times, uint32_t& most) {
  most = __vmaxu2(most, em);
  const uint32_t r = bf16x2_mul((sign & 0x80008000u) | em, up);
  return times == 0x3f803f80u ? r : bf16x2_mul(r, times);
}
// Four codes come out in the order 0, 2, 1, 3: even ones and odd ones are two masks of the word.
__device__ __forceinline__ uint4 widen8_bf16(uint32_t a, uint32_t b, uint32_t up, uint32_t times, uint32_t& most) {
  constexpr uint32_t kMask = 0x07f007f0u;
  return make_uint4(widen2_bf16((a << 4) & kMask, a << 8, up, times, most), widen2_bf16((a >> 4) & kMask, a, up, times, most),
                    widen2_bf16((b << 4) & kMask, b << 8, up, times, most), widen2_bf16((b >> 4) & kMask, b, up, times, most));
}
// The same, in the same order, by conversions, which know NaN.
__device__ __forceinline__ uint4 widen8_any(uint32_t a, uint32_t b, float s) {
  uint4 r = widen8_half(__byte_perm(a, 0, 0x3120), __byte_perm(b, 0, 0x3120));
  float lo, hi;
  unpack16<true>(r.x, lo, hi); r.x = pack16<false>(lo * s, hi * s);
  unpack16<true>(r.y, lo, hi); r.y = pack16<false>(lo * s, hi * s);
  unpack16<true>(r.z, lo, hi); r.z = pack16<false>(lo * s, hi * s);
  unpack16<true>(r.w, lo, hi); r.w = pack16<false>(lo * s, hi * s);
  return r;
}

// ---- two floats at a time ----
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void split(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 2^x of two values of at most 127, without the special-function unit: x = n + f with n nearest to x, 2^f a polynomial (interpolation of
// (2^f - 1) / f at the five Chebyshev nodes of [-1/2, 1/2]: off by at most 2^-22, relative), 2^n by its exponent.  Below 2^-126 it
// comes out as 0 or as something below 2^-126; NaN stays.
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
  float x0, x1, t0, t1;
  split(x, x0, x1);
  x = pair_of(max_nan(x0, -127.0f), max_nan(x1, -127.0f));
  const float kMagic = 12582912.0f + 127.0f;              // 1.5 * 2^23: the sum's low bits are n, here with the exponent's bias
  const uint64_t t = add2(x, pair_of(kMagic, kMagic));
  const uint64_t n = add2(t, pair_of(-kMagic, -kMagic));
  const uint64_t f = fma2(n, pair_of(-1.0f, -1.0f), x);
  uint64_t y = fma2(f, pair_of(0x1.5ec866p-10f, 0x1.5ec866p-10f), pair_of(0x1.3cbf6p-7f, 0x1.3cbf6p-7f));
  y = fma2(y, f, pair_of(0x1.c6afeep-5f, 0x1.c6afeep-5f));
  y = fma2(y, f, pair_of(0x1.ebfa4cp-3f, 0x1.ebfa4cp-3f));
  y = fma2(y, f, pair_of(0x1.62e43p-1f, 0x1.62e43p-1f));
  y = fma2(y, f, pair_of(1.0f, 1.0f));
  split(t, t0, t1);
  return mul2(y, pair_of(__uint_as_float(__float_as_uint(t0) << 23), __uint_as_float(__float_as_uint(t1) << 23)));
}

template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

}  // namespace

template <int D, bool kE4M3, bool kOne>
__global__ void __launch_bounds__(PrefixCfg<D, kE4M3, kOne>::kThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                   const __grid_constant__ CUtensorMap tmap_v, const PrefixParams p) {
  using Cfg = PrefixCfg<D, kE4M3, kOne>;
  constexpr int NK = Cfg::kKTiles, NV = Cfg::kVTiles, NR = Cfg::kRaw, KH = Cfg::KH, kThreads = Cfg::kThreads, kWarps = Cfg::kWarps;
  extern __shared__ __align__(1024) uint8_t smem[];       // the tiles need 1024-byte alignment (128-byte swizzle atoms)
  uint8_t* const sK = smem;
  uint8_t* const sQ = sK + NK * Cfg::kKBytes;             // one or two row tiles
  uint8_t* const sV = sQ + Cfg::kQTiles * Cfg::kTileBytes;
  uint8_t* const sRaw = sV + NV * Cfg::kTileBytes;
  // 8-bit pages: the power of two that a row of Q was shifted by, and the scales of a chunk's pages
  long long* const scan = reinterpret_cast<long long*>(sRaw + (kE4M3 ? NR * Cfg::kRawBytes : 0));
  int8_t* const row_shift = reinterpret_cast<int8_t*>(scan) + Cfg::kScanBytes;                    // [tile][row]
  float* const page_scale = reinterpret_cast<float*>(row_shift + 2 * kTile);                      // [kScaleSlots][kScales]
  using Barriers = PrefixBarriers<NR>;
  static_assert(sizeof(Barriers) <= 896, "what is set aside for the barriers");
  Barriers* const bars = reinterpret_cast<Barriers*>(page_scale + kScaleSlots * kScales);

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
  long long u = 0, u_end = 0;                             // in chunks and what units cost, along all units
  int cost;
  Segment first;
  long long in_group;
  if (p.n_prefixes == 1) {                                // nothing to scan
    first.group = 0;
    first.of = group_of(p, 0);
    const long long units = static_cast<long long>(first.of.pairs) * Hkv;
    cost = unit_cost(p, units * first.of.chunks);
    const long long total = units * (first.of.chunks + cost);
    const int ctas = sharing_ctas(p, total);
    if (blockIdx.x == 0 && t == 0) {
      if (first.of.len != __ldcg(p.lens)) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_LEN);
      if (p.cu_seqs != nullptr) {
        const int a = __ldcg(p.cu_seqs), b = __ldcg(p.cu_seqs + 1);
        if (a < 0 || b < a || b > p.c.batch) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_GROUP);
      }
    }
    if (static_cast<int>(blockIdx.x) < ctas) {
      u = quotient(total * blockIdx.x, ctas);
      u_end = quotient(total * (blockIdx.x + 1), ctas);
    }
    if (u >= u_end) {                                     // nothing for this CTA (uniform)
      pdl_wait();
      return;
    }
    in_group = u;
  } else {
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
    if (lane == 31) { scan[warp] = before; scan[32 + warp] = before_u; }
    if (t == 0) bars->first_group = -1;
    __syncthreads();
    before -= mine;
    before_u -= units;
    long long total = 0, total_u = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) { before += scan[w]; before_u += scan[32 + w]; }
      total += scan[w];
      total_u += scan[32 + w];
    }
    cost = unit_cost(p, total);
    total += cost * total_u;
    before += cost * before_u;
    mine += cost * units;
    if (total_u > p.max_units) {                          // groups that overlap: there is no room for their pieces
      if (blockIdx.x == 0 && t == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_GROUP);
      total = 0;
    }
    const int ctas = sharing_ctas(p, total);
    if (static_cast<int>(blockIdx.x) < ctas) {
      u = quotient(total * blockIdx.x, ctas);
      u_end = quotient(total * (blockIdx.x + 1), ctas);
    }
    if (u < u_end && before <= u && u < before + mine) {
      long long at = before, at_u = before_u;
      for (int i = i0; i < i1; ++i) {
        const Group g = group_of(p, i);
        const long long k = static_cast<long long>(g.pairs) * Hkv * (g.chunks + cost);
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
    in_group = u - bars->first_chunk;
  }
  first.unit = static_cast<int>(quotient(in_group, first.of.chunks + cost));
  in_group -= static_cast<long long>(first.unit) * (first.of.chunks + cost);            // in the unit
  const long long next_unit = u - in_group + first.of.chunks + cost;
  first.c0 = static_cast<int>(max(in_group - cost, 0ll));
  first.c1 = static_cast<int>(min(static_cast<long long>(first.of.chunks), in_group - cost + (u_end - u)));
  if (first.c1 <= first.c0) {                             // no chunk (uniform)
    pdl_wait();
    return;
  }
  first.g = first.unit / first.of.pairs;                  // (of the prefix's units, so far)
  first.pair = first.unit - first.g * first.of.pairs;
  if (p.n_prefixes > 1) first.unit += bars->first_unit;
  first.n0 = 0;
  first.set(p);
  // Moves on to the next segment of the share, `at` where its unit starts; false when there is none.
  auto advance = [&](Segment& s, long long& at) -> bool {
    s.n0 += s.c1 - s.c0;
    if (u_end - at <= cost) return false;
    ++s.unit;
    if (++s.pair == s.of.pairs) {
      s.pair = 0;
      if (++s.g == Hkv) {
        s.g = 0;
        do { s.of = group_of(p, ++s.group); } while (s.of.pairs == 0);                 // at + cost < u_end: there is one
      }
    }
    s.c0 = 0;
    s.c1 = static_cast<int>(min(static_cast<long long>(s.of.chunks), u_end - at - cost));
    at += s.of.chunks + cost;
    s.set(p);
    return true;
  };

  if (t == 0) {
    mbar_init(&bars->q_full, 1);
    mbar_init(&bars->q_empty, 2 + 2 * kSoftmaxWarps);
    mbar_init(&bars->q_wide, kWideWarps);
    mbar_init(&bars->v_tail, 1);
    for (int i = 0; i < kBars; ++i) {
      mbar_init(&bars->k_full[i], 1); mbar_init(&bars->k_empty[i], 2);
      mbar_init(&bars->v_full[i], kE4M3 ? kWideWarps : 1); mbar_init(&bars->v_empty[i], 2);
    }
    for (int i = 0; i < NR; ++i) { mbar_init(&bars->raw_full[i], 1); mbar_init(&bars->raw_empty[i], kWideWarps); }
    for (int i = 0; i < 2; ++i) {
      for (int h = 0; h < 2; ++h) { mbar_init(&bars->s_full[i][h], 1); mbar_init(&bars->p_full[i][h], kSoftmaxWarps); }
      mbar_init(&bars->o_step[i], 1);
      mbar_init(&bars->o_done[i], 1);
      mbar_init(&bars->o_free[i], kSoftmaxWarps);
    }
    mbar_init(&bars->drained[0], 1);
    mbar_init(&bars->drained[1], 1);
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
  long long at = next_unit;
  // Id of page j of the chunk c of a prefix of `len` entries; kNoPage behind its end.  Whoever asks looks at the answer a chunk later: what is
  // done with a loaded value at once waits for it.
  constexpr int kNoPage = static_cast<int>(0x80000000u);
  auto page_of = [&](int group, int len, int c, int j) -> int {
    const int key = c * kTile + (j << p.c.page_log2);
    return j < pages && key < len ? __ldcg(p.table + static_cast<size_t>(group) * p.max_pages + (key >> p.c.page_log2)) : kNoPage;
  };
  // Its block (page * Hkv + g): -1 for none, page 0 for one outside the pool.
  auto block_of = [&](int page, int g) -> int {
    if (page == kNoPage) return -1;
    const long long blk = pool_block(page, p.c.n_pages, Hkv, g);
    if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PREFIX_PAGE); return g; }
    return static_cast<int>(blk);
  };

  if (warp == 0) {
    // ---------------- loader of K and V ----------------
    if constexpr (kE4M3) give_registers<Cfg::kCtrlRegs>();
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
      // (8-bit pages: page, then scale, a chain of two loads; kCols is 1 and lane = page)
      int blk = block_of(page_of(s.group, s.of.len, s.c0, lane / kCols), s.g);
      int next = page_of(s.group, s.of.len, s.c0 + 1, lane / kCols);
      float scale = kE4M3 && blk >= 0 ? __ldcg(p.c.k_scales + blk) : 0.0f, scale_v = kE4M3 && blk >= 0 ? __ldcg(p.c.v_scales + blk) : 0.0f;
      for (int c = s.c0; c < s.c1 && ok; ++c, ++n) {
        const int bar = n % kBars;
        if (n >= NK) ok = wait(&bars->k_empty[(n - NK) % kBars], (n - NK) / kBars & 1);
        if (!ok) break;
        if (kE4M3) {
          if (lane < 8) {
            page_scale[n % kScaleSlots * kScales + lane] = scale;
            page_scale[n % kScaleSlots * kScales + 8 + lane] = scale_v;
          }
          __syncwarp();
        }
        bring(&tmap_k, sK + n % NK * Cfg::kKBytes, &bars->k_full[bar], blk);
        k_out = n + 1;
        const int blk_v = blk;
        blk = block_of(next, s.g);
        next = page_of(s.group, s.of.len, c + 2, lane / kCols);
        if (kE4M3) {
          scale = blk >= 0 ? __ldcg(p.c.k_scales + blk) : 0.0f;
          scale_v = blk >= 0 ? __ldcg(p.c.v_scales + blk) : 0.0f;
        }
        if constexpr (kE4M3) {
          const int slot = n % NR;
          if (n >= NR) ok = wait(&bars->raw_empty[slot], (n / NR - 1) & 1);
          if (!ok) break;
          bring(&tmap_v, sRaw + slot * Cfg::kRawBytes, &bars->raw_full[slot], blk_v);
          v_out = n + 1;
        } else {
          if (n >= NV) ok = wait(&bars->v_empty[(n - NV) % kBars], (n - NV) / kBars & 1);
          if (!ok) break;
          const int have = s.of.len - c * kTile;
          uint8_t* const dst = sV + n % NV * Cfg::kTileBytes;
          if (have >= kTile) {
            bring(&tmap_v, dst, &bars->v_full[bar], blk_v);
            v_out = n + 1;
          } else {
            // the prefix's last entries: a zero weight does not silence a NaN behind them, so those rows are cleared
            bring(&tmap_v, dst, &bars->v_tail, blk_v);
            ok = wait(&bars->v_tail, tails & 1);
            if (!ok) { mbar_wait_drain(&bars->v_tail, tails & 1, p.hdr, SITE_PREFIX_DRAIN, limit); break; }
            ++tails;
            for (int i = lane; i < (kTile - have) * 8 * KH; i += 32) {
              const int col = i / ((kTile - have) * 8), rest = i - col * (kTile - have) * 8;
              *reinterpret_cast<uint4*>(dst + col * kHalfBytes + have * 128 + rest * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->v_full[bar]);
          }
        }
      }
    } while (ok && advance(s, at));
    // nothing may still be landing in shared memory when the CTA ends
    if (!ok && lane == 0) {
      for (int j = max(0, k_out - NK); j < k_out; ++j) mbar_wait_drain(&bars->k_full[j % kBars], j / kBars & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      if constexpr (kE4M3) {
        for (int j = max(0, v_out - NR); j < v_out; ++j) mbar_wait_drain(&bars->raw_full[j % NR], (j / NR) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      } else {
        for (int j = max(0, v_out - NV); j < v_out; ++j) mbar_wait_drain(&bars->v_full[j % kBars], j / kBars & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      }
    }
  } else if (warp == 3) {
    // ---------------- loader of Q, which tells the other roles what a segment is ----------------
    if constexpr (kE4M3) give_registers<Cfg::kCtrlRegs>();
    const uint64_t pol_q = l2_policy_evict_first();
    const uint32_t q_bytes = static_cast<uint32_t>(KH) * 128 * G * p.tile_tokens;
    bool ok = true;
    int segs = 0;
    do {
      if (segs > 0) ok = __all_sync(0xffffffffu, mbar_wait_parked(&bars->q_empty, (segs - 1) & 1, abort_flag, p.hdr, SITE_PREFIX_Q, limit));
      if (!ok) break;
      if (lane == 0) {
        bars->brief[segs & 1] = Brief{s.unit, s.n0, s.c1 - s.c0, s.of.len - s.c0 * kTile, s.tokens, s.dual ? 1 : 0, s.group, s.g, s.c0, s.of.len};
        mbar_arrive_expect_tx(&bars->q_full, (s.dual ? 2 : 1) * q_bytes);
        for (int x = 0; x < (s.dual ? 2 : 1); ++x)
          for (int c = 0; c < KH; ++c)
            tma_load_3d(sQ + x * Cfg::kTileBytes + c * kHalfBytes, &tmap_q, &bars->q_full, c * 64, s.g * G, s.token0 + x * p.tile_tokens, pol_q);
      }
      __syncwarp();
      ++segs;
    } while (advance(s, at));
    // the end of the share: nothing more to come
    if (ok) ok = __all_sync(0xffffffffu, mbar_wait_parked(&bars->q_empty, (segs - 1) & 1, abort_flag, p.hdr, SITE_PREFIX_Q, limit));
    if (lane == 0) {
      mbar_wait_drain(&bars->q_full, (segs - 1) & 1, p.hdr, SITE_PREFIX_DRAIN, limit);
      if (ok) {
        bars->brief[segs & 1].chunks = 0;
        mbar_arrive(&bars->q_full);
      }
    }
  } else if (warp < 3) {
    // ---------------- issuer of one row tile ----------------
    // One lane issues a tile's contractions, so that they execute in the order they are issued in: O += P V of a step, then S of the step
    // that takes P's place.  The whole warp walks the loop, with values that the compiler can see to be the same in every lane (a shuffle
    // from lane 0), so that descriptors live in uniform registers: in a branch of one lane a contraction took twice as long to
    // issue.  What is between two contractions is one warp's chain of dependent instructions, some ten cycles each: ring positions are
    // carried along, not worked out.
    if constexpr (kE4M3) give_registers<Cfg::kCtrlRegs>();
    const int x = __shfl_sync(0xffffffffu, warp, 0) - 1;
    // 8-bit pages: Q (its two terms) and K are e4m3 (formats 0), P and V bf16
    constexpr uint32_t idesc_s = umma_idesc_bf16_f32(kTile, kStep) & ~(kE4M3 ? (1u << 7) | (1u << 10) : 0u);
    constexpr uint32_t idesc_o = umma_idesc_bf16_f32(kTile, D) | (1u << 16);    // B (V) is MN-major
    // from a tile's first 64 entries to its second, in a descriptor's units
    constexpr uint64_t kHalfTile = kStep * 128 >> 4, kHalfKTile = kE4M3 ? kStep * D >> 4 : kHalfTile;
    constexpr uint64_t kTileStep = Cfg::kTileBytes >> 4, kBlockStep = kHalfBytes >> 4;
    const bool leader = elect_one();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    const uint32_t s_tmem = tmem + x * kTile, o_tmem = tmem + 256 + x * D;
    const uint64_t q_desc = umma_desc_k_sw128(smem_u32(sQ)), k_desc = kE4M3 && D == 64 ? umma_desc_k_sw64(smem_u32(sK)) : umma_desc_k_sw128(smem_u32(sK)),
                   v_desc = umma_desc_mn_sw128(smem_u32(sV), kHalfBytes);
    bool ok = true, issued = false, again = false;        // again: the tile has had a segment with chunks
    uint32_t q_phase = 0, p_phase = 0, o_phase = 0;       // (p_phase: the same for both buffers, they alternate)
    auto wait = [&](uint64_t* bar, uint32_t parity, int site) -> bool {
      return __all_sync(0xffffffffu, mbar_wait_nap(bar, parity, abort_flag, p.hdr, site, limit));
    };
    while (true) {
      ok = wait(&bars->q_full, q_phase, SITE_PREFIX_Q);
      if (!ok) break;
      const Brief& shared = bars->brief[q_phase];
      Brief br;
      br.chunks = __shfl_sync(0xffffffffu, shared.chunks, 0);
      br.n0 = __shfl_sync(0xffffffffu, shared.n0, 0);
      br.dual = kOne ? 0 : __shfl_sync(0xffffffffu, shared.dual, 0);
      br.tokens = __shfl_sync(0xffffffffu, shared.tokens, 0);
      if (br.chunks == 0) break;
      if (kE4M3) ok = wait(&bars->q_wide, q_phase, SITE_PREFIX_Q);
      q_phase ^= 1;
      const int chunks = br.chunks_of(x), stride = br.dual ? 1 : 2;
      const uint64_t a0 = q_desc + (br.dual ? x : 0) * kTileStep - static_cast<uint64_t>(br.ahead(x, G) * 128 >> 4);
      int n = br.chunk(x, 0), k_at = n % NK, v_at = n % NV, before = 0;   // the chunk whose S is next; its tiles; the one before it
      int v_before = 0;
      for (int j = 0; j <= chunks && chunks > 0 && ok; ++j) {
        uint64_t* const k_full = &bars->k_full[n % kBars];
        uint64_t* const v_full = &bars->v_full[before % kBars];
        const uint32_t k_phase = n / kBars & 1, v_phase = before / kBars & 1;
        const uint64_t kb = k_desc + k_at * static_cast<uint64_t>(Cfg::kKBytes >> 4), vb = v_desc + v_before * kTileStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (j > 0) {                                    // O (+)= P V of the chunk before
            if (h == 0) {
              ok = wait(v_full, v_phase, SITE_PREFIX_V);
              if (ok && j == 1 && again) {
                ok = wait(&bars->o_free[x], o_phase, SITE_PREFIX_O);
                o_phase ^= 1;
              }
            }
            ok = ok && wait(&bars->p_full[x][h], p_phase, SITE_PREFIX_P);
            if (!ok) break;
            tc_fence_after_sync();
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < kStep / 16; ++kk)     // 16 entries = 8 packed columns of P, 2048 bytes of V
                tc_mma_bf16_ts(o_tmem, s_tmem + h * kStep + kk * 8, vb + h * kHalfTile + static_cast<uint64_t>(kk * (2048 >> 4)), idesc_o,
                               (j > 1 || h > 0 || kk > 0) ? 1u : 0u);
              tc_commit(&bars->o_step[x]);
              if (h == 1) {                               // a tile is free when both row tiles have released it
                tc_commit(&bars->v_empty[before % kBars]);
                if (!br.dual) tc_commit(&bars->v_empty[before % kBars]);
                if (j == chunks) tc_commit(&bars->o_done[x]);
              }
            }
            __syncwarp();
          }
          if (j < chunks) {                               // S = Q K^T
            if (h == 0) {
              ok = wait(k_full, k_phase, SITE_PREFIX_K);
              if (!ok) break;
              tc_fence_after_sync();
              issued = true;
            }
            if (leader) {
              if constexpr (kE4M3) {
                // the terms of Q: the leading one's tile, then the other's (head dimension 64: the halves of a row)
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  const int term = kk / (D / 32), step = kk % (D / 32) * 2;             // 32 elements, 32 bytes a step
                  tc_mma_e4m3(s_tmem + h * kStep, a0 + term * (D == 128 ? kBlockStep : 4) + step, kb + h * kHalfKTile + step, idesc_s, kk > 0 ? 1u : 0u);
                }
              } else {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {     // 64-element block kk / 4, 32 bytes per step inside it
                  const uint64_t step = (kk >> 2) * kBlockStep + (kk & 3) * 2;
                  tc_mma_bf16(s_tmem + h * kStep, a0 + step, kb + h * kHalfTile + step, idesc_s, kk > 0 ? 1u : 0u);
                }
              }
              if (!(x == 0 && n == p.skip_commit)) tc_commit(&bars->s_full[x][h]);    // (test hook: a completion that is never signalled)
              if (h == 1) {
                tc_commit(&bars->k_empty[n % kBars]);
                if (!br.dual) tc_commit(&bars->k_empty[n % kBars]);
              }
            }
            __syncwarp();
          }
        }
        if (j > 0) p_phase ^= 1;
        before = n;
        v_before = v_at;
        n += stride;
        k_at = NK == 1 ? 0 : n % NK;
        v_at += stride;
        if (v_at >= NV) v_at -= NV;
      }
      if (!ok) break;
      if (leader) {
        if (chunks > 0) tc_commit(&bars->q_empty); else mbar_arrive(&bars->q_empty);
      }
      __syncwarp();
      again = again || chunks > 0;
    }
    // every contraction issued has finished before tensor memory is released
    if (issued) {
      if (leader) tc_commit(&bars->drained[x]);
      __syncwarp();
      mbar_wait_drain(&bars->drained[x], 0, p.hdr, SITE_PREFIX_DRAIN, limit);
    }
  } else if (warp < kCtrlWarps + 2 * kSoftmaxWarps) {
    // ---------------- softmax: four warps per row tile, a thread per row ----------------
    if constexpr (kE4M3) take_registers<Cfg::kSoftmaxRegs>();
    // Every kPoly-th pair of exponentials does without the special-function unit, which does 16 a cycle and SM: with 256 rows it would be
    // busy for 1024 cycles a step otherwise.  (0: none)
    constexpr int kPoly = kOne ? 0 : 4;
    const int gw = warp - kCtrlWarps;
    const int x = gw >> 2, quarter = gw & 3;              // row tile; lane quarter (warp % 4: the control warps are four)
    const int at_lane = quarter * 32 + lane;              // tensor-memory lane
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + x * kTile, o_addr = lane_addr + 256 + x * D;
    bool ok = true;
    int sn = 0, o_segs = 0, segs = 0;                     // this tile's steps, its segments with steps, and all segments so far
    while (ok) {
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars->q_full, segs & 1, abort_flag, p.hdr, SITE_PREFIX_Q, limit));
      if (!ok) break;
      const Brief& br = bars->brief[segs & 1];
      if (br.chunks == 0) break;
      const int dual = kOne ? 0 : br.dual, steps = 2 * br.chunks_of(x), n_first = br.chunk(x, 0), n_step = dual ? 1 : 2;
      const int tokens = dual ? (x == 0 ? p.tile_tokens : br.tokens - p.tile_tokens) : br.tokens, rows = tokens * G;
      const int r = at_lane - (kOne || !dual ? br.ahead(x, G) : 0);      // row of the tile
      int seen = br.seen - (n_first - br.n0) * kTile;     // entries from the step's first one to the prefix's end
      const long long piece = static_cast<long long>(br.unit) + blockIdx.x;
      ++segs;
      // what the warp needs of the segment that the next one writes over has been read: as far as it goes, the next one may come
      auto taken = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->q_empty);
      };
      if (r - lane < 0 || r - lane >= rows) {
        taken();
        // no rows: the warp only keeps step (nobody may run ahead of a barrier by two phases)
        for (int i = 0; i < steps && ok; ++i, ++sn) {
          ok = __all_sync(0xffffffffu, mbar_wait_nap(&bars->s_full[x][sn & 1], (sn >> 1) & 1, abort_flag, p.hdr, SITE_PREFIX_S, limit));
          if (ok && lane == 0) mbar_arrive(&bars->p_full[x][sn & 1]);
        }
        if (steps > 0 && ok) {
          ok = __all_sync(0xffffffffu, mbar_wait_nap(&bars->o_done[x], o_segs & 1, abort_flag, p.hdr, SITE_PREFIX_O, limit));
          if (ok && lane == 0) mbar_arrive(&bars->o_free[x]);
          ++o_segs;
        }
        continue;
      }
      float by_row = p.scale_log2;                        // what a logit is multiplied by
      if (kE4M3) {
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars->q_wide, (segs - 1) & 1, abort_flag, p.hdr, SITE_PREFIX_Q, limit));
        if (!ok) break;
        by_row *= __uint_as_float(pow2_bits(-row_shift[(dual ? x : 0) * kTile + r]));
      }
      taken();
      float m_ref = -INFINITY, l = 0.0f, lr = 0.0f;       // sums of the weights, and of the weights as rounded
      for (int i = 0; i < steps; ++i, ++sn) {
        const int h = i & 1, n = n_first + n_step * (i >> 1);         // (a segment's steps are even in number: sn & 1 == h)
        ok = mbar_wait_bounded(&bars->s_full[x][h], (sn >> 1) & 1, abort_flag, p.hdr, SITE_PREFIX_S, limit);
        if (kE4M3 && ok) ok = mbar_wait_bounded(&bars->k_full[n % kBars], n / kBars & 1, abort_flag, p.hdr, SITE_PREFIX_K, limit);   // the scales (long there)
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after_sync();
        float v[kStep / 32][32];
        float f[kE4M3 ? kStep / 16 : 1];                  // what 16 logits (of one page) are multiplied by
        float most = -INFINITY;
        f[0] = by_row;
#pragma unroll
        for (int c = 0; c < kStep / 32; ++c) tmem_ld_32x32(s_addr + h * kStep + c * 32, v[c]);
        if (seen < kStep) {
#pragma unroll
          for (int c = 0; c < kStep / 32; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e) v[c][e] = c * 32 + e < seen ? v[c][e] : -INFINITY;
        }
        seen -= h == 0 ? kStep : (n_step * 2 - 1) * kStep;
#pragma unroll
        for (int c = 0; c < kStep / 32; ++c)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            // positive, so that masked logits stay -infinity
            if (kE4M3) f[c * 2 + z] = fmaxf(by_row * page_scale[n % kScaleSlots * kScales + ((h * kStep + c * 32 + z * 16) >> p.c.page_log2)], 1.17549435e-38f);
            float mx[2] = {v[c][z * 16], v[c][z * 16 + 1]};
#pragma unroll
            for (int e = 2; e < 16; e += 2) { mx[0] = fmaxf(mx[0], v[c][z * 16 + e]); mx[1] = fmaxf(mx[1], v[c][z * 16 + e + 1]); }
            most = fmaxf(most, fmaxf(mx[0], mx[1]) * f[kE4M3 ? c * 2 + z : 0]);
          }
        // the reference moves only when a logit comes close to it (or at a row's first logits)
        const bool move = most > m_ref - kRoomLog2;
        if (__any_sync(0xffffffffu, move)) {
          const float to = most + (kSlackLog2 + kRoomLog2), alpha = move ? ex2(m_ref - to) : 1.0f;
          if (move) { m_ref = to; l *= alpha; lr *= alpha; }
          if (i >= 1) {
            // The step before this one may still be on its way into O.  (The one before that is in it: S of this step was issued behind it.  So
            // the barrier is at this phase or through with it, never further.)
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars->o_step[x], (sn - 1) & 1, abort_flag, p.hdr, SITE_PREFIX_O, limit));
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              float o[16];
              tmem_ld_32x16(o_addr + c * 16, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] *= alpha;
              tmem_st_32x16(o_addr + c * 16, o);
            }
          }
        }
        const float neg_ref = m_ref == -INFINITY ? 0.0f : -m_ref;   // nothing seen yet: every weight is 2^-inf
        const uint64_t neg2 = pair_of(neg_ref, neg_ref);
        uint64_t ls = 0, lrs = 0;
#pragma unroll
        for (int c = 0; c < kStep / 32; ++c) {
          float packed[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float by = f[kE4M3 ? (c * 32 + e) / 16 : 0];
            uint64_t w = fma2(pair_of(v[c][e], v[c][e + 1]), pair_of(by, by), neg2);
            float e0, e1;
            if (kPoly > 0 && e / 2 % kPoly == kPoly - 1) {
              w = exp2_pair(w);
              split(w, e0, e1);
            } else {
              split(w, e0, e1);
              e0 = ex2(e0);
              e1 = ex2(e1);
              w = pair_of(e0, e1);
            }
            ls = add2(ls, w);
            const uint32_t pair = pack16<false>(e0, e1);
            lrs = add2(lrs, pair_of(__uint_as_float(pair << 16), __uint_as_float(pair & 0xffff0000u)));
            packed[e / 2] = __uint_as_float(pair);
          }
          tmem_st_32x16(s_addr + h * kStep + c * 16, packed);
        }
        float l0, l1;
        split(ls, l0, l1);
        l += l0 + l1;
        split(lrs, l0, l1);
        lr += l0 + l1;
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->p_full[x][h]);
      }
      if (!ok) break;
      // ---- the segment's piece: four columns of O by rows, so that a warp's stores are whole lines ----
      float4* const ml = p.part_ml + (piece * 2 + x) * p.tile_rows + r;
      if (steps == 0) {
        if (r < rows) *ml = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
        continue;
      }
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars->o_done[x], o_segs & 1, abort_flag, p.hdr, SITE_PREFIX_O, limit));
      ++o_segs;
      if (!ok) break;
      tc_fence_after_sync();
      if (r < rows) __stcg(ml, make_float4(m_ref, lr, l, 0.0f));
      float4* po = reinterpret_cast<float4*>(p.part_o) + (piece * 2 + x) * (D / 4) * p.tile_rows + r;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float o[32];
        tmem_ld_32x32(o_addr + c * 32, o);
#pragma unroll
        for (int e = 0; e < 8; ++e, po += p.tile_rows)
          if (r < rows) __stcg(po, make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]));
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->o_free[x]);
    }
  } else {
    // ---------------- widening (8-bit pages): Q into two e4m3 terms, V's codes to bf16 ----------------
    if constexpr (kE4M3) {
      give_registers<Cfg::kWideRegs>();
      const int w = warp - kCtrlWarps - 2 * kSoftmaxWarps;
      bool ok = true;
      int n = 0, segs = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity, int site) -> bool {
        return __all_sync(0xffffffffu, mbar_wait_nap(bar, parity, abort_flag, p.hdr, site, limit));
      };
      const int first = w * (kTile / kWideWarps);         // the warp's 16 rows of every tile of V
      constexpr int kPieces = D / 16;                     // 16-byte pieces of a row of codes
      constexpr int kRowsAt = 32 / kPieces;               // rows of a warp's step
      // Eight lanes (what shared memory serves at a time) take four pieces of one column block of two neighbouring rows: the
      // swizzle puts their 16-byte stores into eight different places of a line.
      const int c4 = lane & 3, block = D == 128 ? (lane >> 3) & 1 : 0;
      const int row_in = ((lane >> 2) & 1) + (D == 128 ? (lane >> 4) * 2 : (lane >> 3) * 2);
      while (true) {
        ok = wait(&bars->q_full, segs & 1, SITE_PREFIX_Q);
        if (!ok) break;
        const Brief br = bars->brief[segs & 1];
        if (br.chunks == 0) break;
        // ---- Q: two threads per row, in place.  After a power-of-two shift that brings the row's largest element to [2^7, 2^8), an element is
        // the sum of its nearest e4m3 value and the e4m3 value nearest to the rest: exact down to 2^-9 of the largest (8 bits are 4 and 4),
        // and what is smaller is off by at most 2^-17 of the largest. ----
        for (int tile = 0; tile < (!kOne && br.dual ? 2 : 1); ++tile) {
          const int row = w * 16 + (lane >> 1), half = lane & 1;
          uint8_t* const at_row = sQ + tile * Cfg::kTileBytes + row * 128;
          auto piece_at = [&](int i) -> uint4* {          // 16 bytes, number i of the row's lines (one or two)
            return reinterpret_cast<uint4*>(at_row + (i >> 3) * kHalfBytes + (((i & 7) ^ (row & 7)) << 4));
          };
          uint32_t q[D / 4];                              // half a row
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const uint4 v = *piece_at(half * (D / 16) + i);
            q[4 * i] = v.x; q[4 * i + 1] = v.y; q[4 * i + 2] = v.z; q[4 * i + 3] = v.w;
          }
          uint32_t most = 0;                              // the largest element's bits (bf16, without the sign)
#pragma unroll
          for (int i = 0; i < D / 4; ++i) most = __vmaxu2(most, q[i] & 0x7fff7fffu);
          most = max(most & 0xffffu, most >> 16);
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));                      // (and nobody of the warp reads elements any more)
          int up = most > 0 ? 7 - scale_log2(most << 16) : 0;
          up = up > 120 ? 120 : up;                       // of a subnormal row; otherwise within [-120, 120] as it stands
          const float f = __uint_as_float(pow2_bits(up));
          const bool finite = most < 0x7f80u;
          if (half == 0) row_shift[tile * kTile + row] = static_cast<int8_t>(up);
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {              // 16 elements
            uint32_t high[4], low[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t hi2[2], lo2[2];
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                float x, y, u, v;
                unpack16<false>(q[8 * i + 2 * e + z], x, y);
                x *= f;
                y *= f;
                hi2[z] = pack_e4m3(x, y);
                unpack16<true>(widen_lo(hi2[z]), u, v);
                lo2[z] = pack_e4m3(x - u, y - v);
              }
              high[e] = finite ? hi2[0] | hi2[1] << 16 : 0x7f7f7f7fu;                   // an infinite or NaN row becomes NaN
              low[e] = lo2[0] | lo2[1] << 16;
            }
            // the leading terms, and in the row's other line (head dimension 64: its line's other half) the rests
            *piece_at(half * (D / 32) + i) = make_uint4(high[0], high[1], high[2], high[3]);
            *piece_at(D / 16 + half * (D / 32) + i) = make_uint4(low[0], low[1], low[2], low[3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->q_wide);
        ++segs;
        for (int c = br.c0; c < br.c0 + br.chunks && ok; ++c, ++n) {
          const int have = br.len - c * kTile;
          const int slot = n % NR, gone = n - NV;         // gone: the chunk whose tile this one takes
          ok = wait(&bars->raw_full[slot], (n / NR) & 1, SITE_PREFIX_RAW);
          if (ok && gone >= 0) ok = wait(&bars->v_empty[gone % kBars], gone / kBars & 1, SITE_PREFIX_RAW);
          if (!ok) break;
          const uint8_t* const src = sRaw + slot * Cfg::kRawBytes + (first + row_in) * D + (block * 4 + c4) * 16;
          uint8_t* const tile = sV + n % NV * Cfg::kTileBytes + block * kHalfBytes;
          // row y * kRowsAt + row_in of the warp's: where its two 16-byte pieces go
          auto put = [&](int y, const uint4& a, const uint4& b) {
            const int r = first + y * kRowsAt + row_in;
            *reinterpret_cast<uint4*>(tile + r * 128 + (((2 * c4) ^ (r & 7)) << 4)) = a;
            *reinterpret_cast<uint4*>(tile + r * 128 + (((2 * c4 + 1) ^ (r & 7)) << 4)) = b;
          };
          constexpr int kSteps = kTile / kWideWarps / kRowsAt;
          const float f = page_scale[n % kScaleSlots * kScales + 8 + (first >> p.c.page_log2)];         // the warp's 16 rows are one page's
          // 2^120 f in one factor, unless that is too large for one
          const bool two = f > 128.0f;
          const uint32_t up = __byte_perm(__float_as_uint(two ? 1.329227995784916e36f : f * 1.329227995784916e36f), 0, 0x3232);
          const uint32_t times = __byte_perm(__float_as_uint(two ? f : 1.0f), 0, 0x3232);
          uint32_t most = 0;
          uint4 q[kSteps];
#pragma unroll
          for (int y = 0; y < kSteps; ++y) q[y] = *reinterpret_cast<const uint4*>(src + y * kRowsAt * D);
#pragma unroll
          for (int y = 0; y < kSteps; ++y) put(y, widen8_bf16(q[y].x, q[y].y, up, times, most), widen8_bf16(q[y].z, q[y].w, up, times, most));
          // NaN among the codes, or the prefix's end among the rows: those again
          if (__any_sync(0xffffffffu, (most & 0xffffu) == 0x7f0u || most >> 16 == 0x7f0u) || have < kTile) {
#pragma unroll 1
            for (int y = 0; y < kSteps; ++y) {
              uint4 q = *reinterpret_cast<const uint4*>(src + y * kRowsAt * D);
              if (first + y * kRowsAt + row_in >= have) q = make_uint4(0u, 0u, 0u, 0u);          // behind the end: zeros
              put(y, widen8_any(q.x, q.y, f), widen8_any(q.z, q.w, f));
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&bars->v_full[n % kBars]);
            mbar_arrive(&bars->raw_empty[slot]);
          }
        }
        if (!ok) break;
      }
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

// Joins a query row's pieces and the attention over its own entries.  A block takes 32 rows (lane = row; the pieces hold columns by rows),
// a warp some columns of them.  SPLIT: warps that share the pieces out and meet once in shared memory; 1: a warp has all of them, and the
// block every column.  All of it is latency: every load that can be is in flight before the first is used, the row's own entries are
// what the sum starts from, and up to 32 prefixes are scanned without a barrier.
template <int D, int SPLIT>
struct MergeCfg {
  static constexpr int kCols = SPLIT > 8 ? 8 : 16;        // columns of a warp
  static constexpr int kAhead = SPLIT > 8 ? 3 : 2;        // pieces whose loads are in flight
  static constexpr int kWarps = SPLIT == 1 ? D / kCols : SPLIT;
  static constexpr int kResident = SPLIT > 8 ? 32 : 24;   // warps on an SM
};
template <int D, bool kE4M3, int SPLIT>
__global__ void __launch_bounds__(32 * MergeCfg<D, SPLIT>::kWarps, MergeCfg<D, SPLIT>::kResident / MergeCfg<D, SPLIT>::kWarps)
prefix_merge_kernel(const PrefixParams p) {
  using Cfg = MergeCfg<D, SPLIT>;
  constexpr int kWarps = Cfg::kWarps, kMergeThreads = 32 * kWarps, kMergeCols = Cfg::kCols;
  // chunks and units of the prefixes before (more than 32 of them), later the warps' sums
  constexpr int kSums = SPLIT == 1 ? 0 : kWarps * 32 * (kMergeCols + 1) * 4, kScan = kMaxPrefixes * 12;
  __shared__ __align__(16) uint8_t space[kSums > kScan ? kSums : kScan];
  auto acc_of = reinterpret_cast<float (*)[32][kMergeCols + 1]>(space);
  long long* const chunk0 = reinterpret_cast<long long*>(space);
  int* const unit0 = reinterpret_cast<int*>(chunk0 + kMaxPrefixes);
  __shared__ float2 ml_of[SPLIT == 1 ? 1 : kWarps][32];
  __shared__ long long scratch[kWarps], scratch_u[kWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len, n = p.n_prefixes;
  pdl_launch_dependents();
  // (what is read here was there before the kernel before this one began)
  const bool few = n <= 32;                               // then every warp scans the prefixes for itself, a lane each
  long long total, before = 0, before_u = 0;              // of prefix `lane` (few), or of the block's scan
  Group mine_of = {};
  int cost;
  int first_seq = 0x7fffffff;
  {
    const int threads = few ? 32 : kMergeThreads, at = few ? lane : t;
    const int per = few ? 1 : (n + threads - 1) / threads, i0 = min(at * per, n), i1 = min(i0 + per, n);
    long long mine = 0, units = 0;
    for (int i = i0; i < i1; ++i) {
      const Group g = group_of(p, i);
      if (few) { mine_of = g; first_seq = p.cu_seqs != nullptr ? __ldcg(p.cu_seqs + i) : 0; }
      units += static_cast<long long>(g.pairs) * Hkv;
      mine += static_cast<long long>(g.pairs) * Hkv * g.chunks;
    }
    before = mine;
    before_u = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, before, o), z = __shfl_up_sync(0xffffffffu, before_u, o);
      if (lane >= o) { before += y; before_u += z; }
    }
    long long all = __shfl_sync(0xffffffffu, before, 31), all_u = __shfl_sync(0xffffffffu, before_u, 31);
    if (!few) {
      if (lane == 31) { scratch[warp] = before; scratch_u[warp] = before_u; }
      __syncthreads();
      all = all_u = 0;
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) { before += scratch[w]; before_u += scratch_u[w]; }
        all += scratch[w];
        all_u += scratch_u[w];
      }
    }
    before -= mine;
    before_u -= units;
    cost = unit_cost(p, all);
    all += cost * all_u;
    before += cost * before_u;
    if (!few) {
      long long c = before, z = before_u;
      for (int i = i0; i < i1; ++i) {
        const Group g = group_of(p, i);
        chunk0[i] = c;
        unit0[i] = static_cast<int>(z);
        c += static_cast<long long>(g.pairs) * Hkv * (g.chunks + cost);
        z += static_cast<long long>(g.pairs) * Hkv;
      }
      __syncthreads();
    }
    total = all_u > p.max_units ? 0 : all;
  }
  const int rows = p.c.batch * T * G;                     // of a KV head
  const int R = blockIdx.x * 32 + lane, g = blockIdx.y, col0 = (SPLIT == 1 ? warp : blockIdx.z) * kMergeCols;
  const int token = R / G, b = token / T;
  // ---- this row's pieces: `count` of them from `piece` on, and the same rows' other half of the chunks where one tile took both ----
  int count = 0, both = 1;
  const float4* ml = p.part_ml;
  const float4* po = reinterpret_cast<const float4*>(p.part_o);
  int lo = 0;                                             // the last prefix that starts at or before the row's sequence
  Group gr;
  long long chunk_at, unit_at;
  if (few) {
    for (int i = 1; i < n; ++i)
      if (__shfl_sync(0xffffffffu, first_seq, i) <= b) lo = i;
    gr.seq0 = __shfl_sync(0xffffffffu, mine_of.seq0, lo);
    gr.tokens = __shfl_sync(0xffffffffu, mine_of.tokens, lo);
    gr.chunks = __shfl_sync(0xffffffffu, mine_of.chunks, lo);
    gr.pairs = __shfl_sync(0xffffffffu, mine_of.pairs, lo);
    chunk_at = __shfl_sync(0xffffffffu, before, lo);
    unit_at = __shfl_sync(0xffffffffu, before_u, lo);
  } else {
    int hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldcg(p.cu_seqs + mid) <= b) lo = mid; else hi = mid;
    }
    gr = group_of(p, lo);
    chunk_at = chunk0[lo];
    unit_at = unit0[lo];
    __syncthreads();                                      // (the sums go there)
  }
  if (R < rows && total > 0) {
    const int in = token - gr.seq0 * T;
    if (in >= 0 && in < gr.tokens && gr.pairs > 0) {
      const int pair = in / (2 * p.tile_tokens), rest = in - pair * 2 * p.tile_tokens;
      const bool dual = min(gr.tokens - pair * 2 * p.tile_tokens, 2 * p.tile_tokens) > p.tile_tokens;
      const int tile = rest / p.tile_tokens, row = (rest - tile * p.tile_tokens) * G + R - token * G;
      const long long unit = static_cast<long long>(g) * gr.pairs + pair, q0 = chunk_at + unit * (gr.chunks + cost) + cost, q1 = q0 + gr.chunks;
      const int ctas = sharing_ctas(p, total);
      const int ca = static_cast<int>(quotient((q0 + 1) * ctas - 1, total)), cb = static_cast<int>(quotient(q1 * ctas - 1, total));
      const long long piece = unit_at + unit + ca;
      both = dual ? 1 : 2;
      count = (cb - ca + 1) * both;
      ml += (piece * 2 + tile) * p.tile_rows + row;
      po += ((piece * 2 + tile) * (D / 4) + col0 / 4) * p.tile_rows + row;
    }
  }
  const int most = __reduce_max_sync(0xffffffffu, count);
  pdl_wait();
  // ---- the sum starts with the row's own entries (8-bit pages: the pieces' columns 1 and 2 of four have changed places), at half their
  // size: next to values at the end of the range there is room for the pieces' ----
  constexpr int k1 = kE4M3 ? 2 : 1, k2 = kE4M3 ? 1 : 2;
  const int sub = SPLIT == 1 ? 0 : warp;
  const size_t at = static_cast<size_t>(token) * p.n_q_heads + g * G + R - token * G;
  float M = -INFINITY, L = 0.0f, E = 0.0f, acc[kMergeCols];        // reference, what the output is divided by, sum of the weights
#pragma unroll
  for (int i = 0; i < kMergeCols; ++i) acc[i] = 0.0f;
  if (R < rows && sub == 0) {
    const float own = __ldcg(p.own_lse + at);
    const float4* from = reinterpret_cast<const float4*>(p.own_out + at * D + col0);
#pragma unroll
    for (int i = 0; i < kMergeCols; i += 4) {
      const float4 y = __ldcg(from + i / 4);
      acc[i] = 0.5f * y.x; acc[i + k1] = 0.5f * y.y; acc[i + k2] = 0.5f * y.z; acc[i + 3] = 0.5f * y.w;
    }
    M = fmaf(own, 1.4426950408889634f, 1.0f);
    L = E = own == -INFINITY ? 0.0f : 0.5f;               // (without entries its output is zeros)
  }
  const size_t step_ml = static_cast<size_t>(p.tile_rows), step_o = static_cast<size_t>(D / 4) * p.tile_rows;
  constexpr int kAhead = Cfg::kAhead;
  for (int s0 = sub; s0 < most; s0 += kAhead * SPLIT) {
    float4 v[kAhead];
    float o[kAhead][kMergeCols];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = s0 + k * SPLIT;
      v[k] = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
      if (s < count) {
        const size_t tile = both == 2 ? s : 2 * s;        // tiles of a piece lie side by side
        v[k] = __ldcg(ml + tile * step_ml);
        const float4* at = po + tile * step_o;
#pragma unroll
        for (int i = 0; i < kMergeCols; i += 4, at += p.tile_rows) {
          const float4 y = __ldcg(at);
          o[k][i] = y.x; o[k][i + 1] = y.y; o[k][i + 2] = y.z; o[k][i + 3] = y.w;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (v[k].y == 0.0f) continue;                       // nothing seen; NaN stays
      const float top = fmaxf(M, v[k].x), ref = top == -INFINITY ? 0.0f : top;
      const float a = ex2(M - ref), w = ex2(v[k].x - ref);
      M = top;
      L = fmaf(L, a, v[k].y * w);
      E = fmaf(E, a, v[k].z * w);
#pragma unroll
      for (int i = 0; i < kMergeCols; ++i) acc[i] = fmaf(acc[i], a, o[k][i] * w);
    }
  }
  if constexpr (SPLIT == 1) {
    if (R >= rows) return;
    const float f = L != 0.0f ? 1.0f / L : 0.0f;
    uint32_t o[kMergeCols / 2];
#pragma unroll
    for (int i = 0; i < kMergeCols; i += 4) {
      o[i / 2] = pack16<false>(acc[i] * f, acc[i + k1] * f);
      o[i / 2 + 1] = pack16<false>(acc[i + k2] * f, acc[i + 3] * f);
    }
    uint4* to = reinterpret_cast<uint4*>(p.out + at * D + col0);
    to[0] = make_uint4(o[0], o[1], o[2], o[3]);
    to[1] = make_uint4(o[4], o[5], o[6], o[7]);
    if (p.lse != nullptr && col0 == 0) p.lse[at] = L != 0.0f ? (M + log2f(E)) * 0.6931471805599453f : -INFINITY;
  } else {
    ml_of[warp][lane] = make_float2(M, L);
#pragma unroll
    for (int i = 0; i < kMergeCols; ++i) acc_of[warp][lane][i] = acc[i];
    acc_of[warp][lane][kMergeCols] = E;
    __syncthreads();
    // ---- now a thread for some columns of a row ----
    constexpr int kMine = SPLIT > 8 ? 2 : kMergeCols / SPLIT, kEach = kMergeCols / kMine;
    const int r = t / kEach, c = t % kEach * kMine, R2 = blockIdx.x * 32 + r;
    if (r >= 32 || R2 >= rows) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < SPLIT; ++w) top = fmaxf(top, ml_of[w][r].x);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, weights = 0.0f, out[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) out[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < SPLIT; ++w) {
      const float2 x = ml_of[w][r];
      if (x.y == 0.0f) continue;
      const float by = ex2(x.x - ref);
      sum = fmaf(x.y, by, sum);
      weights = fmaf(acc_of[w][r][kMergeCols], by, weights);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int z = (c + i) & 3;
        out[i] = fmaf(acc_of[w][r][kE4M3 && z == 1 ? c + i + 1 : kE4M3 && z == 2 ? c + i - 1 : c + i], by, out[i]);
      }
    }
    const float f = sum != 0.0f ? 1.0f / sum : 0.0f;
    const int token2 = R2 / G;
    const size_t at2 = static_cast<size_t>(token2) * p.n_q_heads + g * G + R2 - token2 * G;
    uint32_t* const to = reinterpret_cast<uint32_t*>(p.out + at2 * D + col0 + c);
#pragma unroll
    for (int i = 0; i < kMine; i += 2) to[i / 2] = pack16<false>(out[i] * f, out[i + 1] * f);
    if (p.lse != nullptr && col0 + c == 0) p.lse[at2] = sum != 0.0f ? (top + log2f(weights)) * 0.6931471805599453f : -INFINITY;
  }
}

namespace {

template <int D, bool kE4M3, bool kOne>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, cudaStream_t stream, int* launches) {
  using Cfg = PrefixCfg<D, kE4M3, kOne>;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(prefix_attn_kernel<D, kE4M3, kOne>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
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
  e = cudaLaunchKernelEx(&cfg, prefix_attn_kernel<D, kE4M3, kOne>, tq, tk, tv, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  const long long rows = static_cast<long long>(p.c.batch) * p.q_len * p.group;
  cfg.dynamicSmemBytes = 0;
  // As many warps share a row's pieces out as one wave has room for: what a block does before its first load and behind its last is most
  // of the time.  (Eight everywhere: 48 x 4 tokens, 1536 blocks in 3.5 waves, 16 us; rule: 8.7.)  More than eight where a row has as many
  // pieces (7 rows of one head over 66101 entries, 296 pieces a row: whole call 39 us with eight, 26 with 32).
  const long long tokens = static_cast<long long>(p.c.batch) * p.q_len, row_blocks = (rows + 31) / 32 * p.c.n_kv_heads;
  const long long units = p.c.n_kv_heads * max(static_cast<long long>(p.n_prefixes), (tokens + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens));
  const long long pieces = (p.ctas / units + 1) * 2;      // of a row, two tiles each
  auto merge = [&](auto split_) {
    constexpr int kSplit = decltype(split_)::value;
    using Cfg = MergeCfg<D, kSplit>;
    cfg.gridDim = dim3(static_cast<unsigned>((rows + 31) / 32), p.c.n_kv_heads, kSplit == 1 ? 1 : D / Cfg::kCols);
    cfg.blockDim = dim3(32 * Cfg::kWarps);
    return cudaLaunchKernelEx(&cfg, prefix_merge_kernel<D, kE4M3, kSplit>, p);
  };
  auto fits = [&](int split) { return row_blocks * (D / (split > 8 ? 8 : 16)) * split <= 148ll * (split > 8 ? 32 : 24); };
  e = pieces >= 32 && fits(32)   ? merge(std::integral_constant<int, 32>{})
      : pieces >= 16 && fits(16) ? merge(std::integral_constant<int, 16>{})
      : fits(8)                  ? merge(std::integral_constant<int, 8>{})
      : fits(4)                  ? merge(std::integral_constant<int, 4>{})
      : fits(2)                  ? merge(std::integral_constant<int, 2>{})
                                 : merge(std::integral_constant<int, 1>{});
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <int D, bool kE4M3>
cudaError_t launch_d(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const PrefixParams& p, cudaStream_t stream, int* launches) {
  if (static_cast<long long>(p.c.batch) * p.q_len <= p.tile_tokens) return launch_t<D, kE4M3, true>(tq, tk, tv, p, stream, launches);
  return launch_t<D, kE4M3, false>(tq, tk, tv, p, stream, launches);
}

}  // namespace

cudaError_t launch_prefix_attn(const CUtensorMap& tmap_q, const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, const PrefixParams& p,
                               int head_dim, bool e4m3, cudaStream_t stream, int* launches) {
  if (head_dim == 128) return e4m3 ? launch_d<128, true>(tmap_q, tmap_k, tmap_v, p, stream, launches) : launch_d<128, false>(tmap_q, tmap_k, tmap_v, p, stream, launches);
  if (head_dim == 64) return e4m3 ? launch_d<64, true>(tmap_q, tmap_k, tmap_v, p, stream, launches) : launch_d<64, false>(tmap_q, tmap_k, tmap_v, p, stream, launches);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
