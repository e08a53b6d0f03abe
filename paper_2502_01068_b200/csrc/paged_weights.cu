// The attention weight that every cached entry draws, accumulated over decode steps (what an eviction ranks entries by):
//
//   w[b, g, t] = decay * w[b, g, t] + sum over query tokens i and heads h of group g that see t of
//                exp(scale <q[b, i, h], K[t, g]> - lse[b, i, h])
//
// with the log-sum-exp lse of the attention over the same entries.  Entries 0 .. len_b - q_len - 1 have a weight from before; the
// last q_len are the query tokens' own and start here.
//
// Memory-bound: every K row is read once (2 d bytes per entry and KV head, d in 8 bits), next to 8 bytes of weight.  So the kernel is
// a stream: K goes from memory straight into the registers that the tensor cores read it from (the contraction runs over the head
// dimension in whatever order the 16-byte loads bring it, as long as the queries come in the same one), 4 KB a warp and step (2 KB in 8
// bits), the next step's in flight while this one is computed; no shared memory, no barrier, and every CTA an even share of all entries.
//   S [16 entries x 8 rows] = K Q^T: A = K rows, B = the query rows; a lane holds 2 entries x 2 rows, and the sum over rows ends
//   with two shuffles.  Each entry belongs to one lane: no atomics, and the order of the sums is fixed.
// 32 query heads over 8 KV heads of 128, one B200: 64 sequences of 2048 bf16 entries 45 us, 250 MB at 5.5 TB/s (85 % of a copy); 16 of 500
// to 40000 in 8 bits with four query tokens 84 us, 375 MB at 4.5 TB/s (79 to 88 by the lengths drawn): there half of the issue slots are taken (products,
// conversions and exponentials of 16 rows an entry) and the rest is lost to waits that four warps a scheduler, all that the registers
// allow, do not cover.  64 sequences of 2048: one query token in 8 bits 31 us (65 % of a copy), two in bf16 46, four (16 rows) 60 in bf16, where
// the fragments of 16 rows and two steps spill (172 bytes a thread), and 37 in 8 bits.  More than 16 rows are slow: their fragments do not stay
// in registers and are read (in 8 bits also converted) again for every step, eight query tokens (32 rows) 109 us in bf16 and 158 in 8 bits.
// 8-bit codes widen exactly to fp16 in registers, one conversion for two of them (an SM does 16 of those a cycle, and two for a pair,
// through bf16, were what bounded the kernel: 118 us for the ragged batch against 109, with one step a unit both times).  The queries go into
// fp16 after a power-of-two shift per row that brings the row's largest element to [2^14, 2^15): exact down to 2^-28 of it, and what is
// smaller is off by at most 2^-39 of the largest.  K's scale and the shift multiply the logits.  Logits, exponentials and sums are fp32.
#include <type_traits>

#include "paged.cuh"
#include "paged_mma.cuh"

namespace fastkv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

template <int D, bool kE4M3>
struct WeightsCfg {
  // 16-byte loads of a lane per step: 4 KB a warp, in 8 bits 2 KB (with 4 KB the two steps do not fit the registers next to the queries).
  // Two steps are a pair, whose weights are read and written together; one or more pairs in a row are what a warp has of a unit, so that
  // the walk over sequences and pages is paid for once (at one step a unit it was half of all instructions in 8 bits: 109 us, now 80).
  static constexpr int kLoads = kE4M3 ? 4 : 8;
  static constexpr int kRowBytes = D * (kE4M3 ? 1 : 2);
  static constexpr int kPieces = kRowBytes / 64;         // loads of a row by its four lanes
  static constexpr int kTiles = kLoads / (2 * kPieces);  // 16-entry tiles of a step
  static constexpr int kPair = 2 * 16 * kTiles;          // entries of a pair: 32 or 64
  static constexpr int kPairLog2 = kPair == 32 ? 5 : 6;
};

__device__ __forceinline__ int entries_of(const PagedWeightsParams& p, int b) {
  const int len = usable_len(p.lens[b], p.c.max_pages, p.c.page_log2);
  return static_cast<int>(min(static_cast<long long>(len), p.stride));
}

}  // namespace

// NT: tiles of 8 query rows whose fragments stay in registers (rows <= 8 NT); 0: any number, fragments read again (from L1) for every
// step.  kFull: rows == 8 NT, so that no row is padding and none has to be left out (16 of 500 to 40000, 16 rows in 8 bits: 86.1 us, with the
// selection 87.8).
template <int D, bool kE4M3, int NT, bool kFull>
__global__ void __launch_bounds__(kThreads, 2) paged_weights_kernel(const PagedWeightsParams p) {
  using Cfg = WeightsCfg<D, kE4M3>;
  constexpr int KS = D / 16, kTiles = Cfg::kTiles, kLoads = Cfg::kLoads, kPieces = Cfg::kPieces;
  constexpr int kHeld = NT > 0 ? NT : 2;       // tiles of 8 query rows at a time
  __shared__ long long scratch[kWarps];
  __shared__ int s_first;
  __shared__ long long s_base;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, quad = lane >> 2, c = lane & 3;
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len;
  const int span_log2 = Cfg::kPairLog2 + p.pairs_log2, log2 = span_log2 + 3;       // entries of a unit: a warp's, the CTA's
  pdl_launch_dependents();
  pdl_wait();

  // ---- this CTA's share: units of a row of (sequence, KV head, chunk) ----
  int b = 0;
  long long u, u_end, base = 0;
  {
    const int B = p.c.batch;
    if (t == 0) s_first = -1;
    long long mine = 0, before = 0, total;
    const int per = (B + kThreads - 1) / kThreads, b0 = min(t * per, B), b1 = min(b0 + per, B);
    if (B == 1) {
      total = static_cast<long long>(chunk_count(entries_of(p, 0), log2)) * Hkv;
    } else {
      for (int x = b0; x < b1; ++x) mine += chunk_count(entries_of(p, x), log2);
      before = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
      }
      if (lane == 31) scratch[warp] = before;
      before -= mine;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += scratch[w];
        total += scratch[w];
      }
      total *= Hkv;
    }
    u = total * blockIdx.x / gridDim.x;
    u_end = total * (blockIdx.x + 1) / gridDim.x;
    if (blockIdx.x == 0)                        // a length that was cut is reported once
      for (int x = t; x < B; x += kThreads)
        if (p.lens[x] != entries_of(p, x)) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_WEIGHTS_LEN);
    if (u >= u_end) return;
    if (B > 1) {
      if (before * Hkv <= u && u < (before + mine) * Hkv) {
        long long at = before;
        for (int x = b0; x < b1; ++x) {
          const int n = chunk_count(entries_of(p, x), log2);
          if (u < (at + n) * Hkv) { s_first = x; s_base = at * Hkv; break; }
          at += n;
        }
      }
      __syncthreads();
      b = s_first;
      base = s_base;
    }
  }

  // A warp's place in the share: sequence, KV head, chunk of it.
  struct Place { int b, g, c, len; };
  Place at;
  at.b = b;
  at.len = entries_of(p, b);
  {
    const int n = chunk_count(at.len, log2);
    at.g = static_cast<int>((u - base) / n);
    at.c = static_cast<int>((u - base) - static_cast<long long>(at.g) * n);
  }
  int left = static_cast<int>(u_end - u);       // units of the share that are not done
  auto next = [&](Place x) -> Place {           // the caller knows that there is one
    if (++x.c < chunk_count(x.len, log2)) return x;
    x.c = 0;
    if (++x.g < Hkv) return x;
    x.g = 0;
    do { x.len = entries_of(p, ++x.b); } while (x.len == 0);
    return x;
  };
  // Lane y: page of tile y of what the warp has of a unit, kNoPage behind the end; then its block (page * Hkv + g), -1 for none and page 0
  // for one outside the pool.  (Two parts, since what is done with a loaded value at once waits for it.)
  constexpr int kNoPage = static_cast<int>(0x80000000u);
  auto first_of = [&](const Place& x) -> int { return (x.c << log2) + (warp << span_log2); };
  auto pages_of = [&](const Place& x) -> int {
    const int key = first_of(x) + lane * 16;
    return lane * 16 < (1 << span_log2) && key < x.len ? __ldg(p.c.block_table + static_cast<size_t>(x.b) * p.c.max_pages + (key >> p.c.page_log2)) : kNoPage;
  };
  auto blocks_of = [&](const Place& x, int page) -> int {
    if (page == kNoPage) return -1;
    const long long blk = pool_block(page, p.c.n_pages, Hkv, x.g);
    if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_WEIGHTS_PAGE); return x.g; }
    return static_cast<int>(blk);
  };
  // The entry of tile pair z of the pair of steps at `key0` that this lane writes: lanes c = 0, 1 take tile 2 z, c = 2, 3 tile 2 z + 1, each
  // one of its halves.
  auto my_key = [&](int key0, int z) -> int { return key0 + (2 * z + (c >> 1)) * 16 + (c & 1) * 8 + quad; };
  auto row_of = [&](const Place& x) -> float* { return p.weights + (static_cast<long long>(x.b) * Hkv + x.g) * p.stride; };
  // K's rows of a step whose first tile is `tile` of the warp's; blk: lane y has the block of tile y
  auto load = [&](int tile, int blk, uint4 (&k)[kLoads]) {
    // (a warp's entries start on a multiple of their number, as pages do)
    const int row = (warp << span_log2) + tile * 16;
#pragma unroll
    for (int y = 0; y < kTiles; ++y) {
      const int by = __shfl_sync(0xffffffffu, blk, tile + y);
      const int first = (row + y * 16) & ((1 << p.c.page_log2) - 1);
      const uint8_t* src = p.c.k_pages + ((static_cast<long long>(max(by, 0)) << p.c.page_log2) + first + quad) * Cfg::kRowBytes + c * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < kPieces; ++j)               // [tile][half][piece]
          k[(y * 2 + h) * kPieces + j] = by < 0 ? make_uint4(0u, 0u, 0u, 0u)
              : __ldg(reinterpret_cast<const uint4*>(src + h * 8 * Cfg::kRowBytes + j * 64));
    }
  };

  // ---- query fragments: row quad of each tile of 8, 16-byte pieces in the order K's come in ----
  uint32_t qf[kHeld][2 * KS];
  float lse[kHeld][2];                          // of rows 2c, 2c + 1
  float shift[kHeld][2];                        // 8-bit pages: what a logit is multiplied by besides the scales
  int sees[kHeld][2];                           // entries the row sees; 0 for rows that are not there or saw nothing
  auto take_rows = [&](const Place& x, int nt, uint32_t (&f)[2 * KS], float (&l)[2], float (&by)[2], int (&n)[2]) {
    const int r = nt * 8 + quad, i = r / G, h = x.g * G + r - i * G;
    const uint16_t* src = p.q + ((static_cast<size_t>(x.b) * T + i) * p.n_q_heads + h) * D;
#pragma unroll
    for (int j = 0; j < D / (kE4M3 ? 64 : 32); ++j) {
      // bf16: elements 8 (c + 4 j) .. + 7; 8-bit: 16 (c + 4 j) .. + 15
      if constexpr (kE4M3) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u), w = v;
        if (r < p.rows) {
          v = __ldg(reinterpret_cast<const uint4*>(src + 16 * (c + 4 * j)));
          w = __ldg(reinterpret_cast<const uint4*>(src + 16 * (c + 4 * j) + 8));
        }
        f[8 * j] = v.x; f[8 * j + 1] = v.y; f[8 * j + 2] = v.z; f[8 * j + 3] = v.w;
        f[8 * j + 4] = w.x; f[8 * j + 5] = w.y; f[8 * j + 6] = w.z; f[8 * j + 7] = w.w;
      } else {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (r < p.rows) v = __ldg(reinterpret_cast<const uint4*>(src + 8 * (c + 4 * j)));
        f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
      }
    }
    int up = 0;
    if constexpr (kE4M3) {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
        float lo, hi;
        unpack16<false>(f[i], lo, hi);
        m = fmaxf(m, fmaxf(fabsf(lo), fabsf(hi)));
      }
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      up = m > 0.0f ? 14 - scale_log2(__float_as_uint(m)) : 0;
      up = up > 120 ? 120 : up;                 // of a subnormal row; otherwise within [-113, 120] as it stands
      const float times = __uint_as_float(pow2_bits(up));
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
        float lo, hi;
        unpack16<false>(f[i], lo, hi);
        f[i] = pack16<true>(lo * times, hi * times);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (kE4M3) by[e] = __uint_as_float(pow2_bits(-__shfl_sync(0xffffffffu, up, (2 * c + e) * 4)));
      const int s = nt * 8 + 2 * c + e, si = s / G, sh = x.g * G + s - si * G;
      l[e] = s < p.rows ? __ldg(p.lse + (static_cast<size_t>(x.b) * T + si) * p.n_q_heads + sh) : 0.0f;
      n[e] = s >= p.rows || l[e] == -INFINITY ? 0 : max(x.len - (T - 1 - si), 0);
    }
  };

  int all_see = 0;
  // whether row 2c + e of a tile is there (the last tile's may be padding, with queries of zeros)
  auto is_row = [&](int nt, int e) -> bool { return kFull || nt * 8 + 2 * c + e < p.rows; };
  // the fewest entries that a row sees which is there
  auto least = [&]() -> int {
    int n = 0x7fffffff;
#pragma unroll
    for (int nt = 0; nt < kHeld; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) n = min(n, is_row(nt, e) ? sees[nt][e] : n);
    return __reduce_min_sync(0xffffffffu, n);
  };
  // what the entries of the step from `key0` on draw from the lane's rows
  auto compute = [&](const Place& x, int key0, int tile, const uint4 (&k)[kLoads], float scales, float* sum) {
#pragma unroll
    for (int y = 0; y < 2 * kTiles; ++y) sum[y] = 0.0f;
    if (key0 >= x.len) return;
    // the rows of kHeld tiles: K's fragments (widened once) serve them all.  kAll: every row that is there sees the whole step; those that are
    // not are left out by selection, because a query of zeros meets an infinite key as NaN.
    auto draw = [&](auto all_) {
      constexpr bool kAll = decltype(all_)::value;
#pragma unroll
      for (int y = 0; y < kTiles; ++y) {
        float d[kHeld][4];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          const uint4 a = k[(y * 2) * kPieces + j], e = k[(y * 2 + 1) * kPieces + j];
          const uint32_t av[4] = {a.x, a.y, a.z, a.w}, ev[4] = {e.x, e.y, e.z, e.w};
          if constexpr (kE4M3) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t a0 = widen_lo(av[w]), a1 = widen_lo(ev[w]), a2 = widen_hi(av[w]), a3 = widen_hi(ev[w]);
#pragma unroll
              for (int nt = 0; nt < kHeld; ++nt)
                mma16<true>(d[nt], j == 0 && w == 0, a0, a1, a2, a3, qf[nt][8 * j + 2 * w], qf[nt][8 * j + 2 * w + 1]);
            }
          } else {
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int nt = 0; nt < kHeld; ++nt)
                mma16<false>(d[nt], j == 0 && w == 0, av[2 * w], ev[2 * w], av[2 * w + 1], ev[2 * w + 1], qf[nt][4 * j + 2 * w], qf[nt][4 * j + 2 * w + 1]);
          }
        }
        const float times = p.scale * (kE4M3 ? __shfl_sync(0xffffffffu, scales, tile + y) : 1.0f);
#pragma unroll
        for (int nt = 0; nt < kHeld; ++nt) {
          const float by[2] = {kE4M3 ? times * shift[nt][0] : times, kE4M3 ? times * shift[nt][1] : times};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // what a row does not see must not reach the sum, NaN included
            const float w = ex2(fmaf(d[nt][e], by[e & 1], -lse[nt][e & 1]) * 1.4426950408889634f);
            if (kAll ? is_row(nt, e & 1) : key0 + y * 16 + quad + (e >> 1) * 8 < sees[nt][e & 1]) sum[2 * y + (e >> 1)] += w;
          }
        }
      }
    };
    if constexpr (NT > 0) {
      if (key0 + 16 * kTiles <= all_see) draw(std::true_type{}); else draw(std::false_type{});
    } else {
#pragma unroll 1
      for (int nt = 0; nt * 8 < p.rows; nt += kHeld) {
#pragma unroll
        for (int z = 0; z < kHeld; ++z) take_rows(x, nt + z, qf[z], lse[z], shift[z], sees[z]);
        draw(std::false_type{});
      }
    }
  };

  // ---- the stream: two steps' rows in flight or being computed, the pages of the next unit being looked up.  Two buffers that take
  // turns, not one that is copied: a copy would wait for the loads. ----
  const int pairs = 1 << p.pairs_log2;
  uint4 even[kLoads], odd[kLoads];
  int blk = blocks_of(at, pages_of(at));
  float scales = kE4M3 && blk >= 0 ? __ldg(p.c.k_scales + blk) : 1.0f;
  load(0, blk, even);
  load(kTiles, blk, odd);
  bool fresh = true;
  while (true) {
    if (NT > 0 && fresh) {
#pragma unroll
      for (int nt = 0; nt < kHeld; ++nt) take_rows(at, nt, qf[nt], lse[nt], shift[nt], sees[nt]);
      all_see = least();
    }
    const bool more = --left > 0;
    Place far = at;
    int page = kNoPage, far_blk = -1;
    float far_scales = 1.0f;
    if (more) {
      far = next(at);
      page = pages_of(far);
    }
#pragma unroll 1
    for (int i = 0; i < pairs; ++i) {
      const bool last = i + 1 == pairs;
      const int key0 = first_of(at) + i * Cfg::kPair, tile = i * 2 * kTiles, tile_next = last ? 0 : tile + 2 * kTiles;
      float old[kTiles];
#pragma unroll
      for (int z = 0; z < kTiles; ++z) old[z] = my_key(key0, z) < at.len - T ? row_of(at)[my_key(key0, z)] : 0.0f;
      float sum[4 * kTiles];                    // [tile][half]
      compute(at, key0, tile, even, scales, sum);
      if (last) {
        far_blk = blocks_of(far, page);
        if (kE4M3 && far_blk >= 0) far_scales = __ldg(p.c.k_scales + far_blk);
      }
      load(tile_next, last ? far_blk : blk, even);
      compute(at, key0 + 16 * kTiles, tile + kTiles, odd, scales, sum + 2 * kTiles);
      load(tile_next + kTiles, last ? far_blk : blk, odd);
#pragma unroll
      for (int y = 0; y < 4 * kTiles; ++y) {
        sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 1);
        sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 2);
      }
#pragma unroll
      for (int z = 0; z < kTiles; ++z) {
        const float a = (c & 1) ? sum[4 * z + 1] : sum[4 * z], d = (c & 1) ? sum[4 * z + 3] : sum[4 * z + 2];
        const int key = my_key(key0, z);
        const float drew = c >= 2 ? d : a;
        if (key < at.len) row_of(at)[key] = key < at.len - T ? fmaf(p.decay, old[z], drew) : drew;
      }
    }
    if (!more) return;
    fresh = far.c == 0;                         // another KV head or sequence
    at = far;
    blk = far_blk;
    scales = far_scales;
  }
}

namespace {

template <int D, bool kE4M3, int NT, bool kFull>
cudaError_t launch_nt(PagedWeightsParams& p, cudaStream_t stream) {
  // CTAs: what is resident at once (two per SM), or one for every unit of a short call.  Units: two or four pairs a warp as long as there
  // are six for every CTA, so that the uneven last one costs little (64 x 2048 bf16: one pair 46.5 us, two 45.2); one in shorter calls.
  constexpr int kLog2 = WeightsCfg<D, kE4M3>::kPairLog2 + 3;
  const long long pairs = p.total_len * p.c.n_kv_heads >> kLog2;
  p.pairs_log2 = 0;
  while (p.pairs_log2 < 2 && pairs >> (p.pairs_log2 + 1) >= 6ll * 2 * 148) ++p.pairs_log2;
  const long long chunks = (p.total_len >> (kLog2 + p.pairs_log2)) + p.c.batch;
  p.ctas = static_cast<int>(min(chunks * p.c.n_kv_heads, 2ll * 148));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_weights_kernel<D, kE4M3, NT, kFull>, static_cast<const PagedWeightsParams&>(p));
}

template <int D, bool kE4M3>
cudaError_t launch_d(PagedWeightsParams& p, cudaStream_t stream) {
  if (p.rows <= 8) return p.rows == 8 ? launch_nt<D, kE4M3, 1, true>(p, stream) : launch_nt<D, kE4M3, 1, false>(p, stream);
  if (p.rows <= 16) return p.rows == 16 ? launch_nt<D, kE4M3, 2, true>(p, stream) : launch_nt<D, kE4M3, 2, false>(p, stream);
  return launch_nt<D, kE4M3, 0, false>(p, stream);
}

}  // namespace

cudaError_t launch_paged_weights(PagedWeightsParams& p, int head_dim, bool e4m3, cudaStream_t stream) {
  if (head_dim == 128) return e4m3 ? launch_d<128, true>(p, stream) : launch_d<128, false>(p, stream);
  if (head_dim == 64) return e4m3 ? launch_d<64, true>(p, stream) : launch_d<64, false>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
