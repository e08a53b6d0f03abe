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
// dimension in whatever order the 16-byte loads bring it, as long as the queries come in the same one), 4 KB a warp and step, the next
// step's in flight while this one is computed; no shared memory, no barrier, and every CTA an even share of all entries.
//   S [16 entries x 8 rows] = K Q^T: A = K rows, B = the query rows; a lane holds 2 entries x 2 rows, and the sum over rows ends
//   with two shuffles.  Each entry belongs to one lane: no atomics, and the order of the sums is fixed.
// 8-bit codes widen exactly to fp16 in registers, one conversion for two of them (an SM does 16 of those a cycle, and two for a pair,
// through bf16, were what bounded the kernel: 118 us for the ragged 16 x 500 to 40000 with four query tokens).  The queries go into
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
  // 16-byte loads of a lane per step: 4 KB a warp, in 8 bits 2 KB (with 4 KB the two steps do not fit the registers next to the queries)
  static constexpr int kLoads = kE4M3 ? 4 : 8;
  static constexpr int kRowBytes = D * (kE4M3 ? 1 : 2);
  static constexpr int kPieces = kRowBytes / 64;         // loads of a row by its four lanes
  static constexpr int kTiles = kLoads / (2 * kPieces);  // 16-entry tiles of a step
  static constexpr int kStep = 16 * kTiles;
  static constexpr int kChunk = kWarps * kStep;          // entries of a CTA's step: 128, 256 or 512
  static constexpr int kChunkLog2 = kChunk == 128 ? 7 : kChunk == 256 ? 8 : 9;
};

__device__ __forceinline__ int entries_of(const PagedWeightsParams& p, int b) {
  const int len = usable_len(p.lens[b], p.c.max_pages, p.c.page_log2);
  return static_cast<int>(min(static_cast<long long>(len), p.stride));
}

}  // namespace

// NT: tiles of 8 query rows whose fragments stay in registers (rows <= 8 NT); 0: any number, fragments read again (from L1) for every
// step.
template <int D, bool kE4M3, int NT>
__global__ void __launch_bounds__(kThreads, 2) paged_weights_kernel(const PagedWeightsParams p) {
  using Cfg = WeightsCfg<D, kE4M3>;
  constexpr int KS = D / 16, kTiles = Cfg::kTiles, kLoads = Cfg::kLoads, kPieces = Cfg::kPieces, kLog2 = Cfg::kChunkLog2;
  constexpr int kHeld = NT > 0 ? NT : 2;       // tiles of 8 query rows at a time
  __shared__ long long scratch[kWarps];
  __shared__ int s_first;
  __shared__ long long s_base;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, quad = lane >> 2, c = lane & 3;
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len;
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
      total = static_cast<long long>(chunk_count(entries_of(p, 0), kLog2)) * Hkv;
    } else {
      for (int x = b0; x < b1; ++x) mine += chunk_count(entries_of(p, x), kLog2);
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
          const int n = chunk_count(entries_of(p, x), kLog2);
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
  struct Place { int b, g, c, n_chunks, len; };
  Place at;
  at.b = b;
  at.len = entries_of(p, b);
  at.n_chunks = chunk_count(at.len, kLog2);
  at.g = static_cast<int>((u - base) / at.n_chunks);
  at.c = static_cast<int>((u - base) - static_cast<long long>(at.g) * at.n_chunks);
  auto next = [&](Place x) -> Place {           // the caller knows that there is one
    if (++x.c < x.n_chunks) return x;
    x.c = 0;
    if (++x.g < Hkv) return x;
    x.g = 0;
    do {
      x.len = entries_of(p, ++x.b);
      x.n_chunks = chunk_count(x.len, kLog2);
    } while (x.n_chunks == 0);
    return x;
  };
  // Lane y < kTiles: block (page * Hkv + g) of tile y of the warp's step, -1 behind the end.
  auto blocks = [&](const Place& x) -> int {
    const int key = (x.c << kLog2) + warp * Cfg::kStep + lane * 16;
    if (lane >= kTiles || key >= x.len) return -1;
    const long long blk = pool_block(p.c.block_table[static_cast<size_t>(x.b) * p.c.max_pages + (key >> p.c.page_log2)], p.c.n_pages, Hkv, x.g);
    if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_WEIGHTS_PAGE); return x.g; }      // page 0 instead
    return static_cast<int>(blk);
  };
  struct Step {
    uint4 k[kLoads];                            // [tile][half][piece]
    float scale;                                // lane y < kTiles: K's scale of tile y
    float old[(kTiles + 1) / 2];                // weights so far, of the entries this lane writes
  };
  // The entry of tile pair z that this lane writes: lanes c = 0, 1 take tile 2 z, c = 2, 3 tile 2 z + 1, each one of its halves.
  auto my_key = [&](const Place& x, int z) -> int {
    return (x.c << kLog2) + warp * Cfg::kStep + (2 * z + (c >> 1)) * 16 + (c & 1) * 8 + quad;
  };
  auto writes = [&](const Place& x, int z) -> bool { return 2 * z + (c >> 1) < kTiles && my_key(x, z) < x.len; };
  auto row_of = [&](const Place& x) -> float* { return p.weights + (static_cast<long long>(x.b) * Hkv + x.g) * p.stride; };
  auto load = [&](const Place& x, int blk, Step& s) {
    const int row = (((x.c << kLog2) + warp * Cfg::kStep) & ((1 << p.c.page_log2) - 1));
#pragma unroll
    for (int y = 0; y < kTiles; ++y) {
      const int by = __shfl_sync(0xffffffffu, blk, y);
      const int first = (row + y * 16) & ((1 << p.c.page_log2) - 1);
      const uint8_t* src = p.c.k_pages + ((static_cast<long long>(max(by, 0)) << p.c.page_log2) + first + quad) * Cfg::kRowBytes + c * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
          s.k[(y * 2 + h) * kPieces + j] = by < 0 ? make_uint4(0u, 0u, 0u, 0u)
              : __ldg(reinterpret_cast<const uint4*>(src + h * 8 * Cfg::kRowBytes + j * 64));
    }
    s.scale = kE4M3 && blk >= 0 ? __ldg(p.c.k_scales + blk) : 1.0f;
#pragma unroll
    for (int z = 0; z < (kTiles + 1) / 2; ++z)
      s.old[z] = writes(x, z) && my_key(x, z) < x.len - T ? row_of(x)[my_key(x, z)] : 0.0f;
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
      l[e] = s < p.rows ? __ldg(p.lse + (static_cast<size_t>(x.b) * T + si) * p.n_q_heads + sh) : INFINITY;
      n[e] = s >= p.rows || l[e] == -INFINITY ? 0 : max(x.len - (T - 1 - si), 0);
    }
  };

  int have_b = -1, have_g = -1, all_see = 0;
  // the fewest entries that a row sees which is there
  auto least = [&]() -> int {
    int n = 0x7fffffff;
#pragma unroll
    for (int nt = 0; nt < kHeld; ++nt) n = min(n, min(lse[nt][0] == INFINITY ? n : sees[nt][0], lse[nt][1] == INFINITY ? n : sees[nt][1]));
    return __reduce_min_sync(0xffffffffu, n);
  };
  auto compute = [&](const Place& x, const Step& s) {
    const int key0 = (x.c << kLog2) + warp * Cfg::kStep;
    if (NT > 0 && (x.b != have_b || x.g != have_g)) {
      have_b = x.b;
      have_g = x.g;
#pragma unroll
      for (int nt = 0; nt < kHeld; ++nt) take_rows(x, nt, qf[nt], lse[nt], shift[nt], sees[nt]);
      all_see = least();
    }
    if (key0 >= x.len) return;
    float sum[kTiles][2];
#pragma unroll
    for (int y = 0; y < kTiles; ++y) sum[y][0] = sum[y][1] = 0.0f;
    // the rows of kHeld tiles: K's fragments (widened once) serve them all.  kAll: every row that is there sees the whole step (rows that
    // are not there have an lse of +infinity).
    auto draw = [&](auto all_) {
      constexpr bool kAll = decltype(all_)::value;
#pragma unroll
      for (int y = 0; y < kTiles; ++y) {
        float d[kHeld][4];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          const uint4 a = s.k[(y * 2) * kPieces + j], e = s.k[(y * 2 + 1) * kPieces + j];
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
        const float k = p.scale * (kE4M3 ? __shfl_sync(0xffffffffu, s.scale, y) : 1.0f);
#pragma unroll
        for (int nt = 0; nt < kHeld; ++nt) {
          const float by[2] = {kE4M3 ? k * shift[nt][0] : k, kE4M3 ? k * shift[nt][1] : k};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // what a row does not see must not reach the sum, NaN included
            const float w = ex2(fmaf(d[nt][e], by[e & 1], -lse[nt][e & 1]) * 1.4426950408889634f);
            if (kAll || key0 + y * 16 + quad + (e >> 1) * 8 < sees[nt][e & 1]) sum[y][e >> 1] += w;
          }
        }
      }
    };
    if constexpr (NT > 0) {
      if (key0 + Cfg::kStep <= all_see) draw(std::true_type{}); else draw(std::false_type{});
    } else {
#pragma unroll 1
      for (int nt = 0; nt * 8 < p.rows; nt += kHeld) {
#pragma unroll
        for (int z = 0; z < kHeld; ++z) take_rows(x, nt + z, qf[z], lse[z], shift[z], sees[z]);
        draw(std::false_type{});
      }
    }
#pragma unroll
    for (int y = 0; y < kTiles; ++y)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[y][h] += __shfl_xor_sync(0xffffffffu, sum[y][h], 1);
        sum[y][h] += __shfl_xor_sync(0xffffffffu, sum[y][h], 2);
      }
#pragma unroll
    for (int z = 0; z < (kTiles + 1) / 2; ++z) {
      const int hi = 2 * z + 1 < kTiles ? 2 * z + 1 : 2 * z;
      const float a = (c & 1) ? sum[2 * z][1] : sum[2 * z][0], d = (c & 1) ? sum[hi][1] : sum[hi][0];
      if (writes(x, z)) {
        const int key = my_key(x, z);
        const float drew = c >= 2 ? d : a;
        row_of(x)[key] = key < x.len - T ? fmaf(p.decay, s.old[z], drew) : drew;
      }
    }
  };

  // ---- the stream: two steps' rows in flight or being computed, the pages of the one after being looked up.  Two buffers that take
  // turns, not one that is copied: a copy would wait for the loads. ----
  Step even, odd;
  Place at_even = at, at_odd = at, far = at;
  long long left = u_end - u;                   // units from the next one to compute on
  load(at_even, blocks(at_even), even);
  if (left > 1) {
    at_odd = next(at_even);
    load(at_odd, blocks(at_odd), odd);
  }
  int blk = -1;
  if (left > 2) {
    far = next(at_odd);
    blk = blocks(far);
  }
  // computes x and starts the loads of what is two units ahead into its place
  auto turn = [&](Place& x, Step& s) {
    compute(x, s);
    if (left > 2) {
      x = far;
      load(x, blk, s);
      if (left > 3) {
        far = next(far);
        blk = blocks(far);
      }
    }
    --left;
  };
  while (left > 0) {
    turn(at_even, even);
    if (left > 0) turn(at_odd, odd);
  }
}

namespace {

template <int D, bool kE4M3, int NT>
cudaError_t launch_nt(PagedWeightsParams& p, cudaStream_t stream) {
  // CTAs: what is resident at once (two per SM), or one for every chunk of a short call
  const long long chunks = (p.total_len >> WeightsCfg<D, kE4M3>::kChunkLog2) + p.c.batch;
  p.ctas = static_cast<int>(min(chunks * p.c.n_kv_heads, 2ll * 148));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_weights_kernel<D, kE4M3, NT>, static_cast<const PagedWeightsParams&>(p));
}

template <int D, bool kE4M3>
cudaError_t launch_d(PagedWeightsParams& p, cudaStream_t stream) {
  if (p.rows <= 8) return launch_nt<D, kE4M3, 1>(p, stream);
  if (p.rows <= 16) return launch_nt<D, kE4M3, 2>(p, stream);
  return launch_nt<D, kE4M3, 0>(p, stream);
}

}  // namespace

cudaError_t launch_paged_weights(PagedWeightsParams& p, int head_dim, bool e4m3, cudaStream_t stream) {
  if (head_dim == 128) return e4m3 ? launch_d<128, true>(p, stream) : launch_d<128, false>(p, stream);
  if (head_dim == 64) return e4m3 ? launch_d<64, true>(p, stream) : launch_d<64, false>(p, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
