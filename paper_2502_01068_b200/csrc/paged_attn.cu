// Attention of a few new query tokens per sequence over the paged cache, in bf16 or in 8-bit codes with a power-of-two scale
// for each (page, KV head).
//
//   out[b, i, h] = sum_t softmax_t(scale <q[b, i, h], K[t, h / G]>) V[t, h / G],   t < len_b - (q_len - 1 - i)
//
// Memory-bound: every cached K and V row is read once (2 d bytes per entry and KV head in 8 bits, 4 d in bf16) for the G * q_len
// query rows that share it.  The products run as warp-level m16n8k16 tensor-core products, whose only job is to keep the
// instruction count per entry low; a tcgen05 tile has 128 rows and these have 8 or 16.
//
// Split-KV: one CTA per (split of the entries, KV head, sequence, tile of query rows); inside it every warp owns a ring of
// shared-memory stages (16 entries of K and of V each, filled by one lane with tiled TMA copies) and its own online softmax.
//   S [rows x 16 entries] = Q K^T: A = the query rows, B = K rows as stored;
//   O^T [d x rows] += V^T P^T:     A = V through the transposing matrix load, B = P in the layout S comes out in.
// Pages hold 16 rows or more, so that a chunk of 16 entries never straddles two pages; each lane keeps the page and the scales
// of one of the next 32 chunks, fetched a batch ahead, because the table -> scale chain would cost two trips to memory.
//
// 8-bit pages: a code is exact in fp16, so K and V are widened in registers and the products are fp16 x fp16 -> fp32.  The
// queries (bf16) go into fp16 exactly after a power-of-two shift per row that brings the row's largest element to [2^14, 2^15).
// K's scale multiplies the logits.  V's scale 2^v is an addend of the exponent: the outputs accumulate 2^(l + v - R) * code
// against their own running reference R = max(l + v), the sum of exponentials 2^(l - M) against M = max(l) as usual, and
// out = O / L * 2^(R - M): the weights of the second product stay in (0, 1] whatever the pages' scales are.
// P goes in as two 16-bit terms (value and rounding remainder), so the result carries fp32-level error.
#include "paged.cuh"

namespace fastkv {

namespace {

constexpr int kChunk = 16;          // entries per stage
constexpr float kShift = 14.0f;     // 8-bit pages: the weights of the second product are 2^14 times too large, so that the
                                    // remainder term of the largest of them is far from fp16's subnormals

__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// D[16x8] += A[16x16] B[16x8], fp32 accumulators.
template <bool kHalf>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (kHalf)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

template <int D, bool kE4M3, int RT, int kWarps>
struct PagedCfg {
  static constexpr int kItem = kE4M3 ? 1 : 2;
  static constexpr int kRowBytes = D * kItem;
  static constexpr int kBoxes = kRowBytes > 128 ? kRowBytes / 128 : 1;     // 128-byte column blocks of a row (or one of 64)
  static constexpr int kBoxRow = kRowBytes / kBoxes;
  static constexpr int kBoxBytes = kChunk * kBoxRow;
  static constexpr int kHalfBytes = kBoxes * kBoxBytes;                    // K (or V) rows of one stage
  static constexpr int kStageBytes = 2 * kHalfBytes;
  static constexpr int kStages = kE4M3 ? 6 : 3;
  static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
  static constexpr int kRows = 8 * RT;
  static constexpr int kMergeBytes = kWarps * kRows * (D * 4 + 16);        // the warps' outputs and (max, sum, reference)
  static constexpr int kSmem = (kRingBytes > kMergeBytes ? kRingBytes : kMergeBytes) + 1024;
};

}  // namespace

template <int D, bool kE4M3, int RT, int kWarps>
__global__ void __launch_bounds__(32 * kWarps)
paged_attn_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const PagedAttnParams p) {
  using Cfg = PagedCfg<D, kE4M3, RT, kWarps>;
  constexpr int KS = D / 16, MT = D / 16, kRows = Cfg::kRows, kStages = Cfg::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint64_t full[kWarps][kStages];
  __shared__ int abort_flag;

  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int quad = lane >> 2, c = lane & 3;     // fragment coordinates
  const int Hkv = p.c.n_kv_heads, G = p.group, T = p.q_len, n_splits = p.splits;
  // block -> (split, KV head, tile of query rows, sequence), splits fastest
  unsigned rest = blockIdx.x;
  const int split = rest % n_splits; rest /= n_splits;
  const int g = rest % Hkv; rest /= Hkv;
  const int tile = rest % p.row_tiles;
  const int b = rest / p.row_tiles;
  const int row_base = tile * kRows;

  if (t == 0) {
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (t == 0) abort_flag = 0;
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();

  const int asked = p.lens[b];
  const int len = usable_len(asked, p.c.max_pages, p.c.page_log2);
  if (t == 0 && split == 0 && g == 0 && tile == 0 && asked != len) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PAGED_LEN);
  const int n_chunks_all = (len + kChunk - 1) / kChunk;
  const int per = (n_chunks_all + n_splits - 1) / n_splits;
  const int c0 = split * per, c1 = min(n_chunks_all, c0 + per);
  const int my_chunks = c1 - c0 > warp ? (c1 - c0 - warp + kWarps - 1) / kWarps : 0;

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
  float m_run[RT], l_part[RT], r_run[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m_run[rt] = r_run[rt] = -INFINITY;
    l_part[rt] = 0.0f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[rt][mt][e] = 0.0f;
  }

  uint8_t* const ring_ptr = smem + warp * kStages * Cfg::kStageBytes;
  const uint32_t ring = smem_u32(ring_ptr);
  const uint64_t policy = l2_policy_evict_first();
  const int* const table = p.c.block_table + static_cast<size_t>(b) * p.c.max_pages;
  const int page_chunks_log2 = p.c.page_log2 - 4;          // chunks of 16 entries in a page

  // Page and scales of the warp's chunk i for lane i % 32, fetched for 32 chunks at a time.
  auto page_of = [&](int i) -> int {                       // block (page * Hkv + g) of this lane's chunk i
    if (i >= my_chunks) return 0;
    const int pid = table[(c0 + warp + i * kWarps) >> page_chunks_log2];
    const long long blk = pool_block(pid, p.c.n_pages, Hkv, g);
    if (blk < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_PAGED_PAGE); return g; }   // page 0 instead
    return static_cast<int>(blk);
  };
  int blk_cur = page_of(lane), blk_next = page_of(32 + lane);
  float sk_cur = 1.0f, sv_cur = 1.0f, sk_next = 1.0f, sv_next = 1.0f;
  if constexpr (kE4M3) {
    sk_cur = p.c.k_scales[blk_cur]; sv_cur = p.c.v_scales[blk_cur];
    sk_next = p.c.k_scales[blk_next]; sv_next = p.c.v_scales[blk_next];
  }
  auto issue = [&](int i, int blk) {                       // lane 0 only
    const int row = ((c0 + warp + i * kWarps) & ((1 << page_chunks_log2) - 1)) * kChunk;
    uint64_t* bar = &full[warp][i % kStages];
    uint8_t* stage = ring_ptr + (i % kStages) * Cfg::kStageBytes;
    mbar_arrive_expect_tx(bar, Cfg::kStageBytes);
#pragma unroll
    for (int x = 0; x < Cfg::kBoxes; ++x) {
      tma_load_3d(stage + x * Cfg::kBoxBytes, &tmap_k, bar, x * 64, row, blk, policy);
      tma_load_3d(stage + Cfg::kHalfBytes + x * Cfg::kBoxBytes, &tmap_v, bar, x * 64, row, blk, policy);
    }
  };
  int issued = 0;
  for (; issued < kStages - 1 && issued < my_chunks; ++issued) {
    const int blk = __shfl_sync(0xffffffffu, blk_cur, issued);
    if (lane == 0) issue(issued, blk);
  }
  const uint32_t row7 = lane & 7;
  const uint32_t swz = Cfg::kBoxRow == 128 ? row7 : (row7 >> 1);      // 16-byte piece p of row r sits at p ^ swz
  bool ok = true;
  int done = 0;
  for (int i = 0; i < my_chunks; ++i) {
    if ((i & 31) == 0 && i > 0) {                          // the next batch of 32 chunks becomes the current one
      blk_cur = blk_next;
      sk_cur = sk_next; sv_cur = sv_next;
      blk_next = page_of(i + 32 + lane);
      if constexpr (kE4M3) { sk_next = p.c.k_scales[blk_next]; sv_next = p.c.v_scales[blk_next]; }
    }
    if (issued < my_chunks) {                              // the stage it goes to was consumed last iteration
      const int blk = (issued >> 5) == (i >> 5) ? __shfl_sync(0xffffffffu, blk_cur, issued & 31)
                                                : __shfl_sync(0xffffffffu, blk_next, issued & 31);
      if (lane == 0) issue(issued, blk);
      ++issued;
    }
    ok = mbar_wait_bounded(&full[warp][i % kStages], (i / kStages) & 1, &abort_flag, p.hdr, SITE_PAGED_WAIT);
    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
    const uint32_t ks_addr = ring + (i % kStages) * Cfg::kStageBytes;
    const uint32_t vs_addr = ks_addr + Cfg::kHalfBytes;
    const int key0 = (c0 + warp + i * kWarps) * kChunk;
    const int rows = min(kChunk, len - key0);
    if (rows < kChunk) {
      // the sequence's last chunk: what lies behind its end in the page is not its own.  The logits are masked below, but
      // a zero weight does not silence a NaN in V, so those V rows are cleared.
      uint8_t* vs = ring_ptr + (i % kStages) * Cfg::kStageBytes + Cfg::kHalfBytes;
      constexpr int kPieces = Cfg::kBoxRow / 16;
      const int n = (kChunk - rows) * kPieces;
      for (int j = lane; j < Cfg::kBoxes * n; j += 32) {
        const int x = j / n, rem = j - x * n;
        *reinterpret_cast<uint4*>(vs + x * Cfg::kBoxBytes + rows * Cfg::kBoxRow + rem * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      __syncwarp();
    }
    // ---- S = Q K^T: two tiles of 8 entries; lane holds (row quad, entries nt * 8 + 2c, + 1) in [0], [1], row quad + 8 in [2], [3] ----
    float s[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] = 0.0f;
    }
    if constexpr (kE4M3) {
#pragma unroll
      for (int k4 = 0; k4 < KS / 4; ++k4) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          uint32_t kb[4];                       // four 16-element steps of eight K rows
          const uint32_t piece = k4 * 4 + (lane >> 3);
          ldsm_x4(kb, ks_addr + (nt * 8 + row7) * Cfg::kBoxRow + ((piece ^ swz) << 4));
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int ks = k4 * 4 + y;
            mma16<true>(s[nt], qa[ks][0], RT == 2 ? qa[ks][RT - 1] : 0u, qa[ks][RT], RT == 2 ? qa[ks][2 * RT - 1] : 0u,
                        widen_lo(kb[y]), widen_hi(kb[y]));
          }
        }
      }
    } else {
#pragma unroll
      for (int k2 = 0; k2 < KS / 2; ++k2) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          uint32_t kb[4];
          const uint32_t piece = (k2 & 1) * 4 + (lane >> 3);
          ldsm_x4(kb, ks_addr + (k2 >> 1) * Cfg::kBoxBytes + (nt * 8 + row7) * 128 + ((piece ^ swz) << 4));
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int ks = k2 * 2 + y;
            mma16<false>(s[nt], qa[ks][0], RT == 2 ? qa[ks][RT - 1] : 0u, qa[ks][RT], RT == 2 ? qa[ks][2 * RT - 1] : 0u,
                         kb[2 * y], kb[2 * y + 1]);
          }
        }
      }
    }
    float sk = 1.0f, ev = 0.0f;
    if constexpr (kE4M3) {
      sk = __shfl_sync(0xffffffffu, sk_cur, i & 31);
      ev = static_cast<float>(scale_log2(__float_as_uint(__shfl_sync(0xffffffffu, sv_cur, i & 31))));
    }
    uint32_t ph[RT][2], pl[RT][2];
    float alpha[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // ---- online softmax of row quad (+ 8 rt): its 16 logits sit in the four lanes of the quad ----
      const float f = q_scale[rt] * sk;
      float sv[4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          sv[nt * 2 + e] = key0 + nt * 8 + c * 2 + e < sees[rt] ? s[nt][rt * 2 + e] * f : -INFINITY;
      float mx = fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float m_new = fmaxf(m_run[rt], mx);
      const float ref = m_new == -INFINITY ? 0.0f : m_new;             // nothing seen yet: everything stays at zero
      const float alpha_l = ex2(m_run[rt] - ref);
      float pr[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) pr[e] = ex2(sv[e] - ref);
      l_part[rt] = l_part[rt] * alpha_l + ((pr[0] + pr[1]) + (pr[2] + pr[3]));
      m_run[rt] = m_new;
      if constexpr (kE4M3) {
        const float r_new = fmaxf(r_run[rt], mx + ev);
        const float refo = r_new == -INFINITY ? 0.0f : r_new;
        alpha[rt] = ex2(r_run[rt] - refo);
        r_run[rt] = r_new;
        const float shift = ev - refo + kShift;
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[e] = ex2(sv[e] + shift);
      } else {
        alpha[rt] = alpha_l;
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        ph[rt][y] = pack16<kE4M3>(pr[2 * y], pr[2 * y + 1]);
        float a, d;
        unpack16<kE4M3>(ph[rt][y], a, d);
        pl[rt][y] = pack16<kE4M3>(pr[2 * y] - a, pr[2 * y + 1] - d);
      }
    }
    bool moved = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) moved |= alpha[rt] != 1.0f;
    if (__any_sync(0xffffffffu, moved)) {        // the running maxima settle after a few chunks
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float a0 = __shfl_sync(0xffffffffu, alpha[rt], 8 * c), a1 = __shfl_sync(0xffffffffu, alpha[rt], 8 * c + 4);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          o[rt][mt][0] *= a0; o[rt][mt][1] *= a1; o[rt][mt][2] *= a0; o[rt][mt][3] *= a1;
        }
      }
    }
    // ---- O^T += V^T P^T ----
    if constexpr (kE4M3) {
#pragma unroll
      for (int m2 = 0; m2 < MT / 2; ++m2) {
        uint32_t vb[4];                         // entries 0..7 and 8..15 of pieces 2 m2 and 2 m2 + 1
        const uint32_t piece = m2 * 2 + (lane >> 4);
        ldsm_x4_trans(vb, vs_addr + (((lane >> 3) & 1) * 8 + row7) * Cfg::kBoxRow + ((piece ^ swz) << 4));
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          // a word holds elements (2 quad, 2 quad + 1) of entry 2c, then of entry 2c + 1: bring equal elements together
          const uint32_t w0 = __byte_perm(vb[2 * y], 0, 0x3120), w1 = __byte_perm(vb[2 * y + 1], 0, 0x3120);
          const uint32_t a0 = widen_lo(w0), a1 = widen_hi(w0), a2 = widen_lo(w1), a3 = widen_hi(w1);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            mma16<true>(o[rt][2 * m2 + y], a0, a1, a2, a3, ph[rt][0], ph[rt][1]);
            mma16<true>(o[rt][2 * m2 + y], a0, a1, a2, a3, pl[rt][0], pl[rt][1]);
          }
        }
      }
    } else {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t va[4];
        const uint32_t piece = (mt & 3) * 2 + ((lane >> 3) & 1);
        ldsm_x4_trans(va, vs_addr + (mt >> 2) * Cfg::kBoxBytes + ((lane >> 4) * 8 + row7) * 128 + ((piece ^ swz) << 4));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          mma16<false>(o[rt][mt], va[0], va[1], va[2], va[3], ph[rt][0], ph[rt][1]);
          mma16<false>(o[rt][mt], va[0], va[1], va[2], va[3], pl[rt][0], pl[rt][1]);
        }
      }
    }
    __syncwarp();                                // every lane is done with the stage before it is refilled
    done = i + 1;
  }
  if (lane == 0)                                 // after a wait that gave up: no copy may still be in flight
    for (int j = done; j < issued; ++j)
      mbar_wait_drain(&full[warp][j % kStages], (j / kStages) & 1, p.hdr, SITE_PAGED_WAIT);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l_part[rt] += __shfl_xor_sync(0xffffffffu, l_part[rt], 1);
    l_part[rt] += __shfl_xor_sync(0xffffffffu, l_part[rt], 2);
    if constexpr (!kE4M3) r_run[rt] = m_run[rt];
  }
  // ---- the warps of the CTA merge through shared memory (the rings are idle: every copy was waited for) ----
  __syncthreads();
  float* mo = reinterpret_cast<float*>(smem);                                  // [warps][rows][D]
  float4* mml = reinterpret_cast<float4*>(mo + kWarps * kRows * D);            // [warps][rows]: max, sum, reference
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int d0 = mt * 16 + (kE4M3 ? 2 * quad : quad), d1 = d0 + (kE4M3 ? 1 : 8);
      float* row0 = mo + (warp * kRows + rt * 8 + 2 * c) * D;
      row0[d0] = o[rt][mt][0]; row0[D + d0] = o[rt][mt][1]; row0[d1] = o[rt][mt][2]; row0[D + d1] = o[rt][mt][3];
    }
    if (c == 0) mml[warp * kRows + rt * 8 + quad] =
        make_float4(ok ? m_run[rt] : -INFINITY, ok ? l_part[rt] : 0.0f, ok ? r_run[rt] : -INFINITY, 0.0f);
  }
  __syncthreads();
  const int n_rows = min(kRows, p.rows - row_base);
  for (int x = t; x < n_rows * D; x += 32 * kWarps) {
    const int r = x / D, col = x - r * D;
    float M = -INFINITY, R = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      M = fmaxf(M, mml[w * kRows + r].x);
      R = fmaxf(R, mml[w * kRows + r].z);
    }
    float L = 0.0f, acc = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 ml = mml[w * kRows + r];
      if (ml.x == -INFINITY) continue;                                          // warps without entries weigh nothing
      L = fmaf(ml.y, ex2(ml.x - M), L);
      acc = fmaf(mo[(w * kRows + r) * D + col], ex2(ml.z - R), acc);
    }
    const int row = row_base + r;
    if (n_splits == 1) {
      const int i = row / G, h = g * G + row - i * G;
      const size_t at = (static_cast<size_t>(b) * T + i) * p.n_q_heads + h;
      p.out[at * D + col] = L > 0.0f ? acc / L * ex2(R - M - (kE4M3 ? kShift : 0.0f)) : 0.0f;
      if (p.lse != nullptr && col == 0) p.lse[at] = L > 0.0f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
    } else {
      const size_t part = ((static_cast<size_t>(b) * Hkv + g) * n_splits + split) * p.rows + row;
      if (col == 0) p.part_ml[part] = make_float4(M, L, R, 0.0f);
      p.part_o[part * D + col] = acc;
    }
  }
}

// Merges the splits of one query row: one block of D threads each.
template <int D, bool kE4M3>
__global__ void __launch_bounds__(D) paged_merge_kernel(const PagedAttnParams p) {
  __shared__ float f_o[kPagedMaxSplits], f_l[kPagedMaxSplits];
  pdl_wait();
  pdl_launch_dependents();
  const int t = threadIdx.x, n = p.splits, G = p.group;
  // block -> (query token of the batch, head)
  const unsigned bi = blockIdx.x / p.n_q_heads;
  const int h = blockIdx.x - bi * p.n_q_heads, b = bi / p.q_len, i = bi - b * p.q_len, g = h / G;
  const int row = i * G + h - g * G;
  const size_t base = (static_cast<size_t>(b) * p.c.n_kv_heads + g) * n * p.rows + row;
  float4 ml = make_float4(-INFINITY, 0.0f, -INFINITY, 0.0f);
  if (t < n) ml = p.part_ml[base + static_cast<size_t>(t) * p.rows];
  if (t < n) { f_o[t] = ml.z; f_l[t] = ml.x; }
  __syncthreads();
  float M = -INFINITY, R = -INFINITY;
  for (int s = 0; s < n; ++s) { M = fmaxf(M, f_l[s]); R = fmaxf(R, f_o[s]); }
  __syncthreads();
  if (t < n) {
    f_o[t] = ml.x == -INFINITY ? 0.0f : ex2(ml.z - R);
    f_l[t] = ml.x == -INFINITY ? 0.0f : ml.y * ex2(ml.x - M);
  }
  __syncthreads();
  float L = 0.0f, acc = 0.0f;
  for (int s = 0; s < n; ++s) L += f_l[s];
  const float* o = p.part_o + base * D + t;
#pragma unroll 8
  for (int s = 0; s < n; ++s) acc = fmaf(__ldg(o + static_cast<size_t>(s) * p.rows * D), f_o[s], acc);
  const size_t at = (static_cast<size_t>(b) * p.q_len + i) * p.n_q_heads + h;
  p.out[at * D + t] = L > 0.0f ? acc / L * ex2(R - M - (kE4M3 ? kShift : 0.0f)) : 0.0f;
  if (p.lse != nullptr && t == 0) p.lse[at] = L > 0.0f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

PagedAttnPlan plan_paged_attn(int batch, int n_kv_heads, int rows, int head_dim, bool e4m3, int max_len, long long total_len) {
  (void)head_dim; (void)e4m3; (void)total_len;
  constexpr int kSms = 148;
  PagedAttnPlan pl;
  pl.row_tiles_of_8 = rows <= 8 ? 1 : 2;
  pl.row_tiles = (rows + 8 * pl.row_tiles_of_8 - 1) / (8 * pl.row_tiles_of_8);
  const long long pairs = static_cast<long long>(batch) * n_kv_heads * pl.row_tiles;
  pl.warps = pairs > kSms ? 4 : 8;
  const long long capacity = pairs > kSms ? 2 * kSms : kSms;
  long long splits = capacity / pairs;
  const long long chunks = (max_len + kChunk - 1) / kChunk;
  const long long useful = (chunks + pl.warps - 1) / pl.warps;
  if (splits > useful) splits = useful;
  if (splits > kPagedMaxSplits) splits = kPagedMaxSplits;
  if (splits < 1) splits = 1;
  pl.splits = static_cast<int>(splits);
  return pl;
}

size_t paged_attn_workspace_bytes(const PagedAttnPlan& plan, int batch, int n_kv_heads, int rows, int head_dim) {
  if (plan.splits == 1) return sizeof(WorkspaceHeader);
  const size_t parts = static_cast<size_t>(batch) * n_kv_heads * plan.splits * rows;
  return sizeof(WorkspaceHeader) + (parts * sizeof(float4) + 255) / 256 * 256 + parts * head_dim * sizeof(float);
}

template <int D, bool kE4M3, int RT, int kWarps>
static cudaError_t launch_w(const CUtensorMap& tk, const CUtensorMap& tv, PagedAttnParams& p, cudaStream_t stream, int* launches) {
  using Cfg = PagedCfg<D, kE4M3, RT, kWarps>;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(paged_attn_kernel<D, kE4M3, RT, kWarps>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem);
    if (e != cudaSuccess) return e;
    configured.set(dev);
  }
  const long long blocks = static_cast<long long>(p.c.batch) * p.row_tiles * p.c.n_kv_heads * p.splits;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, paged_attn_kernel<D, kE4M3, RT, kWarps>, tk, tv, static_cast<const PagedAttnParams&>(p));
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (p.splits == 1) return cudaSuccess;
  cfg.gridDim = dim3(static_cast<unsigned>(p.c.batch) * p.q_len * p.n_q_heads);
  cfg.blockDim = dim3(D);
  cfg.dynamicSmemBytes = 0;
  e = cudaLaunchKernelEx(&cfg, paged_merge_kernel<D, kE4M3>, static_cast<const PagedAttnParams&>(p));
  if (e == cudaSuccess) *launches = 2;
  return e;
}

template <int D, bool kE4M3>
static cudaError_t launch_f(const CUtensorMap& tk, const CUtensorMap& tv, PagedAttnParams& p, const PagedAttnPlan& plan,
                            cudaStream_t stream, int* launches) {
  if (plan.row_tiles_of_8 == 1)
    return plan.warps == 8 ? launch_w<D, kE4M3, 1, 8>(tk, tv, p, stream, launches) : launch_w<D, kE4M3, 1, 4>(tk, tv, p, stream, launches);
  return plan.warps == 8 ? launch_w<D, kE4M3, 2, 8>(tk, tv, p, stream, launches) : launch_w<D, kE4M3, 2, 4>(tk, tv, p, stream, launches);
}

cudaError_t launch_paged_attn(const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, PagedAttnParams& p, const PagedAttnPlan& plan,
                              int head_dim, bool e4m3, cudaStream_t stream, int* launches) {
  *launches = 0;
  p.row_tiles = plan.row_tiles;
  p.splits = plan.splits;
  if (head_dim == 128)
    return e4m3 ? launch_f<128, true>(tmap_k, tmap_v, p, plan, stream, launches) : launch_f<128, false>(tmap_k, tmap_v, p, plan, stream, launches);
  if (head_dim == 64)
    return e4m3 ? launch_f<64, true>(tmap_k, tmap_v, p, plan, stream, launches) : launch_f<64, false>(tmap_k, tmap_v, p, plan, stream, launches);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
