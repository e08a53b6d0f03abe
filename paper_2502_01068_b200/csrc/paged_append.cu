// Appending rows to the paged cache: new tokens' keys and values (the keys, and the queries beside them, rotated by their
// positions), or the rows that the selection kept (Alg. 1: C <- update(K, V)), into pages of bf16 or of 8-bit codes with
// a power-of-two scale for each (page, KV head).
//
// Rotation: for pair i of a head's first rot_dim elements, angle a = pos * inv_freq[i],
//   y1 = x1 cos a - x2 sin a,   y2 = x2 cos a + x1 sin a      (in fp32, one rounding a product and one a sum, then the one of the cache).
// The angle is formed and reduced in fp64: in fp32 a position of 100 000 leaves 2^-7 of an angle's bits.
//
// Eight lanes (four for head_dim 64) handle one row of one head: sixteen elements each, as two 16-byte pieces chosen so
// that both halves of every rotated pair are the lane's own.
//   Row role   (bf16 pages; queries of either format): a lane group takes one token and a run of heads, so that the
//              angles are formed once per run.  A prompt of 8192 tokens, 32 query and 8 KV heads of 128, bf16: 34.4 us, 89 % of a
//              plain copy's rate over what it reads and writes; 13107 kept rows, 23.6 us, 70 %.
//   Page role  (8-bit pages, calls of more than 8 rows per sequence): a block takes one page and walks a run of heads, whose rows
//              of the page wait in shared memory while their largest absolute value is found and are encoded from there.
//              some 36 900 rows in eight ragged prompts, rotated, with their queries: 148 us, 86 %; 13107 kept rows of 8 heads,
//              gathered: 18 us, 69 % (launch and the chain length -> table -> index -> row take 4 of them).
//   Small role (8-bit pages, up to 8 rows per sequence): a lane group for each new row of a (page, head); 64 sequences, one row
//              each: 3.6 us, as good as launching and three dependent trips to memory; 10 us where every page of 64 takes a larger
//              scale, so that its old rows are encoded again.
// Rows that were in a page before keep their codes unless the new rows need a larger scale; then the codes are re-encoded
// by the ratio, a power of two, which is exact but for codes that become subnormal.
#include "paged.cuh"

namespace fastkv {

namespace {

constexpr int kHeads = 2;            // page role: heads of a round
// What a call does to its rows on the way.
enum Mode { kPlain = 0, kRotated = 1, kGathered = 2 };
// Page role: rounds of heads on their way while one is in use.  Two for tiled copies (51 us against 58 with one, some 36 900 rows of
// 8 heads); one for gathered rows, so that three blocks fit an SM (18 us against 25.5 with two rounds and two blocks, 13107 rows
// of 8 heads).
template <int kMode> constexpr int kRoundsAhead = kMode == kGathered ? 1 : 2;
template <int kMode> constexpr int kSlotsOf = (kRoundsAhead<kMode> + 1) * kHeads;
constexpr int kRowStages = 8;        // row role: heads whose rows are on their way or in use
constexpr int kSmallRows = 8;        // rows per sequence up to which the small role is used

struct Row16 {                       // a lane's sixteen elements of one row: the pieces at `lo` and `hi`
  uint4 lo, hi;
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Four floats to four e4m3 codes (round to nearest even, saturating), the first in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
// Four codes times a power of two, encoded again.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float ratio) {
  uint32_t h0, h1;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h0) : "h"(static_cast<uint16_t>(w & 0xffffu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h1) : "h"(static_cast<uint16_t>(w >> 16)));
  float f[4];
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f[0]), "=f"(f[1]) : "r"(h0));
  asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f[2]), "=f"(f[3]) : "r"(h1));
  return pack_e4m3(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
}

// Where lane j's two pieces start in a head's row of `dim` elements, and whether they are rotated.  Halves: the pieces lie half of
// the rotated part (or half of the rest) apart, which keeps neighbouring lanes on neighbouring 16 bytes.
struct Pieces {
  int lo, hi;
  bool turned;
};
__device__ __forceinline__ Pieces pieces_of(int j, int dim, int rot_dim, int adjacent) {
  Pieces q;
  q.turned = 16 * j < rot_dim;
  const int base = q.turned ? 0 : rot_dim, part = q.turned ? rot_dim : dim - rot_dim;
  q.lo = base + 8 * (j - base / 16);
  q.hi = q.lo + part / 2;
  if (q.turned && adjacent) {        // pairs (2 i, 2 i + 1) of sixteen elements in a row
    q.lo = 16 * j;
    q.hi = 16 * j + 8;
  }
  return q;
}

// cos and sin of the eight pairs 8j .. 8j + 7 at position `pos`.  The angle is formed in fp64 in quarter turns, pos * f * 2 / pi,
// with the rounding errors of both products (pos * f alone needs 55 bits) added back after the whole quarters are gone; what is
// left, at most an eighth of a turn, goes through the Taylor series of sin and cos (to x^13 and x^14: off by 2e-14 and 1e-15, so
// that the one rounding to fp32 is the right one but for one value in millions).  26 fp64 instructions a pair.
__device__ __forceinline__ void angles_of(int pos, const float* inv_freq, int j, float (&cs)[8], float (&sn)[8]) {
  const double kQuarters = 0.6366197723675814, kQuartersLow = -3.935735335036497e-17;      // 2 / pi, high and low part
  const double kHalfPi = 1.5707963267948966;
  const double kRound = 6755399441055744.0;       // 1.5 * 2^52: adding it leaves the nearest integer in the low bits
  const float4 f0 = *reinterpret_cast<const float4*>(inv_freq + 8 * j), f1 = *reinterpret_cast<const float4*>(inv_freq + 8 * j + 4);
  const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
  const double dpos = static_cast<double>(pos);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double freq = static_cast<double>(f[e]), a = dpos * freq, a_low = fma(dpos, freq, -a);
    const double t = a * kQuarters, whole = t + kRound;
    const double rest = (t - (whole - kRound)) + fma(a_low, kQuarters, fma(a, kQuartersLow, fma(a, kQuarters, -t)));
    const double x = rest * kHalfPi, z = x * x;
    double s = fma(z, 1.0 / 6227020800.0, -1.0 / 39916800.0);
    s = fma(z, s, 1.0 / 362880.0); s = fma(z, s, -1.0 / 5040.0); s = fma(z, s, 1.0 / 120.0); s = fma(z, s, -1.0 / 6.0);
    s = fma(x * z, s, x);
    double c = fma(z, -1.0 / 87178291200.0, 1.0 / 479001600.0);
    c = fma(z, c, -1.0 / 3628800.0); c = fma(z, c, 1.0 / 40320.0); c = fma(z, c, -1.0 / 720.0); c = fma(z, c, 1.0 / 24.0);
    c = fma(z, c, -0.5);
    c = fma(z, c, 1.0);
    const int quarter = __double2loint(whole);
    const float fs = static_cast<float>(s), fc = static_cast<float>(c);
    const float u = (quarter & 1) ? fs : fc, v = (quarter & 1) ? fc : fs;       // |cos|, |sin| of the whole angle
    cs[e] = ((quarter + 1) & 2) ? -u : u;
    sn[e] = (quarter & 2) ? -v : v;
  }
}

__device__ __forceinline__ void turn(float& x1, float& x2, float c, float s) {
  const float y1 = __fsub_rn(__fmul_rn(x1, c), __fmul_rn(x2, s));
  const float y2 = __fadd_rn(__fmul_rn(x2, c), __fmul_rn(x1, s));
  x1 = y1;
  x2 = y2;
}

// The sixteen values, lo piece first.
__device__ __forceinline__ void unpack(const Row16& r, float (&x)[16]) {
  const uint32_t w[8] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w, r.hi.x, r.hi.y, r.hi.z, r.hi.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = bf_lo(w[i]);
    x[2 * i + 1] = bf_hi(w[i]);
  }
}
// Pairs of fp32 products and sums.
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void rotate16(float (&x)[16], const float (&cs)[8], const float (&sn)[8], int adjacent) {
  if (adjacent) {
#pragma unroll
    for (int m = 0; m < 8; ++m) turn(x[2 * m], x[2 * m + 1], cs[m], sn[m]);
  } else {
#pragma unroll
    for (int m = 0; m < 8; m += 2) {              // two pairs at a time
      const unsigned long long x1 = pair_of(x[m], x[m + 1]), x2 = pair_of(x[8 + m], x[9 + m]);
      const unsigned long long c = pair_of(cs[m], cs[m + 1]), s = pair_of(sn[m], sn[m + 1]), ns = pair_of(-sn[m], -sn[m + 1]);
      const unsigned long long y1 = add2(mul2(x1, c), mul2(x2, ns)), y2 = add2(mul2(x2, c), mul2(x1, s));
      asm("mov.b64 {%0, %1}, %2;" : "=f"(x[m]), "=f"(x[m + 1]) : "l"(y1));
      asm("mov.b64 {%0, %1}, %2;" : "=f"(x[8 + m]), "=f"(x[9 + m]) : "l"(y2));
    }
  }
}
__device__ __forceinline__ float amax16(const float (&x)[16]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
  return m;
}
__device__ __forceinline__ Row16 load_row(const uint16_t* row, const Pieces& at) {
  Row16 r;
  r.lo = *reinterpret_cast<const uint4*>(row + at.lo);
  r.hi = *reinterpret_cast<const uint4*>(row + at.hi);
  return r;
}
__device__ __forceinline__ void store_codes(uint8_t* row, const Pieces& at, const float (&x)[16], float inv) {
  uint2 lo, hi;
  lo.x = pack_e4m3(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  lo.y = pack_e4m3(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
  hi.x = pack_e4m3(x[8] * inv, x[9] * inv, x[10] * inv, x[11] * inv);
  hi.y = pack_e4m3(x[12] * inv, x[13] * inv, x[14] * inv, x[15] * inv);
  *reinterpret_cast<uint2*>(row + at.lo) = lo;
  *reinterpret_cast<uint2*>(row + at.hi) = hi;
}

// The source row of new row `row` of head h: itself, or the kept row that idx names (-1: none such).  The index is fetched
// apart from its use, so that a caller can have it under way before it is needed.
__device__ __forceinline__ int fetch_index(const AppendParams& p, int row, int h) {
  if (p.idx == nullptr) return row;
  return p.idx[static_cast<long long>(h) * p.total + row];
}
__device__ __forceinline__ long long source_row(const AppendParams& p, int i, int b) {
  if (p.idx == nullptr) return i;
  const int s0 = p.cu_src ? p.cu_src[b] : 0;
  const int L = p.cu_src ? p.cu_src[b + 1] - s0 : p.total_src;
  if (i < 0 || i >= L || s0 < 0 || static_cast<long long>(s0) + i >= p.total_src) {
    raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_INDEX);
    return -1;
  }
  return static_cast<long long>(s0) + i;
}

// The sequence that owns new row t: the last b with cu_new[b] <= t.
__device__ __forceinline__ int owner_of_row(const AppendParams& p, int t) {
  if (p.cu_new == nullptr) return t / p.uniform;
  int lo = 0, hi = p.c.batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.cu_new[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace

__device__ __forceinline__ void copy16_async(uint32_t smem_dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
  return r;
}

// Row role: unit u = (slice of heads, token); heads in the order queries, keys, values.  Every lane copies the pieces of the
// next heads' rows that it will need into shared-memory slots of its own: seven heads in flight a lane, no registers held,
// nothing to synchronise.
template <int D, bool kE4M3, int kMode>
__device__ void append_rows(const AppendParams& p, int block) {
  constexpr bool kRot = kMode == kRotated;
  constexpr int GL = D / 16;                      // lanes of a row
  extern __shared__ __align__(128) uint8_t ring[];   // [kRowStages][2 pieces][threads][16 bytes]
  const int j = threadIdx.x % GL;
  const long long u = static_cast<long long>(block) * (blockDim.x / GL) + threadIdx.x / GL;
  if (u >= static_cast<long long>(p.row_slices) * p.total) return;
  const int slice = static_cast<int>(u / p.total), t = static_cast<int>(u - static_cast<long long>(slice) * p.total);
  const int h0 = slice * p.heads_per_unit, h1 = min(h0 + p.heads_per_unit, p.row_heads);
  const int Hq = p.n_q_heads, Hkv = p.c.n_kv_heads;
  const Pieces turned = pieces_of(j, D, kRot ? p.rot_dim : 0, p.adjacent), plain = pieces_of(j, D, 0, 0);
  pdl_wait();
  int b = 0, slot = -1;
  long long page = -1;                            // of bf16 pages: where row t goes; -1: nowhere
  if (!kE4M3 && h1 > Hq) {
    b = owner_of_row(p, t);
    RowRange r;
    const int len = p.lens[b];
    new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
    if (t >= r.first && t - r.first < r.count) {
      slot = len + (t - r.first);
      const int pid = p.c.block_table[static_cast<long long>(b) * p.c.max_pages + (slot >> p.c.page_log2)];
      page = pool_block(pid, p.c.n_pages, Hkv, 0);
      if (page < 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_PAGE);
    }
  }
  const int in_page = slot & ((1 << p.c.page_log2) - 1);
  const uint32_t slots = smem_u32(ring) + threadIdx.x * 16, piece = blockDim.x * 16;
  auto slot_of = [&](int h) -> uint32_t { return slots + static_cast<uint32_t>(h - h0) % kRowStages * 2 * piece; };
  auto kv_head = [&](int h) -> int { return h < Hq + Hkv ? h - Hq : h - Hq - Hkv; };
  uint32_t here = 0;                              // by stage: whether the row exists
  int index = 0;                                  // source row of the head that starts next
  auto fetch = [&](int h) { if (!kE4M3 && h < h1 && h >= Hq && page >= 0) index = kMode == kGathered ? fetch_index(p, t, kv_head(h)) : t; };
  auto start = [&](int h) {
    const uint32_t bit = 1u << (static_cast<uint32_t>(h - h0) % kRowStages);
    here &= ~bit;
    if (h < h1) {
      const uint16_t* x = nullptr;
      if (h < Hq) {
        x = p.q + static_cast<long long>(t) * p.q_tok + h * p.q_head;
      } else if (!kE4M3 && page >= 0) {
        const long long src = kMode == kGathered ? source_row(p, index, b) : index;
        const int g = kv_head(h);
        if (src >= 0) x = h < Hq + Hkv ? p.k + src * p.k_tok + g * p.k_head : p.v + src * p.v_tok + g * p.v_head;
      }
      if (x != nullptr) {
        const Pieces& at = h < Hq + Hkv ? turned : plain;
        here |= bit;
        copy16_async(slot_of(h), x + at.lo);
        copy16_async(slot_of(h) + piece, x + at.hi);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    fetch(h + 1);
  };
  fetch(h0);
#pragma unroll 1
  for (int h = h0; h < h0 + kRowStages - 1; ++h) start(h);
  float cs[8], sn[8];
  if (kRot && turned.turned && h0 < Hq + Hkv) angles_of(p.pos[t], p.inv_freq, j, cs, sn);      // while the first rows are on their way
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    start(h + kRowStages - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(kRowStages - 1) : "memory");
    if (!((here >> (static_cast<uint32_t>(h - h0) % kRowStages)) & 1u)) continue;
    Row16 raw;
    raw.lo = shared16(slot_of(h));
    raw.hi = shared16(slot_of(h) + piece);
    const bool is_v = h >= Hq + Hkv;
    uint16_t* dst = h < Hq ? p.q_out + (static_cast<long long>(t) * Hq + h) * D
                           : reinterpret_cast<uint16_t*>(is_v ? p.c.v_pages : p.c.k_pages) + (((page + kv_head(h)) << p.c.page_log2) + in_page) * D;
    if (kRot && !is_v && turned.turned) {
      float x[16];
      unpack(raw, x);
      rotate16(x, cs, sn, p.adjacent);
      raw.lo = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
      raw.hi = make_uint4(pack_bf16(x[8], x[9]), pack_bf16(x[10], x[11]), pack_bf16(x[12], x[13]), pack_bf16(x[14], x[15]));
    }
    const Pieces& at = is_v ? plain : turned;
    *reinterpret_cast<uint4*>(dst + at.lo) = raw.lo;
    *reinterpret_cast<uint4*>(dst + at.hi) = raw.hi;
  }
}

// Small role: unit u = (sequence, which of its touched pages, head of K or V), a lane group for each new row it may have (a power
// of two, 2^small_log2).  Every row is read and its angles formed once, all of them side by side: what costs here is the chain
// from the length to the codes (five rows took 8.6 us when one lane group went through them, now 3.6, one row 3.1).  The
// groups of a unit share out the old rows that have to be encoded again.  Idle units walk through with nothing to do, because
// every thread takes part in the shuffles and the meeting.
template <int D>
__device__ void append_small(const AppendParams& p, int block) {
  constexpr int GL = D / 16;
  __shared__ float warp_top[8];
  const int grp = threadIdx.x / GL, j = threadIdx.x % GL, Hkv = p.c.n_kv_heads, jobs = 2 * Hkv;
  const int mates = 1 << p.small_log2, mine = grp & (mates - 1);
  const long long u = static_cast<long long>(block) * ((blockDim.x / GL) >> p.small_log2) + (grp >> p.small_log2);
  const long long units = static_cast<long long>(p.c.batch) * p.pages_per_seq * jobs;
  const bool live = u < units;
  const long long item = live ? u / jobs : 0;
  const int job = live ? static_cast<int>(u - item * jobs) : 0;
  const int b = static_cast<int>(item / p.pages_per_seq), which = static_cast<int>(item - static_cast<long long>(b) * p.pages_per_seq);
  const bool is_v = job >= Hkv;
  const int g = is_v ? job - Hkv : job;
  const Pieces at = is_v ? pieces_of(j, D, 0, 0) : pieces_of(j, D, p.rot_dim, p.adjacent);
  const int P = 1 << p.c.page_log2;
  pdl_wait();
  int len = 0, lo = 0, hi = 0, row0 = 0;           // slots [lo, hi) of the sequence are this unit's new rows
  long long block_row = -1;
  int pg = 0;
  if (live) {
    len = p.lens[b];
    RowRange r;
    new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
    row0 = r.first;
    if (r.count > 0) {
      pg = (len >> p.c.page_log2) + which;
      lo = max(len, pg << p.c.page_log2);
      hi = min(len + r.count, (pg + 1) << p.c.page_log2);
      if (hi > lo) {
        const int pid = p.c.block_table[static_cast<long long>(b) * p.c.max_pages + pg];
        block_row = pool_block(pid, p.c.n_pages, Hkv, g);
        if (block_row < 0) { raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_PAGE); hi = lo; }
      } else {
        hi = lo;
      }
    }
  }
  float* const scales = is_v ? p.c.v_scales : p.c.k_scales;
  const int n_old = block_row >= 0 ? max(0, min(len - (pg << p.c.page_log2), P)) : 0;
  const float old_scale = n_old > 0 ? scales[block_row] : 0.0f;
  float x[16], m = 0.0f;
  bool got = false;
  if (lo + mine < hi) {
    const int row = row0 + (lo + mine - len);
    const long long src = source_row(p, fetch_index(p, row, g), b);
    if (src >= 0) {
      got = true;
      unpack(load_row((is_v ? p.v + g * p.v_head : p.k + g * p.k_head) + src * (is_v ? p.v_tok : p.k_tok), at), x);
      if (at.turned) {
        float cs[8], sn[8];
        angles_of(p.pos[row], p.inv_freq, j, cs, sn);
        rotate16(x, cs, sn, p.adjacent);
      }
      m = amax16(x);
    }
  }
  const int lanes = GL << p.small_log2;            // of a unit: 4 to 64, in a row
  for (int o = 1; o < min(lanes, 32); o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lanes > 32) {                                // a unit of two warps; the same for the whole call
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) warp_top[warp] = m;
    __syncthreads();                               // also: both have read the old scale
    m = fmaxf(m, warp_top[warp ^ 1]);
  }
  if (hi <= lo) return;
  int e = scale_exponent(__float_as_uint(m));
  const int e_old = scale_log2(__float_as_uint(old_scale));
  if (n_old > 0 && e_old > e) e = e_old;
  uint8_t* const rows = (is_v ? p.c.v_pages : p.c.k_pages) + (block_row << p.c.page_log2) * D;
  if (got) store_codes(rows + ((lo + mine) & (P - 1)) * D, at, x, __uint_as_float(pow2_bits(-e)));
  if (n_old > 0 && e > e_old) {                    // the rows that were there take the larger scale
    const float ratio = __uint_as_float(pow2_bits(max(e_old - e, -126)));
    uint4* const w = reinterpret_cast<uint4*>(rows + 16 * j);
    for (int r0 = mine; r0 < n_old; r0 += 8 * mates) {             // eight rows' loads under way together
      uint4 c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i * mates < n_old) c[i] = w[(r0 + i * mates) * GL];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (r0 + i * mates >= n_old) continue;
        c[i].x = rescale_e4m3(c[i].x, ratio); c[i].y = rescale_e4m3(c[i].y, ratio);
        c[i].z = rescale_e4m3(c[i].z, ratio); c[i].w = rescale_e4m3(c[i].w, ratio);
        w[(r0 + i * mates) * GL] = c[i];
      }
    }
  }
  if (mine == 0 && j == 0) scales[block_row] = __uint_as_float(pow2_bits(e));
}

// The larger of two pairs of bf16 magnitudes (a NaN gives way, as with fmaxf).
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t m, uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b32 a;\n\tabs.bf16x2 a, %2;\n\tmax.bf16x2 %0, %1, a;\n\t}" : "=r"(r) : "r"(m), "r"(w));
  return r;
}
__device__ __forceinline__ float amax_raw(const Row16& r) {
  uint32_t m = 0;
  m = max_abs_bf16x2(m, r.lo.x); m = max_abs_bf16x2(m, r.lo.y); m = max_abs_bf16x2(m, r.lo.z); m = max_abs_bf16x2(m, r.lo.w);
  m = max_abs_bf16x2(m, r.hi.x); m = max_abs_bf16x2(m, r.hi.y); m = max_abs_bf16x2(m, r.hi.z); m = max_abs_bf16x2(m, r.hi.w);
  return fmaxf(bf_lo(m), bf_hi(m));
}

// Page role: a block takes one page of one sequence and a slice of the 2 * Hkv heads, kHeads of them a round.  A head's rows of
// the page come into shared memory rounds ahead, by one tiled copy (whoever starts it is held up for some 500 cycles, so the
// heads of a round are started from different warps), or, when they are gathered, by 16-byte copies that every lane asks for
// itself (a bulk copy for every row: 20.7 us against 18, 13107 rows).  The block meets over the largest absolute value of each
// head's rows; the rows are read from shared memory once for it and once more to be encoded, which leaves the registers to more
// blocks per SM.
template <int D, int NS, int kMode>
__device__ void append_page(const AppendParams& p, const CUtensorMap* map_k, const CUtensorMap* map_v, int block) {
  constexpr int GL = D / 16, kPageSlots = kSlotsOf<kMode>;
  constexpr bool kRot = kMode == kRotated, gather = kMode == kGathered;
  extern __shared__ __align__(128) uint8_t ring[];   // [kPageSlots][rows of a slot][D] bf16
  __shared__ uint64_t full[kPageSlots];
  __shared__ uint32_t top[3][kHeads][4];          // by round: the bits of the largest absolute value, per head (and side by side)
  __shared__ int abort_flag;
  const int P = 1 << p.c.page_log2, Hkv = p.c.n_kv_heads, jobs = 2 * Hkv;
  const int threads = blockDim.x, groups = threads / GL, j = threadIdx.x % GL, grp = threadIdx.x / GL;
  const int lane = threadIdx.x & 31;
  const int side = groups > P ? groups / P : 1;   // heads that a small page lets a slot hold side by side (4 at most)
  const int mine = grp >> p.c.page_log2;          // which of them (0 when side == 1)
  const int n_rows = groups * NS;                 // rows of a slot
  const int item = block / p.job_slices, slice = block - item * p.job_slices;
  const int b = item / p.pages_per_seq, which = item - b * p.pages_per_seq;
  pdl_wait();
  const int len = p.lens[b];
  RowRange r;
  new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
  if (r.count <= 0) return;
  const int pg = (len >> p.c.page_log2) + which, slot0 = pg << p.c.page_log2;
  const int lo = max(len, slot0), hi = min(len + r.count, slot0 + P);
  if (hi <= lo) return;
  const int pid = p.c.block_table[static_cast<long long>(b) * p.c.max_pages + pg];
  if (pool_block(pid, p.c.n_pages, Hkv, 0) < 0) {
    if (threadIdx.x == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_PAGE);
    return;
  }
  if (threadIdx.x < kHeads * 4) (&top[0][0][0])[threadIdx.x] = 0u;
  if (!gather && threadIdx.x == 0) {
    abort_flag = 0;
    tma_prefetch_desc(map_k);
    tma_prefetch_desc(map_v);
    for (int i = 0; i < kPageSlots; ++i) mbar_init(&full[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  const int n_old = max(0, min(len - slot0, P));
  const int job0 = slice * p.jobs_per_slice, job1 = min(job0 + p.jobs_per_slice, jobs);
  const int fills = (job1 - job0 + side - 1) / side;            // slots to be filled in all
  const int rounds = (fills + kHeads - 1) / kHeads;
  const Pieces turned = pieces_of(j, D, kRot ? p.rot_dim : 0, p.adjacent), plain = pieces_of(j, D, 0, 0);

  // ---- what this thread brings of round k ----
  bool fresh[NS];                                 // this lane group's rows of a slot: which of them are new
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int slot = slot0 + ((grp + n * groups) & (P - 1));    // side == 1 whenever NS > 1
    fresh[n] = slot >= lo && slot < hi;
  }
  // Tiled: fill m of every kHeads is started by lane 0 of warp m % kHeads, a box of the page's rows for each head side by side.
  const uint64_t policy = l2_policy_evict_first();
  const int my_fill = static_cast<int>(threadIdx.x) / 32;
  auto start_boxes = [&](int k) {
    const int m = k * kHeads + my_fill;
    if (my_fill >= kHeads || lane != 0 || m >= fills || m == p.skip_copy) return;
    const int st = m % kPageSlots;
    const int first = job0 + m * side, n = min(side, job1 - first);
    mbar_arrive_expect_tx(&full[st], static_cast<uint32_t>(n) << (p.c.page_log2 + (D == 128 ? 8 : 7)));
    for (int z = 0; z < n; ++z) {
      const bool is_v = first + z >= Hkv;
      tma_load_3d(ring + ((static_cast<uint32_t>(st) * n_rows + (z << p.c.page_log2)) * (D * 2)), is_v ? map_v : map_k, &full[st], 0,
                  is_v ? first + z - Hkv : first + z, r.first + (slot0 - len), policy);
    }
  };
  // Gathered: every lane brings the two pieces of each row that it will encode itself, into 16 bytes of its own: nothing to wait
  // for but its own copies.
  const int src0 = gather && p.cu_src ? p.cu_src[b] : 0;          // where the sequence's source rows start, and how many
  const int src_n = gather ? min(p.cu_src ? p.cu_src[b + 1] - src0 : p.total_src, src0 >= 0 ? p.total_src - src0 : 0) : 0;
  const uint32_t own = smem_u32(ring) + threadIdx.x * 16, piece = threads * 16;
  auto own_slot = [&](int st, int n) -> uint32_t { return own + (st * NS + n) * 2 * piece; };
  int index[kHeads][NS];                          // source rows of the round that starts next
  auto fetch = [&](int k) {
#pragma unroll
    for (int z = 0; z < kHeads; ++z) {
      const int job = job0 + (k * kHeads + z) * side + mine, g = job >= Hkv ? job - Hkv : job;
#pragma unroll
      for (int n = 0; n < NS; ++n)
        if (fresh[n] && job < job1) index[z][n] = p.idx[static_cast<long long>(g) * p.total + r.first + (slot0 + ((grp + n * groups) & (P - 1)) - len)];
    }
  };
  auto start_rows = [&](int k) -> uint32_t {      // bit z * NS + n: row n of head z is on its way
    uint32_t coming = 0;
#pragma unroll
    for (int z = 0; z < kHeads; ++z) {
      const int m = k * kHeads + z, job = job0 + m * side + mine;
      const bool is_v = job >= Hkv;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        if (!fresh[n] || job >= job1) continue;
        if (index[z][n] < 0 || index[z][n] >= src_n) {
          if (j == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_INDEX);
          continue;
        }
        const int g = is_v ? job - Hkv : job, src = src0 + index[z][n];
        const uint16_t* x = is_v ? p.v + g * p.v_head + src * p.v_tok : p.k + g * p.k_head + src * p.k_tok;
        coming |= 1u << (z * NS + n);
        const uint32_t to = own_slot(m % kPageSlots, n);
        copy16_async(to, x + plain.lo);
        copy16_async(to + piece, x + plain.hi);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    fetch(k + 1);
    return coming;
  };
  uint32_t coming[kRoundsAhead<kMode> + 1];       // gathered: rows of the rounds ahead, nearest first
  if constexpr (gather) {
    fetch(0);
#pragma unroll
    for (int k = 0; k < kRoundsAhead<kMode>; ++k) coming[k] = start_rows(k);
  }
  __syncthreads();                                // barriers and top[0] are set
  if constexpr (!gather)
    for (int k = 0; k < kRoundsAhead<kMode>; ++k) start_boxes(k);

  // ---- the rows this lane group computes ----
  float cs[NS][8], sn[NS][8];
  if constexpr (kRot) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (fresh[n] && turned.turned && job0 < Hkv)
        angles_of(p.pos[r.first + (slot0 + ((grp + n * groups) & (P - 1)) - len)], p.inv_freq, j, cs[n], sn[n]);
  }
  auto row_at = [&](int st, int n, const Pieces& at) -> Row16 {
    if constexpr (gather) {
      Row16 raw;
      raw.lo = shared16(own_slot(st, n));
      raw.hi = shared16(own_slot(st, n) + piece);
      return raw;
    } else {
      return load_row(reinterpret_cast<const uint16_t*>(ring + (static_cast<uint32_t>(st) * n_rows + grp + n * groups) * (D * 2)), at);
    }
  };
  int ok = 1;                                     // of the whole block, once it has met
  int now = 0;                                    // k % 3
  int k = 0;
  for (; k < rounds; ++k) {
    float old_scale[kHeads];
    uint32_t here = 0;                            // bit z * NS + n: this lane group has row n of head z
    const int next = now == 2 ? 0 : now + 1;
    if constexpr (gather) {
      coming[kRoundsAhead<kMode>] = start_rows(k + kRoundsAhead<kMode>);
      asm volatile("cp.async.wait_group %0;" ::"n"(kRoundsAhead<kMode>) : "memory");
      here = coming[0];
#pragma unroll
      for (int i = 0; i < kRoundsAhead<kMode>; ++i) coming[i] = coming[i + 1];
    }
#pragma unroll
    for (int z = 0; z < kHeads; ++z) {
      const int m = k * kHeads + z, st = m % kPageSlots, job = job0 + m * side + mine;
      const bool on = job < job1, is_v = job >= Hkv;
      old_scale[z] = on && n_old > 0 ? (is_v ? p.c.v_scales : p.c.k_scales)[static_cast<long long>(pid) * Hkv + (is_v ? job - Hkv : job)] : 0.0f;
      if (!gather && m < fills && ok) ok = mbar_wait_bounded(&full[st], (m / kPageSlots) & 1, &abort_flag, p.hdr, SITE_APPEND_WAIT, p.wait_limit);
      const Pieces& at = is_v ? plain : turned;
      float big = 0.0f;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        if (!gather && ok && on && fresh[n]) here |= 1u << (z * NS + n);
        if (!((here >> (z * NS + n)) & 1u)) continue;
        const Row16 raw = row_at(st, n, at);
        if (kRot && !is_v) {
          float x[16];
          unpack(raw, x);
          if (at.turned) rotate16(x, cs[n], sn[n], p.adjacent);
          big = fmaxf(big, amax16(x));
        } else {
          big = fmaxf(big, amax_raw(raw));
        }
      }
      // magnitudes order like their bits
      const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(big));
      if (lane == 0 && most != 0u) atomicMax(&top[now][z][mine], most);
    }
    if (threadIdx.x < kHeads * 4) (&top[next][0][0])[threadIdx.x] = 0u;             // last read two rounds ago
    // Every thread has read the old scales, and is done with the round before.  Tiled: the block agrees on whether the round's rows
    // are there, so that a head is written by all of it or by none; after a wait that gave up nothing more is started, because
    // nobody would wait for the copies before it in the same slots.
    if constexpr (gather) {
      __syncthreads();
    } else {
      ok = __syncthreads_and(ok);
      if (!ok) break;
      start_boxes(k + kRoundsAhead<kMode>);       // into the slots of the round before
    }
#pragma unroll
    for (int z = 0; z < kHeads; ++z) {
      const int m = k * kHeads + z, st = m % kPageSlots, job = job0 + m * side + mine;
      if (job >= job1) continue;
      const bool is_v = job >= Hkv;
      const int g = is_v ? job - Hkv : job;
      const Pieces& at = is_v ? plain : turned;
      const long long block_row = static_cast<long long>(pid) * Hkv + g;
      int e = scale_exponent(top[now][z][mine]);
      const int e_old = scale_log2(__float_as_uint(old_scale[z]));
      if (n_old > 0 && e_old > e) e = e_old;
      const float inv = __uint_as_float(pow2_bits(-e));
      uint8_t* const rows = (is_v ? p.c.v_pages : p.c.k_pages) + (block_row << p.c.page_log2) * D;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int in_page = (grp + n * groups) & (P - 1);
        if ((here >> (z * NS + n)) & 1u) {
          float x[16];
          unpack(row_at(st, n, at), x);
          if (kRot && !is_v && at.turned) rotate16(x, cs[n], sn[n], p.adjacent);
          store_codes(rows + in_page * D, at, x, inv);
        }
        if (n_old > 0 && e > e_old && in_page < n_old) {
          const float ratio = __uint_as_float(pow2_bits(max(e_old - e, -126)));
          uint4* w = reinterpret_cast<uint4*>(rows + in_page * D + 16 * j);
          uint4 c = *w;
          c.x = rescale_e4m3(c.x, ratio); c.y = rescale_e4m3(c.y, ratio);
          c.z = rescale_e4m3(c.z, ratio); c.w = rescale_e4m3(c.w, ratio);
          *w = c;
        }
      }
      if ((grp & (P - 1)) == 0 && j == 0) ((is_v ? p.c.v_scales : p.c.k_scales))[block_row] = __uint_as_float(pow2_bits(e));
    }
    now = next;
  }
  if (!ok)                                        // round k's copies and those ahead of it may be in flight: none when the block leaves
    for (int m = k * kHeads; m < min(fills, (k + kRoundsAhead<kMode>) * kHeads); ++m)
      if (m != p.skip_copy) mbar_wait_drain(&full[m % kPageSlots], (m / kPageSlots) & 1, p.hdr, SITE_APPEND_WAIT);
}

// kKind: 0 bf16 pages (row role only), 1 8-bit pages with the small role, 2 and 3 with the page role (one, two rows per lane
// group).  The blocks from page_blocks on take the row role.
template <int D, int kKind, int kMode>
__global__ void __launch_bounds__(kKind == 3 ? 512 : 256, kKind <= 1 ? 2 : 0)
paged_append_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AppendParams p) {
  pdl_launch_dependents();                        // every role waits for earlier kernels once it knows what it is to do
  if (blockIdx.x == 0) {
    pdl_wait();                                   // and with this block's, who waits for this kernel waits for them, too
    for (int b = threadIdx.x; b < p.c.batch; b += blockDim.x) {
      RowRange r;
      const int len = p.lens[b];
      const bool ok = new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
      if (p.new_lens != nullptr) p.new_lens[b] = max(len, 0) + r.count;
      if (!ok) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_ROWS);
    }
  }
  // the long blocks of the page role come first, so that the short ones of the row role fill the gaps they leave
  const int block = static_cast<int>(blockIdx.x);
  if (block >= p.page_blocks) append_rows<D, kKind != 0, kMode>(p, block - p.page_blocks);
  else if constexpr (kKind == 1) append_small<D>(p, block);
  else if constexpr (kKind == 2) append_page<D, 1, kMode>(p, &map_k, &map_v, block);
  else if constexpr (kKind == 3) append_page<D, 2, kMode>(p, &map_k, &map_v, block);
}

template <int D, int kKind, int kMode>
static cudaError_t launch_kind(const AppendParams& p, const CUtensorMap (&maps)[2], int blocks, int threads, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  constexpr int kEach = kKind == 3 ? 2 * kSlotsOf<kMode> : kKind == 2 ? kSlotsOf<kMode> : 0;    // page role: rows of 32 bytes a thread
  const int rows = p.row_heads == 0 ? kEach : kEach > kRowStages ? kEach : kRowStages;
  static PerDeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(paged_append_kernel<D, kKind, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (kEach > kRowStages ? kEach : kRowStages) * 32 * (kKind == 3 ? 512 : 256));
    if (e != cudaSuccess) return e;
    configured.set(dev);
  }
  cfg.dynamicSmemBytes = rows * 32 * threads;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_append_kernel<D, kKind, kMode>, maps[0], maps[1], p);
}

template <int D, int kMode>
static cudaError_t launch_mode(const AppendParams& p, const CUtensorMap (&maps)[2], bool e4m3, bool two_rows, int blocks, int threads,
                               cudaStream_t stream) {
  if (!e4m3) return launch_kind<D, 0, kMode>(p, maps, blocks, threads, stream);
  return two_rows ? launch_kind<D, 3, kMode>(p, maps, blocks, threads, stream) : launch_kind<D, 2, kMode>(p, maps, blocks, threads, stream);
}

template <int D>
static cudaError_t launch_d(AppendParams& p, const CUtensorMap (&maps)[2], bool e4m3, cudaStream_t stream) {
  constexpr int GL = D / 16, kSms = 148;
  const int P = 1 << p.c.page_log2, jobs = 2 * p.c.n_kv_heads;
  const bool small = p.max_new <= kSmallRows;
  const int per_page = P * GL;                    // lanes that hold a page's rows of one head, one row per lane group
  const int threads = e4m3 && !small && per_page > 512 ? 512 : 256;
  // Row role: a token's heads are split over as many lane groups as it takes to put two blocks on every SM (what their registers
  // allow); a long call keeps them together, so that a token's angles are formed once.
  p.row_heads = p.n_q_heads + (e4m3 ? 0 : jobs);
  const long long groups = static_cast<long long>(kSms) * 2 * (256 / GL);
  long long hpu = p.row_heads > 0 ? (static_cast<long long>(p.total) * p.row_heads + groups - 1) / groups : 1;
  if (hpu < 1) hpu = 1;
  if (hpu > p.row_heads && p.row_heads > 0) hpu = p.row_heads;
  p.row_slices = p.row_heads > 0 ? (p.row_heads + static_cast<int>(hpu) - 1) / static_cast<int>(hpu) : 0;
  p.heads_per_unit = p.row_slices > 0 ? (p.row_heads + p.row_slices - 1) / p.row_slices : 1;        // alike
  const long long units = static_cast<long long>(p.row_slices) * p.total;
  const long long row_blocks = (units + threads / GL - 1) / (threads / GL);
  long long page_blocks = 0;
  if (e4m3) {
    // pages a sequence's new rows can touch
    p.pages_per_seq = p.max_new == 1 ? 1 : (p.max_new + P - 2) / P + 1;
    const long long items = static_cast<long long>(p.c.batch) * p.pages_per_seq;
    if (small) {
      p.small_log2 = p.max_new == 1 ? 0 : p.max_new == 2 ? 1 : p.max_new <= 4 ? 2 : 3;
      const int units = (threads / GL) >> p.small_log2;            // of a block
      page_blocks = (items * jobs + units - 1) / units;
    } else {
      // Page role: a block walks all heads of its page; with fewer pages than the SMs hold blocks (as far as the slots' shared
      // memory goes), the heads are split over as many blocks as still run at once (13107 gathered rows, pages of 64: 18 us in 410
      // blocks; 20.3 in 820, 22.6 in 1640).
      long long slices = static_cast<long long>(kSms) * (threads == 512 ? 1 : per_page > threads ? (p.idx ? 3 : 2) : 4) / items;
      const int side = per_page < threads ? threads / per_page : 1;
      if (slices > jobs / side) slices = jobs / side;
      if (slices < 1) slices = 1;
      p.jobs_per_slice = static_cast<int>((jobs + slices - 1) / slices);
      p.jobs_per_slice = (p.jobs_per_slice + side - 1) / side * side;
      p.job_slices = (jobs + p.jobs_per_slice - 1) / p.jobs_per_slice;
      page_blocks = items * p.job_slices;
    }
  }
  if (page_blocks + row_blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  p.page_blocks = static_cast<int>(page_blocks);
  const int blocks = static_cast<int>(page_blocks + row_blocks);
  if (e4m3 && small) return launch_kind<D, 1, kRotated>(p, maps, blocks, threads, stream);       // the small role looks for itself
  const bool two_rows = e4m3 && per_page > threads;
  if (p.rot_dim) return launch_mode<D, kRotated>(p, maps, e4m3, two_rows, blocks, threads, stream);
  if (p.idx) return launch_mode<D, kGathered>(p, maps, e4m3, two_rows, blocks, threads, stream);
  return launch_mode<D, kPlain>(p, maps, e4m3, two_rows, blocks, threads, stream);
}

bool paged_append_uses_maps(const AppendParams& p, bool e4m3) { return e4m3 && p.max_new > kSmallRows && p.idx == nullptr; }

cudaError_t launch_paged_append(AppendParams& p, const CUtensorMap (&maps)[2], int head_dim, bool e4m3, cudaStream_t stream) {
  if (head_dim == 128) return launch_d<128>(p, maps, e4m3, stream);
  if (head_dim == 64) return launch_d<64>(p, maps, e4m3, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
