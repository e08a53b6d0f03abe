// Appending rows to the paged cache: new tokens' keys and values (the keys, and the queries beside them, rotated by their
// positions), or the rows that the selection kept (Alg. 1: C <- update(K, V)), into pages of bf16 or of 8-bit codes with
// a power-of-two scale for each (page, KV head).
//
// Rotation: for pair i of a head's first rot_dim elements, angle a = pos * inv_freq[i],
//   y1 = x1 cos a - x2 sin a,   y2 = x2 cos a + x1 sin a      (three roundings each in fp32, then the one of the cache).
// The angle is formed and reduced in fp64: in fp32 a position of 100 000 leaves 2^-7 of an angle's bits.
//
// Eight lanes (four for head_dim 64) handle one row of one head: sixteen elements each, as two 16-byte pieces chosen so
// that both halves of every rotated pair are the lane's own.
//   Row role   (bf16 pages; queries of either format): a lane group takes one token and a run of heads, so that the
//              angles are formed once per run.
//   Page role  (8-bit pages, calls of more than 8 rows per sequence): a block takes one page and walks a run of heads; the
//              page's rows of one head sit in registers while their largest absolute value is found.
//   Small role (8-bit pages, up to 8 rows per sequence): a lane group takes one (page, head) and its few new rows.
// Rows that were in a page before keep their codes unless the new rows need a larger scale; then the codes are re-encoded
// by the ratio, a power of two, which is exact but for codes that become subnormal.
#include "paged.cuh"

namespace fastkv {

namespace {

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

// Where lane j's two pieces start in a head's row, and whether they are rotated.
struct Pieces {
  int lo, hi;
  bool turned;
};
__device__ __forceinline__ Pieces pieces_of(int j, int rot_dim, int adjacent) {
  Pieces q;
  q.turned = 16 * j < rot_dim;
  q.lo = 16 * j;
  q.hi = 16 * j + 8;
  if (q.turned && !adjacent) {       // halves: elements i and i + rot_dim / 2
    q.lo = 8 * j;
    q.hi = rot_dim / 2 + 8 * j;
  }
  return q;
}

// cos and sin of the eight pairs 8j .. 8j + 7 at position `pos`.  The angle in turns, pos * f / (2 pi), is formed in fp64
// with the rounding error of the product added back after the whole turns are gone.
__device__ __forceinline__ void angles_of(int pos, const float* inv_freq, int j, float (&cs)[8], float (&sn)[8]) {
  const double kInv2Pi = 0.15915494309189535, kInv2PiLow = -9.839338337591243e-18;
  const float4 f0 = *reinterpret_cast<const float4*>(inv_freq + 8 * j), f1 = *reinterpret_cast<const float4*>(inv_freq + 8 * j + 4);
  const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double a = static_cast<double>(pos) * static_cast<double>(f[e]);
    const double t = a * kInv2Pi;
    const double r = (t - rint(t)) + (fma(a, kInv2Pi, -t) + a * kInv2PiLow);
    double s, c;
    sincospi(2.0 * r, &s, &c);
    cs[e] = static_cast<float>(c);
    sn[e] = static_cast<float>(s);
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
__device__ __forceinline__ void rotate16(float (&x)[16], const float (&cs)[8], const float (&sn)[8], int adjacent) {
  if (adjacent) {
#pragma unroll
    for (int m = 0; m < 8; ++m) turn(x[2 * m], x[2 * m + 1], cs[m], sn[m]);
  } else {
#pragma unroll
    for (int m = 0; m < 8; ++m) turn(x[m], x[8 + m], cs[m], sn[m]);
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

// The source row of new row `row` of head h: itself, or the kept row that idx names (-1: none such).
__device__ __forceinline__ long long source_row(const AppendParams& p, int row, int b, int h) {
  if (p.idx == nullptr) return row;
  const int i = p.idx[static_cast<long long>(h) * p.total + row];
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

// Row role: unit u = (slice of heads, token); heads in the order queries, keys, values.
template <int D, bool kE4M3>
__device__ void append_rows(const AppendParams& p) {
  constexpr int GL = D / 16;                      // lanes of a row
  constexpr int kBatch = 4;                       // rows loaded before the first is used
  const int j = threadIdx.x % GL;
  const long long u = static_cast<long long>(blockIdx.x) * (blockDim.x / GL) + threadIdx.x / GL;
  if (u >= static_cast<long long>(p.row_slices) * p.total) return;
  const int slice = static_cast<int>(u / p.total), t = static_cast<int>(u - static_cast<long long>(slice) * p.total);
  const int h0 = slice * p.heads_per_unit, h1 = min(h0 + p.heads_per_unit, p.row_heads);
  const int Hq = p.n_q_heads, Hkv = p.c.n_kv_heads;
  const Pieces turned = pieces_of(j, p.rot_dim, p.adjacent), plain = pieces_of(j, 0, 0);
  float cs[8], sn[8];
  if (turned.turned && h0 < Hq + Hkv) angles_of(p.pos[t], p.inv_freq, j, cs, sn);
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
  for (int hb = h0; hb < h1; hb += kBatch) {
    Row16 raw[kBatch];
    bool have[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = hb + i;
      have[i] = false;
      if (h >= h1) continue;
      if (h < Hq) {
        raw[i] = load_row(p.q + static_cast<long long>(t) * p.q_tok + h * p.q_head, turned);
        have[i] = true;
      } else if (!kE4M3 && page >= 0) {
        const bool is_k = h < Hq + Hkv;
        const int g = is_k ? h - Hq : h - Hq - Hkv;
        const long long src = source_row(p, t, b, g);
        if (src < 0) continue;
        have[i] = true;
        if (is_k) raw[i] = load_row(p.k + src * p.k_tok + g * p.k_head, turned);
        else raw[i] = load_row(p.v + src * p.v_tok + g * p.v_head, plain);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (!have[i]) continue;
      const int h = hb + i;
      const bool is_v = h >= Hq + Hkv;
      uint16_t* dst;
      if (h < Hq) {
        dst = p.q_out + (static_cast<long long>(t) * Hq + h) * D;
      } else {
        const int g = is_v ? h - Hq - Hkv : h - Hq;
        dst = reinterpret_cast<uint16_t*>(is_v ? p.c.v_pages : p.c.k_pages) + (((page + g) << p.c.page_log2) + in_page) * D;
      }
      if (!is_v && turned.turned) {
        float x[16];
        unpack(raw[i], x);
        rotate16(x, cs, sn, p.adjacent);
        raw[i].lo = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        raw[i].hi = make_uint4(pack_bf16(x[8], x[9]), pack_bf16(x[10], x[11]), pack_bf16(x[12], x[13]), pack_bf16(x[14], x[15]));
      }
      const Pieces& at = is_v ? plain : turned;
      *reinterpret_cast<uint4*>(dst + at.lo) = raw[i].lo;
      *reinterpret_cast<uint4*>(dst + at.hi) = raw[i].hi;
    }
  }
}

// Small role: unit u = (sequence, which of its touched pages, head of K or V); one lane group each.  Every lane of the
// warp takes part in the shuffles, so idle units walk through with nothing to do.
template <int D>
__device__ void append_small(const AppendParams& p, int block) {
  constexpr int GL = D / 16;
  const int j = threadIdx.x % GL, Hkv = p.c.n_kv_heads, jobs = 2 * Hkv;
  const long long u = static_cast<long long>(block) * (blockDim.x / GL) + threadIdx.x / GL;
  const long long units = static_cast<long long>(p.c.batch) * p.pages_per_seq * jobs;
  const bool live = u < units;
  const long long item = live ? u / jobs : 0;
  const int job = live ? static_cast<int>(u - item * jobs) : 0;
  const int b = static_cast<int>(item / p.pages_per_seq), which = static_cast<int>(item - static_cast<long long>(b) * p.pages_per_seq);
  const bool is_v = job >= Hkv;
  const int g = is_v ? job - Hkv : job;
  const Pieces at = is_v ? pieces_of(j, 0, 0) : pieces_of(j, p.rot_dim, p.adjacent);
  const int P = 1 << p.c.page_log2;
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
  const uint16_t* const base = is_v ? p.v + g * p.v_head : p.k + g * p.k_head;
  const long long tok = is_v ? p.v_tok : p.k_tok;
  float x[16];
  auto load = [&](int slot) -> bool {
    const int row = row0 + (slot - len);
    const long long src = source_row(p, row, b, g);
    if (src < 0) return false;
    unpack(load_row(base + src * tok, at), x);
    if (at.turned) {
      float cs[8], sn[8];
      angles_of(p.pos[row], p.inv_freq, j, cs, sn);
      rotate16(x, cs, sn, p.adjacent);
    }
    return true;
  };
  float m = 0.0f;
  bool got = false;
  for (int s = lo; s < hi; ++s) {
    got = load(s);
    if (got) m = fmaxf(m, amax16(x));
  }
#pragma unroll
  for (int o = 1; o < GL; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (hi <= lo) return;
  int e = scale_exponent(__float_as_uint(m));
  const int e_old = scale_log2(__float_as_uint(old_scale));
  if (n_old > 0 && e_old > e) e = e_old;
  const float inv = __uint_as_float(pow2_bits(-e));
  uint8_t* const rows = (is_v ? p.c.v_pages : p.c.k_pages) + (block_row << p.c.page_log2) * D;
  if (n_old > 0 && e > e_old) {                    // the rows that were there take the larger scale
    const float ratio = __uint_as_float(pow2_bits(max(e_old - e, -126)));
    for (int r = 0; r < n_old; ++r) {
      uint4* w = reinterpret_cast<uint4*>(rows + r * D + 16 * j);
      uint4 c = *w;
      c.x = rescale_e4m3(c.x, ratio); c.y = rescale_e4m3(c.y, ratio);
      c.z = rescale_e4m3(c.z, ratio); c.w = rescale_e4m3(c.w, ratio);
      *w = c;
    }
  }
  if (j == 0) scales[block_row] = __uint_as_float(pow2_bits(e));
  for (int s = lo; s < hi; ++s) {
    if (hi - lo > 1) got = load(s);
    if (got) store_codes(rows + (s & (P - 1)) * D, at, x, inv);
  }
}

// Page role: a block takes one page of one sequence and a slice of the 2 * Hkv heads; NS rows per lane group.
template <int D, int NS>
__device__ void append_page(const AppendParams& p, int block) {
  constexpr int GL = D / 16;
  __shared__ float top[2][16];                    // per warp: largest absolute value of the rows it holds
  const int P = 1 << p.c.page_log2, Hkv = p.c.n_kv_heads, jobs = 2 * Hkv;
  const int groups = blockDim.x / GL, j = threadIdx.x % GL, grp = threadIdx.x / GL;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int side = groups > P ? groups / P : 1;   // heads that a small page lets the block take side by side
  const int mine = grp / P;                       // which of them (0 when side == 1)
  const int item = block / p.job_slices, slice = block - item * p.job_slices;
  const int b = item / p.pages_per_seq, which = item - b * p.pages_per_seq;
  const int len = p.lens[b];
  RowRange r;
  new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
  if (r.count <= 0) return;
  const int pg = (len >> p.c.page_log2) + which;
  const int lo = max(len, pg << p.c.page_log2), hi = min(len + r.count, (pg + 1) << p.c.page_log2);
  if (hi <= lo) return;
  const int pid = p.c.block_table[static_cast<long long>(b) * p.c.max_pages + pg];
  if (pool_block(pid, p.c.n_pages, Hkv, 0) < 0) {
    if (threadIdx.x == 0) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_PAGE);
    return;
  }
  const int n_old = max(0, min(len - (pg << p.c.page_log2), P));
  const int job0 = slice * p.jobs_per_slice, job1 = min(job0 + p.jobs_per_slice, jobs);
  const Pieces turned = pieces_of(j, p.rot_dim, p.adjacent), plain = pieces_of(j, 0, 0);
  int in_page[NS], row[NS];
  bool fresh[NS];
  float cs[NS][8], sn[NS][8];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    in_page[n] = grp % P + n * groups;            // side == 1 whenever NS > 1
    const int slot = (pg << p.c.page_log2) + in_page[n];
    fresh[n] = in_page[n] < P && slot >= lo && slot < hi;
    row[n] = r.first + (slot - len);
    if (fresh[n] && turned.turned && job0 < Hkv) angles_of(p.pos[row[n]], p.inv_freq, j, cs[n], sn[n]);
  }
  int turnstile = 0;
  for (int jb = job0; jb < job1; jb += side, turnstile ^= 1) {
    const int job = jb + mine;
    const bool on = job < job1;
    const bool is_v = job >= Hkv;
    const int g = is_v ? job - Hkv : job;
    const Pieces& at = is_v ? plain : turned;
    const long long block_row = static_cast<long long>(pid) * Hkv + g;
    float* const scales = is_v ? p.c.v_scales : p.c.k_scales;
    const float old_scale = on && n_old > 0 ? scales[block_row] : 0.0f;
    float x[NS][16];
    bool got[NS];
    float m = 0.0f;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      got[n] = false;
      if (!on || !fresh[n]) continue;
      const long long src = source_row(p, row[n], b, g);
      if (src < 0) continue;
      got[n] = true;
      unpack(load_row((is_v ? p.v + g * p.v_head + src * p.v_tok : p.k + g * p.k_head + src * p.k_tok), at), x[n]);
    }
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (!got[n]) continue;
      if (at.turned) rotate16(x[n], cs[n], sn[n], p.adjacent);
      m = fmaxf(m, amax16(x[n]));
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) top[turnstile][warp] = m;
    __syncthreads();                              // also: every thread has read the old scale
    const int warps_each = (blockDim.x >> 5) / side, w0 = mine * warps_each;
    m = 0.0f;
    for (int w = 0; w < warps_each; ++w) m = fmaxf(m, top[turnstile][w0 + w]);
    if (!on) continue;
    int e = scale_exponent(__float_as_uint(m));
    const int e_old = scale_log2(__float_as_uint(old_scale));
    if (n_old > 0 && e_old > e) e = e_old;
    const float inv = __uint_as_float(pow2_bits(-e));
    uint8_t* const rows = (is_v ? p.c.v_pages : p.c.k_pages) + (block_row << p.c.page_log2) * D;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (got[n]) store_codes(rows + in_page[n] * D, at, x[n], inv);
      if (n_old > 0 && e > e_old && in_page[n] < n_old) {
        const float ratio = __uint_as_float(pow2_bits(max(e_old - e, -126)));
        uint4* w = reinterpret_cast<uint4*>(rows + in_page[n] * D + 16 * j);
        uint4 c = *w;
        c.x = rescale_e4m3(c.x, ratio); c.y = rescale_e4m3(c.y, ratio);
        c.z = rescale_e4m3(c.z, ratio); c.w = rescale_e4m3(c.w, ratio);
        *w = c;
      }
    }
    if (grp % P == 0 && j == 0) scales[block_row] = __uint_as_float(pow2_bits(e));
  }
}

// kPage: 0 bf16 pages (row role only), 1 8-bit pages with the small role, 2 and 3 with the page role (one, two rows per
// lane group).  The first row_blocks blocks take the row role.
template <int D, int kKind>
__global__ void __launch_bounds__(kKind == 3 ? 512 : 256) paged_append_kernel(const AppendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && p.new_lens != nullptr) {
    for (int b = threadIdx.x; b < p.c.batch; b += blockDim.x) {
      RowRange r;
      const int len = p.lens[b];
      const bool ok = new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, len, p.c.max_pages, p.c.page_log2, &r);
      p.new_lens[b] = max(len, 0) + r.count;
      if (!ok) raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_ROWS);
    }
  } else if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b < p.c.batch; b += blockDim.x) {
      RowRange r;
      if (!new_rows_of(p.cu_new, p.uniform, p.total, p.max_new, b, p.lens[b], p.c.max_pages, p.c.page_log2, &r))
        raise_status(p.hdr, FASTKV_ERR_DEVICE_INDEX, SITE_APPEND_ROWS);
    }
  }
  const int block = static_cast<int>(blockIdx.x) - p.row_blocks;
  if (block < 0) {
    append_rows<D, kKind != 0>(p);
    return;
  }
  if constexpr (kKind == 1) append_small<D>(p, block);
  if constexpr (kKind == 2) append_page<D, 1>(p, block);
  if constexpr (kKind == 3) append_page<D, 2>(p, block);
}

template <int D, int kKind>
static cudaError_t launch_kind(const AppendParams& p, int blocks, int threads, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  fill_pdl_attribute(&attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_append_kernel<D, kKind>, p);
}

template <int D>
static cudaError_t launch_d(AppendParams& p, bool e4m3, cudaStream_t stream) {
  constexpr int GL = D / 16, kSms = 148;
  const int P = 1 << p.c.page_log2, jobs = 2 * p.c.n_kv_heads;
  const bool small = p.max_new <= kSmallRows;
  const int per_page = P * GL;                    // lanes that hold a page's rows of one head, one row per lane group
  const int threads = e4m3 && !small && per_page > 512 ? 512 : 256;
  // Row role: a token's heads are split over as many lane groups as it takes to put about eight blocks on every SM; a
  // long call keeps them together, so that a token's angles are formed once.
  p.row_heads = p.n_q_heads + (e4m3 ? 0 : jobs);
  const long long groups = static_cast<long long>(kSms) * 8 * (threads / GL);
  long long hpu = p.row_heads > 0 ? (static_cast<long long>(p.total) * p.row_heads + groups - 1) / groups : 1;
  if (hpu < 1) hpu = 1;
  if (hpu > p.row_heads && p.row_heads > 0) hpu = p.row_heads;
  p.heads_per_unit = static_cast<int>(hpu);
  p.row_slices = p.row_heads > 0 ? (p.row_heads + p.heads_per_unit - 1) / p.heads_per_unit : 0;
  const long long units = static_cast<long long>(p.row_slices) * p.total;
  p.row_blocks = static_cast<int>((units + threads / GL - 1) / (threads / GL));
  if (!e4m3) return launch_kind<D, 0>(p, p.row_blocks, threads, stream);
  // pages a sequence's new rows can touch
  p.pages_per_seq = (p.max_new + P - 2) / P + 1;
  const long long items = static_cast<long long>(p.c.batch) * p.pages_per_seq;
  if (small) {
    if (p.max_new == 1) p.pages_per_seq = 1;
    const long long n = static_cast<long long>(p.c.batch) * p.pages_per_seq * jobs;
    const long long blocks = (n + threads / GL - 1) / (threads / GL);
    return launch_kind<D, 1>(p, p.row_blocks + static_cast<int>(blocks), threads, stream);
  }
  // Page role: a block walks all heads of its page when there are pages enough for about four blocks on every SM.
  long long slices = (4LL * kSms + items - 1) / items;
  const int side = per_page < threads ? threads / per_page : 1;
  if (slices > jobs / side) slices = jobs / side;
  if (slices < 1) slices = 1;
  p.jobs_per_slice = static_cast<int>((jobs + slices - 1) / slices);
  p.jobs_per_slice = (p.jobs_per_slice + side - 1) / side * side;
  p.job_slices = (jobs + p.jobs_per_slice - 1) / p.jobs_per_slice;
  const long long blocks = p.row_blocks + items * p.job_slices;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  if (per_page > threads) return launch_kind<D, 3>(p, static_cast<int>(blocks), threads, stream);
  return launch_kind<D, 2>(p, static_cast<int>(blocks), threads, stream);
}

cudaError_t launch_paged_append(AppendParams& p, int head_dim, bool e4m3, cudaStream_t stream) {
  if (head_dim == 128) return launch_d<128>(p, e4m3, stream);
  if (head_dim == 64) return launch_d<64>(p, e4m3, stream);
  return cudaErrorInvalidValue;
}

}  // namespace fastkv
