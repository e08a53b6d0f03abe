// Index arithmetic of the paged cache, shared by the kernels and by a host test: which page and row an entry sits in,
// which rows a call may touch, and the power-of-two scale of a block.  Plain C++ apart from the function qualifiers.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define FASTKV_HD __host__ __device__ __forceinline__
#else
#define FASTKV_HD inline
#endif

namespace fastkv {

// 448 is the largest e4m3 value.  A block's scale is 2^e with e in this range: 2^120 * 448 is beyond every finite
// float, and below 2^-64 nothing that a model computes is lost (2^-64 * 2^-9 is the smallest step kept).
constexpr int kScaleMinExp = -64, kScaleMaxExp = 120;

// The smallest e (within the range) with 448 * 2^e >= m, from the bits of m >= 0: with m = 1.f * 2^E the answer is
// E - 8 as long as 1.f <= 1.75 (448 = 1.75 * 2^8), else E - 7.  Zero and subnormals give the smallest scale; infinity
// the largest.
FASTKV_HD int scale_exponent(uint32_t m_bits) {
  const int E = static_cast<int>((m_bits >> 23) & 0xffu) - 127;
  int e = E - 8 + ((m_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  if (e < kScaleMinExp) e = kScaleMinExp;
  if (e > kScaleMaxExp) e = kScaleMaxExp;
  return e;
}
// 2^e for e in [-126, 127], as the bits of a float.
FASTKV_HD uint32_t pow2_bits(int e) { return static_cast<uint32_t>(e + 127) << 23; }
// The exponent of a scale read back from a pool (a power of two).
FASTKV_HD int scale_log2(uint32_t s_bits) { return static_cast<int>((s_bits >> 23) & 0xffu) - 127; }

// Entries of a sequence that a call may use: what the caller's length says, cut to what its block-table row can hold.
FASTKV_HD int usable_len(int len, int max_pages, int page_log2) {
  const long long room = static_cast<long long>(max_pages) << page_log2;
  if (len < 0) return 0;
  return len > room ? static_cast<int>(room) : len;
}

// Chunks of 2^chunk_log2 entries that hold `len` >= 0 entries, without a sum that could pass 2^31 - 1.
FASTKV_HD int chunk_count(int len, int chunk_log2) { return len <= 0 ? 0 : ((len - 1) >> chunk_log2) + 1; }
// The first chunks of them that every one of q_len query tokens sees all of.
FASTKV_HD int chunks_all_see(int len, int q_len, int chunk_log2) {
  const int all = len - (q_len - 1);
  return all <= 0 ? 0 : all >> chunk_log2;
}

// New rows of sequence b: [first, first + count) of the call's rows, cut to the rows that exist and to the room behind
// `len` entries.  Returns whether nothing had to be cut.
struct RowRange {
  int first, count;
};
FASTKV_HD bool new_rows_of(const int* cu_new, int uniform, int total, int max_new, int b, int len, int max_pages,
                           int page_log2, RowRange* r) {
  long long first = cu_new ? cu_new[b] : static_cast<long long>(b) * uniform;
  long long count = cu_new ? static_cast<long long>(cu_new[b + 1]) - first : uniform;
  const long long asked = count, capacity = static_cast<long long>(max_pages) << page_log2;
  bool ok = len >= 0 && len <= capacity && first >= 0 && count >= 0 && count <= max_new && first + count <= total;
  if (!ok) {
    if (len < 0 || first < 0 || first > total) { first = 0; count = 0; }
    if (count > max_new) count = max_new;
    if (first + count > total) count = total - first;
    if (count < 0) count = 0;
  }
  const long long room = capacity - (len < 0 ? 0 : len);
  if (count > room) count = room < 0 ? 0 : room;
  r->first = static_cast<int>(first);
  r->count = static_cast<int>(count);
  return ok && count == asked;
}

// Row of the pool ([pages * heads] blocks of 2^page_log2 rows) that holds entry `slot` of the sequence; -1 if the block
// table names a page that does not exist.  64-bit: a pool may hold more than 2^31 rows.
FASTKV_HD long long pool_block(int page, int n_pages, int n_kv_heads, int head) {
  if (page < 0 || page >= n_pages) return -1;
  return static_cast<long long>(page) * n_kv_heads + head;
}

}  // namespace fastkv
