// Operators on a cache kept in pages: what the host side (paged_api.hip) hands to the kernels (kernels_paged.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace flk {

constexpr int kRowTile = 16;        // query rows (token x head of a group) of a block of the streaming kernel
inline int row_keys(int dtype) { return dtype == 0 ? 16 : 32; }    // keys of a step of it: 32 of 16-bit caches, 16 of fp32 ones
constexpr int kTileRows = 128, kTileKeys = 64;                     // the same of the tile kernel (16-bit types)

// Quotients by a number known on the host: x / d = floor(x m / 2^(31 + l)) for 0 <= x < 2^31, with l = ceil(log2 d), m = ceil(2^(31 + l) / d), since
// m d exceeds 2^(31 + l) by less than d <= 2^l (division by invariant multiplication; Granlund and Montgomery, PLDI 1994).
struct Divisor {
  uint32_t m;
  int l;
};
inline Divisor divisor(int d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  return {(uint32_t)(((1ull << (31 + l)) + d - 1) / d), l};
}
__device__ __forceinline__ int quotient(int x, const Divisor& d) { return (int)(__umulhi((uint32_t)x << 1, d.m) >> d.l); }

// A sequence of the plan.
struct PagedSeq {
  int first;      // its first new token's row in q, k, v and out
  int fresh;      // new tokens
  int len;        // cached rows with them
  int pages;      // its first entry in the page list
};
// A block's work: rows [row0, row0 + tile) of one key head of a sequence over steps [u0, u1) of the keys that some row sees.  Step u is
// keys step * u .. while u < gap, and step * (u + skip) .. behind: the keys between first tokens and window are left out.
struct PagedItem {
  PagedSeq s;
  int row0, u0, u1, gap, skip;
  int part;       // first row of its partial result (key head h: h * tile rows further), -1: it has all keys, and writes the output
  int pad[2];
  // rows in the cache, of key head 0, that the block loads first, so that no list has to be read before: of wave w the 16-key groups of its first
  // step, [2 * w], [2 * w + 1] (streaming kernel), or its group of step u0, [w] (tile kernel)
  uint32_t place[8];
};
// Up to 16 rows whose keys are shared out to `parts` items: partial rows at `part`, `stride` rows from part to part, `tile` from key head to
// key head.
struct PagedMerge {
  PagedSeq s;
  int row0, part, stride, parts, tile, pad[3];
};

// 128 positions of a sequence for the weights' tile kernel, those with the most rows of queries to go through first.
struct PagedKeys {
  int seq, key0;
};
constexpr int kWeighKeys = 128;

struct PagedView {     // device memory of a plan, and the shape
  const PagedSeq* seqs;
  const int* pages;
  const uint32_t* places;      // [T] row of a new token in the cache, key head 0
  float *pm, *po;              // partial results: (max, sum) of a row, its [head_dim]
  int n_seq, tokens, longest;
  int n_head, n_kv, group, d, page_size;
  Divisor by_group, by_page;
  int window, sinks;
  float scale;
};

hipError_t paged_append(int dtype, const PagedView& v, const void* k, int64_t ks, const void* vv, int64_t vs, void* kc, void* vc, hipStream_t st);
// most_parts, most_rows: of any entry of merges
hipError_t paged_attention(int dtype, const PagedView& v, const PagedItem* rows, int n_rows, const PagedItem* tiles, int n_tiles, const PagedMerge* merges, int n_merges,
                           int most_parts, int most_rows, const void* q, int64_t qs, const void* kc, const void* vc, void* out, float* lse, hipStream_t st);
// few: whether there are sequences of the streaming kernel (those without new tokens among them); many: the tile kernel's work; few_blocks, split:
// whether it has few blocks
hipError_t paged_weights(int dtype, const PagedView& v, const void* q, int64_t qs, const void* kc, const float* lse, float decay, float* w,
                         int64_t ws, bool few, bool few_blocks, const PagedKeys* many, int n_many, bool split, hipStream_t st);
hipError_t paged_evict(int dtype, const PagedView& v, void* kc, void* vc, const float* w, int64_t ws, int budget, int first, int recent,
                       float* wo, int64_t os, int* kept, hipStream_t st);

}  // namespace flk
