// The paged key-value cache: keys and values of many sequences in pages of `1 << shift` tokens, placed anywhere;
// table[s][i] is the page with tokens i << shift .. of sequence s.  A page number outside [0, n_pages) is no page:
// its tokens are not seen and not written.
#pragma once

#include "common.hpp"

namespace gformer {

struct PagedDecodeArgs {
  const void *q, *k, *v;       // one token of every sequence; k, v: null where it is in the cache already
  void* out;
  void *kpages, *vpages;
  const int32_t *table, *lens; // [B, width], [B]
  float *sums, *stats;         // splits > 1: [B, H, splits, d] and [B, H, splits, 2] (maximum, sum)
  int B, H, Hkv, d, n_pages, width, shift;
  int room;                    // keys a sequence may have: the table's, or the bound the caller named
  int chunk, splits;           // keys per workgroup, workgroups along a sequence
  float scale;
  int64_t qs[2], ks[2], vs[2], os[2];   // (sequence, head) strides
  int64_t kps[3], vps[3];               // (page, head, token) strides
};
struct PagedFillArgs {
  const void *k, *v;           // [total, Hkv, d], packed
  void *kpages, *vpages;
  const int32_t *table, *start, *cu;
  int n_seqs, total, Hkv, d, n_pages, width, shift;
  int64_t ks[2], vs[2], kps[3], vps[3];
};
struct PagesCopyArgs {
  void *kpages, *vpages;
  const int32_t *src, *dst;
  int n_copies, Hkv, d, n_pages, page;
  int64_t kps[3], vps[3];
};
struct PagedSplit {
  int chunk, splits;
};
constexpr int kPagedHeads = 16;        // query heads of one key head that a workgroup takes
constexpr int kPagedThreads = 256;     // of a workgroup, in all of these kernels
PagedSplit paged_split(int B, int H, int Hkv, int64_t max_len);
// Whether the launches are within what one may have.
bool paged_decode_fits(int B, int H, int Hkv, PagedSplit s);
bool paged_fill_fits(int total, int n_seqs, int Hkv);
hipError_t launch_paged_decode(const PagedDecodeArgs& a, bool bf16, hipStream_t s);
hipError_t launch_paged_fill(const PagedFillArgs& a, bool bf16, hipStream_t s);
hipError_t launch_pages_copy(const PagesCopyArgs& a, bool bf16, hipStream_t s);

}  // namespace gformer
