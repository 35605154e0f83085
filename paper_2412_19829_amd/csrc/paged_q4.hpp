// The paged cache in 4 bits a value.  A row, one token of one head, is d / 2 bytes of codes, channel c in bits 4 (c % 2) .. of byte c / 2,
// and behind them a scale s and a lowest value l, both bf16, for each 32 channels: code n stands for l + s n.  Pages are
// those of paged.hpp; their strides are in bytes.
//
// Of 32 values x, l is the largest bf16 at or below their minimum and s the smallest with l + 15 s at or above their maximum, so that
// every value has a code, n the integer nearest to (x - l) / s (of two as near the even one), and no value is off by more than s / 2.
// A group with a value that is no number, or of magnitude 2^127 or more, has s and l that are none.
#pragma once

#include "paged.hpp"

namespace gformer {

constexpr int kQ4Group = 32;
constexpr int q4_row(int d) { return d / 2 + d / 8; }        // bytes
constexpr int q4_piece(int d) { return d / 8; }              // bytes: what rows are read in, and aligned to

struct PagedReadArgs {
  const void *kpages, *vpages;
  void *k, *v;                 // [total, Hkv, d], packed
  const int32_t *table, *start, *cu;
  int n_seqs, total, Hkv, d, n_pages, width, shift;
  int64_t ks[2], vs[2], kps[3], vps[3];
};

// Workgroups that share the sequences' tokens, for each set of heads: PagedDecodeArgs::splits (chunk is not used).  Where they are more than one
// and may cut a sequence, sums and stats hold parts + B rows, [parts + B, H, d] and [parts + B, H, 2]; else both are null.
int paged_q4_parts(bool bf16, int B, int H, int Hkv, int d, int64_t max_len);
bool paged_q4_cuts(int64_t max_len);
bool paged_q4_decode_fits(bool bf16, int B, int H, int Hkv, int d, int64_t max_len);
bool paged_q4_rows_fit(int total, int n_seqs, int Hkv, int d);
hipError_t launch_paged_q4_decode(const PagedDecodeArgs& a, bool bf16, hipStream_t s);
hipError_t launch_paged_q4_fill(const PagedFillArgs& a, bool bf16, hipStream_t s);
hipError_t launch_paged_q4_read(const PagedReadArgs& a, bool bf16, hipStream_t s);
hipError_t launch_pages_q4_copy(const PagesCopyArgs& a, hipStream_t s);

}  // namespace gformer
