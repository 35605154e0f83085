// Attention over packed sequences: declarations and the pieces its passes share.
//
// Sequences lie one behind another in [rows, heads, D] tensors; cu[s] is sequence s's first row.  Query i of a
// sequence (nq queries, nk keys) sees the keys j <= i + nk - nq, so the last query sees all of them:
//   x_ij = scale q_i.k_j,  p_ij = exp(x_ij - lse_i),  lse_i = log sum_j exp(x_ij),  o_i = sum_j p_ij v_j
// and with the output's gradient g_i, delta_i = g_i.o_i (= sum_j p_ij g_i.v_j):
//   t_ij = p_ij (g_i.v_j - delta_i),  dq_i = scale sum_j t_ij k_j,  dk_j = scale sum_i t_ij q_i,  dv_j = sum_i p_ij g_i
// where dk and dv of a key head sum over the H / Hkv query heads that share it.
//
// All three passes keep 32 rows a wave resident (queries, or keys in the pass that gives dk and dv) and stream the
// others through LDS, tile by tile, loaded straight into it ahead of their use.  The products are taken with the
// streamed rows as the A operand's, so a lane holds one resident row and 16 streamed rows of each 32x32 score tile, and
// the weights feed the next product from their registers (mfma.hpp has the layouts).
#pragma once

#include <type_traits>

#include "common.hpp"
#include "mfma.hpp"

namespace gformer {

struct PackedArgs {
  const void *q, *k, *v, *dout;   // dout: backward pass only
  void *out, *dq, *dk, *dv;       // out: written by the forward pass, read by the backward pass
  void* rest;                     // what rounding took from out, in bf16 and laid out like it; may be null
  float* lse;                     // [H, total_q], natural logarithm; may be null in the forward pass
  float* stats;                   // [2, H, total_q], workspace of the backward pass: lse in base 2, and -delta
  float* sums;                    // [groups, 2, total_k, Hkv, d]: dk and dv of every part of the heads
  const int32_t *cu_q, *cu_k;     // [n_seqs + 1]
  int n_seqs, total_q, total_k, H, Hkv, d;
  int zero_tail;                  // rows behind the last sequence are set to zero
  float scale;
  int64_t qs[2], ks[2], vs[2], os[2];        // (row, head) strides
  int64_t gs[2], dqs[2], dks[2], dvs[2];     // of dout, dq, dk, dv
};
hipError_t launch_packed_fwd(const PackedArgs& a, bool bf16, hipStream_t s);
hipError_t launch_packed_bwd(const PackedArgs& a, bool bf16, hipStream_t s);
// What the backward pass keeps beside a query's statistics: the query heads of a key head in `groups` parts, whose dk and dv
// are added up by a kernel of their own (1: there is none).
int packed_head_groups(int total_k, int H, int Hkv);
// The streams of the passes that hold queries (packed_fwd.hip has the figures).
int packed_streams(bool fp32, int d, int total_q, int H, int n_seqs);
// Whether the launches of the passes that hold queries, and of the pass that holds keys, are within what one may have.
bool packed_queries_fit(bool fp32, int d, int total_q, int H, int n_seqs);
bool packed_keys_fit(bool fp32, int d, int total_k, int H, int Hkv, int n_seqs);
inline size_t packed_stats_bytes(int total_q, int H) { return ((size_t)total_q * H * 2 * sizeof(float) + 255) / 256 * 256; }
inline size_t packed_sums_bytes(int total_k, int H, int Hkv, int d) {
  const int groups = packed_head_groups(total_k, H, Hkv);
  return groups == 1 ? 0 : (size_t)groups * total_k * Hkv * d * 2 * sizeof(float);
}

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kPackedRows = 128;   // resident rows of a workgroup, where the streamed ones are not split over its waves
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// How a workgroup's waves share its work: RW of them side by side, 32 resident rows each, and S such sets ("streams") that
// take the streamed tiles in turn and join their sums at the end.  R streamed rows a tile, BUF tiles of a stream in LDS
// (one in use, the others on their way); registers are kept down for PER_SIMD waves on a SIMD.
template <int RW_, int S_, int R_, int BUF_, int PER_SIMD_> struct Shape {
  static constexpr int RW = RW_, S = S_, R = R_, BUF = BUF_, PER_SIMD = PER_SIMD_, ROWS = 32 * RW, THREADS = 64 * RW * S;
};
// Of a workgroup that holds queries, by its streams.
constexpr int kQueryThreads = 256;
constexpr int query_rows(int streams) { return kPackedRows / streams; }
// Tiles of R rows over all sequences, none straddling two: sequence s owns tiles cu[s] / R + s up to the next
// one's.  That is at least as many as it needs (floor(b / R) + 1 - floor(a / R) >= ceil((b - a) / R)), takes no
// prefix sum and no look at the offsets on the host; the few tiles too many end at once.  The rows behind the last sequence
// count as sequence n_seqs.
inline int64_t packed_tiles(int total, int n_seqs, int rows) { return (int64_t)total / rows + n_seqs + 1; }

struct SeqTile {
  int seq;     // n_seqs: the rows behind the last sequence
  int first;   // the tile's first row inside the sequence; negative or past the end: nothing to do
};
__device__ __forceinline__ int packed_row(const int32_t* cu, int s, int total) { return min(max(cu[s], 0), total); }

// The sequence that owns `tile`: the last s with cu[s] / R + s <= tile, by 64 probes at a time.
template <int R> __device__ __forceinline__ SeqTile find_tile(const int32_t* cu, int n_seqs, int total, int tile, int lane) {
  int lo = 0, hi = n_seqs + 1;
  do {
    const int step = (hi - lo + 63) / 64;
    const int s = lo + lane * step;
    const bool in = s < hi && packed_row(cu, min(s, n_seqs), total) / R + s <= tile;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(in));
    if (n == 0) return {n_seqs, -1};   // in front of the first sequence
    lo = __builtin_amdgcn_readfirstlane(lo + (n - 1) * step);
    hi = __builtin_amdgcn_readfirstlane(min(hi, lo + step));
  } while (hi - lo > 1);
  return {lo, (tile - lo - packed_row(cu, lo, total) / R) * R};
}

// The same with the longest work first, which evens out the end of a launch: a tile's level is how many tiles of R keys its
// queries see (FIRST_IS_LONG: how many tiles of the sequence lie behind it, for keys, which the later queries see), and tile
// number `rank` is taken in order of falling levels.  The sequences' tiles are counted for 64 levels at a time, in as many
// steps as there are sequences; with more than kRanked the order is the tensors'.  One long sequence among short ones does not tell the
// two apart: 8192 rows, 32 / 8 heads, d = 128 beside 31 of 10 rows 572 us (backward 2407), beside 32 553 in front of them and 560 behind
// (2389, 2370).
constexpr int kRanked = 32;
template <int R, bool FIRST_IS_LONG>
__device__ __forceinline__ SeqTile ranked_tile(const int32_t* cu, int total, const int32_t* cu_seen, int total_seen, int n_seqs, int rank,
                                               int tiles, int lane) {
  if (n_seqs > kRanked) return find_tile<R>(cu, n_seqs, total, FIRST_IS_LONG ? rank : tiles - 1 - rank, lane);
  const int s = min(lane, n_seqs - 1);
  int nt = 0, from = 0;   // this lane's sequence: its tiles, and the first one's level
  if (lane < n_seqs) {
    const int len = max(packed_row(cu, s + 1, total) - packed_row(cu, s, total), 0);
    nt = (len + R - 1) / R;
    if (!FIRST_IS_LONG) from = max(packed_row(cu_seen, s + 1, total_seen) - packed_row(cu_seen, s, total_seen) - len, 0) / R;
  }
  int lo = 0, hi = 1;
  for (int i = 0; i < n_seqs; ++i) hi = max(hi, __builtin_amdgcn_readlane(nt, i) + __builtin_amdgcn_readlane(from, i));
  // tiles of level l and above
  auto above = [&](int l) {
    int n = 0;
    for (int i = 0; i < n_seqs; ++i) {
      const int x = __builtin_amdgcn_readlane(nt, i);
      n += min(max(x + __builtin_amdgcn_readlane(from, i) - l, 0), x);
    }
    return n;
  };
  do {
    const int step = (hi - lo + 63) / 64, l = lo + lane * step;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(l < hi && above(l) > rank));
    if (n == 0) {   // lane 0 knows all tiles: what is left are the rows behind the last sequence
      const int all = __builtin_amdgcn_readfirstlane(above(0));
      return {n_seqs, (rank - all) * R};
    }
    lo = __builtin_amdgcn_readfirstlane(lo + (n - 1) * step);
    hi = __builtin_amdgcn_readfirstlane(min(hi, lo + step));
  } while (hi - lo > 1);
  uint64_t at = __builtin_amdgcn_ballot_w64(from <= lo && lo < nt + from);   // the sequences with a tile of this level
  for (int i = rank - __builtin_amdgcn_readfirstlane(above(lo + 1)); i > 0; --i) at &= at - 1;
  const int seq = __builtin_ctzll(at);
  const int tile = FIRST_IS_LONG ? __builtin_amdgcn_readlane(nt, seq) - 1 - lo : lo - __builtin_amdgcn_readlane(from, seq);
  return {seq, tile * R};
}

// What scores are multiplied by for base-2 exponents, without the scale's sign.  Not let down to zero, where a masked score (-infinity)
// would lose its weight of zero: the smallest number in its place changes no exponent by more than 5e-7.
__device__ __forceinline__ float base2_scale(float scale) { return fmaxf(fabsf(scale) * kLog2e, 0x1p-149f); }

// Offsets of a pointer of either element type.
template <typename T> __device__ __forceinline__ const T* rows_of(const void* p, const int64_t (&st)[2], int64_t row, int head) {
  return reinterpret_cast<const T*>(p) + row * st[0] + head * st[1];
}
template <typename T> __device__ __forceinline__ T* rows_of(void* p, const int64_t (&st)[2], int64_t row, int head) {
  return reinterpret_cast<T*>(p) + row * st[0] + head * st[1];
}

// The largest of three (v_maximum3_f32), or no number.  Left to the compiler, which knows how long after a matrix
// instruction its result may be read: an asm statement would hide the reader from it.
__device__ __forceinline__ float maximum3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// A tile of R streamed rows in LDS: rows one behind another with no padding, as a load into LDS writes them (64 lanes, 16
// bytes each, in lane order), the 16-byte pieces of row r at places that differ by swz(r).  swz moves bits of r about, so
// swz(a ^ b) = swz(a) ^ swz(b), and keeps both ways of reading off each other's banks (256 bytes a cycle):
//   rows, 16 bytes a lane    lanes 0-3, 12-15, 20-23, 24-27 go together, then the others of the half: 16 different pieces
//   transposed, bf16         a half's lanes: two neighbouring pairs of pieces in each of 4 rows, which the low bits of r set apart
//   transposed, fp32         8 pieces of a row and of the one 4 further on, which bit 2 of r sets apart
template <typename T, int D> constexpr size_t kTileAlign = D * sizeof(T);   // a row's bytes (lds_lane())
constexpr size_t kLdsAlign = 512;                                           // the longest row's
template <typename T, int D, int R> struct Tile {
  static constexpr int E = 16 / (int)sizeof(T), C = D / E;   // elements a piece, pieces a row
  static constexpr int RPI = 64 / C;                          // rows an instruction loads
  static constexpr int SIZE = R * D;
  __host__ __device__ static constexpr int swz(int r) {
    if (sizeof(T) == 4) return ((r & 7) << 1) | ((r >> 3) & 1);
    return (C == 8 ? ((r >> 1) & 1) << 2 : (r & 3) << 2) | ((r >> 2) & 3);
  }
  static constexpr int loads(int waves) { return R / (RPI * waves); }
  // Rows r0 .. r0 + R - 1 of [rows, D] at `base`, by W waves; those past `last` are row `last`: in bounds, and masked later.
  // A uniform base and an offset of the lane's own; a tile's rows lie within 2^28 bytes (a row stride is at most 2^20 elements).
  template <int W> static __device__ __forceinline__ void load(T* tile, const T* base, int64_t stride, int r0, int last, int wave, int lane) {
    static_assert(loads(W) * RPI * W == R, "whole rows");
    const uint32_t bytes = (uint32_t)stride * (int)sizeof(T);
    const int row = RPI * wave + lane / C, left = min(last - r0, R - 1);
    const uint32_t piece = (lane % C) ^ swz(row);
    const char* from = reinterpret_cast<const char*>(base + r0 * stride);
#pragma unroll
    for (int j = 0; j < loads(W); ++j) {
      const int first = min(RPI * W * j, left);   // uniform
      const uint32_t off = (uint32_t)min(row, left - first) * bytes + 16 * (piece ^ swz(RPI * W * j));
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + (size_t)first * bytes + off),
                                       (__attribute__((address_space(3))) void*)(tile + (wave + W * j) * 64 * E), 16, 0, 0);
    }
  }
  // Whether 32 rows hold a value that is infinite or no number; the answer is the wave's.
  static __device__ __forceinline__ bool odd(const T* rows, int lane) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 32 * C / 64; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(rows + (64 * i + lane) * E);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) r |= ((x[j] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
        else r |= ((x[j] & 0x7fffffffu) + 0x00800000u) & 0x80000000u;
      }
    }
    return __builtin_amdgcn_ballot_w64(r != 0) != 0;
  }
};

// Whether any wave of the workgroup says so (all have passed a barrier since `flag`'s place was last in use).
__device__ __forceinline__ bool any_wave(int* flag, bool x) {
  if (threadIdx.x == 0) *flag = 0;
  lds_barrier();
  if (x) *flag = 1;
  lds_barrier();
  x = *flag != 0;
  lds_barrier();   // the flag's place may be written again
  return x;
}

// Every load of this wave has arrived but the latest N (loads return in order).
template <int N> __device__ __forceinline__ void loads_left() {
  static_assert(N < 64);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A wave is done reading a tile that it alone uses: what it loads into it next comes behind.
__device__ __forceinline__ void tile_read() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// LDS by its byte addresses.  A tile starts at a multiple of a row's bytes (kTileAlign), so the pieces of a row (and of the rows
// 16 further on) differ from a lane's first one by an exclusive or: one instruction a read, where addresses kept ready would take
// the registers of the sums.  lds_lane() keeps the compiler from doing that.
__device__ __forceinline__ uint32_t lds_lane(const void* tile, int bytes) {
  uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)tile + bytes;
  asm volatile("" : "+v"(at));
  return at;
}
template <typename V> __device__ __forceinline__ V lds_get(uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>(at);
}
// Transposed reads (mfma.hpp) at x and y, the latter OFF bytes further on, 64 bytes apart by exclusive or for the tiles of sums.
// One statement that also waits for them: the compiler takes the builtin for a read of what the loads into LDS still write,
// and would wait for those, tiles ahead, each time.
template <int N, int X, int OFF> __device__ __forceinline__ void lds_get_turned(bf16x8 (&to)[N], uint32_t at, uint32_t other) {
  u32x2 x[N], y[N];
  if constexpr (N == 4)
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %4, %12 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %1, %9 offset:%16\n\tds_read_b64_tr_b16 %5, %13 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %2, %10 offset:%16\n\tds_read_b64_tr_b16 %6, %14 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %3, %11 offset:%16\n\tds_read_b64_tr_b16 %7, %15 offset:%17\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
                 : "v"(at), "v"(at ^ 64), "v"(at ^ 128), "v"(at ^ 192), "v"(other), "v"(other ^ 64), "v"(other ^ 128), "v"(other ^ 192),
                   "n"(X), "n"(X + OFF)
                 : "memory");
  else
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %2, %6 offset:%9\n\t"
                 "ds_read_b64_tr_b16 %1, %5 offset:%8\n\tds_read_b64_tr_b16 %3, %7 offset:%9\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(y[0]), "=&v"(y[1])
                 : "v"(at), "v"(at ^ 64), "v"(other), "v"(other ^ 64), "n"(X), "n"(X + OFF)
                 : "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) to[i] = as_bf16x8(u32x4{x[i][0], x[i][1], y[i][0], y[i][1]});
}

// The matrix products of one wave, for 32 resident and 32 streamed rows.
template <typename T, int D> struct Products;
constexpr f32x16 kZeroTile = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

template <int D> struct Products<uint16_t, D> {
  using T = uint16_t;
  using L = Tile<T, D, 32>;
  struct Resident { bf16x8 x[D / 16]; };
  struct Weights { bf16x8 x[2]; };
  // this lane's resident row: elements 16 ks + 8 lh .. +7; `flip` changes its sign
  static __device__ __forceinline__ void load(Resident& r, const T* row, int lane, bool flip) {
    const uint32_t sign = flip ? 0x80008000u : 0u;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      u32x4 x = *reinterpret_cast<const u32x4*>(row + 16 * ks + 8 * (lane >> 5));
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] ^= sign;
      r.x[ks] = as_bf16x8(x);
    }
  }
  static __device__ __forceinline__ float dot(const Resident& a, const Resident& b) {
    float s = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const u32x4 x = as_u32x4(a.x[ks]), y = as_u32x4(b.x[ks]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s = fmaf(bf16_lo(x[i]), bf16_lo(y[i]), fmaf(bf16_hi(x[i]), bf16_hi(y[i]), s));
    }
    return sum_over_halves(s);
  }
  // where a lane reads, in bytes: row l % 32, piece 2 ks + lh; and of the transposed reads, piece 4 mt + l / 16 % 2 * 2 + l / 2 % 2
  // of row 4 lh + l / 4 % 4
  static __device__ __forceinline__ int row_at(int lane) { return 2 * ((lane & 31) * D + 8 * ((lane >> 5) ^ L::swz(lane & 31))); }
  static __device__ __forceinline__ int turned_at(int lane) {
    const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), piece = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    return 2 * (row * D + 8 * (piece ^ L::swz(row)) + 4 * (lane & 1));
  }
  template <int KB> static __device__ __forceinline__ void turned(bf16x8 (&x)[D / 32], uint32_t at) {
    lds_get_turned<D / 32, 32 * KB * D, 16 * D>(x, at, at ^ (16 * L::swz(8)));
  }
  static __device__ __forceinline__ bf16x8 piece(uint32_t at, int ks) { return as_bf16x8(lds_get<u32x4>(at ^ (32 * ks))); }
  // 32 streamed rows against the resident ones, added to s
  static __device__ __forceinline__ f32x16 scores(const T* rows, const Resident& r, int lane, f32x16 s = kZeroTile) {
    const uint32_t at = lds_lane(rows, row_at(lane));
    // all reads first: left alone, the compiler has each product wait for its own
    bf16x8 x[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) x[ks] = piece(at, ks);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = mfma32(x[ks], r.x[ks], s);
    return s;
  }
  // the same with the resident rows in a tile of LDS too
  static __device__ __forceinline__ f32x16 scores_lds(const T* rows, const T* own, int lane, f32x16 s) {
    const uint32_t at = lds_lane(rows, row_at(lane)), own_at = lds_lane(own, row_at(lane));
#pragma unroll
    for (int k0 = 0; k0 < D / 16; k0 += 2) {
      bf16x8 x[2], y[2];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        x[ks] = piece(at, k0 + ks);
        y[ks] = piece(own_at, k0 + ks);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) s = mfma32(x[ks], y[ks], s);
    }
    return s;
  }
  static __device__ __forceinline__ void to_lds(const Resident& r, T* own, int lane) {
    const int at = row_at(lane) / 2;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) *reinterpret_cast<u32x4*>(own + (at ^ (16 * ks))) = as_u32x4(r.x[ks]);
  }
  static __device__ __forceinline__ Weights weights(const float (&p)[16]) {
    Weights w;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      u32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = pack_bf16(p[8 * kb + 2 * i], p[8 * kb + 2 * i + 1]);
      w.x[kb] = as_bf16x8(x);
    }
    return w;
  }
  // what rounding took from them
  static __device__ __forceinline__ Weights rests(const float (&p)[16], const Weights& w) {
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t y = as_u32x4(w.x[i / 8])[i % 8 / 2];
      x[i] = p[i] - (i % 2 ? bf16_hi(y) : bf16_lo(y));
    }
    return weights(x);
  }
  // acc += rows^T weights
  static __device__ __forceinline__ void product(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int lane) {
    const uint32_t at = lds_lane(rows, turned_at(lane));
    bf16x8 x[D / 32];
    turned<0>(x, at);
#pragma unroll
    for (int mt = 0; mt < D / 32; ++mt) acc[mt] = mfma32(x[mt], w.x[0], acc[mt]);
    turned<1>(x, at);
#pragma unroll
    for (int mt = 0; mt < D / 32; ++mt) acc[mt] = mfma32(x[mt], w.x[1], acc[mt]);
  }
  // The same row by row, for tiles that hold values which are not finite: zero times such a value is no number, so a row is
  // left out of a lane's sums, not weighted with zero, where first <= row < end does not hold.  The kernels look for such
  // values in the tiles that some of a wave's rows see in part, and where they find one take the whole workgroup's sums again
  // in a second loop that has this: in the first one it would cost registers.
  static __device__ __forceinline__ void product_by_rows(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int first, int end,
                                                         int lane) {
    const uint32_t at = lds_lane(rows, turned_at(lane));
    auto half = [&](auto kb) {
      constexpr int KB = decltype(kb)::value;
      bf16x8 x[D / 32];
      turned<KB>(x, at);
#pragma unroll 1
      for (int e = 0; e < 16; ++e) {                      // row 16 KB + e: half e / 4 % 2, slot 4 (e / 8) + e % 4
        const int slot = 4 * (e / 8) + e % 4, row = 16 * KB + e;
        const bool mine = (lane >> 5) == ((e / 4) & 1);
        u32x4 keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = mine && slot / 2 == i ? (slot & 1 ? 0xffff0000u : 0x0000ffffu) : 0u;
#pragma unroll
        for (int mt = 0; mt < D / 32; ++mt) {
          const f32x16 with = mfma32(as_bf16x8(as_u32x4(x[mt]) & keep), as_bf16x8(as_u32x4(w.x[KB]) & keep), acc[mt]);
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[mt][r] = row >= first && row < end ? with[r] : acc[mt][r];
        }
      }
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 1>{});
  }
  static __device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
    u32x2 x;
    x[0] = pack_bf16(a, b);
    x[1] = pack_bf16(c, d);
    *reinterpret_cast<u32x2*>(p) = x;
  }
  static __device__ __forceinline__ float rest(float x) { return x - bf16_lo(pack_bf16(x, 0.f)); }   // what rounding takes
};

// Single precision, on v_mfma_f32_32x32x2_f32: a k-step has one slot for each half of the wave.  A contraction along
// rows takes elements 8 s + 4 lh + j (j = 0..3) in four steps; one over the 32 streamed rows takes the rows that
// register r of both halves stands for, 8 (r / 4) + 4 lh + r % 4.
template <int D> struct Products<float, D> {
  using T = float;
  using L = Tile<T, D, 32>;
  struct Resident { f32x4_t x[D / 8]; };
  struct Weights { float x[16]; };
  static __device__ __forceinline__ f32x16 mfma(float a, float b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ void load(Resident& r, const T* row, int lane, bool flip) {
    const float sign = flip ? -1.f : 1.f;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) r.x[s] = *reinterpret_cast<const f32x4_t*>(row + 8 * s + 4 * (lane >> 5)) * sign;
  }
  static __device__ __forceinline__ float dot(const Resident& a, const Resident& b) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = fmaf(a.x[i][j], b.x[i][j], s);
    return sum_over_halves(s);
  }
  static __device__ __forceinline__ f32x16 scores(const T* rows, const Resident& r, int lane, f32x16 s = kZeroTile) {
    const uint32_t at = lds_lane(rows, 4 * ((lane & 31) * D + 4 * ((lane >> 5) ^ L::swz(lane & 31))));
#pragma unroll
    for (int i0 = 0; i0 < D / 8; i0 += 4) {
      f32x4_t a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = lds_get<f32x4_t>(at ^ (32 * (i0 + i)));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s = mfma(a[i][j], r.x[i0 + i][j], s);
    }
    return s;
  }
  static __device__ __forceinline__ Weights weights(const float (&p)[16]) {
    Weights w;
#pragma unroll
    for (int i = 0; i < 16; ++i) w.x[i] = p[i];
    return w;
  }
  // column 32 mt + l % 32 of row 8 (r / 4) + 4 lh + r % 4
  static __device__ __forceinline__ int turned_at(int lane) {
    return 4 * (4 * (lane >> 5) * D + 4 * (((lane & 31) >> 2) ^ L::swz(4 * (lane >> 5))) + (lane & 3));
  }
  static __device__ __forceinline__ float turned(uint32_t at, int r, int mt) {
    const int row = 8 * (r / 4) + r % 4;
    return lds_get<float>((at ^ (128 * mt) ^ (16 * L::swz(row))) + 4 * row * D);
  }
  static __device__ __forceinline__ void product(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int lane) {
    const uint32_t at = lds_lane(rows, turned_at(lane));
    // some reads ahead of their products; all at once would take the registers of the sums
    constexpr int AHEAD = 4;
#pragma unroll
    for (int r0 = 0; r0 < 16; r0 += AHEAD) {
      float x[AHEAD][D / 32];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r)
#pragma unroll
        for (int mt = 0; mt < D / 32; ++mt) x[r][mt] = turned(at, r0 + r, mt);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < AHEAD; ++r)
#pragma unroll
        for (int mt = 0; mt < D / 32; ++mt) acc[mt] = mfma(x[r][mt], w.x[r0 + r], acc[mt]);
    }
  }
  static __device__ __forceinline__ void product_by_rows(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int first, int end,
                                                         int lane) {
    const uint32_t at = lds_lane(rows, turned_at(lane));
#pragma unroll
    for (int mt = 0; mt < D / 32; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r)
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const int row = 8 * (r / 4) + 4 * half + r % 4;
          const bool mine = (lane >> 5) == half;
          const f32x16 with = mfma(mine ? turned(at, r, mt) : 0.f, mine ? w.x[r] : 0.f, acc[mt]);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[mt][i] = row >= first && row < end ? with[i] : acc[mt][i];
        }
  }
  static __device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{a, b, c, d};
  }
  static __device__ __forceinline__ float rest(float) { return 0.f; }
};

// A wave's 32 resident rows of sums (lane: one row; register (mt, 4 g + i): column 32 mt + 8 g + 4 lh + i) times `by`,
// through kPutRow 32 elements of LDS that are its own, to whole rows in memory.  REST: what rounding takes from them instead.
template <typename T, int D> constexpr int kPutRow = D + 16 / (int)sizeof(T);
template <typename T, int D, bool REST = false>
__device__ __forceinline__ void put_rows(const f32x16 (&acc)[D / 32], float by, T* own, T* to, int64_t stride, int rows, int lane) {
  using P = Products<T, D>;
  T* p = own + (lane & 31) * kPutRow<T, D> + 4 * (lane >> 5);
  auto value = [&](int mt, int r) { return REST ? P::rest(acc[mt][r] * by) : acc[mt][r] * by; };
#pragma unroll
  for (int mt = 0; mt < D / 32; ++mt)
#pragma unroll
    for (int g = 0; g < 4; ++g) P::put4(p + 32 * mt + 8 * g, value(mt, 4 * g), value(mt, 4 * g + 1), value(mt, 4 * g + 2), value(mt, 4 * g + 3));
  wave_sync();
  constexpr int C = D * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 32 * C / 64; ++i) {
    const int row = lane / C + i * (64 / C);
    if (row < rows)
      *reinterpret_cast<u32x4*>(to + row * stride + E * (lane % C)) = *reinterpret_cast<const u32x4*>(own + row * kPutRow<T, D> + E * (lane % C));
  }
  wave_sync();
}

// Zeros in rows [0, rows) of a workgroup's tile.
template <typename T, int D> __device__ __forceinline__ void zero_rows(T* to, int64_t stride, int rows, int tid, int threads) {
  constexpr int C = D * (int)sizeof(T) / 16;
  for (int r = tid / C; r < rows; r += threads / C)
    *reinterpret_cast<u32x4*>(to + r * stride + (16 / (int)sizeof(T)) * (tid % C)) = u32x4{0, 0, 0, 0};
}

}  // namespace
}  // namespace gformer
