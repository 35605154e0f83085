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
// others through LDS.  The products are taken with the streamed rows as the A operand's, so a lane holds one
// resident row and 16 streamed rows of each 32x32 score tile, and the weights feed the next product from their
// registers (mfma.hpp has the layouts).
#pragma once

#include <type_traits>

#include "common.hpp"
#include "mfma.hpp"

namespace gformer {

struct PackedArgs {
  const void *q, *k, *v, *dout;   // dout: backward pass only
  void *out, *dq, *dk, *dv;       // out: written by the forward pass, read by the backward pass
  float* lse;                     // [H, total_q], natural logarithm; may be null in the forward pass
  float* delta;                   // [H, total_q], workspace of the backward pass
  const int32_t *cu_q, *cu_k;     // [n_seqs + 1]
  int n_seqs, total_q, total_k, H, Hkv, d;
  int zero_tail;                  // rows behind the last sequence are set to zero
  float scale;
  int64_t qs[2], ks[2], vs[2], os[2];        // (row, head) strides
  int64_t gs[2], dqs[2], dks[2], dvs[2];     // of dout, dq, dk, dv
};
hipError_t launch_packed_fwd(const PackedArgs& a, bool bf16, hipStream_t s);
hipError_t launch_packed_bwd(const PackedArgs& a, bool bf16, hipStream_t s);

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kPackedThreads = 256;
constexpr int kPackedRows = kPackedThreads / 64 * 32;   // resident rows per workgroup
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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

// Offsets of a pointer of either element type.
template <typename T> __device__ __forceinline__ const T* rows_of(const void* p, const int64_t (&st)[2], int64_t row, int head) {
  return reinterpret_cast<const T*>(p) + row * st[0] + head * st[1];
}
template <typename T> __device__ __forceinline__ T* rows_of(void* p, const int64_t (&st)[2], int64_t row, int head) {
  return reinterpret_cast<T*>(p) + row * st[0] + head * st[1];
}

// Whether any of 16 bytes' elements is infinite or no number.
template <typename T> __device__ __forceinline__ uint32_t not_finite(u32x4 x) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) r |= ((x[i] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
    else r |= ((x[i] & 0x7fffffffu) + 0x00800000u) & 0x80000000u;
  }
  return r;
}

// A tile of R streamed rows on its way from memory to LDS, 16 bytes a lane: a uniform base and an offset of the thread's
// own that never changes, so a load costs no address registers.  Rows past `last` re-read it: in bounds, and masked
// later.
template <typename T, int D, int R> struct Stage {
  static constexpr int C = D * (int)sizeof(T) / 16, STEP = kPackedThreads / C, N = R / STEP;
  static_assert(N * STEP == R, "whole rows");
  u32x4 x[N];
  // rows r0 .. r0 + R - 1; r0 <= last.  A tile's rows lie within 2^28 bytes (the row stride is at most 2^20 elements)
  __device__ __forceinline__ void load(const T* base, int64_t stride, int r0, int last, int tid) {
    const uint32_t bytes = (uint32_t)stride * sizeof(T), col = 16 * (tid % C), off = tid / C * bytes + col;
    const char* from = reinterpret_cast<const char*>(base + r0 * stride);
    const int left = min(last - r0, R - 1);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int first = min(i * STEP, left);   // uniform
      x[i] = *reinterpret_cast<const u32x4*>(from + (size_t)first * bytes + (size_t)min(off, (left - first) * bytes + col));
    }
  }
  template <int ROW> __device__ __forceinline__ void store(T* tile, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      *reinterpret_cast<u32x4*>(tile + (tid / C + i * STEP) * ROW + (16 / (int)sizeof(T)) * (tid % C)) = x[i];
  }
  __device__ __forceinline__ bool odd() const {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) r |= not_finite<T>(x[i]);
    return r != 0;
  }
};

// The largest of three (v_maximum3_f32), or no number.  Left to the compiler, which knows how long after a matrix
// instruction its result may be read: an asm statement would hide the reader from it.
__device__ __forceinline__ float maximum3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The matrix products of one wave, for 32 resident and 32 streamed rows.
template <typename T, int D> struct Products;

template <int D> struct Products<uint16_t, D> {
  using T = uint16_t;
  static constexpr int R = 64;                               // streamed rows per tile
  // row strides in LDS of tiles read by rows, transposed, and both ways (mfma.hpp): 4, 16 and 12 dwords mod 64 at d = 128,
  // 36, 48 and 36 at d = 64
  static constexpr int BY_ROWS = D + 8, TURNED = D + 32, BOTH = D == 128 ? D + 24 : D + 8;
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
  // 32 streamed rows from `rows` against the resident ones
  template <int ROW> static __device__ __forceinline__ f32x16 scores(const T* rows, const Resident& r, int lane) {
    const T* p = rows + (lane & 31) * ROW + 8 * (lane >> 5);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = mfma32(lds_read16(p + 16 * ks), r.x[ks], s);
    return s;
  }
  // the same with the resident rows in LDS too, at `own`
  template <int ROW> static __device__ __forceinline__ f32x16 scores_lds(const T* rows, const T* own, int lane) {
    const int at = (lane & 31) * ROW + 8 * (lane >> 5), own_at = (lane & 31) * BY_ROWS + 8 * (lane >> 5);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = mfma32(lds_read16(rows + at + 16 * ks), lds_read16(own + own_at + 16 * ks), s);
    return s;
  }
  static __device__ __forceinline__ void to_lds(const Resident& r, T* own, int lane) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      *reinterpret_cast<u32x4*>(own + (lane & 31) * BY_ROWS + 8 * (lane >> 5) + 16 * ks) = as_u32x4(r.x[ks]);
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
  // acc += rows^T weights
  template <int ROW> static __device__ __forceinline__ void product(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int lane) {
    const T* p = rows + 4 * (lane >> 5) * ROW + lds_operand_tr_lane_offset(ROW, lane);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int mt = 0; mt < D / 32; ++mt)
        acc[mt] = mfma32(lds_operand_tr_at(p, ROW, 16 * kb, 16 * kb + 8, 32 * mt), w.x[kb], acc[mt]);
  }
  // The same row by row, for tiles that hold values which are not finite: zero times such a value is no number, so a row is
  // left out of a lane's sums, not weighted with zero, where first <= row < end does not hold.
  template <int ROW>
  static __device__ __forceinline__ void product_by_rows(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int first, int end,
                                                         int lane) {
    const T* p = rows + 4 * (lane >> 5) * ROW + lds_operand_tr_lane_offset(ROW, lane);
#pragma unroll
    for (int mt = 0; mt < D / 32; ++mt)                   // one tile of sums at a time: this is rare, and must not cost registers
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll 1
        for (int e = 0; e < 16; ++e) {                    // row 16 kb + e: half e / 4 % 2, slot 4 (e / 8) + e % 4
          const int slot = 4 * (e / 8) + e % 4, row = 16 * kb + e;
          const bool mine = (lane >> 5) == ((e / 4) & 1);
          u32x4 keep;
#pragma unroll
          for (int i = 0; i < 4; ++i) keep[i] = mine && slot / 2 == i ? (slot & 1 ? 0xffff0000u : 0x0000ffffu) : 0u;
          const bf16x8 a = as_bf16x8(as_u32x4(lds_operand_tr_at(p, ROW, 16 * kb, 16 * kb + 8, 32 * mt)) & keep);
          const f32x16 with = mfma32(a, as_bf16x8(as_u32x4(w.x[kb]) & keep), acc[mt]);
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[mt][r] = row >= first && row < end ? with[r] : acc[mt][r];
        }
  }
  static __device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
    u32x2 x;
    x[0] = pack_bf16(a, b);
    x[1] = pack_bf16(c, d);
    *reinterpret_cast<u32x2*>(p) = x;
  }
};

// Single precision, on v_mfma_f32_32x32x2_f32: a k-step has one slot for each half of the wave.  A contraction along
// rows takes elements 8 s + 4 lh + j (j = 0..3) in four steps; one over the 32 streamed rows takes the rows that
// register r of both halves stands for, 8 (r / 4) + 4 lh + r % 4.
template <int D> struct Products<float, D> {
  using T = float;
  static constexpr int R = 32;
  static constexpr int BY_ROWS = D + 4, TURNED = D + 4, BOTH = D + 4;   // 4 dwords mod 64: 16-byte row reads without conflicts
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
  template <int ROW> static __device__ __forceinline__ f32x16 scores(const T* rows, const Resident& r, int lane) {
    const T* p = rows + (lane & 31) * ROW + 4 * (lane >> 5);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p + 8 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = mfma(a[j], r.x[i][j], s);
    }
    return s;
  }
  static __device__ __forceinline__ Weights weights(const float (&p)[16]) {
    Weights w;
#pragma unroll
    for (int i = 0; i < 16; ++i) w.x[i] = p[i];
    return w;
  }
  template <int ROW> static __device__ __forceinline__ void product(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int lane) {
    const T* p = rows + 4 * (lane >> 5) * ROW + (lane & 31);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int mt = 0; mt < D / 32; ++mt) acc[mt] = mfma(p[(8 * (r / 4) + r % 4) * ROW + 32 * mt], w.x[r], acc[mt]);
  }
  template <int ROW>
  static __device__ __forceinline__ void product_by_rows(f32x16 (&acc)[D / 32], const T* rows, const Weights& w, int first, int end,
                                                         int lane) {
    const T* p = rows + 4 * (lane >> 5) * ROW + (lane & 31);
#pragma unroll
    for (int mt = 0; mt < D / 32; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r)
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const int row = 8 * (r / 4) + 4 * half + r % 4;
          const bool mine = (lane >> 5) == half;
          const f32x16 with = mfma(mine ? p[(8 * (r / 4) + r % 4) * ROW + 32 * mt] : 0.f, mine ? w.x[r] : 0.f, acc[mt]);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[mt][i] = row >= first && row < end ? with[i] : acc[mt][i];
        }
  }
  static __device__ __forceinline__ void put4(T* p, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{a, b, c, d};
  }
};

// A wave's 32 resident rows of sums (lane: one row; register (mt, 4 g + i): column 32 mt + 8 g + 4 lh + i) times `by`,
// through 32 BY_ROWS elements of LDS that are its own, to whole rows in memory.
template <typename T, int D>
__device__ __forceinline__ void put_rows(const f32x16 (&acc)[D / 32], float by, T* own, T* to, int64_t stride, int rows, int lane) {
  using P = Products<T, D>;
  T* p = own + (lane & 31) * P::BY_ROWS + 4 * (lane >> 5);
#pragma unroll
  for (int mt = 0; mt < D / 32; ++mt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      P::put4(p + 32 * mt + 8 * g, acc[mt][4 * g] * by, acc[mt][4 * g + 1] * by, acc[mt][4 * g + 2] * by, acc[mt][4 * g + 3] * by);
  wave_sync();
  constexpr int C = D * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 32 * C / 64; ++i) {
    const int row = lane / C + i * (64 / C);
    if (row < rows)
      *reinterpret_cast<u32x4*>(to + row * stride + E * (lane % C)) = *reinterpret_cast<const u32x4*>(own + row * P::BY_ROWS + E * (lane % C));
  }
  wave_sync();
}

// Zeros in rows [0, rows) of a workgroup's tile.
template <typename T, int D> __device__ __forceinline__ void zero_rows(T* to, int64_t stride, int rows, int tid) {
  constexpr int C = D * (int)sizeof(T) / 16;
  for (int r = tid / C; r < rows; r += kPackedThreads / C)
    *reinterpret_cast<u32x4*>(to + r * stride + (16 / (int)sizeof(T)) * (tid % C)) = u32x4{0, 0, 0, 0};
}

template <typename T, int R, int XROW, int YROW> struct alignas(16) PackedTiles {
  T x[2][R * XROW], y[2][R * YROW];   // K and V, or Q and dO, in rows of XROW and YROW elements
  float lse[2][R], delta[2][R];   // statistics of the streamed queries (dk and dv)
  int odd[3];                     // tile it holds values that are not finite: odd[it % 3]
};

}  // namespace
}  // namespace gformer
