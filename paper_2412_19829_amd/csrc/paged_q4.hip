// The paged cache in 4 bits a value: what writes its rows, reads them back and moves its pages, and one new token of every sequence
// over it.
//
// decode: with codes n, scales s and lowest values l of the keys' groups g of 32 channels c, and Q_g the sum of a query's channels there,
//   q.k_j = sum_g ( s_jg sum_c q_c n_jc + l_jg Q_g ),   sum_j p_j v_jc = sum_j (p_j s_jg) n_jc + sum_j p_j l_jg
// so that codes are the matrix operands, which bf16 holds exactly, and scales meet 16 x 16 tiles.  The tiles' columns are pairs
// (query head, group): a column's query is zero outside its group; its scores' parts are added over the columns of a head, which leaves every
// token's score in one of them; and a weight, handed back to all of them, takes their groups' scales for the second product, whose rows
// (channels) count in their own group's columns alone.  16 columns are 4 heads of 128 channels, or 8 of 64.
// A code becomes an operand by way of fp8: the byte n is n 2^-9 for n < 16, two of which one instruction converts.
// Memory bounds it up to 4 query heads of 128 channels a key head, beyond that the instructions that these columns take: codes are widened
// anew for every eight heads.  us, kernel alone: 220,039 keys of 8 sequences, 32 / 8 heads, d = 128, bf16 (282 MB) 56.6, 5.0 TB/s; 88,074 in 32
// ragged ones (114 MB) 28.7; 48 of 16000, 32 / 1 heads (123 MB) 121: 468 vector instructions (73 us) and 48 products (30) a tile of 32 keys and eight
// heads; over a cache of bf16 118.  d = 64, 8 of 16000, 16 heads (164 MB) 45.6: 270 vector and 144 scalar instructions a tile, which at d = 128 are
// 339 and 146 for twice the bytes; in fp32 56.8, and 44.0 for 32 / 8 heads, d = 128.  Six fp32 sequences of 10,167 keys in all, 16 heads, d = 64 11.8;
// one of 2047, 12 heads, d = 64 6.9, and 4.5 to join.
#include "paged_q4.hpp"

#include "f32_mfma.hpp"
#include "mfma.hpp"
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

constexpr int kWaves = kPagedThreads / 64;
constexpr uint32_t kNibbles = 0x0f0f0f0fu;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A value of the lane whose number differs in bit 0 or bit 1.
template <int BIT> __device__ __forceinline__ uint32_t beside(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, BIT == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true);
}
template <int BIT> __device__ __forceinline__ float beside(float x) { return __uint_as_float(beside<BIT>(__float_as_uint(x))); }

// The value of lane `from` of this lane's GR neighbours.
template <int GR> __device__ __forceinline__ float of_group(float x, int from) {
  const int v = __float_as_int(x);
  if (GR == 2) return __int_as_float(from == 0 ? __builtin_amdgcn_mov_dpp(v, 0xa0, 0xf, 0xf, true) : __builtin_amdgcn_mov_dpp(v, 0xf5, 0xf, 0xf, true));
  return __int_as_float(from == 0   ? __builtin_amdgcn_mov_dpp(v, 0x00, 0xf, 0xf, true)
                        : from == 1 ? __builtin_amdgcn_mov_dpp(v, 0x55, 0xf, 0xf, true)
                        : from == 2 ? __builtin_amdgcn_mov_dpp(v, 0xaa, 0xf, 0xf, true)
                                    : __builtin_amdgcn_mov_dpp(v, 0xff, 0xf, 0xf, true));
}

// The largest, or the sum, of all lanes' values.
template <bool MAX> __device__ __forceinline__ float over_lanes(float x) {
  auto with = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
  x = with(x, beside<1>(x));
  x = with(x, beside<2>(x));
  x = with(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xf, 0xf, true)));   // halves of a row of 16, mirrored
  x = with(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xf, 0xf, true)));   // rows, mirrored
  return MAX ? max_over_groups(x) : sum_over_groups(x);
}

// The sum of the lanes up to this one.
__device__ __forceinline__ int sum_up_to(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // from 1, 2, 4 and 8 lanes before in the row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the last of the row before, to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // the last of row 1, to rows 2 and 3
  return x;
}

// ---- rows -------------------------------------------------------------------------------------------

// Codes of 8 of 32 values that four neighbouring lanes hold, and the group's (scale, lowest value).
struct Codes {
  uint32_t n, pair;
};

// What the scale and codes are by their definition, in 64 bits, for any sound values: x - l and the quotients are exact or nearly.
__device__ __forceinline__ uint32_t scale_of(double range) {
  // the quotient's first guess may be a step short of what reaches the range, or two where the guess itself was rounded down
  uint32_t scale = __float_as_uint((float)(range * (1.0 / 15.0))) & 0xffff0000u;
#pragma unroll
  for (int i = 0; i < 2; ++i) scale += 15.0 * (double)__uint_as_float(scale) < range ? 0x10000u : 0u;
  return scale;
}
__device__ __forceinline__ uint32_t careful_codes(const float (&x)[8], float low, uint32_t scale) {
  const double l = (double)low, s = (double)__uint_as_float(scale), half = 0.5 * s, by = scale ? __builtin_amdgcn_rcp(s) : 0.0;
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double at = (double)x[i] - l;
    const double n = rint(at * by), rest = fma(-n, s, at);   // exact: s has 8 bits
    int k = (int)n;
    if (rest > half || (rest == half && (k & 1))) ++k;
    else if (rest < -half || (rest == -half && (k & 1))) --k;
    codes |= (uint32_t)k << (4 * i);
  }
  return codes;
}

// In 32 bits where that gives the same.  Differences of bf16 values are exact where none is below 2^-15 of the largest, and then
// so is a quotient that is half way between two codes: the guess's remainder is exact (at most 9 bits), and the corrected quotient is off by
// 2^-45 of it before its rounding.  An fp32 difference is rounded, so that quotients within 2^-18 of half way are not told from it.  Those
// waves, and ones of steps or ranges near the ends of the exponents, take 64 bits for all of their values.
template <typename T> __device__ __forceinline__ Codes quantised(const float (&x)[8]) {
  constexpr bool BF16 = sizeof(T) == 2;
  float lo = min3(x[0], x[1], x[2]), hi = max3(x[0], x[1], x[2]);   // no number stays none
  float least = min3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2]));
#pragma unroll
  for (int i = 3; i < 7; i += 2) {
    lo = min3(lo, x[i], x[i + 1]);
    hi = max3(hi, x[i], x[i + 1]);
    if (BF16) least = min3(least, fabsf(x[i]), fabsf(x[i + 1]));
  }
  lo = min3(lo, x[7], beside<1>(min3(lo, x[7], x[7])));
  lo = min3(lo, beside<2>(lo), lo);
  hi = max3(hi, x[7], beside<1>(max3(hi, x[7], x[7])));
  hi = max3(hi, beside<2>(hi), hi);
  if (BF16) {
    least = min3(least, fabsf(x[7]), beside<1>(min3(least, fabsf(x[7]), fabsf(x[7]))));
    least = min3(least, beside<2>(least), least);
  }
  const float most = max3(fabsf(lo), fabsf(hi), fabsf(hi));
  const bool sound = most < 0x1p127f;
  uint32_t low = __float_as_uint(lo + 0.f);             // zero without its sign
  if (!BF16) low = (low & 0xffff0000u) + ((low & 0x8000ffffu) > 0x80000000u ? 0x10000u : 0u);   // negative with bits behind: one step away from zero
  const float l = __uint_as_float(low), top = hi + 0.f;
  bool careful = !(most < 0x1p126f) || (BF16 && least < most * 0x1p-15f);
  uint32_t scale;
  if (BF16) {
    const float range = top - l;
    scale = __float_as_uint(range * (1.f / 15.f)) & 0xffff0000u;
#pragma unroll
    for (int i = 0; i < 2; ++i) scale += 15.f * __uint_as_float(scale) < range ? 0x10000u : 0u;
  } else {
    scale = scale_of((double)top - (double)l);
  }
  const float s = __uint_as_float(scale), by = __builtin_amdgcn_rcpf(s);
  careful = (careful && lo != hi) || s < 0x1p-100f;     // a step of zero among them
  uint32_t codes = 0;
  float nearest = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float at = x[i] - l, guess = at * by, quotient = fmaf(fmaf(-guess, s, at), by, guess), n = rintf(quotient);
    if (!BF16) nearest = max3(nearest, fabsf(quotient - n), nearest);
    codes |= (uint32_t)n << (4 * i);
  }
  careful = careful || (!BF16 && !(nearest < 0.5f - 0x1p-18f));
  if (__builtin_amdgcn_ballot_w64(careful && sound)) {
    if (BF16) scale = scale_of((double)top - (double)l);
    codes = careful_codes(x, l, scale);
  }
  return sound ? Codes{codes, low | scale >> 16} : Codes{0u, 0x7fc07fc0u};
}

// 8 values of a row; what a kernel reads or writes for the last time may pass the caches by.
template <bool ONCE = false, typename V> __device__ __forceinline__ V take(const V* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; }
template <typename V> __device__ __forceinline__ void put(V* p, V x, bool once) {
  if (once) __builtin_nontemporal_store(x, p);
  else *p = x;
}
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  u32x4 w;
  template <bool ONCE = false> __device__ __forceinline__ void get(const uint16_t* p) { w = take<ONCE>(reinterpret_cast<const u32x4*>(p)); }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
};
template <> struct Eight<float> {
  f32x4 a, b;
  template <bool ONCE = false> __device__ __forceinline__ void get(const float* p) {
    a = take<ONCE>(reinterpret_cast<const f32x4*>(p));
    b = take<ONCE>(reinterpret_cast<const f32x4*>(p + 4));
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
};
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8], bool once) {
  put(reinterpret_cast<u32x4*>(p), u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}, once);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8], bool once) {
  put(reinterpret_cast<f32x4*>(p), f32x4{x[0], x[1], x[2], x[3]}, once);
  put(reinterpret_cast<f32x4*>(p + 4), f32x4{x[4], x[5], x[6], x[7]}, once);
}

// Lane c of a row's D / 8 puts its codes, and the first of four the group's pair.
template <int D> __device__ __forceinline__ void put_codes(uint32_t* row, int c, Codes x) {
  row[c] = x.n;
  if (c % 4 == 0) row[D / 8 + c / 4] = x.pair;
}

// Packed rows into their slots, or out of them: a workgroup takes ROWS rows of HB heads, a lane 8 channels of N of them.  Four heads where they
// come in fours, which leaves fewer lanes idle where sequences have few rows each; at thousands of rows it makes no difference.
constexpr int kReadRows = 2, kFillRows = 2;
template <int D, int N_, int HB> struct RowShape {
  static constexpr int C = D / 8, STEP = kPagedThreads / C, N = N_, ROWS = N * STEP / HB;   // lanes a row; rows of all lanes, of one
};
// Where a lane's rows are: rows of the packed tensors (negative: none), and their slots (page negative: none).
template <int D, int N, int HB> struct Slots {
  int row[N], head[N], page[N], slot[N];
  template <typename A> __device__ __forceinline__ bool find(const A& a, int block, int tid) {
    using S = RowShape<D, N, HB>;
    const int sets = (a.Hkv + HB - 1) / HB;
    const int tile = block / sets, lane = tid & 63;
    int seq, base, n;
    int64_t from;
    if (a.n_seqs < 64) {   // find_tile's search, with the starts on their way beside the offsets
      const int cu = packed_row(a.cu, min(lane, a.n_seqs), a.total), start = a.start[min(lane, a.n_seqs - 1)];
      seq = __popcll(__builtin_amdgcn_ballot_w64(lane <= a.n_seqs && cu / S::ROWS + lane <= tile)) - 1;
      if (seq < 0 || seq >= a.n_seqs) return false;
      base = __builtin_amdgcn_readlane(cu, seq);
      n = __builtin_amdgcn_readlane(cu, seq + 1) - base;
      from = __builtin_amdgcn_readlane(start, seq);
    } else {
      const SeqTile at = find_tile<S::ROWS>(a.cu, a.n_seqs, a.total, tile, lane);
      if (at.first < 0 || at.seq == a.n_seqs) return false;
      seq = at.seq;
      base = packed_row(a.cu, seq, a.total);
      n = packed_row(a.cu, seq + 1, a.total) - base;
      from = a.start[seq];
    }
    const int first = (tile - seq - base / S::ROWS) * S::ROWS;
    if (first < 0) return false;
    const int64_t room = (int64_t)a.width << a.shift;
    const int32_t* table = a.table + (int64_t)seq * a.width;
#pragma unroll
    for (int i = 0; i < S::N; ++i) {
      const int u = tid / S::C + i * S::STEP, r = first + u / HB;
      const int64_t pos = from + r;
      head[i] = block % sets * HB + u % HB;
      const bool real = r < n && head[i] < a.Hkv;
      row[i] = real ? base + r : -1;
      page[i] = real && pos >= 0 && pos < room ? table[pos >> a.shift] : -1;
      slot[i] = (int)pos & ((1 << a.shift) - 1);
      if ((unsigned)page[i] >= (unsigned)a.n_pages) page[i] = -1;
    }
    return true;
  }
  __device__ __forceinline__ int64_t at(const int64_t (&st)[3], int i) const { return page[i] * st[0] + head[i] * st[1] + slot[i] * st[2]; }
};

// Keys and values in workgroups of their own, which halves what a lane quantises in turn: 128 tokens of 12 heads, d = 64 5.2 us (6.6 in
// the same ones).  7206 rows of 8 heads, d = 128, bf16 (39 MB read and written): 13.5 us, of which vector instructions take 8.6 and the
// memory would take 7.9 (20 with all of them in 64 bits; 15.9 with one row a lane, 14.2 with four); fp32, whose scales are always taken in
// 64 bits (68 MB) 17.4, the memory 13.9.
template <typename T, int D, int HB> __global__ __launch_bounds__(kPagedThreads) void q4_fill_kernel(PagedFillArgs a) {
  constexpr int N = kFillRows;
  const int tid = threadIdx.x, c = tid % (D / 8);
  const bool values = blockIdx.x & 1;
  Slots<D, N, HB> s;
  if (!s.find(a, blockIdx.x >> 1, tid)) return;
  const T* rows = reinterpret_cast<const T*>(values ? a.v : a.k) + 8 * c;
  char* pages = reinterpret_cast<char*>(values ? a.vpages : a.kpages);
  const int64_t* from = values ? a.vs : a.ks;
  const int64_t* to = values ? a.vps : a.kps;
  Eight<T> x[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (s.page[i] >= 0) x[i].template get<true>(rows + s.row[i] * from[0] + s.head[i] * from[1]);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (s.page[i] >= 0) {
      float y[8];
      x[i].values(y);
      put_codes<D>(reinterpret_cast<uint32_t*>(pages + s.page[i] * to[0] + s.head[i] * to[1] + s.slot[i] * to[2]), c, quantised<T>(y));
    }
}

// l + s n in 32 bits.  s n has 12 bits and l has 8, so that the sum is half way between two bf16 values and should not be in one case alone:
// where s n is, and l too small to be seen beside it (below 2^-24 of it).  HIDDEN: then a step towards l, which is on the right side.
template <bool HIDDEN> __device__ __forceinline__ void values8(float (&x)[8], Codes y) {
  const float s = bf16_lo(y.pair), l = bf16_hi(y.pair);
  const uint32_t step = l == 0.f ? 0u : l < 0.f ? ~0u : 1u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float n = (float)(y.n >> (4 * i) & 15u);
    x[i] = fmaf(s, n, l);
    if (HIDDEN && x[i] == s * n) x[i] = __uint_as_float(__float_as_uint(x[i]) + step);
  }
}
__device__ __forceinline__ bool hides(Codes y) { return bf16_hi(y.pair) != 0.f && fabsf(bf16_hi(y.pair)) < bf16_lo(y.pair) * 0x1p-20f; }
template <int D> __device__ __forceinline__ Codes codes_of(const void* pages, int64_t at, int c) {
  const uint32_t* row = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(pages) + at);
  return {row[c], row[D / 8 + c / 4]};
}
// 56866 rows of 8 heads, d = 128, bf16 (306 MB read and written): 60.9 us, 5.0 TB/s; 6066 of 16 heads, d = 64, fp32 (57 MB) 17.5 with two
// rows a lane, 18.3 with one.  `once`: the rows are more than the last cache holds, so that nobody finds them there: 4 x 32767 tokens
// with an attention of 32 queries each behind them 442 us (475 without), but 7 x 8192 with 64 queries 240 (234).
constexpr int64_t kLastCache = (int64_t)256 << 20;   // bytes
template <typename T, int D, int HB> __global__ __launch_bounds__(kPagedThreads) void q4_read_kernel(PagedReadArgs a) {
  constexpr int N = kReadRows;
  const int tid = threadIdx.x, c = tid % (D / 8);
  const bool once = (int64_t)a.total * a.Hkv * (2 * D * (int)sizeof(T)) > kLastCache;
  Slots<D, N, HB> s;
  if (!s.find(a, blockIdx.x, tid)) return;
  Codes k[N], v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    k[i] = v[i] = {0u, 0u};
    if (s.page[i] >= 0) {
      k[i] = codes_of<D>(a.kpages, s.at(a.kps, i), c);
      v[i] = codes_of<D>(a.vpages, s.at(a.vps, i), c);
    }
  }
  const auto write = [&](auto hidden) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (s.row[i] >= 0) {
        float x[8];
        values8<hidden>(x, k[i]);
        store8(rows_of<T>(a.k, a.ks, s.row[i], s.head[i]) + 8 * c, x, once);
        values8<hidden>(x, v[i]);
        store8(rows_of<T>(a.v, a.vs, s.row[i], s.head[i]) + 8 * c, x, once);
      }
  };
  write(std::false_type());
  if (sizeof(T) == 2) {   // once more where it matters; 61.0 us where 60.6 were without, and 61.8 asked in front of the stores
    bool any = false;
#pragma unroll
    for (int i = 0; i < N; ++i) any = any || hides(k[i]) || hides(v[i]);
    if (__builtin_amdgcn_ballot_w64(any)) write(std::true_type());
  }
}

// Whole pages: a workgroup copies one head of one page, keys and values, in five pieces a row.  2000 pages of 64 tokens, 8 heads, d = 128 (328 MB
// read and written): 68.5 us, 4.8 TB/s; 4000 of 16 tokens, 12 heads, d = 64 (123 MB) 37.0: a workgroup there is 80 pieces; one page 2.5.
template <int D> __global__ __launch_bounds__(kPagedThreads) void q4_copy_kernel(PagesCopyArgs a) {
  typedef typename std::conditional<D == 128, u32x4, u32x2>::type Piece;
  const int copy = blockIdx.x / a.Hkv, head = blockIdx.x % a.Hkv;
  const int src = a.src[copy], dst = a.dst[copy];
  if ((unsigned)src >= (unsigned)a.n_pages || (unsigned)dst >= (unsigned)a.n_pages || src == dst) return;
  const char* ks = reinterpret_cast<const char*>(a.kpages) + src * a.kps[0] + head * a.kps[1];
  const char* vs = reinterpret_cast<const char*>(a.vpages) + src * a.vps[0] + head * a.vps[1];
  char* kd = reinterpret_cast<char*>(a.kpages) + dst * a.kps[0] + head * a.kps[1];
  char* vd = reinterpret_cast<char*>(a.vpages) + dst * a.vps[0] + head * a.vps[1];
  for (int i = threadIdx.x; i < 5 * a.page; i += kPagedThreads) {
    const int r = i / 5, c = (int)sizeof(Piece) * (i % 5);
    const Piece k = *reinterpret_cast<const Piece*>(ks + r * a.kps[2] + c), v = *reinterpret_cast<const Piece*>(vs + r * a.vps[2] + c);
    *reinterpret_cast<Piece*>(kd + r * a.kps[2] + c) = k;
    *reinterpret_cast<Piece*>(vd + r * a.vps[2] + c) = v;
  }
}

// ---- the decode step --------------------------------------------------------------------------------

template <int D> struct Shape4 {
  static constexpr int GR = D / kQ4Group, HC = 16 / GR;   // groups of a row, query heads of a workgroup
  static constexpr int ST = D / 32;                       // products of a score tile: lane group L takes channels D / 4 L ..
  static constexpr int E = D / 16;                        // channels of a value row that a lane takes: E i ..
  typedef typename std::conditional<D == 128, u32x4, u32x2>::type KeyCodes;
  typedef typename std::conditional<D == 128, uint32_t, uint16_t>::type ValueCodes;
};
// Whether the next tile's keys are loaded ahead, and the workgroups that a compute unit runs at once, by the registers that the sums and queries
// take.  us: 8 x 16000 tokens, 32 / 8 heads, d = 128, bf16 40.8 ahead with three, 50.9 without and with four (spilled); 8 x 16000, 16 heads,
// d = 64 52.8 ahead and 49.8 without, with four; 57.7 with five (spilled).  fp32, d = 128 47.9 with two, 57.5 with three.
template <int D> constexpr bool kAhead = D == 128;
template <typename T, int D, int C> constexpr int kAtOnce = sizeof(T) == 2 ? (D == 128 ? 4 - C : 4) : (D == 128 ? 2 : 3);
// Parts in bf16 that a factor of the products is taken in.  Queries: bf16 is one, fp32 the three that hold its 24 bits.  Weights times scales: two
// for bf16 calls and three for fp32.  In one part their rounding meets codes from 0 to 15, whose sum the lowest values' cancels nearly:
// the output of 2048 to 32768 random tokens is then off by 1.8 to 2.4 times one rounding of it, in two by one.
template <typename T> constexpr int kQueryParts = sizeof(T) == 2 ? 1 : 3;
template <typename T> constexpr int kWeightParts = sizeof(T) == 2 ? 2 : 3;
// fp32 sums would lose bits to that cancelling too: there the first part meets codes less kMiddle, which goes to the lowest values.
constexpr float kMiddle = 7.5f;
constexpr uint32_t kMinusMiddle = 0xc0f0c0f0u;

// Two values' first bf16 parts, cut off; what they leave stays in a and b.
__device__ __forceinline__ uint32_t take_part(float& a, float& b) {
  const uint32_t w = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
  b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
  return w;
}
// Their N parts, the last one rounded.
template <int N> __device__ __forceinline__ void parts_of(uint32_t (&w)[N], float a, float b) {
#pragma unroll
  for (int p = 0; p < N - 1; ++p) w[p] = take_part(a, b);
  w[N - 1] = pack_bf16(a, b);
}

__device__ __forceinline__ uint32_t codes_bf16(uint32_t bytes, bool upper) {
  return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.f, true)
                                            : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.f, false));
}

__device__ __forceinline__ int seen_tokens(const PagedDecodeArgs& a, int b) {
  const int t = a.lens[b], own = a.k ? 1 : 0;
  return t < 0 || t > a.room - own ? 0 : t + own;
}

// The sequences' tokens lie one behind another in blocks of kBlock, at least one for each, and `parts` workgroups take equal shares of the
// blocks, whatever the lengths are, which are known on the device alone.  A share may hold several sequences, or a part of one; what
// part p finds of sequence b has row p + b of the workspace to itself, since from one such piece to the next p or b grows.
constexpr int kBlock = 32 * kWaves;   // a tile for each wave
// What beginning a sequence costs, in blocks: counted in front of its own.  us with none, one, two and four: 32 ragged sequences of up to 8191,
// 32 / 8 heads, d = 128 36.1, 32.3, 32.3, 33.1; 16 of 8000 and 200 of 50 78.0, 60.7, 54.2, 58.1; 255 of 100 and one of 1000 27.6, 27.8, 26.4, 29.3; 64 of
// 0 to 1000 21.8, 20.7, 22.8, 23.2.  A row that sees nothing counts as one of a block, and is worked through like it: 8 of 16000 take 40.9, among 248
// idle rows 54.1.
constexpr int kSetUp = 2;
__host__ __device__ constexpr int64_t blocks_of(int64_t tokens) { return tokens < 1 ? 1 : (tokens + kBlock - 1) / kBlock; }
__device__ __forceinline__ int units_of(int tokens) { return kSetUp + (int)blocks_of(tokens); }
__device__ __forceinline__ int first_unit(int part, int parts, int total) { return (int)((int64_t)part * total / parts); }
// The part that holds a unit.
__device__ __forceinline__ int part_of(int unit, int parts, int total) { return (int)((((int64_t)unit + 1) * parts + total - 1) / total) - 1; }

struct Cut {
  int total, parts;     // units, and workgroups that have any
  int b, base;          // the sequence that holds the part's first unit, and that sequence's first unit
  int from, known, tokens;   // what this lane's sequence, from + lane, sees, for the first `known` lanes
  __device__ __forceinline__ int seen(const PagedDecodeArgs& a, int seq) const {
    return __builtin_amdgcn_readfirstlane(seq - from < known ? __builtin_amdgcn_readlane(tokens, seq - from) : seen_tokens(a, seq));
  }
};
__device__ __forceinline__ Cut cut_at(const PagedDecodeArgs& a, int part, int lane) {
  Cut x = {-1, 0, 0, 0, 0, 0, 0};
  int count = a.B, target = 0;
  for (;;) {   // a 64th of the sequences a lane
    const int per = (count + 63) / 64;
    int sum = 0;
    for (int j = 0; j < per; ++j)
      if (lane * per + j < count) sum += units_of(x.tokens = seen_tokens(a, x.b + lane * per + j));
    if (per == 1) {
      x.from = x.b;
      x.known = count;
    }
    sum = sum_up_to(sum);
    if (x.total < 0) {
      x.total = __builtin_amdgcn_readlane(sum, 63);
      x.parts = min(a.splits, x.total);
      if (part >= x.parts) return x;
      target = first_unit(part, x.parts, x.total);
    }
    // lanes whose sequences lie in front; never all, also where somebody changes the lengths meanwhile
    const int before = min(__popcll(__builtin_amdgcn_ballot_w64(x.base + sum <= target)), (count - 1) / per);
    if (before > 0) x.base += __builtin_amdgcn_readlane(sum, before - 1);
    x.b += before * per;
    if (per == 1) return x;
    count = min(per, count - before * per);
  }
}

// ONE: a page holds whole tiles of 16 keys (pages of 8 tokens do not), so that their pages and addresses are the same for all lanes, which
// then add nothing but a fixed offset to them: with addresses of their own they took 193 of 572 vector instructions a tile of 32 keys, d = 128
// (339 are left).
template <typename T, int D, bool ONE, int C> __global__ __launch_bounds__(kPagedThreads, (kAtOnce<T, D, C>)) void q4_decode_kernel(PagedDecodeArgs a) {
  using S = Shape4<D>;
  typedef typename S::KeyCodes KeyCodes;
  typedef typename S::ValueCodes ValueCodes;
  constexpr int GR = S::GR, HC = S::HC, HW = C * HC, ST = S::ST, E = S::E, PARTS = kQueryParts<T>, WPARTS = kWeightParts<T>, ROW = q4_row(D), U = 2, R = 16 * U, NS = 4 / GR;
  constexpr bool AHEAD = kAhead<D>;
  __shared__ float sm_o[kWaves][HW][D + 4], sm_m[kWaves][HW], sm_l[kWaves][HW];
  __shared__ __align__(16) uint32_t sm_new[2][ROW / 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, L = lane >> 4;
  const int G = a.H / a.Hkv, tiles = (G + HW - 1) / HW;
  // workgroups that read the same rows for other query heads are eight apart: on one XCD
  const int work = a.Hkv * a.splits, even = work / 8 * 8 * tiles, id = blockIdx.x;
  const int tile = id < even ? id / 8 % tiles : (id - even) % tiles, w = id < even ? id / (8 * tiles) * 8 + id % 8 : work / 8 * 8 + (id - even) / tiles;
  const int kvh = w % a.Hkv, part = w / a.Hkv;
  const int h0 = kvh * G + tile * HW, heads = min(G - tile * HW, HW);
  Cut cut;
  int unit, last_unit;
  if (a.room <= kBlock) {   // a sequence each
    cut = {0, 0, part, 0, 0, 0, 0};
    unit = 0;
    last_unit = kSetUp + 1;
  } else {
    cut = cut_at(a, part, lane);
    if (part >= cut.parts) return;
    unit = first_unit(part, cut.parts, cut.total);
    last_unit = first_unit(part + 1, cut.parts, cut.total);
  }
  const char* kc = reinterpret_cast<const char*>(a.kpages) + kvh * a.kps[1];
  const char* vc = reinterpret_cast<const char*>(a.vpages) + kvh * a.vps[1];
  const int in_page = (1 << a.shift) - 1;

  // a part that ends while it sets a sequence up leaves it to the next one
  while (cut.base + kSetUp < last_unit && cut.b < a.B) {
    const int b = cut.b, n = cut.seen(a, b), first = cut.base + kSetUp;
    const int from = max(unit - first, 0) * kBlock, to = (int)min((int64_t)n, (int64_t)(last_unit - first) * kBlock);   // at most 2^30
    const bool whole_sequence = unit <= first && last_unit - cut.base >= units_of(n);
    unit = cut.base += units_of(n);
    ++cut.b;
    const int own = a.k && n > 0 ? n - 1 : -1;   // the new token's position
    const int32_t* table = a.table + (int64_t)b * a.width;

    // pages of the tile at t0: of its 16-key parts, or of the key that this lane loads and of its four value rows
    struct Pages { int k[U], v[U]; };
    auto page_of = [&](int token) { return token < to ? table[token >> a.shift] : -1; };
    auto pages = [&](int t0) {
      Pages p;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        p.k[u] = page_of(t0 + 16 * u + (ONE ? 0 : i));
        p.v[u] = ONE ? 0 : page_of(t0 + 16 * u + 4 * L);
      }
      return p;
    };
    auto there = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
    // Everything that the first tile waits for sets out at once.  Pages are looked up two tiles ahead.
    const int step = kWaves * R;
    int t0 = from + wave * R;
    Pages here = pages(t0), next = pages(t0 + step);
    // column i of set c: query head HC c + i / GR, group i % GR
    const int h = i / GR, g = i % GR, mine = L * GR / 4;   // mine: the group of this lane's channels
    Eight<T> raw[C][ST];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        raw[c][t] = {};
        if (HC * c + h < heads && g == mine) raw[c][t].get(rows_of<T>(a.q, a.qs, b, h0 + HC * c + h) + D / 4 * L + 8 * t);
      }
    const bool brings_own = own >= from && own < to, my_own = brings_own && wave < 2 && lane < D / 8;
    Eight<T> fresh = {};
    int own_page = -1;
    if (my_own) {
      fresh.get((wave == 0 ? rows_of<T>(a.k, a.ks, b, kvh) : rows_of<T>(a.v, a.vs, b, kvh)) + 8 * lane);
      own_page = table[own >> a.shift];
    }

    // rows that are not there are read from page 0: in bounds, and masked
    const uint32_t k_codes = (uint32_t)(i * a.kps[2]) + q4_piece(D) * L, k_pairs = (uint32_t)(4 * L * a.kps[2]) + D / 2 + 4 * g;
    const uint32_t v_codes = (uint32_t)(4 * L * a.vps[2]) + (uint32_t)sizeof(ValueCodes) * i, v_pairs = (uint32_t)(4 * L * a.vps[2]) + D / 2 + 4 * g;
    auto row_at = [&](const char* pages, const int64_t (&st)[3], int page, int token) {
      return pages + (there(page) ? page * st[0] + (token & in_page) * st[2] : 0);
    };
    struct Keys {
      KeyCodes codes[U];
      uint32_t pair[U][4];     // of tokens 4 L + r
    };
    auto load_keys = [&](Keys& x, const Pages& p, int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (ONE) {
          // opaque here, or their extensions to 64 bits leave the loop and take a vector addition each
          uint32_t codes = k_codes, pairs = k_pairs;
          asm volatile("" : "+v"(codes), "+v"(pairs));
          const char* at = row_at(kc, a.kps, p.k[u], t0 + 16 * u);
          x.codes[u] = *reinterpret_cast<const KeyCodes*>(at + codes);
#pragma unroll
          for (int r = 0; r < 4; ++r) x.pair[u][r] = *reinterpret_cast<const uint32_t*>(at + r * a.kps[2] + pairs);
        } else {
          x.codes[u] = *reinterpret_cast<const KeyCodes*>(row_at(kc, a.kps, p.k[u], t0 + 16 * u + i) + q4_piece(D) * L);
          const char* at = row_at(kc, a.kps, p.v[u], t0 + 16 * u + 4 * L);
#pragma unroll
          for (int r = 0; r < 4; ++r) x.pair[u][r] = reinterpret_cast<const uint32_t*>(at + r * a.kps[2])[D / 8 + g];
        }
      }
    };
    struct Values {
      uint32_t codes[U][4], pair[U][4];
    };
    auto load_values = [&](Values& x, const Pages& p, int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t codes = v_codes, pairs = v_pairs;
        if (ONE) asm volatile("" : "+v"(codes), "+v"(pairs));
        const char* at = ONE ? row_at(vc, a.vps, p.k[u], t0 + 16 * u) : row_at(vc, a.vps, p.v[u], t0 + 16 * u + 4 * L) - 4 * L * a.vps[2];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x.pair[u][r] = *reinterpret_cast<const uint32_t*>(at + r * a.vps[2] + pairs);
          x.codes[u][r] = *reinterpret_cast<const ValueCodes*>(at + r * a.vps[2] + codes);
        }
      }
    };

    auto settle = [&](Pages& p) {
      if (ONE) {
#pragma unroll
        for (int u = 0; u < U; ++u) p.k[u] = __builtin_amdgcn_readfirstlane(p.k[u]);
      }
    };
    settle(here);
    Keys keys;
    if (AHEAD) load_keys(keys, here, t0);

    // the new token's row, for its slot and for the tile that sees it: nobody reads the slot in this call
    if (brings_own) {
      if (my_own) {
        float x[8];
        fresh.values(x);
        const Codes y = quantised<T>(x);
        put_codes<D>(sm_new[wave], lane, y);
        if (tile == 0 && there(own_page)) {
          char* row = wave == 0 ? reinterpret_cast<char*>(a.kpages) + own_page * a.kps[0] + kvh * a.kps[1] + (own & in_page) * a.kps[2]
                                : reinterpret_cast<char*>(a.vpages) + own_page * a.vps[0] + kvh * a.vps[1] + (own & in_page) * a.vps[2];
          put_codes<D>(reinterpret_cast<uint32_t*>(row), lane, y);
        }
      }
      lds_barrier();
    }

    bf16x8 q[C][PARTS][ST];
    float qsum[C], m[C], l[C], low[C];
    f32x4 o[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      qsum[c] = l[c] = low[c] = 0.f;
      m[c] = -INFINITY;
#pragma unroll
      for (int t = 0; t < ST; ++t) {
        float x[8];
        raw[c][t].values(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) qsum[c] += x[e];
        u32x4 w[PARTS];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = j < 2 ? 4 * j : 4 * j - 7;   // the order that codes_bf16 leaves them in: 0 2 4 6 1 3 5 7
          uint32_t y[PARTS];
          parts_of(y, x[e], x[e + 2]);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) w[p][j] = y[p];
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) q[c][p][t] = as_bf16x8(w[p]);
      }
      qsum[c] = sum_over_groups(qsum[c]);
#pragma unroll
      for (int e = 0; e < E; ++e) o[c][e] = kZeroF4;
    }
    const float sc = a.scale * kLog2e;

    // A tile's values are on their way while its scores are taken, the next tile's keys, in the registers of this one's, from then on.
    for (; t0 < to; t0 += step) {
      Values x;
      if (!AHEAD) load_keys(keys, here, t0);
      load_values(x, here, t0);
      settle(next);
      const Pages later = pages(t0 + 2 * step);
      const bool has_own = (unsigned)(own - t0) < (unsigned)R;   // this tile holds the new token
      if (has_own) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (t0 + 16 * u + i == own) keys.codes[u] = *reinterpret_cast<const KeyCodes*>(reinterpret_cast<const char*>(sm_new[0]) + q4_piece(D) * L);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t0 + 16 * u + 4 * L + r == own) keys.pair[u][r] = sm_new[0][D / 8 + g];
        }
      }
      // scores: this lane keeps those of tokens 4 L + g + GR n, n < NS
      float w[C][U][NS];
      // tokens of part u that are there, as bits
      auto there_of = [&](int u) {
        const int key = t0 + 16 * u + i;
        if (!ONE) return (uint32_t)__builtin_amdgcn_ballot_w64(key < to && (there(here.k[u]) || key == own)) & 0xffffu;
        const int left = min(max(to - t0 - 16 * u, 0), 16), mine_at = own - t0 - 16 * u;
        return (there(here.k[u]) ? (1u << left) - 1u : 0u) | ((unsigned)mine_at < 16u ? 1u << mine_at : 0u);
      };
      bool whole = t0 + R <= to;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        whole = whole && (ONE ? there(here.k[u]) : there_of(u) == 0xffffu);
        f32x4 s[C];
#pragma unroll
        for (int c = 0; c < C; ++c) s[c] = kZeroF4;
#pragma unroll
        for (int t = 0; t < ST; ++t) {
          const uint32_t even = keys.codes[u][t] & kNibbles, odd = keys.codes[u][t] >> 4 & kNibbles;
          const bf16x8 codes = as_bf16x8(u32x4{codes_bf16(even, false), codes_bf16(even, true), codes_bf16(odd, false), codes_bf16(odd, true)});
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) s[c] = mfma16(codes, q[c][p][t], s[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float y[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) y[r] = fmaf(bf16_lo(keys.pair[u][r]), s[c][r], bf16_hi(keys.pair[u][r]) * qsum[c]);
          // the groups' parts added up: of two tokens a lane keeps one and hands the other to the lane beside it
          const float first = (g & 1 ? y[1] : y[0]) + beside<1>(g & 1 ? y[0] : y[1]), second = (g & 1 ? y[3] : y[2]) + beside<1>(g & 1 ? y[2] : y[3]);
          if constexpr (GR == 4) {
            w[c][u][0] = ((g & 2 ? second : first) + beside<2>(g & 2 ? first : second)) * sc;
          } else {
            w[c][u][0] = first * sc;
            w[c][u][1] = second * sc;
          }
        }
      }
      if (AHEAD && t0 + step < to) load_keys(keys, next, t0 + step);
      if (has_own) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t0 + 16 * u + 4 * L + r == own) {
              x.pair[u][r] = sm_new[1][D / 8 + g];
              x.codes[u][r] = reinterpret_cast<const ValueCodes*>(sm_new[1])[i];
            }
      }
      if (!whole) {
        // what is not there gets no weight, and its values, which may be anything, become zero
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t in = there_of(u);
#pragma unroll
          for (int n = 0; n < NS; ++n)
            if (!(in >> (4 * L + g + GR * n) & 1u)) {
#pragma unroll
              for (int c = 0; c < C; ++c) w[c][u][n] = -INFINITY;
            }
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(in >> (4 * L + r) & 1u)) x.pair[u][r] = 0u;
        }
      }
      u32x4 weights[C][WPARTS];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int n = 0; n < NS; ++n) top = fmaxf(top, w[c][u][n]);
        top = fmaxf(top, beside<1>(top));
        if (GR == 4) top = fmaxf(top, beside<2>(top));
        top = max_over_groups(top);
        if (__builtin_amdgcn_ballot_w64(top > m[c] + 8.f) != 0) {   // weights stay below 2^8 (packed_fwd.hip)
          const float up = fmaxf(m[c], top), by = __builtin_amdgcn_exp2f(m[c] - (up == -INFINITY ? 0.f : up));
          m[c] = up;
          l[c] *= by;
          low[c] *= by;
#pragma unroll
          for (int e = 0; e < E; ++e) o[c][e] *= by;
        }
        const float ref = m[c] == -INFINITY ? 0.f : m[c];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            w[c][u][n] = __builtin_amdgcn_exp2f(w[c][u][n] - ref);
            l[c] += w[c][u][n];
          }
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            float y[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float p = of_group<GR>(w[c][u][(r + z) / GR], (r + z) % GR);
              low[c] = fmaf(p, bf16_hi(x.pair[u][r + z]), low[c]);
              y[z] = p * bf16_lo(x.pair[u][r + z]);
            }
            uint32_t z[WPARTS];
            parts_of(z, y[0], y[1]);
#pragma unroll
            for (int p = 0; p < WPARTS; ++p) weights[c][p][2 * u + r / 2] = z[p];
            if (sizeof(T) == 4) low[c] = fmaf(kMiddle, bf16_lo(z[0]), fmaf(kMiddle, bf16_hi(z[0]), low[c]));
          }
        }
      }
      // channels of the same byte's half and parity at a time: a byte of each of two tokens, then one of the next
#pragma unroll
      for (int half = 0; half < E / 4; ++half) {
        uint32_t two[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          two[j] = __builtin_amdgcn_perm(x.codes[j / 2][2 * (j % 2) + 1], x.codes[j / 2][2 * (j % 2)], half ? 0x07030602u : 0x05010400u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          u32x4 codes;
#pragma unroll
          for (int j = 0; j < 4; ++j) codes[j] = codes_bf16(two[j] >> (4 * (e % 2)) & kNibbles, e >= 2);
#pragma unroll
          for (int c = 0; c < C; ++c) {
            f32x4& sum = o[c][4 * half + e];
            if (sizeof(T) == 4)
              sum = mfma16(as_bf16x8(u32x4{kMinusMiddle, kMinusMiddle, kMinusMiddle, kMinusMiddle}), as_bf16x8(weights[c][0]), sum);
#pragma unroll
            for (int p = WPARTS - 1; p >= 0; --p) sum = mfma16(as_bf16x8(codes), as_bf16x8(weights[c][p]), sum);
          }
        }
      }
      here = next;
      next = later;
    }
    // join the waves: a channel counts in its own group's column
#pragma unroll
    for (int c = 0; c < C; ++c) {
      l[c] += beside<1>(l[c]);
      if (GR == 4) l[c] += beside<2>(l[c]);
      l[c] = sum_over_groups(l[c]);
      low[c] = sum_over_groups(low[c]);
      if (L == 0 && g == 0) {
        sm_m[wave][HC * c + h] = m[c];
        sm_l[wave][HC * c + h] = l[c];
      }
      if (g == mine) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) sm_o[wave][HC * c + h][E * (4 * L + r) + e] = o[c][e][r] + low[c];
      }
    }
    lds_barrier();
    const int c = tid % D;
    for (int x = tid / D; x < heads; x += kPagedThreads / D) {
      float top = -INFINITY, sum = 0.f, acc = 0.f;
#pragma unroll
      for (int y = 0; y < kWaves; ++y) top = fmaxf(top, sm_m[y][x]);
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int y = 0; y < kWaves; ++y) {
        const float by = __builtin_amdgcn_exp2f(sm_m[y][x] - ref);
        sum = fmaf(sm_l[y][x], by, sum);
        acc = fmaf(sm_o[y][x][c], by, acc);
      }
      if (whole_sequence) {
        Storage<T>::store(rows_of<T>(a.out, a.os, b, h0 + x), c, sum == 0.f ? 0.f : acc / sum);
      } else {
        const int64_t at = (int64_t)(part + b) * a.H + h0 + x;
        a.sums[at * D + c] = acc;
        if (c == 0) {
          a.stats[2 * at] = top;
          a.stats[2 * at + 1] = sum;
        }
      }
    }
    lds_barrier();   // the next sequence's sums go to the same places
  }
}

// Joins the pieces of a sequence that is cut in front of a part, if that is its first cut: W waves for each head, which take every W-th
// piece, the statistics of 64 at once and their sums eight by eight.
template <typename T, int D, int W> __global__ __launch_bounds__(kPagedThreads) void q4_join_kernel(PagedDecodeArgs a) {
  constexpr int N = D / 64;   // columns of a lane
  typedef float Columns __attribute__((ext_vector_type(N)));
  __shared__ float sm_top[kWaves], sm_sum[kWaves];
  __shared__ __align__(8) float sm_acc[kWaves][D];
  constexpr int HEADS = kWaves / W;   // of a workgroup
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sets = (a.H + HEADS - 1) / HEADS;
  const int h = blockIdx.x % sets * HEADS + wave / W, part = blockIdx.x / sets + 1;
  const Cut cut = cut_at(a, part, lane);
  const int first = cut.base + kSetUp;   // its first block
  if (part >= cut.parts || first >= first_unit(part, cut.parts, cut.total) || first < first_unit(part - 1, cut.parts, cut.total)) return;
  if (W < kWaves && h >= a.H) return;   // no barrier follows
  const int n = cut.seen(a, cut.b);
  const int pieces = min(part_of(cut.base + units_of(n) - 1, cut.parts, cut.total), cut.parts - 1) - (part - 1) + 1;
  const int mine = (pieces - wave % W + W - 1) / W;
  const int64_t at = (int64_t)(part - 1 + cut.b + wave % W) * a.H + h, next = (int64_t)W * a.H;   // this wave's first one, and how far the next is
  float top = -INFINITY, sum = 0.f;
  Columns acc = {};
  for (int s0 = 0; s0 < mine; s0 += 64) {
    const int here = min(64, mine - s0);
    float m = -INFINITY, l = 0.f;
    if (lane < here) {
      m = a.stats[2 * (at + (s0 + lane) * next)];
      l = a.stats[2 * (at + (s0 + lane) * next) + 1];
    }
    Columns x[8];
    auto load = [&](int s) {   // set out beside the statistics
#pragma unroll
      for (int y = 0; y < 8; ++y)
        x[y] = s + y < here ? *reinterpret_cast<const Columns*>(a.sums + (at + (s0 + s + y) * next) * D + N * lane) : Columns{};
    };
    load(0);
    const float up = fmaxf(top, over_lanes<true>(m));
    const float ref = up == -INFINITY ? 0.f : up, keep = __builtin_amdgcn_exp2f(top - ref), by = __builtin_amdgcn_exp2f(m - ref);
    top = up;
    acc *= keep;
    sum = fmaf(sum, keep, over_lanes<false>(l * by));
    for (int s = 0;;) {
#pragma unroll
      for (int y = 0; y < 8; ++y) acc += x[y] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), min(s + y, 63)));
      s += 8;
      if (s >= here) break;
      load(s);
    }
  }
  if constexpr (W > 1) {
    *reinterpret_cast<Columns*>(&sm_acc[wave][N * lane]) = acc;
    if (lane == 0) {
      sm_top[wave] = top;
      sm_sum[wave] = sum;
    }
    __syncthreads();
    if (wave % W != 0) return;
    for (int y = 1; y < W; ++y) top = fmaxf(top, sm_top[wave + y]);
    const float ref = top == -INFINITY ? 0.f : top;
    acc = {};
    sum = 0.f;
    for (int y = 0; y < W; ++y) {
      const float by = __builtin_amdgcn_exp2f(sm_top[wave + y] - ref);
      acc += *reinterpret_cast<const Columns*>(&sm_acc[wave + y][N * lane]) * by;
      sum = fmaf(sm_sum[wave + y], by, sum);
    }
  }
#pragma unroll
  for (int x = 0; x < N; ++x) Storage<T>::store(rows_of<T>(a.out, a.os, cut.b, h), N * lane + x, sum == 0.f ? 0.f : acc[x] / sum);
}

// From so many possible pieces a sequence on, a head's are joined by a workgroup, below by a wave.  us of the step, by a wave and by a workgroup, d = 128:
// 12 pieces (8 x 32767 tokens, 32 / 8 heads) 73.3 and 73.8, 24 (4) 41.8 and 42.0, 48 (2) 27.7 and 26.6, 96 (1) 23.7 and 19.1; 16 (32 x 16000, 8 / 1) 31.6 and
// 34.8, 32 (16) 25.0 and 26.0, 64 (8) 25.1 and 21.0.
constexpr int kManyPieces = 24;

// Sets of columns that a workgroup holds.  Two, which widen a code once for both, where a key head has more query heads than the four of one, in
// calls that fill the compute units all the same.  us, one set and two: 16 x 16000 tokens, 32 / 4 heads, d = 128 65.4 and 55.3; 48 x 16000, 32 / 1 152 and
// 121; one of 16000, 8 / 1 12.3 and 14.1.  At d = 64, where a set is eight heads, 32 x 16000, 16 / 1 35.1 and 40.2.  fp32 has no registers for a second one.
int column_sets(bool bf16, int B, int H, int Hkv, int d, int64_t max_len) {
  constexpr int HC = Shape4<128>::HC;
  const int64_t workgroups = (int64_t)Hkv * ((H / Hkv + 2 * HC - 1) / (2 * HC));
  return bf16 && d == 128 && H / Hkv > HC && workgroups * B * blocks_of(max_len) >= 256 * kAtOnce<uint16_t, 128, 2> ? 2 : 1;
}
// Workgroups of a part: one for the query heads that fit its columns.
int64_t decode_units(bool bf16, int B, int H, int Hkv, int d, int64_t max_len) {
  const int heads = column_sets(bf16, B, H, Hkv, d, max_len) * (d == 128 ? Shape4<128>::HC : Shape4<64>::HC);
  return (int64_t)Hkv * ((H / Hkv + heads - 1) / heads);
}

template <typename T, int D, int C> void decode_pages(const PagedDecodeArgs& a, dim3 grid, hipStream_t s) {
  if (a.shift >= 4) q4_decode_kernel<T, D, true, C><<<grid, dim3(kPagedThreads), 0, s>>>(a);
  else q4_decode_kernel<T, D, false, C><<<grid, dim3(kPagedThreads), 0, s>>>(a);
}
template <typename T, int D> hipError_t decode(const PagedDecodeArgs& a, hipStream_t s) {
  constexpr bool BF16 = sizeof(T) == 2;
  const dim3 grid((unsigned)(decode_units(BF16, a.B, a.H, a.Hkv, D, a.room) * a.splits));
  if (column_sets(BF16, a.B, a.H, a.Hkv, D, a.room) == 2) decode_pages<T, D, BF16 && D == 128 ? 2 : 1>(a, grid, s);
  else decode_pages<T, D, 1>(a, grid, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.stats) return e;
  // many pieces a sequence take a workgroup a head
  if (a.splits >= (int64_t)kManyPieces * a.B) q4_join_kernel<T, D, kWaves><<<dim3((unsigned)(a.splits - 1) * a.H), dim3(kPagedThreads), 0, s>>>(a);
  else q4_join_kernel<T, D, 1><<<dim3((unsigned)(a.splits - 1) * ((a.H + kWaves - 1) / kWaves)), dim3(kPagedThreads), 0, s>>>(a);
  return hipGetLastError();
}

int heads_together(int Hkv) { return Hkv % 4 == 0 ? 4 : 1; }
int64_t row_groups(int total, int n_seqs, int Hkv, int d, int n) {
  const int hb = heads_together(Hkv), rows = n * (d == 128 ? RowShape<128, 1, 1>::ROWS : RowShape<64, 1, 1>::ROWS) / hb;
  return packed_tiles(total, n_seqs, rows) * (Hkv / hb);
}
template <typename T, int D> hipError_t fill(const PagedFillArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(2 * row_groups(a.total, a.n_seqs, a.Hkv, D, kFillRows)));
  if (heads_together(a.Hkv) == 4) q4_fill_kernel<T, D, 4><<<grid, kPagedThreads, 0, s>>>(a);
  else q4_fill_kernel<T, D, 1><<<grid, kPagedThreads, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, int D> hipError_t read(const PagedReadArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)row_groups(a.total, a.n_seqs, a.Hkv, D, kReadRows));
  if (heads_together(a.Hkv) == 4) q4_read_kernel<T, D, 4><<<grid, kPagedThreads, 0, s>>>(a);
  else q4_read_kernel<T, D, 1><<<grid, kPagedThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// As many workgroups as run at once on 256 compute units, and no part without a unit if all sequences are the longest.  Sequences of one
// block, which are not cut, take one each.
int paged_q4_parts(bool bf16, int B, int H, int Hkv, int d, int64_t max_len) {
  if (!paged_q4_cuts(max_len)) return B;
  const int at_once = !bf16      ? (d == 128 ? kAtOnce<float, 128, 1> : kAtOnce<float, 64, 1>)
                      : d == 64 ? kAtOnce<uint16_t, 64, 1>
                      : column_sets(bf16, B, H, Hkv, d, max_len) == 2 ? kAtOnce<uint16_t, 128, 2> : kAtOnce<uint16_t, 128, 1>;
  return (int)std::max<int64_t>(1, std::min(256 * at_once / decode_units(bf16, B, H, Hkv, d, max_len), B * (kSetUp + blocks_of(max_len))));
}
bool paged_q4_cuts(int64_t max_len) { return max_len > kBlock; }
bool paged_q4_decode_fits(bool bf16, int B, int H, int Hkv, int d, int64_t max_len) {
  return decode_units(bf16, B, H, Hkv, d, max_len) * paged_q4_parts(bf16, B, H, Hkv, d, max_len) <= most_workgroups(kPagedThreads) &&
         B * (kSetUp + blocks_of(max_len)) < (1ll << 31);   // units are counted in 32 bits
}
bool paged_q4_rows_fit(int total, int n_seqs, int Hkv, int d) { return 2 * row_groups(total, n_seqs, Hkv, d, std::min(kFillRows, kReadRows)) <= most_workgroups(kPagedThreads); }

hipError_t launch_paged_q4_decode(const PagedDecodeArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? decode<uint16_t, 128>(a, s) : decode<uint16_t, 64>(a, s);
  return a.d == 128 ? decode<float, 128>(a, s) : decode<float, 64>(a, s);
}

hipError_t launch_paged_q4_fill(const PagedFillArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? fill<uint16_t, 128>(a, s) : fill<uint16_t, 64>(a, s);
  return a.d == 128 ? fill<float, 128>(a, s) : fill<float, 64>(a, s);
}

hipError_t launch_paged_q4_read(const PagedReadArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? read<uint16_t, 128>(a, s) : read<uint16_t, 64>(a, s);
  return a.d == 128 ? read<float, 128>(a, s) : read<float, 64>(a, s);
}

hipError_t launch_pages_q4_copy(const PagesCopyArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.n_copies * a.Hkv));
  a.d == 128 ? q4_copy_kernel<128><<<grid, kPagedThreads, 0, s>>>(a) : q4_copy_kernel<64><<<grid, kPagedThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gformer
