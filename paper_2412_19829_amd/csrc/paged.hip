// One new token of every sequence over a paged key-value cache, and what fills and moves its pages.
//
// decode: the query heads that share a key head are the columns of 16x16 score tiles (at most 16 a workgroup), so a key
// or value is read once for all of them, straight from memory into matrix operands.  A sequence is cut along its
// length into chunks of keys, one workgroup each, whose four waves take tiles in turn; every wave keeps a softmax of
// its own (running maximum, sum and weighted values), the waves are joined in LDS and the chunks by a second kernel.
// Memory bounds it, and what hides its latency are waves, three on a SIMD: a tile loaded ahead in registers leaves room
// for two only (4 sequences of up to 32768, 32 / 8 heads, d = 128: 97 us so, 88 with three, 5.4 TB/s; with four the sums spill, 138
// for 32 sequences of up to 8192 that take 73 so).  A call of one user is launches and trips to memory: 2047 tokens, 12 heads, d = 64:
// 4.3 us and 3.0 to join.
//
// Score tile S^T = K Q^T (D = A*B, lane l, i = l % 16, g = l / 16): A row i = key i, B column i = head i, result column
// i = head i, register r = key 4 g + r.  Those registers are the next product's B operand as they are, if its
// contraction index takes the keys in that order; V^T is its A operand, whose row i lane i makes from its own
// columns of the value rows 4 g + r: column E i + e for the e-th product.
#include "paged.hpp"

#include "f32_mfma.hpp"
#include "mfma.hpp"
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

constexpr int kDecodeWaves = kPagedThreads / 64;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// One wave's tile of keys and values in registers, and its products.
template <typename T, int D> struct Cached;

template <int D> struct Cached<uint16_t, D> {
  static constexpr int U = 2;               // 16-key tiles
  static constexpr int E = D / 16, HH = 1;  // columns of a value row that a lane holds: E i .. E i + E - 1
  static constexpr int NO = E;              // result tiles
  typedef typename std::conditional<E == 8, u32x4, u32x2>::type Part;
  struct Query { bf16x8 x[D / 32]; };
  struct Tile {
    u32x4 k[U][D / 32];
    Part v[U][4];
  };
  static __device__ __forceinline__ void query(Query& q, const uint16_t* row, bool real, int g) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q.x[s] = as_bf16x8(real ? *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * g) : u32x4{0, 0, 0, 0});
  }
  static __device__ __forceinline__ void load_k(u32x4 (&k)[D / 32], const uint16_t* row, int g) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) k[s] = *reinterpret_cast<const u32x4*>(row + 32 * s + 8 * g);
  }
  // a value row is read whole, once, and need not stay in the caches (a key row is read in quarters, which share lines)
  static __device__ __forceinline__ void load_v(Part& v, const uint16_t* row, int i) { v = __builtin_nontemporal_load(reinterpret_cast<const Part*>(row + E * i)); }
  static __device__ __forceinline__ f32x4 scores(const u32x4 (&k)[D / 32], const Query& q) {
    f32x4 s = kZeroF4;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) s = mfma16(as_bf16x8(k[t]), q.x[t], s);
    return s;
  }
  static __device__ __forceinline__ void product(f32x4 (&o)[NO], Tile& t, const float (&p)[U][4], float& sum) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16(p[j / 2][2 * (j % 2)], p[j / 2][2 * (j % 2) + 1]);
      sum = dot2_ones_bf16(w[j], sum);   // the sum of what the product sees
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u32x4 a;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        a[j] = __builtin_amdgcn_perm(t.v[j / 2][2 * (j % 2) + 1][e / 2], t.v[j / 2][2 * (j % 2)][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
      o[e] = mfma16(as_bf16x8(a), as_bf16x8(w), o[e]);
    }
  }
  static __device__ __forceinline__ uint16_t put(float x) { return (uint16_t)pack_bf16(x, 0.f); }
};

template <int D> struct Cached<float, D> {
  static constexpr int U = 1;
  static constexpr int E = 4, HH = D / 64;   // columns 64 hh + 4 i .. + 3
  static constexpr int NO = E * HH;
  struct Part { f32x4 x[HH]; };
  struct Query { f32x4 x[D / 16]; };
  struct Tile {
    f32x4 k[U][D / 16];
    Part v[U][4];
  };
  static __device__ __forceinline__ void query(Query& q, const float* row, bool real, int g) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q.x[s] = real ? *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g) : kZeroF4;
  }
  static __device__ __forceinline__ void load_k(f32x4 (&k)[D / 16], const float* row, int g) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) k[s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
  }
  static __device__ __forceinline__ void load_v(Part& v, const float* row, int i) {
#pragma unroll
    for (int hh = 0; hh < HH; ++hh) v.x[hh] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row + 64 * hh + 4 * i));
  }
  static __device__ __forceinline__ f32x4 scores(const f32x4 (&k)[D / 16], const Query& q) {
    f32x4 s = kZeroF4;
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = mfma_f32(k[t][j], q.x[t][j], s);
    return s;
  }
  static __device__ __forceinline__ void product(f32x4 (&o)[NO], Tile& t, const float (&p)[U][4], float& sum) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sum += p[0][r];
#pragma unroll
      for (int n = 0; n < NO; ++n) o[n] = mfma_f32(t.v[0][r].x[n / E][n % E], p[0][r], o[n]);
    }
  }
  static __device__ __forceinline__ float put(float x) { return x; }
};

// Keys that sequence b's token sees: its cached ones and, where the call brings it, its own.  A length that there
// is no room for is an idle row: it sees nothing and writes nothing.
__device__ __forceinline__ int seen_keys(const PagedDecodeArgs& a, int b) {
  const int t = a.lens[b], own = a.k ? 1 : 0;
  return t < 0 || t > a.room - own ? 0 : t + own;
}

template <typename T, int D> __global__ __launch_bounds__(kPagedThreads, 3) void paged_decode_kernel(PagedDecodeArgs a) {
  using C = Cached<T, D>;
  constexpr int U = C::U, R = 16 * U, NO = C::NO, E = C::E;
  __shared__ float sm_o[kDecodeWaves][kPagedHeads][D + 4], sm_m[kDecodeWaves][kPagedHeads], sm_l[kDecodeWaves][kPagedHeads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const int G = a.H / a.Hkv, tiles = (G + kPagedHeads - 1) / kPagedHeads;
  // Chunks slowest: workgroups are dealt to the 8 XCDs in turn, and the chunks behind short sequences' ends, which are none,
  // would leave some XCDs without work.
  int id = blockIdx.x;
  const int tile = id % tiles;
  id /= tiles;
  const int kvh = id % a.Hkv;
  id /= a.Hkv;
  const int b = id % a.B, split = id / a.B;
  const int h0 = kvh * G + tile * kPagedHeads, heads = min(G - tile * kPagedHeads, kPagedHeads);
  const int n = seen_keys(a, b), from = split * a.chunk, to = min(n, from + a.chunk);
  if (split > 0 && from >= n) return;   // the joining kernel knows as much

  const int own = a.k && n > 0 ? n - 1 : -1;   // the new token's position
  const T* kn = rows_of<T>(a.k, a.ks, b, kvh);
  const T* vn = rows_of<T>(a.v, a.vs, b, kvh);
  const T* kc = reinterpret_cast<const T*>(a.kpages) + kvh * a.kps[1];
  const T* vc = reinterpret_cast<const T*>(a.vpages) + kvh * a.vps[1];
  const int32_t* table = a.table + (int64_t)b * a.width;
  const int in_page = (1 << a.shift) - 1;

  // the new token's row goes to its slot: nobody reads it there in this call
  if (own >= from && own < to && tile == 0) {
    const int page = table[own >> a.shift];
    if ((unsigned)page < (unsigned)a.n_pages) {
      T* kw = reinterpret_cast<T*>(a.kpages) + page * a.kps[0] + kvh * a.kps[1] + (own & in_page) * a.kps[2];
      T* vw = reinterpret_cast<T*>(a.vpages) + page * a.vps[0] + kvh * a.vps[1] + (own & in_page) * a.vps[2];
      if (tid < D) kw[tid] = kn[tid];
      else if (tid < 2 * D) vw[tid - D] = vn[tid - D];
    }
  }

  typename C::Query q;
  C::query(q, rows_of<T>(a.q, a.qs, b, h0 + min(i, heads - 1)), i < heads, g);
  const float sc = a.scale * kLog2e;
  f32x4 o[NO];
#pragma unroll
  for (int e = 0; e < NO; ++e) o[e] = kZeroF4;
  float m = -INFINITY, l = 0.f;

  // pages of the tile at t0: of the key that this lane loads (its score row), and of its four value rows (pages hold
  // at least eight tokens)
  struct Pages { int k[U], v[U]; };
  auto pages = [&](int t0) {
    Pages p;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      p.k[u] = t0 + 16 * u + i < to ? table[(t0 + 16 * u + i) >> a.shift] : -1;
      p.v[u] = t0 + 16 * u + 4 * g < to ? table[(t0 + 16 * u + 4 * g) >> a.shift] : -1;
    }
    return p;
  };
  auto there = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
  // rows that are not there are read from page 0: in bounds, and masked
  auto load = [&](typename C::Tile& x, const Pages& p, int t0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key = t0 + 16 * u + i;
      const T* row = kc + (there(p.k[u]) ? p.k[u] * a.kps[0] + (key & in_page) * a.kps[2] : 0);
      C::load_k(x.k[u], key == own ? kn : row, g);
      const T* rows = vc + (there(p.v[u]) ? p.v[u] * a.vps[0] : 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int vkey = t0 + 16 * u + 4 * g + r;
        C::load_v(x.v[u][r], vkey == own ? vn : rows + (vkey & in_page) * a.vps[2], i);
      }
    }
  };

  const int step = kDecodeWaves * R;
  int t0 = from + wave * R;
  Pages here = pages(t0);   // looked up a tile ahead
  for (; t0 < to; t0 += step) {
    typename C::Tile x;
    load(x, here, t0);
    const Pages next = pages(t0 + step);
    float w[U][4];
    float top = -INFINITY;
    uint32_t in[U];
    bool whole = true;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key = t0 + 16 * u + i;
      in[u] = (uint32_t)__builtin_amdgcn_ballot_w64(key < to && (there(here.k[u]) || key == own)) & 0xffffu;
      whole = whole && in[u] == 0xffffu;
      const f32x4 s = C::scores(x.k[u], q);
#pragma unroll
      for (int r = 0; r < 4; ++r) w[u][r] = s[r] * sc;
    }
    if (!whole) {
      // what is not there gets no weight, and its values, which may be anything, become zero
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!(in[u] >> (4 * g + r) & 1u)) {
            w[u][r] = -INFINITY;
            x.v[u][r] = typename C::Part{};
          }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, fmaxf(fmaxf(w[u][0], w[u][1]), fmaxf(w[u][2], w[u][3])));
    top = max_over_groups(top);
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f) != 0) {   // weights stay below 2^8 (packed_fwd.hip)
      const float up = fmaxf(m, top), by = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.f : up));
      m = up;
      l *= by;
#pragma unroll
      for (int e = 0; e < NO; ++e) o[e] *= by;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) w[u][r] = __builtin_amdgcn_exp2f(w[u][r] - ref);
    C::product(o, x, w, l);
    here = next;
  }
  l = sum_over_groups(l);

  // join the waves
  if (g == 0) {
    sm_m[wave][i] = m;
    sm_l[wave][i] = l;
  }
#pragma unroll
  for (int e = 0; e < NO; ++e)
#pragma unroll
    for (int r = 0; r < 4; ++r) sm_o[wave][i][64 * (e / E) + E * (4 * g + r) + e % E] = o[e][r];
  __syncthreads();
  const int c = tid % D;
  for (int h = tid / D; h < heads; h += kPagedThreads / D) {
    float top = -INFINITY, sum = 0.f, acc = 0.f;
#pragma unroll
    for (int x = 0; x < kDecodeWaves; ++x) top = fmaxf(top, sm_m[x][h]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < kDecodeWaves; ++x) {
      const float by = __builtin_amdgcn_exp2f(sm_m[x][h] - ref);
      sum = fmaf(sm_l[x][h], by, sum);
      acc = fmaf(sm_o[x][h][c], by, acc);
    }
    if (a.splits == 1) {
      rows_of<T>(a.out, a.os, b, h0 + h)[c] = C::put(sum == 0.f ? 0.f : acc / sum);
    } else {
      const int64_t at = ((int64_t)b * a.H + h0 + h) * a.splits + split;
      a.sums[at * D + c] = acc;
      if (c == 0) {
        a.stats[2 * at] = top;
        a.stats[2 * at + 1] = sum;
      }
    }
  }
}

// Joins the chunks of one head: a workgroup's threads take 4 columns of every (kPagedThreads / (D / 4))-th chunk.  Latency: 3 to 4 us.
template <typename T, int D> __global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(PagedDecodeArgs a) {
  constexpr int C4 = D / 4, GROUPS = kPagedThreads / C4;
  __shared__ float sm_top[4];
  __shared__ f32x4 sm_o[GROUPS][C4];
  __shared__ float sm_l[GROUPS];
  const int tid = threadIdx.x, b = blockIdx.x / a.H, h = blockIdx.x % a.H;
  const int n = seen_keys(a, b), used = max(1, (n + a.chunk - 1) / a.chunk);
  const int64_t at = ((int64_t)b * a.H + h) * a.splits;
  float top = -INFINITY;
  for (int s = tid; s < used; s += kPagedThreads) top = fmaxf(top, a.stats[2 * (at + s)]);
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
  if ((tid & 63) == 0) sm_top[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(sm_top[0], sm_top[1]), fmaxf(sm_top[2], sm_top[3]));
  const float ref = top == -INFINITY ? 0.f : top;
  f32x4 acc = kZeroF4;
  float sum = 0.f;
  for (int s = tid / C4; s < used; s += GROUPS) {
    const float by = __builtin_amdgcn_exp2f(a.stats[2 * (at + s)] - ref);
    sum = fmaf(a.stats[2 * (at + s) + 1], by, sum);
    acc += *reinterpret_cast<const f32x4*>(a.sums + (at + s) * D + 4 * (tid % C4)) * by;
  }
  sm_o[tid / C4][tid % C4] = acc;
  if (tid % C4 == 0) sm_l[tid / C4] = sum;
  __syncthreads();
  if (tid < D) {
    float s = 0.f, x = 0.f;
#pragma unroll
    for (int y = 0; y < GROUPS; ++y) {
      s += sm_l[y];
      x += sm_o[y][tid / 4][tid % 4];
    }
    rows_of<T>(a.out, a.os, b, h)[tid] = Cached<T, D>::put(s == 0.f ? 0.f : x / s);
  }
}

// Packed rows into their slots: a workgroup moves 32 rows of one head.  Memory: 8192 tokens of 8 heads, d = 128, bf16 (67 MB read and
// written) 11.2 us, 6.0 TB/s with part of them in the caches; 128 tokens of 12 heads, d = 64: 2.6.
constexpr int kFillRows = 32;
template <typename T, int D> __global__ __launch_bounds__(kPagedThreads) void paged_fill_kernel(PagedFillArgs a) {
  constexpr int C = D * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T);
  const int tid = threadIdx.x, head = blockIdx.x % a.Hkv;
  const SeqTile at = find_tile<kFillRows>(a.cu, a.n_seqs, a.total, blockIdx.x / a.Hkv, tid & 63);
  if (at.first < 0 || at.seq == a.n_seqs) return;
  const int base = packed_row(a.cu, at.seq, a.total), n = packed_row(a.cu, at.seq + 1, a.total) - base;
  const int64_t room = (int64_t)a.width << a.shift;
  for (int r = tid / C; r < kFillRows; r += kPagedThreads / C) {
    const int row = at.first + r;
    const int64_t pos = (int64_t)a.start[at.seq] + row;
    if (row >= n || pos < 0 || pos >= room) continue;
    const int page = a.table[(int64_t)at.seq * a.width + (pos >> a.shift)];
    if ((unsigned)page >= (unsigned)a.n_pages) continue;
    const int slot = (int)pos & ((1 << a.shift) - 1), c = E * (tid % C);
    const u32x4 k = *reinterpret_cast<const u32x4*>(rows_of<T>(a.k, a.ks, base + row, head) + c);
    const u32x4 v = *reinterpret_cast<const u32x4*>(rows_of<T>(a.v, a.vs, base + row, head) + c);
    *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.kpages) + page * a.kps[0] + head * a.kps[1] + slot * a.kps[2] + c) = k;
    *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.vpages) + page * a.vps[0] + head * a.vps[1] + slot * a.vps[2] + c) = v;
  }
}

// Whole pages: a workgroup copies one head of one page, keys and values.  Memory: 1024 pages of 64 tokens, 8 heads, d = 128, bf16 (537 MB
// read and written) 102 us, 5.3 TB/s; 16 pages 3.4.
template <typename T, int D> __global__ __launch_bounds__(kPagedThreads) void pages_copy_kernel(PagesCopyArgs a) {
  constexpr int C = D * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T), STEP = kPagedThreads / C;
  const int copy = blockIdx.x / a.Hkv, head = blockIdx.x % a.Hkv;
  const int src = a.src[copy], dst = a.dst[copy];
  if ((unsigned)src >= (unsigned)a.n_pages || (unsigned)dst >= (unsigned)a.n_pages || src == dst) return;
  const int c = E * (threadIdx.x % C);
  const T* ks = reinterpret_cast<const T*>(a.kpages) + src * a.kps[0] + head * a.kps[1] + c;
  const T* vs = reinterpret_cast<const T*>(a.vpages) + src * a.vps[0] + head * a.vps[1] + c;
  T* kd = reinterpret_cast<T*>(a.kpages) + dst * a.kps[0] + head * a.kps[1] + c;
  T* vd = reinterpret_cast<T*>(a.vpages) + dst * a.vps[0] + head * a.vps[1] + c;
  for (int r = threadIdx.x / C; r < a.page; r += STEP) {
    const u32x4 k = *reinterpret_cast<const u32x4*>(ks + r * a.kps[2]), v = *reinterpret_cast<const u32x4*>(vs + r * a.vps[2]);
    *reinterpret_cast<u32x4*>(kd + r * a.kps[2]) = k;
    *reinterpret_cast<u32x4*>(vd + r * a.vps[2]) = v;
  }
}

// Workgroups of an uncut call: 16 query heads of one key head of one sequence each.
int64_t decode_units(int B, int H, int Hkv) { return (int64_t)B * Hkv * (((int64_t)H / Hkv + kPagedHeads - 1) / kPagedHeads); }

template <typename T, int D> hipError_t decode(const PagedDecodeArgs& a, hipStream_t s) {
  const unsigned workgroups = (unsigned)(decode_units(a.B, a.H, a.Hkv) * a.splits);
  paged_decode_kernel<T, D><<<dim3(workgroups), dim3(kPagedThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  paged_join_kernel<T, D><<<dim3((unsigned)((int64_t)a.B * a.H)), dim3(kPagedThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Six workgroups for every compute unit if all sequences were the longest, and no chunk shorter than a tile for each wave.
// us, 512 / 1024 / 1536 / 2048 / 4096 workgroups: 32 sequences of up to 8192, 32 / 8 heads, d = 128, 88,000 keys in all 109 / 90 / 72 / 78 / 74,
// 4 of up to 32768 84 / 88 / 88 / 91 / 94; one of 2048, 12 heads, d = 64, by chunks of 64, 128, 256, 512: 7.8 / 7.0 / 7.9 / 10.7.
// Short of that many workgroups without a cut, a chunk is no longer than max_len (at most 2^30); from there on there is none to make.
PagedSplit paged_split(int B, int H, int Hkv, int64_t max_len) {
  constexpr int64_t kWorkgroups = 1536;
  const int64_t units = decode_units(B, H, Hkv);
  const int64_t share = units < kWorkgroups ? (max_len * units + kWorkgroups - 1) / kWorkgroups : max_len;
  const int64_t chunk = std::max<int64_t>(128, (share + 63) / 64 * 64);
  return {(int)chunk, (int)std::max<int64_t>(1, (max_len + chunk - 1) / chunk)};
}

bool paged_decode_fits(int B, int H, int Hkv, PagedSplit s) {
  return decode_units(B, H, Hkv) * s.splits <= most_workgroups(kPagedThreads) &&
         (s.splits == 1 || (int64_t)B * H <= most_workgroups(kPagedThreads));
}
bool paged_fill_fits(int total, int n_seqs, int Hkv) { return packed_tiles(total, n_seqs, kFillRows) * Hkv <= most_workgroups(kPagedThreads); }

hipError_t launch_paged_decode(const PagedDecodeArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? decode<uint16_t, 128>(a, s) : decode<uint16_t, 64>(a, s);
  return a.d == 128 ? decode<float, 128>(a, s) : decode<float, 64>(a, s);
}

hipError_t launch_paged_fill(const PagedFillArgs& a, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)(packed_tiles(a.total, a.n_seqs, kFillRows) * a.Hkv));
  if (bf16) a.d == 128 ? paged_fill_kernel<uint16_t, 128><<<grid, kPagedThreads, 0, s>>>(a) : paged_fill_kernel<uint16_t, 64><<<grid, kPagedThreads, 0, s>>>(a);
  else a.d == 128 ? paged_fill_kernel<float, 128><<<grid, kPagedThreads, 0, s>>>(a) : paged_fill_kernel<float, 64><<<grid, kPagedThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, bool bf16, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.n_copies * a.Hkv));
  if (bf16) a.d == 128 ? pages_copy_kernel<uint16_t, 128><<<grid, kPagedThreads, 0, s>>>(a) : pages_copy_kernel<uint16_t, 64><<<grid, kPagedThreads, 0, s>>>(a);
  else a.d == 128 ? pages_copy_kernel<float, 128><<<grid, kPagedThreads, 0, s>>>(a) : pages_copy_kernel<float, 64><<<grid, kPagedThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gformer
