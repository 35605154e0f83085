// Forward pass of attention over packed sequences (packed.hpp has the formulas): softmax in one pass over the keys, with a
// running maximum and sum per query.
//
// A workgroup holds 128 queries of one head, 32 a wave, and streams key and value tiles through two LDS buffers: the next
// tile's rows arrive while the present one is used.
#include "packed.hpp"

#include <algorithm>

namespace gformer {
namespace {

template <typename T> constexpr int kFwdTile = sizeof(T) == 2 ? 64 : 32;   // keys per tile
template <typename T, int D> struct alignas(256) FwdTiles {
  T k[2][kFwdTile<T> * D], v[2][kFwdTile<T> * D];
  int flag;
};

template <typename T, int D> __global__ __launch_bounds__(kPackedThreads, (sizeof(T) == 4 && D == 128 ? 1 : D == 64 ? 3 : 2)) void packed_fwd_kernel(PackedArgs a, int tiles) {
  using P = Products<T, D>;
  constexpr int R = kFwdTile<T>, NS = R / 32, MT = D / 32, W = kPackedThreads / 64;
  using L = Tile<T, D, R>;
  extern __shared__ __align__(256) unsigned char smem_raw[];
  auto& sm = *reinterpret_cast<FwdTiles<T, D>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, lh = lane >> 5;

  // Heads fastest, the heads that share keys Hkv apart: workgroups are dealt to the 8 XCDs in turn, so that those of one key
  // head meet in few of them.
  const int hh = blockIdx.x % a.H, kvh = hh % a.Hkv, h = kvh * (a.H / a.Hkv) + hh / a.Hkv;
  const SeqTile at = ranked_tile<kPackedRows, false>(a.cu_q, a.total_q, a.cu_k, a.total_k, a.n_seqs, blockIdx.x / a.H, tiles, lane);
  if (at.first < 0) return;
  const int qbase = packed_row(a.cu_q, at.seq, a.total_q), i0 = at.first;
  if (at.seq == a.n_seqs) {
    if (a.zero_tail && i0 < a.total_q - qbase)
      zero_rows<T, D>(rows_of<T>(a.out, a.os, qbase + i0, h), a.os[0], min(kPackedRows, a.total_q - qbase - i0), tid);
    return;
  }
  const int nq = packed_row(a.cu_q, at.seq + 1, a.total_q) - qbase;
  if (i0 >= nq) return;
  const int kbase = packed_row(a.cu_k, at.seq, a.total_k);
  const int nk = max(packed_row(a.cu_k, at.seq + 1, a.total_k) - kbase, 0), off = nk - nq;

  const int q0 = i0 + 32 * wave;                  // this wave's first query
  const int i = q0 + ln, seen = min(i, nq - 1) + off;   // this lane's query sees keys 0 .. seen
  typename P::Resident q;
  P::load(q, rows_of<T>(a.q, a.qs, qbase + min(i, nq - 1), h), lane, a.scale < 0.f);
  // base-2 exponents are score * sc, the scale's sign is in q; zero is nudged so that a masked score keeps its weight of zero
  const float sc = (a.scale == 0.f ? 1e-30f : fabsf(a.scale)) * kLog2e;

  f32x16 o[MT];
  float m, l;   // running maximum (base 2) and this half's share of the sum

  const T* kp = rows_of<T>(a.k, a.ks, kbase, kvh);
  const T* vp = rows_of<T>(a.v, a.vs, kbase, kvh);
  const int last_key = min(i0 + kPackedRows, nq) - 1 + off;   // of the workgroup; < 0: no query sees any
  const int n_tiles = last_key < 0 ? 0 : last_key / R + 1;
  auto load = [&](int t) {
    L::template load<W>(sm.k[t & 1], kp, a.ks[0], t * R, nk - 1, wave, lane);
    L::template load<W>(sm.v[t & 1], vp, a.vs[0], t * R, nk - 1, wave, lane);
  };
  bool odd = false;
  auto attend = [&](int t, auto by_rows) {
    const int t0 = t * R;
    const bool mask = t0 + R - 1 > q0 + off;   // some query of the wave does not see the whole tile
    const T *kt = sm.k[t & 1], *vt = sm.v[t & 1];
    f32x16 s[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) s[n] = P::scores(kt + 32 * n * D, q, lane);
    if (mask) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = t0 + 32 * n + 8 * (r / 4) + 4 * lh + r % 4 > seen ? -INFINITY : s[n][r];
    }
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int r = 0; r < 16; r += 2) top = maximum3(top, s[n][r], s[n][r + 1]);
    top = max_over_halves(top * sc);
    // The reference follows the maximum lazily: sums are rescaled where it grows by more than 8, so weights stay below 2^8
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f) != 0) {
      const float up = fmaxf(m, top), by = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.f : up));
      m = up;
      l *= by;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[mt][r] *= by;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], sc, -ref));
        l += p[r];   // before it is rounded for the product: the log-sum-exp is kept in 32 bits
      }
      const typename P::Weights w = P::weights(p);
      if (by_rows && mask && L::odd(vt + 32 * n * D, lane)) P::product_by_rows(o, vt + 32 * n * D, w, 0, seen + 1 - t0 - 32 * n, lane);
      else P::product(o, vt + 32 * n * D, w, lane);
      if (!by_rows && mask) odd = odd || L::odd(vt + 32 * n * D, lane);
    }
  };
  auto pass = [&](auto by_rows) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[mt][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
    if (n_tiles) load(0);
    for (int t = 0; t < n_tiles; ++t) {
      loads_left<0>();
      lds_barrier();   // tile t is there, and nobody reads tile t - 1 any more
      if (t + 1 < n_tiles) load(t + 1);
      if (t * R <= min(q0 + 31, nq - 1) + off) attend(t, by_rows);   // else nothing for this wave
    }
    lds_barrier();   // every wave is done with the tiles
  };
  pass(std::false_type{});
  if (any_wave(&sm.flag, odd)) pass(std::true_type{});
  l = sum_over_halves(l);
  if (a.lse && lh == 0 && i < nq)
    a.lse[(int64_t)h * a.total_q + qbase + i] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  if (q0 < nq) {
    T* own = reinterpret_cast<T*>(smem_raw) + wave * 32 * kPutRow<T, D>;
    const float by = l == 0.f ? 0.f : 1.f / l;
    put_rows<T, D>(o, by, own, rows_of<T>(a.out, a.os, qbase + q0, h), a.os[0], min(32, nq - q0), lane);
    if (sizeof(T) == 2 && a.rest) put_rows<T, D, true>(o, by, own, rows_of<T>(a.rest, a.os, qbase + q0, h), a.os[0], min(32, nq - q0), lane);
  }
}

template <typename T, int D> hipError_t launch(const PackedArgs& a, hipStream_t s) {
  constexpr size_t smem = std::max(sizeof(FwdTiles<T, D>), kPackedRows * kPutRow<T, D> * sizeof(T));   // the rows leave through it
  auto kern = packed_fwd_kernel<T, D>;
  if (hipError_t e = allow_lds(kern, smem); e != hipSuccess) return e;
  const int64_t tiles = packed_tiles(a.total_q, a.n_seqs, kPackedRows);
  kern<<<dim3((unsigned)(tiles * a.H)), dim3(kPackedThreads), smem, s>>>(a, (int)tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_fwd(const PackedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d == 128 ? launch<uint16_t, 128>(a, s) : launch<uint16_t, 64>(a, s);
  return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace gformer
